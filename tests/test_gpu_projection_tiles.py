"""Products of E4M3 rows by every kernel that leapquant_matmul has (the sizes are held to their kernels by
tests/test_projection_choice.py): depths of k, values that are not finite, equal calls, rows far apart, and the mean error of the
sums.  Tolerances are those of tests/test_gpu_projection.py; references are made on the GPU in 64 bits."""
import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import projection_reference as R
from tests import projection_sizes as Z
from tests.test_gpu_projection import BF, E4, U

pytestmark = pytest.mark.gpu

NAN8 = 0x7F


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(seed, n, k):
    """Codes of all magnitudes, none of them NaN."""
    c = torch.randint(0, 256, (n, k), generator=generator(seed), dtype=torch.uint8, device="cuda")
    c[(c & 0x7F) == NAN8] = 0x38
    return c.view(E4)


def normal(seed, *shape):
    return torch.randn(shape, generator=generator(seed), device="cuda")


def inputs(t, k, n, seed=0):
    return codes(seed + 1, t, k), normal(seed + 3, t, R.blocks(k)).exp(), codes(seed + 2, n, k), normal(seed + 4, R.blocks(n), R.blocks(k)).exp()


def reference(x, xs, w, ws, bias=None):
    """As projection_reference.matmul, on the GPU."""
    (t, k), n = x.shape, w.shape[0]
    a = x.float().double() * R.spread_rows(xs.double(), k)
    b = (w.float().double() * R.spread_weight(ws.double(), n, k)).t().contiguous()
    y, size = a @ b, a.abs() @ b.abs()
    return (y, size) if bias is None else (y + bias.double(), size + bias.double().abs())


def output(t, n, out):
    """Rows of n, and the NaN behind each."""
    full = torch.full((t, -(-n // 8) * 8 + 8), float("nan"), dtype=out, device="cuda")
    return full[:, :n], full[:, n:]


def product(x, xs, w, ws, out, bias=None):
    y, rest = output(x.shape[0], w.shape[0], out)
    B.leapquant_matmul(x, xs, w, ws, y, bias=bias)
    assert rest.isnan().all()
    return y


def close(got, want, size, k):
    tol = ((256 + R.blocks(k) + 20) * U + (7 * 2.0 ** -13 if got.dtype == BF else 0)) * size
    if got.dtype == BF:
        tol = tol + (want.abs() + tol) * 2.0 ** -8
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]))


def check(t, k, n, out, bias):
    a = inputs(t, k, n)
    b = 1000 * normal(9, n) if bias else None
    close(product(*a, out, b), *reference(*a, b), k)


@pytest.mark.parametrize("k", [16, 112, 128, 144, 1168, 4096])
@pytest.mark.parametrize("case", Z.one_each(), ids=Z.name)
def test_depths(case, k):
    """From an eighth of a block to 32 blocks, ends inside a block among them."""
    _, t, n, out = case
    check(t, k, n, out, bias=n % 2 == 1)


@pytest.mark.parametrize("k", [112, 1168, 2048])
@pytest.mark.parametrize("case", Z.several(), ids=Z.name)
def test_depths_of_workgroups_that_take_several_tiles(case, k):
    _, t, n, out = case
    check(t, k, n, out, bias=True)


@pytest.mark.parametrize("case", Z.one_each(), ids=Z.name)
def test_values_that_are_not_finite_stay_in_their_row_and_channel(case):
    _, t, n, out = case
    k = 1168
    x, xs, w, ws = inputs(t, k, n)
    want = product(x, xs, w, ws, out)
    row, channel = t // 2, n - 2
    x, w = x.clone(), w.clone()
    x.view(torch.uint8)[row, k - 1] = 0x80 | NAN8               # in the last, shorter block
    w.view(torch.uint8)[channel, 130] = NAN8
    got = product(x, xs, w, ws, out)
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[row] = False
    others = [c for c in range(n) if c != channel]
    assert got[row].isnan().all() and got[:, channel].isnan().all()
    assert torch.equal(got[keep][:, others], want[keep][:, others])
    xs = xs.clone()
    xs[t - 1, 0] = float("inf")
    got = product(x, xs, w, ws, out)
    keep[t - 1] = False
    assert not got[t - 1].isfinite().any()
    assert torch.equal(got[keep][:, others], want[keep][:, others])


@pytest.mark.parametrize("case", Z.one_each() + Z.several(), ids=Z.name)
def test_equal_calls_are_equal_and_rows_do_not_depend_on_others(case):
    _, t, n, out = case
    x, xs, w, ws = inputs(t, 2064, n)
    want = product(x, xs, w, ws, out)
    for _ in range(8):
        assert torch.equal(product(x, xs, w, ws, out), want)
    other = codes(20, t, 2064)
    mine = torch.arange(0, t, 5, device="cuda")
    other.view(torch.uint8)[mine] = x.view(torch.uint8)[mine]
    assert torch.equal(product(other, xs, w, ws, out)[mine], want[mine])


@pytest.fixture(scope="module")
def far():
    """Memory for rows as far apart as they may be."""
    tiles = [c for c in Z.one_each() if c[0][0] == "tile"]
    t, n = max(c[1] for c in tiles), max(c[2] for c in tiles)
    size = {"x": ((t - 1 << 23) + 4096, torch.uint8), "w": ((n - 1 << 23) + 4096, torch.uint8), "xs": ((t - 1 << 20) + 64, torch.float32)}
    memory = {name: torch.empty(s, dtype=dtype, device="cuda") for name, (s, dtype) in size.items()}
    yield memory
    memory.clear()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("case", [c for c in Z.one_each() if c[0][0] == "tile"], ids=Z.name)
def test_rows_as_far_apart_as_they_may_be(case, far):
    """Tiles address their rows by 32 bits from the first one on."""
    _, t, n, out = case
    k = 272
    x, xs, w, ws = inputs(t, k, n)
    want = product(x, xs, w, ws, out)
    xf = far["x"].as_strided((t, k), (1 << 23, 1))
    wf = far["w"].as_strided((n, k), (1 << 23, 1))
    sf = far["xs"].as_strided((t, R.blocks(k)), (1 << 20, 1))
    xf.copy_(x.view(torch.uint8))
    wf.copy_(w.view(torch.uint8))
    sf.copy_(xs)
    assert torch.equal(product(xf.view(E4), sf, wf.view(E4), ws, out), want)


@pytest.mark.parametrize("case", Z.one_each(), ids=Z.name)
def test_mean_error_of_the_sums(case):
    """Of normal values as the library encodes them.  The bias takes the exact sum away, so what is left and rounded is the sum's error.
    bf16 outputs: the 1.4e-5 of the sums' size that the 8-bit products were measured at, taken twice and up to a power of two.  fp32:
    roundings of one U each, independent: one a block, and those of the scales and of the bias."""
    _, t, n, out = case
    k = 4096
    w8, ws = torch.empty((n, k), dtype=E4, device="cuda"), torch.empty((R.blocks(n), R.blocks(k)), device="cuda")
    B.leapquant_quantize_weight(normal(1, n, k) / 64, w8, ws)
    x8, xs = torch.empty((3, k), dtype=E4, device="cuda"), torch.empty((3, R.blocks(k)), device="cuda")
    B.leapquant_add_norm(normal(2, 3, k), x8, norm=B.LQ_NORM_NONE, scale=xs)
    y, _ = reference(x8, xs, w8, ws)
    bias = -y.float()
    limit = 2.0 ** -15 if out == BF else (R.blocks(k) ** 0.5 + 2) * U
    for i in range(3):
        x = x8.view(torch.uint8)[i].expand(t, k).contiguous().view(E4)
        got = product(x, xs[i].expand(t, -1).contiguous(), w8, ws, out, bias[i])
        error = got.double() - (y[i] + bias[i].double())
        assert error.square().mean().sqrt() <= limit * y[i].square().mean().sqrt()
        assert torch.equal(got, got[:1].expand(t, -1))          # (equal rows: wherever a token stands, its sum is the same)
