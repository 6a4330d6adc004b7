"""Products of E4M3 rows with scales of any size: a result is lost only where fp32 itself does not hold it, not where the product of
two scales is 0, denormal or infinite on the way.

Tolerances, beside those of tests/test_gpu_projection.py for sums and roundings (the same number of roundings: mantissas' product, its
product with the sum, the addition, where one product and one fused addition stand otherwise): a denormal is rounded by up to
half of 2^-149 at each product and sum, (2 blocks + 1) 2^-150 in all, and a bf16 one by half of 2^-133."""
import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import projection_reference as R
from tests import projection_sizes as Z
from tests.test_gpu_projection import BF, E4, U, encoded, rnd, scales

pytestmark = pytest.mark.gpu

K, BLOCKS = 1168, 10
CLASSES = 5                                                     # of tokens; 3 of blocks of channels


def rows(tokens, seed=0):
    """Token t is of class t % 5: ordinary scales; of 2^-80; of 2^70 with codes of one step; ordinary ones with blocks of zeros whose
    scales are 2^100; scales of 0."""
    x, xs = encoded(seed + 1, tokens, K), torch.exp(0.3 * rnd(seed + 2, tokens, BLOCKS))
    b = x.view(torch.uint8)
    xs[1::CLASSES] *= 2.0 ** -80
    xs[2::CLASSES] *= 2.0 ** 70
    b[2::CLASSES] &= 0x81
    for at in range(1, BLOCKS, 2):
        b[3::CLASSES, 128 * at:128 * (at + 1)] = 0
        xs[3::CLASSES, at] = 2.0 ** 100
    xs[4::CLASSES] = 0
    return x, xs


def weight(n, seed=0):
    """Blocks of channels of ordinary scales, of 2^-60, and of 2^60 with codes of one step."""
    w, ws = encoded(seed + 3, n, K), torch.exp(0.3 * rnd(seed + 4, R.blocks(n), BLOCKS))
    ws[1::3] *= 2.0 ** -60
    ws[2::3] *= 2.0 ** 60
    for i in range(2, R.blocks(n), 3):
        w.view(torch.uint8)[128 * i:128 * (i + 1)] &= 0x81
    return w, ws


def product(x, xs, w, ws, out):
    n = w.shape[0]
    y = torch.full((x.shape[0], -(-n // 8) * 8), float("nan"), dtype=out, device="cuda")[:, :n]
    B.leapquant_matmul(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y)
    return y


@pytest.mark.parametrize("case", Z.one_each() + Z.several(), ids=Z.name)
def test_scales_whose_product_is_no_normal_number(case):
    _, tokens, n, out = case
    (x, xs), (w, ws) = rows(tokens), weight(n)
    y = product(x, xs, w, ws, out)
    a = (x.cuda().float().double() * R.spread_rows(xs.cuda().double(), K)).contiguous()
    b = (w.cuda().float().double() * R.spread_weight(ws.cuda().double(), n, K)).t().contiguous()
    want, size = a @ b, a.abs() @ b.abs()
    assert float(size.max()) < 2.0 ** 127                       # (fp32 holds every sum)
    tol = ((256 + BLOCKS + 20) * U + (7 * 2.0 ** -13 if out == BF else 0)) * size + (2 * BLOCKS + 1) * 2.0 ** -150
    if out == BF:
        tol = tol + (want.abs() + tol) * 2.0 ** -8 + 2.0 ** -134
    bad = ~((y.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(y[bad][0]), float(want[bad][0]))
    assert (y[4::CLASSES] == 0).all()


@pytest.mark.parametrize("case", Z.one_each() + Z.several(), ids=Z.name)
def test_ordinary_rows_keep_their_bits_beside_such_scales(case):
    _, tokens, n, out = case
    (x, xs), (w, ws) = rows(tokens), weight(n)
    y = product(x, xs, w, ws, out)
    other, others = encoded(11, tokens, K), scales(12, tokens, BLOCKS)
    other.view(torch.uint8)[::CLASSES], others[::CLASSES] = x.view(torch.uint8)[::CLASSES], xs[::CLASSES]
    assert torch.equal(y[::CLASSES], product(other, others, w, ws, out)[::CLASSES])


@pytest.mark.parametrize("tokens,n", [(3, 144), (320, 1664)])
def test_infinite_and_nan_scales_reach_their_own_row_only(tokens, n):
    x, xs, w, ws = encoded(1, tokens, K), scales(2, tokens, BLOCKS), encoded(3, n, K), scales(4, R.blocks(n), BLOCKS)
    want = product(x, xs, w, ws, torch.float32)
    xs[0, 3], xs[1, 9] = float("inf"), float("nan")
    got = product(x, xs, w, ws, torch.float32)
    assert not got[0].isfinite().any() and got[1].isnan().all() and torch.equal(got[2:], want[2:])


def test_encoded_rows_of_the_least_scales():
    """Rows and a weight near 2^-100 as the library encodes them: the scales' product is 0, their sums are denormal or 0."""
    x8, xs = torch.empty((5, 256), dtype=E4, device="cuda"), torch.empty((5, 2), device="cuda")
    w8, ws = torch.empty((40, 256), dtype=E4, device="cuda"), torch.empty((1, 2), device="cuda")
    x = rnd(1, 5, 256) * 2.0 ** -99
    x[3] = 0
    for size, least in ((2.0 ** -30, 2.0 ** -126), (2.0 ** -40, 2.0 ** -140)):
        w = rnd(2, 40, 256) * size
        B.leapquant_add_norm(x.cuda(), x8, norm=B.LQ_NORM_NONE, scale=xs)
        B.leapquant_quantize_weight(w.cuda(), w8, ws)
        y = torch.empty((5, 40), device="cuda")
        B.leapquant_matmul(x8, xs, w8, ws, y)
        want, mag = R.matmul(x8, xs, w8, ws)
        assert ((y.double().cpu() - want).abs() <= 300 * U * mag + 5 * 2.0 ** -150).all()
        assert (y[3] == 0).all() and float(want.abs().max()) > least


@pytest.mark.parametrize("tokens,n", [(16, 272), (320, 1664), (8256, 1408)])
def test_a_captured_call_follows_its_scales(tokens, n):
    """Replays with ordinary scales, with such scales and with ordinary ones again, eager calls in between."""
    (x, xs), (w, ws) = rows(tokens), weight(n)
    x, w, plain, plain_w = x.cuda(), w.cuda(), scales(21, tokens, BLOCKS).cuda(), scales(22, R.blocks(n), BLOCKS).cuda()
    turns = [(plain, plain_w), (xs.cuda(), ws.cuda()), (plain, plain_w), (xs.cuda(), plain_w)]
    want = [product(x, a, w, b, torch.float32) for a, b in turns]
    sx, sw, y = plain.clone(), plain_w.clone(), torch.empty((tokens, n), device="cuda")
    B.leapquant_matmul(x, sx, w, sw, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.leapquant_matmul(x, sx, w, sw, y)
    for (a, b), expected in zip(turns, want):
        sx.copy_(a)
        sw.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, expected)
        assert torch.equal(product(x, a, w, b, torch.float32), expected)
