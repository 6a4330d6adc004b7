"""Projection operators (residual and norm, gated norm, weights and products in E4M3) against their definitions in 64 bits.

Tolerances, from the rounding errors of the operations (u = 2^-24, the half ulp of fp32; library functions are within 2 ulp,
4 u):
  add_norm   the sum h one rounding, 1 u of h; the squares' sum over c channels: at most 8 P fused terms in a lane (P pieces of 8,
             32 at most) and a tree of at most 10, (32 + 10) u, half of it after the root; eps, the mean's division, the
             root, the reciprocal and the products with it and with the weight 7 u: under 32 u of |y| in all, beside
             1 u of |x| + |r| (the sum's own), times the norm's factor: 40 u (|y| + the norm's share of |x| + |r|);
  gate_norm  the same, and the gate: exp 4 u of itself, the exponent's argument exact, a sum and a division 2 u, one product:
             under 8 u more, 48 u |y|;
  scale      most is a value of y, the division one rounding: that value's tolerance / 448 and 1 u;
  codes      within half a step of the value over the scale: 2^-4 of it (e4m3's eps / 2) above 2^-6, 2^-10 (half the smallest
             step) below, beside the errors of the value, the factor (2 u) and the product (1 u);
  matmul     fp32: a block's 128 products are exact and summed in the matrix cores: at most 128 roundings (or cuts: twice that)
             of partial sums, so 256 u of the sum of magnitudes; then two products, and a sum a block and for every join of at
             most 16 parts: (blocks + 20) u.  bf16: the 8-bit products are summed in groups of 8 with the bits above 2^-13 of the
             group's largest one, so 7 * 2^-13 of the sum of magnitudes more;
  bf16       half a step, 2^-8 of the value, beside the error of the value that is rounded.
"""
import math

import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import projection_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def rnd(seed, *shape, scale=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g) * scale


def close(got, want, tol):
    """Elementwise within tol plus the rounding of a bf16 result; the same places hold NaN or the same infinity."""
    got_ = got.double().cpu()
    if got.dtype == BF:
        tol = tol + (want.abs() + tol) * 2.0 ** -8
    bad = ~((got_ - want).abs() <= tol) & ~(got_.isnan() & want.isnan()) & ~(got_ == want)
    assert not bad.any(), (int(bad.sum()), bad.numel(), float((got_ - want).abs()[bad].nan_to_num(math.inf).max()),
                           bad.nonzero()[0].tolist())


def close_codes(codes, scale, y, tol, scales):
    """An E4M3 output [rows][channels] of y, each within tol of its exact value; scales: the exact ones, [rows][blocks] or
    spread like y."""
    spread = scales if scales.shape == y.shape else R.spread_rows(scales, y.shape[1])
    assert not codes.float().isnan().any()
    # (the block's largest value decides the scale, with its own error)
    most = tol.max() if tol.dim() else tol
    assert ((scale.double().cpu() - scales).abs() <= most / 448 + 2 * U * scales).all()
    v = y / spread
    got = codes.cpu().float().double()
    err = tol / spread + (v.abs() * (most / (448 * spread) + 4 * U))
    step = torch.where(v.abs() + err >= 2.0 ** -6, (v.abs() + err) * 2.0 ** -4, torch.full_like(v, 2.0 ** -10))
    bad = (got - v).abs() > step + err
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(v[bad][0]))


def rows(t, wide=None, pad=0):
    """t [tokens][..] on the GPU as a slice of wider rows that hold NaN elsewhere."""
    n, c = t.shape[0], t[0].numel() if t.shape[0] else math.prod(t.shape[1:])
    per = 16 // t.element_size()
    extra = per if wide is None else wide
    full = torch.full((n, c + pad + 2 * extra), float("nan"), device="cuda").to(t.dtype)
    part = full[:, extra:extra + c]
    part.copy_(t.reshape(n, c))
    return part.view(t.shape), full


def outside_untouched(full, part_cols, start):
    keep = torch.ones(full.shape[1], dtype=torch.bool)
    keep[start:start + part_cols] = False
    assert full.float()[:, keep.cuda()].isnan().all()


# -------------------------------------------------------------------------------------------------------- add_norm

CHANNELS = [8, 64, 120, 128, 136, 512, 520, 1024, 1544, 2048, 2056, 4096, 4104, 8192, 8200, 16376, 16384]


@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("dtype,rtype,out,residual,norm,weight", [
    (BF, BF, E4, True, True, True), (F32, F32, E4, True, True, False), (BF, F32, E4, True, True, True),
    (F32, BF, BF, True, True, True), (BF, BF, F32, False, True, True), (F32, F32, F32, False, False, False),
    (BF, BF, E4, False, False, False), (BF, BF, BF, True, False, False)])
def test_add_norm(channels, dtype, rtype, out, residual, norm, weight):
    n = 5 if channels > 4096 else 19
    x = rnd(1, n, channels).to(dtype)
    r = (3 * rnd(2, n, channels)).to(rtype) if residual else None
    w = 1 + 0.1 * rnd(3, channels) if weight else None
    h, y = R.add_norm(x, r, w, norm)
    xg, _ = rows(x)
    rg = rows(r)[0] if residual else None
    ro, rfull = rows(torch.zeros(n, channels, dtype=rtype)) if residual else (None, None)
    # (rows of 16-byte multiples; 8 bytes between where the channels leave them)
    og, ofull = rows(torch.zeros(n, channels, dtype=out), pad=8 if out == E4 and channels % 16 else 0)
    scale = torch.full((n, R.blocks(channels) + 1), float("nan"), device="cuda")[:, 1:] if out == E4 else None
    B.leapquant_add_norm(xg, og, residual=rg, residual_out=ro, weight=w.cuda() if weight else None,
                         norm=B.LQ_NORM_RMS if norm else B.LQ_NORM_NONE, scale=scale)
    mag = x.double().abs() + (r.double().abs() if residual else 0)
    factor = (y.abs() / h.abs().clamp(min=1e-30)).clamp(max=1e3)
    tol = 40 * U * (y.abs() + factor * mag)
    if residual:
        close(ro, h, U * mag)
        outside_untouched(rfull, channels, 16 // ro.element_size())
        assert torch.equal(rg.cpu(), r)
    if out == E4:
        close_codes(og, scale, y, tol, R.row_scales(y))
    else:
        close(og, y, tol)
    outside_untouched(ofull, channels, 16 // og.element_size())


def test_add_norm_in_place_and_dense_rows():
    x, r = rnd(1, 33, 1024).bfloat16(), rnd(2, 33, 1024)
    h, y = R.add_norm(x, r)
    xg, rg = x.cuda(), r.cuda()
    B.leapquant_add_norm(xg, xg, residual=rg, residual_out=rg)
    close(rg, h, 2 * U * (x.double().abs() + r.double().abs()))
    close(xg, y, 80 * U * (x.double().abs() + r.double().abs() + 1))
    # without a residual the rows themselves can be kept
    kept = torch.empty((33, 1024), device="cuda")
    B.leapquant_add_norm(x.cuda(), xg, residual_out=kept)
    assert torch.equal(kept.cpu(), x.float())


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 8191, 20011])
@pytest.mark.parametrize("channels", [128, 4096])
def test_add_norm_many_rows(tokens, channels):
    """Rows that the workgroups take in turn."""
    if tokens * channels > 1 << 25:
        tokens = (1 << 25) // channels
    x = rnd(1, tokens, channels).bfloat16()
    _, y = R.add_norm(x)
    og, scale = torch.empty((tokens, channels), dtype=E4, device="cuda"), torch.empty((tokens, channels // 128), device="cuda")
    B.leapquant_add_norm(x.cuda(), og, scale=scale)
    close_codes(og, scale, y, 80 * U * y.abs(), R.row_scales(y))


def test_add_norm_values_that_are_not_finite_stay_in_their_row_or_block():
    x = rnd(1, 6, 512)
    bad = x.clone()
    bad[1, 200], bad[3, 300], bad[4, 0] = float("nan"), float("inf"), float("-inf")
    for norm in (B.LQ_NORM_RMS, B.LQ_NORM_NONE):
        got = []
        for y in (x, bad):
            og, scale = torch.zeros((6, 512), dtype=E4, device="cuda"), torch.zeros((6, 4), device="cuda")
            B.leapquant_add_norm(y.cuda(), og, norm=norm, scale=scale)
            got.append((og.float().cpu(), scale.cpu()))
        for t in (0, 2, 5):
            assert torch.equal(got[0][0][t], got[1][0][t]) and torch.equal(got[0][1][t], got[1][1][t])
        code, scale = got[1]
        if norm == B.LQ_NORM_RMS:
            assert code[1].isnan().all() and scale[1].isnan().all()
            for t, c in ((3, 300), (4, 0)):                     # 1 / inf: zeros, and inf * 0
                assert code[t, c].isnan() and scale[t, c // 128].isnan()
                other = [b for b in range(4) if b != c // 128]
                assert (scale[t, other] == torch.tensor(R.LEAST / 448)).all()
                assert (code[t].view(4, 128)[other] == 0).all()
        else:
            assert code[1, 128:256].isnan().all() and scale[1, 1].isnan()
            assert code[3, 300].isnan() and scale[3, 2] == math.inf
            assert (code[3, 256:384][torch.arange(128) != 44] == 0).all()
            assert torch.equal(code[3, :256], got[0][0][3, :256]) and torch.equal(code[4, 128:], got[0][0][4, 128:])


def test_add_norm_zeros_and_tiny_blocks():
    x = torch.zeros(3, 384)
    x[1, 5] = 2.0 ** -120                                       # below the least scale's smallest code: 0
    x[2, 130] = 2.0 ** -100
    x[2, 131] = -2.0 ** -104
    og, scale = torch.zeros((3, 384), dtype=E4, device="cuda"), torch.zeros((3, 3), device="cuda")
    B.leapquant_add_norm(x.cuda(), og, norm=B.LQ_NORM_NONE, scale=scale)
    least = torch.tensor(R.LEAST, dtype=F32) / 448
    assert (scale.cpu() == least).all()
    want = torch.zeros(3, 384)
    want[2, 130], want[2, 131] = 448.0, -28.0
    assert torch.equal(og.cpu().float(), want)
    o = torch.empty((3, 384), device="cuda")
    B.leapquant_add_norm(torch.zeros((3, 384), device="cuda"), o)
    assert (o == 0).all()


def test_codes_reach_every_value():
    """The codes of a block that holds every E4M3 value are those values."""
    every = torch.arange(256, dtype=torch.uint8).view(E4).float()
    every = every[~every.isnan()]
    x = torch.zeros(2, 256)
    x[0, :254], x[1, 1:255] = every, every
    x[0, 254], x[1, 0] = 448, 448                               # (both blocks' largest)
    x[0, 127], x[1, 128] = 448, -448
    x = x.view(4, 128)
    og, scale = torch.zeros((4, 128), dtype=E4, device="cuda"), torch.zeros((4, 1), device="cuda")
    B.leapquant_add_norm(x.cuda(), og, norm=B.LQ_NORM_NONE, scale=scale)
    assert (scale == 1).all() and torch.equal(og.cpu().float(), x)


# ------------------------------------------------------------------------------------------------------- gate_norm

@pytest.mark.parametrize("heads,d", [(1, 64), (3, 64), (4, 64), (1, 128), (5, 128), (32, 128), (3, 256), (2, 384), (3, 512),
                                     (2, 1024), (1, 1664), (2, 2048), (1, 4096), (1, 8192), (1, 12288), (2, 16384)])
@pytest.mark.parametrize("dtype,gtype,out,act,first,weight", [
    (BF, BF, E4, "silu", False, 1), (F32, BF, E4, "sigmoid", False, 1), (F32, F32, F32, "silu", True, 2),
    (BF, F32, BF, "sigmoid", True, 0), (BF, BF, E4, "silu", True, 2)])
def test_gate_norm(heads, d, dtype, gtype, out, act, first, weight):
    n = 7 if heads * d <= 8192 else 3
    x, z = rnd(1, n, heads, d).to(dtype), (2 * rnd(2, n, heads, d)).to(gtype)
    w = None if weight == 0 else 1 + 0.1 * rnd(3, d) if weight == 1 else 1 + 0.1 * rnd(3, heads, d)
    y = R.gate_norm(x, z, w, act, first)
    og, ofull = rows(torch.zeros(n, heads, d, dtype=out))
    scale = torch.full((n, R.blocks(heads * d)), float("nan"), device="cuda") if out == E4 else None
    B.leapquant_gate_norm(rows(x)[0], rows(z)[0], og, weight=None if w is None else w.cuda(),
                          act=B.LQ_ACT_SILU if act == "silu" else B.LQ_ACT_SIGMOID, gate_first=first, scale=scale)
    tol = 48 * U * y.abs()
    if out == E4:
        flat = y.reshape(n, -1)
        close_codes(og.reshape(n, -1), scale, flat, tol.reshape(n, -1), R.row_scales(flat))
    else:
        close(og, y, tol)
    outside_untouched(ofull, heads * d, 16 // og.element_size())


@pytest.mark.parametrize("tokens,heads,d", [(1, 1, 64), (3001, 3, 64), (2501, 7, 128), (1999, 2, 256), (9000, 1, 384)])
def test_gate_norm_many_rows(tokens, heads, d):
    x, z = rnd(1, tokens, heads, d).bfloat16(), rnd(2, tokens, heads, d).bfloat16()
    y = R.gate_norm(x, z)
    og = torch.empty((tokens, heads, d), dtype=BF, device="cuda")
    B.leapquant_gate_norm(x.cuda(), z.cuda(), og)
    close(og, y, 48 * U * y.abs())


def test_gate_norm_in_place_and_extreme_gates():
    x = rnd(1, 4, 2, 128)
    z = torch.zeros(4, 2, 128)
    z[0], z[1], z[2], z[3] = 200.0, -200.0, float("inf"), -60.0
    for act in ("silu", "sigmoid"):
        y = R.gate_norm(x, z, None, act)
        xg, zg = x.cuda(), z.cuda()
        B.leapquant_gate_norm(xg, zg, xg, act=B.LQ_ACT_SILU if act == "silu" else B.LQ_ACT_SIGMOID)
        close(xg[[0, 2, 3]], y[[0, 2, 3]], 48 * U * y[[0, 2, 3]].abs().clamp(max=1e30))
        assert (xg[1].abs() < 1e-30).all()
        B.leapquant_gate_norm(x.cuda(), zg, zg, act=B.LQ_ACT_SILU if act == "silu" else B.LQ_ACT_SIGMOID)
        assert torch.equal(zg, xg)


def test_gate_norm_nan_stays_in_its_head():
    x, z = rnd(1, 3, 4, 128), rnd(2, 3, 4, 128)
    bad = x.clone()
    bad[1, 2, 7] = float("nan")
    out = []
    for v in (x, bad):
        og, scale = torch.zeros((3, 4, 128), dtype=E4, device="cuda"), torch.zeros((3, 4), device="cuda")
        B.leapquant_gate_norm(v.cuda(), z.cuda(), og, scale=scale)
        out.append((og.float().cpu(), scale.cpu()))
    same = torch.ones(3, 4, dtype=torch.bool)
    same[1, 2] = False
    assert torch.equal(out[0][0][same], out[1][0][same]) and torch.equal(out[0][1][same], out[1][1][same])
    assert out[1][0][1, 2].isnan().all() and out[1][1][1, 2].isnan()


# ------------------------------------------------------------------------------------------------- quantize_weight

@pytest.mark.parametrize("n,k", [(1, 16), (127, 128), (128, 144), (129, 112), (257, 400), (1000, 1552), (5, 4096)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_weight(n, k, dtype):
    w = (rnd(1, n, k) * torch.exp(rnd(2, n, 1))).to(dtype)
    wg, _ = rows(w)
    og, ofull = rows(torch.zeros(n, k, dtype=E4))
    scale = torch.full((R.blocks(n), R.blocks(k)), float("nan"), device="cuda")
    B.leapquant_quantize_weight(wg, og, scale)
    want = R.weight_scales(w)
    assert ((scale.double().cpu() - want).abs() <= U * want).all()
    v = w.double() / R.spread_weight(want, n, k)
    step = torch.where(v.abs() >= 2.0 ** -6, v.abs() * (2.0 ** -4 + 4 * U), torch.full_like(v, 2.0 ** -10 + 2.0 ** -28))
    assert ((og.cpu().float().double() - v).abs() <= step).all()
    outside_untouched(ofull, k, 16)


def test_quantize_weight_not_finite_stays_in_its_block():
    w = rnd(1, 256, 256)
    w[3, 5], w[200, 130] = float("nan"), float("inf")
    og, scale = torch.zeros((256, 256), dtype=E4, device="cuda"), torch.zeros((2, 2), device="cuda")
    B.leapquant_quantize_weight(w.cuda(), og, scale)
    code, scale = og.float().cpu(), scale.cpu()
    assert scale[0, 0].isnan() and code[:128, :128].isnan().all()
    assert scale[1, 1] == math.inf and code[200, 130].isnan() and int((code[128:, 128:] != 0).sum()) == 1
    assert scale[0, 1].isfinite() and scale[1, 0].isfinite()
    assert not code[:128, 128:].isnan().any() and not code[128:, :128].isnan().any()


# ---------------------------------------------------------------------------------------------------------- matmul

def encoded(seed, n, k):
    """Codes of all magnitudes and scales of different sizes, as they come (not only those that an encoder makes)."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (n, k), generator=g, dtype=torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x38
    return codes.view(E4)


def scales(seed, *shape):
    return torch.exp(rnd(seed, *shape))


def check_matmul(t, k, n, out, bias=True, seed=0):
    x, w = encoded(seed + 1, t, k), encoded(seed + 2, n, k)
    xs, ws = scales(seed + 3, t, R.blocks(k)), scales(seed + 4, R.blocks(n), R.blocks(k))
    b = 1000 * rnd(seed + 5, n) if bias else None
    y, size = R.matmul(x, xs, w, ws, b)
    # (float8 tensors are made as bytes: the rows' surroundings are NaN codes)
    xg, wg = rows8(x), rows8(w)
    wide = -(-n // 8) * 8 + 8
    full = torch.full((t, wide), float("nan"), dtype=out, device="cuda")
    og = full[:, :n]
    xsg = torch.full((t, R.blocks(k) + 1), float("nan"), device="cuda")
    xsg[:, :-1] = xs.cuda()
    B.leapquant_matmul(xg, xsg[:, :-1], wg, ws.cuda(), og, bias=b.cuda() if bias else None)
    close(og, y, ((256 + R.blocks(k) + 20) * U + (7 * 2.0 ** -13 if out == BF else 0)) * size)
    assert full[:, n:].isnan().all()


def rows8(t):
    n, c = t.shape
    full = torch.full((n, c + 32), 0x7F, dtype=torch.uint8, device="cuda")
    full[:, 16:16 + c] = t.view(torch.uint8).cuda()
    return full.view(E4)[:, 16:16 + c]


TOKENS = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 257, 300]


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("tokens", TOKENS)
def test_matmul_tokens(tokens, out):
    check_matmul(tokens, 1168, 272, out)                        # (a last block of 16)


@pytest.mark.parametrize("tokens", [1, 40, 150, 300])
@pytest.mark.parametrize("k", [16, 32, 112, 128, 144, 240, 256, 272, 512, 640, 1024, 1040, 2048, 4096, 8192])
def test_matmul_depths(tokens, k):
    check_matmul(tokens, k, 144, F32, bias=False)


@pytest.mark.parametrize("tokens", [3, 70, 259])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 15, 16, 17, 64, 100, 127, 128, 129, 255, 256, 257, 511, 513, 1000])
@pytest.mark.parametrize("out", [BF, F32])
def test_matmul_channels(tokens, n, out):
    check_matmul(tokens, 400, n, out, bias=n % 2 == 1)


@pytest.mark.parametrize("tokens,k,n", [(1, 4096, 12288), (7, 2048, 4100), (64, 4096, 4096), (256, 4096, 2048), (1531, 1552, 1000),
                                        (2048, 1024, 2304), (513, 4096, 513), (4100, 512, 771)])
def test_matmul_large(tokens, k, n):
    check_matmul(tokens, k, n, BF)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("tokens,k,n", [(8200, 256, 2200), (8200, 128, 2200), (8192, 384, 2304), (40000, 256, 64), (30000, 640, 100),
                                        (20000, 128, 200), (9000, 1024, 520), (8200, 144, 2200), (33, 256, 20000), (2100, 128, 2048)])
def test_matmul_workgroups_that_take_several_tiles(tokens, k, n, out):
    """More tiles than workgroups, whole ones and edges in turn, of one block of k and more (and one tile each where k ends
    inside a block)."""
    check_matmul(tokens, k, n, out, bias=n % 8 == 0)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("tokens,k,n", [(1531, 272, 4096), (1530, 144, 4093), (8084, 400, 1291), (3000, 272, 4096), (4381, 144, 5380),
                                        (1924, 400, 8850), (2050, 144, 7196), (8234, 272, 779), (7684, 144, 3100)])
def test_matmul_tiles(tokens, k, n, out):
    """Every size of tile, with one tile a workgroup and with two, whole ones and edges."""
    check_matmul(tokens, k, n, out, bias=n % 2 == 1)


def test_matmul_values_that_are_not_finite_stay_in_their_row_and_channel():
    t, k, n = 70, 400, 300
    x, w = encoded(1, t, k), encoded(2, n, k)
    xs, ws = scales(3, t, 4), scales(4, 3, 4)
    xs[33, 2] = float("nan")
    xs[5, 0] = float("inf")
    x.view(torch.uint8)[69, 399] = 0x7F                         # NaN in the last, shorter block
    w.view(torch.uint8)[299, 390] = 0xFF
    og = torch.empty((t, 304), device="cuda")[:, :n]
    B.leapquant_matmul(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), og)
    got = og.cpu()
    assert got[33].isnan().all() and got[69].isnan().all() and got[:, 299].isnan().all()
    assert not got[5, :299].isfinite().any()
    keep = torch.ones(t, dtype=torch.bool)
    keep[[33, 69, 5]] = False
    y, size = R.matmul(x, xs, w, ws)
    close(got[keep][:, :299], y[keep][:, :299], 300 * U * size[keep][:, :299])


@pytest.mark.parametrize("tokens", [1, 64, 300])
def test_matmul_is_repeatable_and_rows_do_not_depend_on_others(tokens):
    k, n = 2064, 1100
    x, w = encoded(1, tokens, k).cuda(), encoded(2, n, k).cuda()
    xs, ws = scales(3, tokens, R.blocks(k)).cuda(), scales(4, R.blocks(n), R.blocks(k)).cuda()
    out = [torch.empty((tokens, 1104), device="cuda")[:, :n] for _ in range(3)]
    for o in out[:2]:
        B.leapquant_matmul(x, xs, w, ws, o)
    assert torch.equal(out[0], out[1])
    other = encoded(9, tokens, k).cuda()
    other.view(torch.uint8)[0] = x.view(torch.uint8)[0]
    B.leapquant_matmul(other, xs, w, ws, out[2])
    assert torch.equal(out[2][0], out[0][0])


def test_no_tokens():
    e = lambda *s, dtype=F32: torch.empty(s, dtype=dtype, device="cuda")      # noqa: E731
    B.leapquant_add_norm(e(0, 128), e(0, 128, dtype=E4), scale=e(0, 1))
    B.leapquant_gate_norm(e(0, 2, 128), e(0, 2, 128), e(0, 2, 128))
    w, ws = e(64, 256, dtype=E4), e(1, 2)
    B.leapquant_matmul(e(0, 256, dtype=E4), e(0, 2), w, ws, e(0, 64))
    torch.cuda.synchronize()
