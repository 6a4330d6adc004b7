"""Layer operators (convolution, query/key norm, selective scan) against their definitions in 64 bits.

Tolerances, from the rounding errors of the operations (u = 2^-24, the half ulp of fp32):
  convolution  width + 1 roundings of terms whose magnitudes sum to m: 5 u m; the activation adds 4 u |y| and the exponent's
               rounding, together under 1e-6 (m + 1);
  norm         a sum of d squares in 8 fused terms and a tree of up to 5, a root, a division, a product, the weight, and
               two products and a sum of the rotation: under 24 u of the head's largest value of the row;
  scan         every step rounds a running sum twice: (2 t + 16) u of the sum of the terms' magnitudes after t tokens, with
               at most 512 of them counted where the operands are split (a chunk's sum is rounded once per product, so the
               count of tokens only bounds it); bf16 tokens are multiplied from two bf16 terms per 32-bit factor: 2^-17 for
               each of two factors more;
  bf16 output  half an ulp, 2^-8 of the value, beside the error of the value that is rounded.
"""
import math

import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import layer_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def rnd(seed, *shape, scale=1.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g) * scale


def close(got, want, tol):
    """Elementwise within tol plus the rounding of a bf16 result; the same places hold NaN."""
    got_ = got.double().cpu()
    if got.dtype == BF:
        tol = tol + want.abs() * 2.0 ** -8
    bad = ~((got_ - want).abs() <= tol) & ~(got_.isnan() & want.isnan())
    assert not bad.any(), (int(bad.sum()), bad.numel(), float((got_ - want).abs()[bad].nan_to_num(math.inf).max()),
                           bad.nonzero()[0].tolist())


def packed(lens, tail=0):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32), cu[-1] + tail


LENGTHS = [[1], [0], [0, 5, 0], [16], [17, 1, 2, 3, 64, 0, 33], [130, 3, 15, 16, 61], [1] * 70 + [0] * 3 + [2] * 70]


# ------------------------------------------------------------------------------------------------------ convolution

@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("width,dtype,out,silu,bias,carry", [
    (4, BF, BF, True, True, True), (4, BF, F32, False, False, False), (3, F32, F32, True, False, True),
    (2, F32, BF, False, True, False), (2, BF, F32, True, True, True), (3, BF, BF, True, True, False)])
def test_conv_prompt(lens, width, dtype, out, silu, bias, carry):
    cu, n = packed(lens, tail=3)
    seqs, c = len(lens), 264 if dtype == F32 else 520     # a full block of lanes and a few of the next
    x, w = rnd(1, n, c).to(dtype), rnd(2, c, width)
    b = rnd(3, c) if bias else None
    slots = torch.randperm(seqs + 2, generator=torch.Generator().manual_seed(4))[:seqs].int()
    state = rnd(5, seqs + 2, width - 1, c).to(dtype)
    spans = R.lengths(cu, n)
    want, size, new = R.conv(x, w, spans, b, silu, state[slots.long()] if carry else None)
    o = torch.full((n, c), float("nan"), dtype=out, device="cuda")
    st = state.cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.leapquant_conv_prompt(x.cuda(), w.cuda(), o, cu.cuda(), bias=b.cuda() if bias else None, silu=silu, state=st,
                            carry=carry, slots=slots.cuda(), err=err)
    close(o, want, 1e-6 * (size + 1))
    kept = state.double()
    kept[slots.long()] = new
    assert torch.equal(st.cpu().double(), kept)           # the last inputs as they are, other slots untouched
    assert B.leapquant_check_error_word(err) == 0


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("batch", [1, 7])
def test_conv_step_continues_the_prompt(batch, width, dtype, out):
    """Tokens one by one give what the whole sequence gives, bit for bit, and leave the same state."""
    c, n = 2056, 9
    x, w, b = rnd(1, batch, n, c).to(dtype).cuda(), rnd(2, c, width).cuda(), rnd(3, c).cuda()
    cu = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * n
    whole = torch.empty((batch * n, c), dtype=out, device="cuda")
    st0 = torch.zeros((batch, width - 1, c), dtype=dtype, device="cuda")
    B.leapquant_conv_prompt(x.view(-1, c), w, whole, cu, bias=b, state=st0)
    st1 = torch.zeros_like(st0)
    for t in range(n):
        o = torch.empty((batch, c), dtype=out, device="cuda")
        B.leapquant_conv_step(x[:, t], w, o, st1, bias=b)             # (rows n * c apart)
        assert torch.equal(o, whole.view(batch, n, c)[:, t])
    assert torch.equal(st0, st1)


def test_conv_slots_padding_and_bad_ones():
    c, width = 64, 4
    x, w = rnd(1, 4, c).cuda(), rnd(2, c, width).cuda()
    state = rnd(3, 2, width - 1, c)
    for prompt in (False, True):
        st = state.cuda()
        slots = torch.tensor([1, -1, 5, 0], dtype=torch.int32, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        o = torch.empty((4, c), device="cuda")
        if prompt:
            cu = torch.arange(5, dtype=torch.int32, device="cuda")
            B.leapquant_conv_prompt(x, w, o, cu, state=st, carry=True, slots=slots, err=err)
        else:
            B.leapquant_conv_step(x, w, o, st, slots=slots, err=err)
        old = torch.stack([state[1], torch.zeros_like(state[0]), torch.full_like(state[0], float("nan")), state[0]])
        want, size, new = R.conv(x, w, [(i, i + 1) for i in range(4)], None, True, old)
        close(o, want, 1e-6 * (size.nan_to_num(0.0) + 1))
        assert o[2].isnan().all()
        assert torch.equal(st.cpu().double(), torch.stack([new[3], new[0]]))
        assert B.leapquant_check_error_word(err) == B.LQ_DEVERR_BAD_SLOT
        assert B.leapquant_check_error_word(err) == 0


def test_conv_not_finite_stays_in_its_sequence_and_after_its_token():
    c, width = 64, 4
    cu, n = packed([20, 20, 20])
    x, w = rnd(1, n, c), rnd(2, c, width).cuda()
    bad = x.clone()
    bad[25] = float("nan")
    bad[19, ::2] = float("inf")
    got = []
    for y in (x, bad):
        o = torch.empty((n, c), device="cuda")
        B.leapquant_conv_prompt(y.cuda(), w, o, cu.cuda())
        got.append(o)
    same = torch.ones(n, dtype=torch.bool)
    same[25:25 + width] = same[19] = False
    assert torch.equal(got[0][same.cuda()], got[1][same.cuda()])
    assert got[1][25:29].isnan().all()


# ------------------------------------------------------------------------------------------------- query / key norm

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("norm,rot,interleaved", [("l2", 0, False), ("rms", 1, False), ("rms", 4, True), ("none", 2, False),
                                                  ("l2", 1, True), ("none", 4, False)])
def test_qk_norm(d, dtype, out, norm, rot, interleaved):
    n, hq, hk, npos = 37, 5, 3, 50
    q, k = (rnd(i, n, h + 1, d).to(dtype).cuda()[:, :h] for i, h in ((1, hq), (2, hk)))      # rows of a wider array
    q[3, 1] = 0                                            # a head of zeros
    weights = [1 + 0.2 * rnd(i, d) if norm == "rms" else None for i in (3, 4)]
    r = d * rot // 4 if rot > 1 else (16 if rot else 0)
    cos = sin = pos = None
    if r:
        angle = rnd(5, npos, r // 2) * 3
        cos, sin = angle.cos(), angle.sin()
        pos = torch.randint(0, npos, (n,), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
        pos[5], pos[6] = -1, npos
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo, ko = (torch.empty((n, h + 2, d), dtype=out, device="cuda")[:, :h] for h in (hq, hk))
    cuda = lambda t: None if t is None else t.cuda()                                        # noqa: E731
    B.leapquant_qk_norm(q, k, qo, ko, norm={"none": 0, "l2": 1, "rms": 2}[norm], eps=1e-6, q_weight=cuda(weights[0]),
                        k_weight=cuda(weights[1]), q_scale=0.3, cos=cuda(cos), sin=cuda(sin), positions=cuda(pos),
                        interleaved=interleaved, err=err)
    for x, o, w, scale in ((q, qo, weights[0], 0.3), (k, ko, weights[1], 1.0)):
        want = R.qk_norm(x, norm, 1e-6, w, scale, cos, sin, pos, interleaved)
        top = want.nan_to_num(0.0).abs().amax(-1, keepdim=True)
        top = torch.maximum(top, R.qk_norm(x, norm, 1e-6, w, scale).abs().amax(-1, keepdim=True))
        close(o, want, 24 * U * top)
    assert B.leapquant_check_error_word(err) == (B.LQ_DEVERR_BAD_POSITION if r else 0)


def test_qk_norm_in_place_queries_only_and_no_tokens():
    q = rnd(1, 9, 4, 128).cuda()
    want = torch.empty_like(q)
    B.leapquant_qk_norm(q, None, want, None)
    same = q.clone()
    B.leapquant_qk_norm(same, None, same, None)
    assert torch.equal(same, want)
    none = q[:0]
    B.leapquant_qk_norm(none, none, none, none)


# ------------------------------------------------------------------------------------------------------------- scan

def scan_inputs(n, hv, hk, dtype, seed=0, big=False):
    x = {"q": rnd(seed + 1, n, hk, 128), "k": rnd(seed + 2, n, hk, 128), "v": rnd(seed + 3, n, hv, 128)}
    x = {a: (y / y.norm(dim=-1, keepdim=True) if a != "v" else y).to(dtype) for a, y in x.items()}
    x["dt"] = rnd(seed + 4, n, hv).to(dtype)
    x["A"] = -torch.exp(rnd(seed + 5, hv)) * (40.0 if big else 1.0)
    x["dt_bias"] = rnd(seed + 6, hv) - 3.0
    x["D"] = rnd(seed + 7, hv)
    return x


def cu_args(x):
    return {a: (None if y is None else y.cuda()) for a, y in x.items()}


def tolerance(size, t, dtype):
    return ((2 * min(t, 512) + 16) * U + (2.0 ** -16 if dtype == BF else 0.0)) * size + 1e-30


def run_prompt(dims, x, cu, n, dtype, state=None, carry=False, slots=None, max_len=0, err=None, softplus=True):
    o = torch.full((n, dims.heads_v, 128), float("nan"), dtype=dtype, device="cuda")
    y = cu_args(x)
    B.leapquant_scan_prompt(dims, y["q"], y["k"], y["v"], y["dt"], y["A"], o, cu.cuda(), D=y["D"], dt_bias=y["dt_bias"],
                            softplus=softplus, state=state, carry=carry, slots=slots, max_len=max_len, err=err)
    return o


SCAN_LENGTHS = [[1], [0], [2, 0, 1], [31], [32], [33], [63, 64, 65], [128, 1, 129, 0, 200], [300]]


@pytest.mark.parametrize("lens", SCAN_LENGTHS, ids=str)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hv,hk,carry,skip,big", [(2, 2, True, True, False), (6, 2, False, False, True)])
def test_scan_prompt(lens, dtype, hv, hk, carry, skip, big):
    cu, n = packed(lens, tail=2)
    seqs = len(lens)
    x = scan_inputs(n, hv, hk, dtype, big=big)
    if not skip:
        x["D"] = x["dt_bias"] = None
    slots = torch.randperm(seqs + 2, generator=torch.Generator().manual_seed(4))[:seqs].int()
    state = rnd(9, seqs + 2, hv, 128, 128, scale=0.3)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"],
                                    True, state[slots.long()] if carry else None)
    d = B.make_dims(seqs, hv, hk, rule=B.LQ_RULE_ADD)
    for max_len in (0, max(lens)):
        st = state.cuda()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        o = run_prompt(d, x, cu, n, dtype, st, carry, slots.cuda(), max_len, err)
        close(o, want, tolerance(osize, max(lens), dtype))
        got = st.cpu()
        close(got[slots.long()], new, tolerance(size, max(lens), dtype))
        rest = torch.ones(seqs + 2, dtype=torch.bool)
        rest[slots.long()] = False
        assert torch.equal(got[rest], state[rest])
        assert B.leapquant_check_error_word(err) == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[1500], [700, 3, 1100, 0, 64]], ids=str)
def test_scan_prompt_split_over_a_long_sequence(lens, dtype):
    """Few heads and long sequences: the work is split along the sequence and joined."""
    cu, n = packed(lens)
    x = scan_inputs(n, 3, 1, dtype)
    x["dt_bias"] -= 2.0                                   # long memory: the join carries what it should
    state = rnd(9, len(lens), 3, 128, 128, scale=0.3)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"],
                                    True, state)
    d = B.make_dims(len(lens), 3, 1, rule=B.LQ_RULE_ADD)
    first = None
    for max_len in (0, max(lens), 5):
        st = state.cuda()
        o = run_prompt(d, x, cu, n, dtype, st, True, None, max_len)
        close(o, want, tolerance(osize, max(lens), dtype))
        close(st, new, tolerance(size, max(lens), dtype))
        again = state.cuda()
        o2 = run_prompt(d, x, cu, n, dtype, again, True, None, max_len)
        assert torch.equal(o, o2) and torch.equal(st, again)             # the same call gives the same bits
        rel = float((st.double().cpu() - new).norm() / new.norm())
        first = rel if first is None else first
        assert rel < 4e-6


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_prompt_without_softplus_state_or_carry(dtype):
    """dt as it is (also negative: growth), no state array at all; a decay of exactly zero forgets what was before."""
    cu, n = packed([70, 40])
    x = scan_inputs(n, 2, 1, dtype)
    x["dt"] = (x["dt"].float() * 0.05 + 0.02).to(dtype)
    x["dt_bias"] = None
    x["A"] = torch.tensor([-1.0, -1e9])
    x["dt"][:, 1] = x["dt"][:, 1].abs() + 0.01
    want, osize, _, _ = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], None, False)
    o = run_prompt(B.make_dims(2, 2, 1, rule=B.LQ_RULE_ADD), x, cu, n, dtype, softplus=False)
    close(o, want, tolerance(osize, 70, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_not_finite_stays_in_its_sequence_and_after_its_token(dtype):
    cu, n = packed([100, 90])
    x = scan_inputs(n, 2, 2, dtype)
    d = B.make_dims(2, 2, 2, rule=B.LQ_RULE_ADD)
    st = [torch.zeros((2, 2, 128, 128), device="cuda") for _ in range(2)]
    clean = run_prompt(d, x, cu, n, dtype, st[0])
    for name, value in (("v", float("nan")), ("v", float("inf")), ("k", float("nan")), ("q", float("inf")), ("dt", float("nan"))):
        y = {a: (None if z is None else z.clone()) for a, z in x.items()}
        y[name][40, 0] = value
        o = run_prompt(d, y, cu, n, dtype, st[1])
        assert torch.equal(o[:40], clean[:40]), name
        assert torch.equal(o[100:], clean[100:]), name
        assert torch.equal(o[:, 1], clean[:, 1]), name                    # the other head
        assert torch.equal(st[1][1], st[0][1]), name
        assert not o[40, 0].isfinite().all(), name
        if name == "q":
            assert torch.equal(o[41:], clean[41:]) and torch.equal(st[1], st[0])


def test_scan_slots_padding_and_bad_ones_and_bad_lengths():
    cu, n = packed([5, 66, 7])
    x = scan_inputs(n, 2, 1, BF)
    d = B.make_dims(3, 2, 1, rule=B.LQ_RULE_ADD)
    state = rnd(3, 2, 2, 128, 128)
    st, err = state.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = torch.tensor([-1, 1, 2], dtype=torch.int32, device="cuda")
    o = run_prompt(d, x, cu, n, BF, st, True, slots, 0, err)
    old = torch.stack([torch.zeros_like(state[0]), state[1], torch.full_like(state[0], float("nan"))])
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"], True, old)
    close(o, want, tolerance(osize.nan_to_num(0.0), 66, BF))
    assert torch.equal(st[0].cpu(), state[0])
    close(st[1], new[1], tolerance(size[1], 66, BF))
    assert B.leapquant_check_error_word(err) == B.LQ_DEVERR_BAD_SLOT
    # lengths that leave the tokens or fall are reported and stay within the arrays
    for lie in ([0, 5, 3, 78], [0, 5, 71, 1000], [-4, 5, 71, 78]):
        run_prompt(d, x, torch.tensor(lie, dtype=torch.int32), n, BF, None, False, None, 0, err)
        assert B.leapquant_check_error_word(err) == B.LQ_DEVERR_BAD_SEQLENS
        c = rnd(1, n, 64).cuda()
        B.leapquant_conv_prompt(c, rnd(2, 64, 4).cuda(), torch.empty_like(c), torch.tensor(lie, dtype=torch.int32).cuda(),
                                err=err)
        assert B.leapquant_check_error_word(err) == B.LQ_DEVERR_BAD_SEQLENS


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sdt", [F32, BF])
@pytest.mark.parametrize("batch,hv,hk", [(1, 1, 1), (3, 6, 2)])
def test_scan_step(batch, hv, hk, sdt, dtype):
    x = scan_inputs(batch, hv, hk, dtype)
    state = rnd(9, batch + 1, hv, 128, 128).to(sdt)
    slots = torch.arange(batch, 0, -1, dtype=torch.int32)
    slots[0] = -1 if batch > 1 else slots[0]
    old = torch.stack([state[s].float() if s >= 0 else torch.zeros((hv, 128, 128)) for s in slots.tolist()])
    bf = sdt == BF
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(b, b + 1) for b in range(batch)], x["D"],
                                    x["dt_bias"], True, old, state_bf16=bf)
    st, y = state.cuda(), cu_args(x)
    o = torch.empty((batch, hv, 128), dtype=dtype, device="cuda")
    d = B.make_dims(batch, hv, hk, rule=B.LQ_RULE_ADD)
    B.leapquant_scan_step(d, st, y["q"], y["k"], y["v"], y["dt"], y["A"], o, D=y["D"], dt_bias=y["dt_bias"], slots=slots.cuda())
    # (a state value that lies on a rounding boundary may round the other way: one bf16 ulp of one term)
    flips = (2.0 ** -8 * new.abs() * x["q"].double().repeat_interleave(hv // hk, 1).abs()[:, :, None, :]).amax(-1) if bf else 0.0
    close(o, want, (128 + 24) * U * osize + flips)
    for b, s in enumerate(slots.tolist()):
        if s >= 0:
            close(st[s], new[b], 24 * U * size[b])
    assert torch.equal(st[0].cpu(), state[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_step_continues_the_prompt(dtype):
    """A prompt, then tokens one at a time, against the whole sequence as one prompt."""
    n, cut = 96, 77
    x = scan_inputs(n, 4, 2, dtype)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(0, n)], x["D"], x["dt_bias"])
    d, y = B.make_dims(1, 4, 2, rule=B.LQ_RULE_ADD), cu_args(x)
    st = torch.zeros((1, 4, 128, 128), device="cuda")
    head = {a: (z if a in ("A", "dt_bias", "D") else z[:cut]) for a, z in x.items()}
    o = [run_prompt(d, head, torch.tensor([0, cut], dtype=torch.int32), cut, dtype, st)]
    for t in range(cut, n):
        o.append(torch.empty((1, 4, 128), dtype=dtype, device="cuda"))
        B.leapquant_scan_step(d, st, *(y[a][t:t + 1] for a in ("q", "k", "v", "dt")), y["A"], o[-1], D=y["D"],
                              dt_bias=y["dt_bias"])
    close(torch.cat(o), want, tolerance(osize, n, dtype))
    close(st, new, tolerance(size, n, dtype))


def test_scan_gates_feed_the_decode_step():
    """The prompt's state goes into the 8-bit path under LQ_RULE_ADD, and scan_gates' alpha and beta give the scan's step:
    without tokens' quantization (BF16 state, records in FP16) the outputs agree to the records' FP16 rounding."""
    batch, hv = 2, 4
    dims = B.make_dims(batch, hv, hv, window=8, n_comp=0, code=B.LQ_CODE_BF16, smooth=0, rule=B.LQ_RULE_ADD)
    x = scan_inputs(batch, hv, hv, F32)
    y = cu_args(x)
    S = rnd(9, batch, hv, 128, 128).cuda().bfloat16().float()
    alpha, beta = (torch.empty((batch, hv), device="cuda") for _ in range(2))
    B.leapquant_scan_gates(dims, y["dt"], y["A"], alpha, beta, dt_bias=y["dt_bias"])
    raw = x["dt"].double() + x["dt_bias"].double()
    delta = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs()))
    close(beta, delta, 8 * U * delta.abs() + 2 * U * raw.abs())
    close(alpha, torch.exp(delta * x["A"].double()), 1e-6 * (1 + (delta * x["A"].double()).abs()))
    st = B.State.empty(dims)
    B.leapquant_quantize_state(dims, S, st)
    o = torch.empty((batch, hv, 128), device="cuda")
    B.leapquant_decode_step(dims, st, y["q"], y["k"], y["v"], alpha, beta, o)
    o += y["D"][:, None] * y["v"]
    dense = S.clone()
    want = torch.empty_like(o)
    B.leapquant_scan_step(dims, dense, y["q"], y["k"], y["v"], y["dt"], y["A"], want, D=y["D"], dt_bias=y["dt_bias"])
    assert float((o - want).norm() / want.norm()) < 2.0 ** -10


# -------------------------------------------------------------------------------------- streams, graphs, large offsets

def _layer(x, y, s, stream=None, ws=None):
    """All operators on one batch of two prompts; returns what they write."""
    kw = {"stream": stream}
    B.leapquant_conv_prompt(s["x"], s["w"], s["c"], s["cu"], state=s["cs"], carry=True, **kw)
    B.leapquant_qk_norm(y["q"], y["k"], s["q"], s["k"], **kw)
    B.leapquant_scan_prompt(s["dims"], s["q"], s["k"], y["v"], y["dt"], y["A"], s["o"], s["cu"], D=y["D"], dt_bias=y["dt_bias"],
                            state=s["S"], carry=True, workspace=ws, **kw)
    B.leapquant_conv_step(s["x"][:2], s["w"], s["c1"], s["cs"], **kw)
    B.leapquant_scan_step(s["dims"], s["S"], s["q"][:2], s["k"][:2], y["v"][:2], y["dt"][:2], y["A"], s["o1"], **kw)


def _buffers(n, x):
    z = lambda *shape, dt=BF: torch.zeros(shape, dtype=dt, device="cuda")                  # noqa: E731
    return {"x": rnd(20, n, 512).to(BF).cuda(), "w": rnd(21, 512, 4).cuda(), "c": z(n, 512), "cs": z(2, 3, 512), "q": z(n, 1, 128),
            "k": z(n, 1, 128), "o": z(n, 3, 128), "S": z(2, 3, 128, 128, dt=F32), "c1": z(2, 512), "o1": z(2, 3, 128),
            "dims": B.make_dims(2, 3, 1, rule=B.LQ_RULE_ADD), "cu": torch.tensor([0, 900, n], dtype=torch.int32).cuda()}


OUT = ("c", "cs", "q", "k", "o", "S", "c1", "o1")


def test_streams_and_graph_replays_give_the_eager_results():
    n = 1000
    x = scan_inputs(n, 3, 1, BF)
    y = cu_args(x)
    s = _buffers(n, x)
    eager = []
    for _ in range(4):                                    # the states move on from pass to pass
        _layer(x, y, s)
        eager.append({a: s[a].clone() for a in OUT})
    # another stream than the tensors' own, with a workspace of the caller's
    s = _buffers(n, x)
    ws = torch.empty(max(16, B.leapquant_scan_workspace_bytes(s["dims"], n)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for want in eager[:2]:
        _layer(x, y, s, side, ws)
        side.synchronize()
        assert all(torch.equal(s[a], want[a]) for a in OUT)
    if B.leapquant_scan_workspace_bytes(s["dims"], n):
        with pytest.raises(ValueError, match="workspace"):
            _layer(x, y, s, side, None)
    # a captured graph, replayed with eager work in between
    s = _buffers(n, x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _layer(x, y, s)
    for want in eager:
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s[a], want[a]) for a in OUT)
        (s["x"].float() @ s["x"].float().t()).sum().item()


def test_rows_and_slots_past_32_bits():
    """Token rows 2^30 elements apart and a state row past 2^32 bytes."""
    far, n = (1 << 30) + 64, 5
    wide = torch.empty((n - 1) * far + 512, dtype=BF, device="cuda")
    view = torch.as_strided(wide, (n, 256), (far, 1))
    x = rnd(1, n, 256).to(BF).cuda()
    view.copy_(x)
    w, cu = rnd(2, 256, 4).cuda(), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    got, want = (torch.empty((n, 256), dtype=BF, device="cuda") for _ in range(2))
    B.leapquant_conv_prompt(view, w, got, cu)
    B.leapquant_conv_prompt(x, w, want, cu)
    assert torch.equal(got, want)
    heads = torch.as_strided(wide, (n, 2, 128), (far, 128, 1))
    a, b = (torch.empty((n, 2, 128), dtype=BF, device="cuda") for _ in range(2))
    B.leapquant_qk_norm(heads, None, a, None)
    B.leapquant_qk_norm(x.view(n, 2, 128), None, b, None)
    assert torch.equal(a, b)
    y = cu_args(scan_inputs(n, 2, 2, BF))
    d = B.make_dims(1, 2, 2, rule=B.LQ_RULE_ADD)
    st = [torch.zeros((1, 2, 128, 128), device="cuda") for _ in range(2)]
    for v, s, o in ((heads, st[0], a), (x.view(n, 2, 128), st[1], b)):
        B.leapquant_scan_prompt(d, v, v, v, y["dt"], y["A"], o, cu, state=s)
    assert torch.equal(a, b) and torch.equal(st[0], st[1])
    del wide, view, heads
    slots = torch.tensor([40000], dtype=torch.int32, device="cuda")
    many = torch.zeros((40001, 2, 128, 128), device="cuda")                # 128 KiB a row: 5.2 GB
    for rows in (many, st[0].zero_()):
        B.leapquant_scan_step(d, rows, y["q"][:1], y["k"][:1], y["v"][:1], y["dt"][:1], y["A"], a[:1],
                              slots=slots if rows is many else None)
    assert torch.equal(many[40000], st[0][0]) and not many[:40000].any()


# --------------------------------------------------------------------------------------------- the native call path

def test_native_path_takes_regular_calls_and_gives_the_same(monkeypatch):
    n = 1000
    x = scan_inputs(n, 3, 1, BF)
    y = cu_args(x)
    got, taken = [], []
    assert B.lib() and B._M is not B._NoMarshal

    class Native:
        def __getattr__(self, name):
            def call(*args):
                status = getattr(native, name)(*args)
                taken.append((name, status))
                return status
            return call

    native = B._M
    for side in (Native(), B._NoMarshal):
        monkeypatch.setattr(B, "_M", side)
        s = _buffers(n, x)
        for _ in range(2):
            _layer(x, y, s)
        got.append({a: s[a].clone() for a in OUT})
    assert [t[0] for t in taken] == 2 * ["conv", "qk_norm", "scan", "conv", "scan"]
    assert all(t[1] == B.LQ_OK for t in taken)
    assert all(torch.equal(got[0][a], got[1][a]) for a in OUT)


def test_irregular_calls_are_refused_by_the_python_checks():
    n = 8
    y = cu_args(scan_inputs(n, 2, 1, BF))
    d = B.make_dims(1, 2, 1, rule=B.LQ_RULE_ADD)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    o = torch.empty((n, 2, 128), dtype=BF, device="cuda")
    st = torch.zeros((1, 2, 128, 128), device="cuda")

    def prompt(**kw):
        a = dict(y, o=o, cu=cu, state=st, workspace=None)
        a.update(kw)
        B.leapquant_scan_prompt(d, a["q"], a["k"], a["v"], a["dt"], a["A"], a["o"], a["cu"], D=a["D"], state=a["state"])

    prompt()
    for kw, said in (({"q": y["q"].float()}, "q must be"), ({"o": o.half()}, "o must be"), ({"cu": cu.long()}, "cu_seqlens must be"),
                     ({"cu": cu[:1]}, "sequences"), ({"A": y["A"].cpu()}, "device tensor"), ({"D": y["D"][:1]}, "D must have shape"),
                     ({"state": st.transpose(2, 3)}, "state must be contiguous"), ({"dt": y["dt"].t()}, "dt must have shape"),
                     ({"k": y["k"].transpose(1, 2)}, "k must have shape"), ({"v": y["v"][..., :64]}, "v must have shape"),
                     ({"state": st.double()}, "state must be")):
        with pytest.raises(ValueError, match=said):
            prompt(**kw)
    c = rnd(1, n, 64).cuda()
    w = rnd(2, 64, 4).cuda()
    B.leapquant_conv_prompt(c, w, torch.empty_like(c), cu)
    for args, said in (((c.half(), w, torch.empty_like(c), cu), "float32 or bfloat16"), ((c, w[:32], torch.empty_like(c), cu), "weight"),
                       ((c, w, torch.empty_like(c)[:4], cu), "out must have shape")):
        with pytest.raises(ValueError, match=said):
            B.leapquant_conv_prompt(*args)
    with pytest.raises(B.LeapQuantError):
        B.leapquant_conv_prompt(c, rnd(2, 64, 5).cuda(), torch.empty_like(c), cu)      # width 5
    with pytest.raises(B.LeapQuantError):
        B.leapquant_scan_step(d, st, y["q"], y["k"], y["v"], y["dt"], y["A"], o)       # 8 tokens, 1 request


@pytest.mark.parametrize("batch,c", [(513, 64), (1026, 2056)])
def test_conv_step_of_many_requests(batch, c):
    """Several requests per thread, a last group of fewer."""
    x, w, b, state = rnd(1, batch, c).to(BF), rnd(2, c, 4), rnd(3, c), rnd(4, batch, 3, c).to(BF)
    st = state.cuda()
    o = torch.empty((batch, c), device="cuda")
    B.leapquant_conv_step(x.cuda(), w.cuda(), o, st, bias=b.cuda())
    line = torch.cat([state, x[:, None]], 1).double()
    m = (line * w.t().double()).abs().sum(1) + b.double().abs()
    y = (line * w.t().double()).sum(1) + b.double()
    close(o, y / (1 + torch.exp(-y)), 1e-6 * (m + 1))
    assert torch.equal(st.cpu(), line[:, 1:].to(BF))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_step_of_many_tiles(dtype):
    """Enough tiles that a row of the state is a thread's whole share."""
    batch, hv = 128, 17
    x = scan_inputs(batch, hv, 1, dtype)
    state = rnd(9, batch, hv, 128, 128)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(b, b + 1) for b in range(batch)], x["D"],
                                    x["dt_bias"], True, state)
    st, y = state.cuda(), cu_args(x)
    o = torch.empty((batch, hv, 128), dtype=dtype, device="cuda")
    B.leapquant_scan_step(B.make_dims(batch, hv, 1, rule=B.LQ_RULE_ADD), st, y["q"], y["k"], y["v"], y["dt"], y["A"], o,
                          D=y["D"], dt_bias=y["dt_bias"])
    close(o, want, (128 + 24) * U * osize)
    close(st, new, 24 * U * size)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_split_with_slots_and_values_that_are_not_finite(dtype):
    """The split form: a sequence without a slot, one with a bad slot, and a token that is not finite."""
    cu, n = packed([700, 3, 1100, 0])
    x = scan_inputs(n, 2, 1, dtype)
    x["dt_bias"] -= 1.0
    d = B.make_dims(4, 2, 1, rule=B.LQ_RULE_ADD)
    state = rnd(3, 3, 2, 128, 128, scale=0.3)
    slots = torch.tensor([-1, 7, 1, 2], dtype=torch.int32)
    old = torch.stack([torch.zeros_like(state[0]), torch.full_like(state[0], float("nan")), state[1], state[2]])
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"], True, old)
    st, err = state.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    clean = run_prompt(d, x, cu, n, dtype, st, True, slots.cuda(), 0, err)
    close(clean, want, tolerance(osize.nan_to_num(0.0), 1100, dtype))
    close(st[1], new[2], tolerance(size[2], 1100, dtype))
    assert torch.equal(st[0].cpu(), state[0]) and torch.equal(st[2].cpu(), state[2])
    assert B.leapquant_check_error_word(err) == B.LQ_DEVERR_BAD_SLOT
    for name in ("v", "k", "dt"):
        y = {a: z.clone() for a, z in x.items()}
        y[name][500, 0] = float("nan")
        st2 = state.cuda()
        o = run_prompt(d, y, cu, n, dtype, st2, True, slots.cuda())
        assert torch.equal(o[:500], clean[:500]), name
        assert torch.equal(o[703:], clean[703:]) and torch.equal(st2, st), name     # (the faulty sequence keeps no state)
        assert o[500:700, 0].isnan().any()


def test_scan_split_of_many_sequences():
    """One long sequence among hundreds of short ones: the segments' numbers are sums over more sequences than threads."""
    lens = [i % 4 for i in range(270)] + [900] + [1] * 30
    cu, n = packed(lens)
    x = scan_inputs(n, 1, 1, BF)
    state = rnd(9, len(lens), 1, 128, 128, scale=0.3)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"], True, state)
    d = B.make_dims(len(lens), 1, 1, rule=B.LQ_RULE_ADD)
    assert B.leapquant_scan_workspace_bytes(d, n, BF, 900) > 0
    st = state.cuda()
    o = run_prompt(d, x, cu, n, BF, st, True, None, 900)
    close(o, want, tolerance(osize, 900, BF))
    close(st, new, tolerance(size, 900, BF))
