"""Layer operators at values and arguments where a kernel goes wrong easily, against their definitions in 64 bits.

Tolerances as in test_gpu_layer.py (u = 2^-24): after t tokens (2 t + 16) u of the sum of the terms' magnitudes, for bf16
tokens as for fp32 ones: bf16 tokens are exact, and all that is multiplied with them is kept to 2^-23 of its value or
better.  A bf16 output has half an ulp more.
"""
import math

import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import layer_reference as R
from tests.test_gpu_layer import BF, F32, U, close, cu_args, packed, rnd, run_prompt, scan_inputs

pytestmark = pytest.mark.gpu


def fp32_tolerance(size, t):
    return (2 * t + 16) * U * size + 1e-30


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_outputs_where_the_state_cancels(dtype):
    """Sums of two terms that are 2^-12 apart: what is left shows every bit of the state that a product drops."""
    n, hv = 20, 2
    cu, _ = packed([n])
    x = scan_inputs(n, hv, hv, dtype)
    x["v"].zero_()
    x["q"].zero_()
    x["q"][..., 6] = x["q"][..., 77] = rnd(1, n, hv).to(dtype)
    x["D"] = None
    state = rnd(2, 1, hv, 128, 128)
    state[..., 77] = -state[..., 6] * (1 + 2.0 ** -12 * torch.rand((1, hv, 128), generator=torch.Generator().manual_seed(3)))
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(0, n)], None, x["dt_bias"], True, state)
    st = state.cuda()
    o = run_prompt(B.make_dims(1, hv, hv, rule=B.LQ_RULE_ADD), x, cu, n, dtype, st, True)
    close(o, want, fp32_tolerance(osize, n))
    close(st, new, fp32_tolerance(size, n))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scan_outputs_where_the_tokens_cancel(dtype):
    """The same for the weights of a chunk's own tokens: two equal keys, values of opposite sign, a slow decay."""
    n, hv = 20, 16
    cu, _ = packed([n])
    x = scan_inputs(n, hv, hv, dtype)
    x["k"][1] = x["k"][0]
    x["q"][..., 1:] = 0                                   # (one term in q . k)
    x["v"][1] = -x["v"][0]
    x["v"][2:] = 0
    x["dt"].fill_(1.0)
    x["dt_bias"] = x["D"] = None
    x["A"] = torch.full((hv,), -2.0 ** -10)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(0, n)], None, None, False)
    st = torch.empty((1, hv, 128, 128), device="cuda")
    o = run_prompt(B.make_dims(1, hv, hv, rule=B.LQ_RULE_ADD), x, cu, n, dtype, st, softplus=False)
    close(o, want, fp32_tolerance(osize, n))
    close(st, new, fp32_tolerance(size, n))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[70, 1, 40], [700, 20]], ids=str)
def test_a_step_of_minus_infinity_masks(lens, dtype):
    """softplus(-inf) = 0: the token changes nothing and the state keeps; a bias of -inf does that for a whole head."""
    cu, n = packed(lens)
    hv, seqs = 3, len(lens)
    x = scan_inputs(n, hv, 1, dtype)
    x["dt"][::3, 0] = -math.inf
    x["dt"][lens[0] - 1] = -math.inf
    x["dt_bias"][1] = -math.inf
    state = rnd(9, seqs, hv, 128, 128, scale=0.3)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"], True, state)
    assert want.isfinite().all() and new.isfinite().all()
    d = B.make_dims(seqs, hv, 1, rule=B.LQ_RULE_ADD)
    assert (B.leapquant_scan_workspace_bytes(d, n, dtype, max(lens)) > 0) == (max(lens) == 700)       # both forms of the prompt
    st = state.cuda()
    o = run_prompt(d, x, cu, n, dtype, st, True, None, max(lens))
    close(o, want, fp32_tolerance(osize, max(lens)))
    close(st, new, fp32_tolerance(size, max(lens)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_step_of_minus_infinity_masks_single_tokens(dtype):
    batch, hv = 3, 4
    x = scan_inputs(batch, hv, 1, dtype)
    x["dt"][0, 1] = x["dt_bias"][2] = -math.inf
    state = rnd(9, batch, hv, 128, 128)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(b, b + 1) for b in range(batch)], x["D"],
                                    x["dt_bias"], True, state)
    d, y, st = B.make_dims(batch, hv, 1, rule=B.LQ_RULE_ADD), cu_args(x), state.cuda()
    o = torch.empty((batch, hv, 128), dtype=dtype, device="cuda")
    B.leapquant_scan_step(d, st, y["q"], y["k"], y["v"], y["dt"], y["A"], o, D=y["D"], dt_bias=y["dt_bias"])
    close(o, want, (128 + 24) * U * osize)
    close(st, new, 24 * U * size)
    alpha, beta = (torch.empty((batch, hv), device="cuda") for _ in range(2))
    B.leapquant_scan_gates(d, y["dt"], y["A"], alpha, beta, dt_bias=y["dt_bias"])
    for b, h in ((0, 1), (0, 2), (1, 2), (2, 2)):
        assert float(alpha[b, h]) == 1.0 and float(beta[b, h]) == 0.0


def same_values(got, want, tol):
    """NaN and infinities in the same places, the finite ones within tol and the rounding of a bf16 result."""
    g = got.double().cpu()
    if got.dtype == BF:
        tol = tol + want.abs().nan_to_num(0.0, 0.0, 0.0) * 2.0 ** -8
    assert torch.equal(g.isnan(), want.isnan()), (int(g.isnan().sum()), int(want.isnan().sum()))
    assert torch.equal(g[want.isinf()], want[want.isinf()])
    fin = want.isfinite()
    assert g[fin].isfinite().all() and ((g - want).abs()[fin] <= (tol + 0 * want)[fin]).all()


@pytest.mark.parametrize("kind", ["state", "value", "value, strong decay", "key", "query", "step"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[70, 40], [700, 20]], ids=str)
def test_scan_with_infinities_is_the_recurrence(lens, dtype, kind):
    """An infinity stays one in the state, token by token, also where a decay over many tokens rounds to zero."""
    cu, n = packed(lens)
    x = scan_inputs(n, 2, 1, dtype)
    state = rnd(9, 2, 2, 128, 128, scale=0.3)
    x["dt"] *= 0.1
    if "strong" in kind:
        x["A"] = torch.tensor([-200.0, -150.0])           # about e^-9 a token: 16 of them are below fp32's range
    clean_state = state.clone().cuda()
    d = B.make_dims(2, 2, 1, rule=B.LQ_RULE_ADD)
    assert (B.leapquant_scan_workspace_bytes(d, n, dtype, max(lens)) > 0) == (max(lens) == 700)
    clean = run_prompt(d, x, cu, n, dtype, clean_state, True, None, max(lens))
    if kind == "state":
        state[0, 0, 5, 9], state[0, 1, 7, 3], state[1, 0, 100, 127] = math.inf, -math.inf, math.inf
    elif "value" in kind:
        x["v"][10, 0, 5] = math.inf
        x["v"][lens[0] + 17, 1, 90] = -math.inf
    elif kind == "key":
        x["k"][10, 0, 9] = math.inf
    elif kind == "query":
        x["q"][10, 0, 9] = -math.inf
    else:
        x["dt"][10, 1] = math.inf
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"], True, state)
    st = state.cuda()
    o = run_prompt(d, x, cu, n, dtype, st, True, None, max(lens))
    same_values(o, want, fp32_tolerance(osize.nan_to_num(0.0, 0.0, 0.0), max(lens)))
    same_values(st, new, fp32_tolerance(size.nan_to_num(0.0, 0.0, 0.0), max(lens)))
    # what the infinity does not reach keeps its bits
    fin = want.isfinite().cuda()
    assert torch.equal(o[fin], clean[fin])
    fin = new.isfinite().cuda()
    assert torch.equal(st[fin], clean_state[fin])


def test_one_workspace_serves_prompts_of_all_lengths():
    """Sized for the longest prompt; on a stream of the caller's, which has to bring it."""
    hv = 64
    d = B.make_dims(1, hv, 1, rule=B.LQ_RULE_ADD)
    ws = torch.empty(B.leapquant_scan_workspace_bytes(d, 2056), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for n in (1, 256, 512, 520, 1024, 2048, 2056):
        y = cu_args(scan_inputs(n, hv, 1, BF))
        cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        got = []
        for max_len in (0, n, None):
            o = torch.empty((n, hv, 128), dtype=BF, device="cuda")
            torch.cuda.synchronize()
            kw = {"stream": side, "workspace": ws, "max_len": max_len} if max_len is not None else {}
            B.leapquant_scan_prompt(d, y["q"], y["k"], y["v"], y["dt"], y["A"], o, cu, D=y["D"], dt_bias=y["dt_bias"], **kw)
            torch.cuda.synchronize()
            got.append(o)
        assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[2])
    # a call that is not cut needs none, whatever others of its size may
    d = B.make_dims(1, 100, 1, rule=B.LQ_RULE_ADD)
    assert B.leapquant_scan_workspace_bytes(d, 400) > 0 and B.leapquant_scan_workspace_bytes(d, 400, max_len=400) == 0
    y = cu_args(scan_inputs(400, 100, 1, BF))
    o = torch.empty((400, 100, 128), dtype=BF, device="cuda")
    torch.cuda.synchronize()
    B.leapquant_scan_prompt(d, y["q"], y["k"], y["v"], y["dt"], y["A"], o, torch.tensor([0, 400], dtype=torch.int32).cuda(), stream=side)
    side.synchronize()


class NoTruth:
    def __bool__(self):
        raise RuntimeError("no truth value")


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("flag", [2, -1, NoTruth(), "yes", None], ids=["2", "-1", "raises", "text", "none"])
def test_flags_are_refused_alike_by_the_native_and_the_python_path(flag, native, monkeypatch):
    assert B.lib() and B._M is not B._NoMarshal
    if not native:
        monkeypatch.setattr(B, "_M", B._NoMarshal)
    n = 4
    y = cu_args(scan_inputs(n, 2, 2, BF))
    d = B.make_dims(1, 2, 2, rule=B.LQ_RULE_ADD)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    o, st = torch.empty((n, 2, 128), dtype=BF, device="cuda"), torch.zeros((1, 2, 128, 128), device="cuda")
    x, w, cs = rnd(1, n, 64).cuda(), rnd(2, 64, 4).cuda(), torch.zeros((1, 3, 64), device="cuda")
    cos = torch.ones((n, 32), device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    tokens = (y["q"], y["k"], y["v"], y["dt"], y["A"], o)
    for call in (lambda f: B.leapquant_conv_prompt(x, w, torch.empty_like(x), cu, silu=f),
                 lambda f: B.leapquant_conv_prompt(x, w, torch.empty_like(x), cu, state=cs, carry=f),
                 lambda f: B.leapquant_conv_step(x[:1], w, torch.empty_like(x[:1]), cs, silu=f),
                 lambda f: B.leapquant_qk_norm(y["q"], None, o, None, cos=cos, sin=cos, positions=pos, interleaved=f),
                 lambda f: B.leapquant_scan_prompt(d, *tokens, cu, softplus=f),
                 lambda f: B.leapquant_scan_prompt(d, *tokens, cu, state=st, carry=f),
                 lambda f: B.leapquant_scan_step(d, st, *(t[:1] for t in tokens[:4]), y["A"], o[:1], softplus=f)):
        for good in (True, False, 0, 1):
            call(good)
        with pytest.raises(B.LeapQuantError if isinstance(flag, int) else (TypeError, ValueError)):
            call(flag)


@pytest.mark.parametrize("native", [True, False])
def test_prompts_without_cu_seqlens_are_refused_alike(native, monkeypatch):
    assert B.lib() and B._M is not B._NoMarshal
    if not native:
        monkeypatch.setattr(B, "_M", B._NoMarshal)
    y = cu_args(scan_inputs(4, 2, 2, BF))
    o, st = torch.empty((4, 2, 128), dtype=BF, device="cuda"), torch.zeros((1, 2, 128, 128), device="cuda")
    x, w, cs = rnd(1, 4, 64).cuda(), rnd(2, 64, 4).cuda(), torch.zeros((4, 3, 64), device="cuda")
    with pytest.raises(ValueError, match="cu_seqlens is required"):
        B.leapquant_conv_prompt(x, w, torch.empty_like(x), None, state=cs)
    with pytest.raises(ValueError, match="cu_seqlens is required"):
        B.leapquant_scan_prompt(B.make_dims(1, 2, 2, rule=B.LQ_RULE_ADD), y["q"], y["k"], y["v"], y["dt"], y["A"], o, None, state=st)


@pytest.mark.parametrize("carry", [False, True])
def test_conv_of_no_tokens_reports_lengths_that_claim_some(carry):
    x, w = rnd(1, 5, 64).cuda(), rnd(2, 64, 4).cuda()
    state = rnd(3, 2, 3, 64)
    for cu, bits in (([0, 0, 0], 0), ([0, 5, 5], B.LQ_DEVERR_BAD_SEQLENS), ([0, 0, -1], B.LQ_DEVERR_BAD_SEQLENS)):
        for st in (state.cuda(), None):
            if st is None and carry:
                continue
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            B.leapquant_conv_prompt(x[:0], w, x[:0], torch.tensor(cu, dtype=torch.int32).cuda(), state=st, carry=carry, err=err)
            assert B.leapquant_check_error_word(err) == bits
            if st is not None:
                assert torch.equal(st.cpu(), state if carry else torch.zeros_like(state))


@pytest.mark.parametrize("carry", [False, True])
@pytest.mark.parametrize("lens", [[0, 4], [0, 0]], ids=str)
def test_conv_reports_the_bad_slot_of_an_empty_sequence(lens, carry):
    """As the scan does."""
    cu, n = packed(lens)
    x, w = rnd(1, max(n, 1), 64).cuda()[:n], rnd(2, 64, 4).cuda()
    for slots, bits in (([1, 0], 0), ([-1, 0], 0), ([2, 0], B.LQ_DEVERR_BAD_SLOT)):
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.leapquant_conv_prompt(x, w, torch.empty_like(x), cu.cuda(), state=rnd(3, 2, 3, 64).cuda(), carry=carry,
                                slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), err=err)
        assert B.leapquant_check_error_word(err) == bits
        y = cu_args(scan_inputs(max(n, 1), 1, 1, BF))
        tokens = [y[a][:n] for a in ("q", "k", "v", "dt")]
        B.leapquant_scan_prompt(B.make_dims(2, 1, 1, rule=B.LQ_RULE_ADD), *tokens, y["A"], torch.empty_like(tokens[2]), cu.cuda(),
                                state=torch.zeros((2, 1, 128, 128), device="cuda"), carry=carry,
                                slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), err=err)
        assert B.leapquant_check_error_word(err) == bits


def in_terms(x, n):
    """The sum of n bf16 terms cut one after the other from fp32 values, the last one rounded."""
    x, out = x.clone(), torch.zeros_like(x, dtype=torch.float64)
    for i in range(n):
        term = (x.view(torch.int32) & -65536).view(torch.float32) if i < n - 1 else x.bfloat16().float()
        out, x = out + term.double(), x - term
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[1], [5, 1], [40], [700]], ids=str)
def test_scan_state_is_fp32(lens, dtype):
    """No decay, and values in at most three tokens: few roundings, so that a state of fewer bits than fp32's shows.  A sum of
    three products of a step, a key and a value: 4 roundings of each, 2 of the sum, and the step's own (softplus to 4 u)."""
    cu, n = packed(lens)
    seqs, hv = len(lens), 2
    x = scan_inputs(n, hv, 1, dtype)
    x["A"].zero_()
    keep = torch.zeros(n, dtype=torch.bool)
    keep[[0, n // 2, n - 1]] = True
    x["v"][~keep] = 0
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], R.lengths(cu, n), x["D"], x["dt_bias"])
    tol = 16 * U * size
    raw = x["dt"].double() + x["dt_bias"].double()
    wv = ((torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs())))[:, :, None] * x["v"].double()).float()
    for terms, enough in ((2, False), (3, True)):         # what a state from two terms of 16 bits would miss
        ks = x["k"].double().repeat_interleave(hv, 1)
        state = torch.stack([(in_terms(wv, terms)[lo:hi, :, :, None] * ks[lo:hi, :, None, :]).sum(0) for lo, hi in R.lengths(cu, n)])
        assert bool(((state - new).abs() <= tol).all()) == enough
    d = B.make_dims(seqs, hv, 1, rule=B.LQ_RULE_ADD)
    assert (B.leapquant_scan_workspace_bytes(d, n, dtype, max(lens)) > 0) == (max(lens) == 700)
    st = torch.empty((seqs, hv, 128, 128), device="cuda")
    o = run_prompt(d, x, cu, n, dtype, st, max_len=max(lens))
    close(st, new, tol)
    close(o, want, fp32_tolerance(osize, max(lens)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [16, 300], ids=["one chunk", "split"])
def test_scan_decays_keep_their_bits_where_they_are_strong(n, dtype):
    """A state without new values, steps that are exact: each chunk (of at least 16 tokens) or segment multiplies it by one
    power of two, good to 2 u of the exponential, 1 u of its argument and 1 u of the product, however strong the decay."""
    x = scan_inputs(n, 2, 2, dtype)
    x["v"].zero_()
    x["q"].zero_()
    x["q"][..., 9] = 1
    x["dt"] = (0.75 + 0.25 * torch.rand((n, 2), generator=torch.Generator().manual_seed(1))).to(dtype)
    x["A"] = torch.tensor([-0.301, -3.1]) if n == 16 else torch.tensor([-0.011, -0.25])
    x["dt_bias"] = x["D"] = None
    state = rnd(9, 1, 2, 128, 128)
    want, osize, new, size = R.scan(x["q"], x["k"], x["v"], x["dt"], x["A"], [(0, n)], None, None, False, state)
    d = B.make_dims(1, 2, 2, rule=B.LQ_RULE_ADD)
    assert (B.leapquant_scan_workspace_bytes(d, n, dtype, n) > 0) == (n == 300)
    st = state.cuda()
    o = run_prompt(d, x, torch.tensor([0, n], dtype=torch.int32), n, dtype, st, True, None, n, softplus=False)
    factors = 1 if n == 16 else -(-n // 64) + 64 // 16    # a segment's start is a product over segments, then chunks follow
    close(st, new, 4 * U * factors * size)
    close(o, want, 4 * U * (factors + 1) * osize)
