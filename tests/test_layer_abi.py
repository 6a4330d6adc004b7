"""Host-side checks of the layer operators (no GPU needed): refusals of the C entry points and of the binding."""
import ctypes as C

import pytest
import torch

from paper_2609_38166_amd import binding as B

GOOD = 0x10000


def conv(**kw):
    a = dict(seqs=3, channels=256, width=4, dtype=1, out_dtype=1, silu=1, carry=1, n_slots=3, tokens=3, x_stride=256,
             out_stride=256, x=GOOD, weight=GOOD, bias=GOOD, out=GOOD, state=GOOD, cu_seqlens=GOOD)
    a.update(kw)
    return B.lq_conv(**a)


def qk(**kw):
    a = dict(tokens=5, heads_q=4, heads_k=2, d=128, norm=B.LQ_NORM_RMS, rot=64, interleaved=0, dtype=1, out_dtype=0,
             eps=1e-6, q_scale=1.0, q_stride=512, k_stride=256, q_out_stride=512, k_out_stride=256, q=GOOD, k=GOOD,
             q_out=GOOD, k_out=GOOD, q_weight=GOOD, k_weight=GOOD, cos=GOOD, sin=GOOD, positions=GOOD, n_positions=16)
    a.update(kw)
    return B.lq_qk(**a)


def scan(**kw):
    a = dict(tokens=2, dtype=1, state_dtype=0, softplus=1, carry=1, n_slots=2, max_len=0, q_stride=256, k_stride=256,
             v_stride=512, dt_stride=4, o_stride=512, q=GOOD, k=GOOD, v=GOOD, dt=GOOD, A=GOOD, skip=GOOD, dt_bias=GOOD,
             o=GOOD, state=GOOD, cu_seqlens=GOOD)
    a.update(kw)
    return B.lq_scan(**a)


EINVAL, EALIGN, EUNSUP = B.LQ_EINVAL, B.LQ_EALIGN, B.LQ_EUNSUPPORTED

CONV = [
    (dict(seqs=0), EINVAL), (dict(channels=0), EINVAL), (dict(dtype=2), EINVAL), (dict(out_dtype=-1), EINVAL),
    (dict(silu=2), EINVAL), (dict(carry=3), EINVAL), (dict(tokens=-1), EINVAL), (dict(width=1), EUNSUP),
    (dict(width=5), EUNSUP), (dict(channels=252), EUNSUP), (dict(dtype=0, channels=254, x_stride=256), EUNSUP),
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(weight=None), EINVAL), (dict(state=None), EINVAL),
    (dict(x_stride=255), EINVAL), (dict(x_stride=260), EALIGN), (dict(out_stride=257), EALIGN),
    (dict(x=GOOD + 8), EALIGN), (dict(weight=GOOD + 4), EALIGN), (dict(bias=GOOD + 2), EALIGN),
    (dict(state=GOOD + 8), EALIGN), (dict(n_slots=2), EINVAL), (dict(n_slots=0, slots=GOOD), EINVAL),
    (dict(slots=GOOD + 2), EALIGN), (dict(err=GOOD + 1), EALIGN),
]


@pytest.mark.parametrize("kw,status", CONV)
def test_conv_refusals(kw, status):
    L = B.lib()
    assert L.leapquant_conv_step(C.byref(conv(**kw)), None) == status
    assert L.leapquant_conv_prompt(C.byref(conv(**kw)), None) == status


def test_conv_refusals_of_one_form():
    L = B.lib()
    assert L.leapquant_conv_step(None, None) == EINVAL
    assert L.leapquant_conv_prompt(None, None) == EINVAL
    assert L.leapquant_conv_step(C.byref(conv(tokens=4)), None) == EINVAL          # one token per request
    assert L.leapquant_conv_prompt(C.byref(conv(cu_seqlens=None)), None) == EINVAL
    assert L.leapquant_conv_prompt(C.byref(conv(cu_seqlens=GOOD + 2)), None) == EALIGN
    assert L.leapquant_conv_prompt(C.byref(conv(tokens=1 << 31)), None) == EUNSUP
    # workgroups past the grid's limit
    assert L.leapquant_conv_prompt(C.byref(conv(tokens=(1 << 31) - 1, channels=1 << 20, x_stride=1 << 20)), None) == EUNSUP


QK = [
    (dict(tokens=-1), EINVAL), (dict(heads_q=0), EINVAL), (dict(heads_k=-1), EINVAL), (dict(d=96), EUNSUP),
    (dict(norm=3), EINVAL), (dict(norm=B.LQ_NORM_L2), EINVAL), (dict(rot=8), EUNSUP), (dict(rot=144), EUNSUP),
    (dict(rot=-16), EINVAL), (dict(interleaved=2), EINVAL), (dict(dtype=7), EINVAL), (dict(out_dtype=7), EINVAL),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(q=None), EINVAL),
    (dict(k=None), EINVAL), (dict(q_out=None), EINVAL), (dict(k_out=None), EINVAL), (dict(q=GOOD + 2), EALIGN),
    (dict(q_stride=511), EINVAL), (dict(q_stride=516), EALIGN), (dict(k_out_stride=258), EALIGN), (dict(cos=None), EINVAL),
    (dict(sin=None), EINVAL), (dict(positions=None), EINVAL), (dict(n_positions=0), EINVAL), (dict(cos=GOOD + 4), EALIGN),
    (dict(q_weight=GOOD + 4), EALIGN), (dict(k_weight=GOOD + 8), EALIGN), (dict(positions=GOOD + 1), EALIGN),
    (dict(err=GOOD + 2), EALIGN), (dict(tokens=(1 << 31) - 1, heads_q=1 << 19, q_stride=1 << 26, q_out_stride=1 << 26), EUNSUP),
]


@pytest.mark.parametrize("kw,status", QK)
def test_qk_norm_refusals(kw, status):
    assert B.lib().leapquant_qk_norm(C.byref(qk(**kw)), None) == status
    assert B.lib().leapquant_qk_norm(None, None) == EINVAL


SCAN = [
    (dict(dtype=2), EINVAL), (dict(softplus=2), EINVAL), (dict(carry=-1), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(state_dtype=2), EINVAL), (dict(max_len=-1), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(dt=None), EINVAL), (dict(A=None), EINVAL), (dict(o=None), EINVAL), (dict(state=None), EINVAL),
    (dict(q=GOOD + 8), EALIGN), (dict(o=GOOD + 2), EALIGN), (dict(dt=GOOD + 1), EALIGN), (dict(A=GOOD + 2), EALIGN),
    (dict(skip=GOOD + 2), EALIGN), (dict(dt_bias=GOOD + 1), EALIGN), (dict(q_stride=255), EINVAL), (dict(k_stride=260), EALIGN),
    (dict(v_stride=516), EALIGN), (dict(dt_stride=3), EINVAL), (dict(o_stride=4), EINVAL), (dict(n_slots=1), EINVAL),
    (dict(slots=GOOD + 1), EALIGN), (dict(err=GOOD + 1), EALIGN),
]


@pytest.mark.parametrize("kw,status", SCAN)
def test_scan_refusals(kw, status):
    L, d = B.lib(), B.make_dims(2, 4, 2, rule=B.LQ_RULE_ADD)
    assert L.leapquant_scan_step(C.byref(d), C.byref(scan(**kw)), None) == status
    assert L.leapquant_scan_prompt(C.byref(d), C.byref(scan(**kw)), None) == status


def test_scan_refusals_of_shapes_and_rules():
    L, good = B.lib(), B.make_dims(2, 4, 2, rule=B.LQ_RULE_ADD)
    n = C.c_size_t(0)
    for fn in (L.leapquant_scan_step, L.leapquant_scan_prompt, lambda d, s, x: L.leapquant_scan_gates(d, s, GOOD, GOOD, x)):
        assert fn(None, C.byref(scan()), None) == EINVAL
        assert fn(C.byref(good), None, None) == EINVAL
        for kw in (dict(rule=B.LQ_RULE_DELTA), dict(rule=B.LQ_RULE_GENERAL), dict(gate=B.LQ_GATE_DIAG, rule=B.LQ_RULE_ADD),
                   dict(d_k=64, rule=B.LQ_RULE_ADD)):
            assert fn(C.byref(B.make_dims(2, 4, 2, **kw)), C.byref(scan()), None) == EUNSUP, kw
        assert fn(C.byref(B.make_dims(2, 4, 3, rule=B.LQ_RULE_ADD)), C.byref(scan()), None) == EINVAL
    assert L.leapquant_scan_step(C.byref(good), C.byref(scan(tokens=3)), None) == EINVAL
    assert L.leapquant_scan_prompt(C.byref(good), C.byref(scan(cu_seqlens=None)), None) == EINVAL
    assert L.leapquant_scan_prompt(C.byref(good), C.byref(scan(state_dtype=1)), None) == EUNSUP
    assert L.leapquant_scan_gates(C.byref(good), C.byref(scan()), None, GOOD, None) == EINVAL
    assert L.leapquant_scan_gates(C.byref(good), C.byref(scan()), GOOD, GOOD + 2, None) == EALIGN
    assert L.leapquant_scan_workspace_bytes(C.byref(good), None, C.byref(n)) == EINVAL
    assert L.leapquant_scan_workspace_bytes(C.byref(good), C.byref(scan()), None) == EINVAL
    assert L.leapquant_scan_workspace_bytes(None, C.byref(scan()), C.byref(n)) == EINVAL
    assert L.leapquant_scan_workspace_bytes(C.byref(good), C.byref(scan(tokens=-1)), C.byref(n)) == EINVAL
    assert L.leapquant_scan_workspace_bytes(C.byref(good), C.byref(scan()), C.byref(n)) == B.LQ_OK


def test_a_prompt_that_needs_a_workspace_refuses_to_go_without():
    """One long sequence on few heads is split: without its workspace, or with a short or misaligned one, nothing is enqueued."""
    L, d = B.lib(), B.make_dims(1, 4, 2, rule=B.LQ_RULE_ADD)
    n = C.c_size_t(0)
    for tokens, needs in ((64, False), (1 << 16, True)):
        s = scan(tokens=tokens, n_slots=1)
        assert L.leapquant_scan_workspace_bytes(C.byref(d), C.byref(s), C.byref(n)) == B.LQ_OK
        if not n.value:
            assert not needs or tokens == 1 << 16
            continue
        s.workspace_bytes = n.value
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == EINVAL
        s.workspace = GOOD + 8
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == EALIGN
        s.workspace, s.workspace_bytes = GOOD, n.value - 1
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == EINVAL


def test_binding_refuses_host_tensors_and_shapes():
    x = torch.zeros((3, 256), dtype=torch.bfloat16)
    w, cu = torch.zeros((256, 4)), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_conv_prompt(x, w, x, cu)
    with pytest.raises(ValueError, match="state is required"):
        B.leapquant_conv_step(x, w, x, None)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_conv_step(x, w, x, torch.zeros((3, 3, 256), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_qk_norm(x.view(3, 2, 128), None, x.view(3, 2, 128), None)
    d = B.make_dims(1, 2, 2, rule=B.LQ_RULE_ADD)
    t = x.view(3, 2, 128)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_scan_prompt(d, t, t, t, x[:, :2], w[:2, 0], t, cu)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_scan_step(d, torch.zeros((3, 2, 128, 128)), t, t, t, x[:, :2], w[:2, 0], t)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_scan_gates(d, x[:, :2], w[:2, 0], w, w)
    with pytest.raises(ValueError, match="device tensor"):
        B.leapquant_check_error_word(cu)
