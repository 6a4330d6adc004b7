"""Host-side checks of the projection operators (no GPU needed): refusals of the C entry points and of the binding."""
import ctypes as C

import pytest
import torch

from paper_2609_38166_amd import binding as B

GOOD = 0x10000
EINVAL, EALIGN, EUNSUP = B.LQ_EINVAL, B.LQ_EALIGN, B.LQ_EUNSUPPORTED
E4 = torch.float8_e4m3fn


def add(**kw):
    a = dict(tokens=5, channels=256, norm=B.LQ_NORM_RMS, dtype=1, residual_dtype=0, out_dtype=B.LQ_TOKEN_E4M3, eps=1e-6, x_stride=256,
             residual_stride=256, residual_out_stride=256, out_stride=256, scale_stride=2, x=GOOD, residual=GOOD, weight=GOOD,
             residual_out=GOOD, out=GOOD, scale=GOOD)
    a.update(kw)
    return B.lq_add(**a)


def gated(**kw):
    a = dict(tokens=5, heads=3, d=128, act=0, gate_first=0, weight_heads=0, dtype=0, gate_dtype=1, out_dtype=B.LQ_TOKEN_E4M3,
             eps=1e-6, x_stride=384, gate_stride=384, out_stride=384, scale_stride=3, x=GOOD, gate=GOOD, weight=GOOD, out=GOOD,
             scale=GOOD)
    a.update(kw)
    return B.lq_gated(**a)


def weight(**kw):
    a = dict(n=200, k=256, dtype=1, w_stride=256, out_stride=256, w=GOOD, out=GOOD, scale=GOOD)
    a.update(kw)
    return B.lq_weight(**a)


def product(**kw):
    a = dict(tokens=5, n=200, k=256, out_dtype=1, x_stride=256, x_scale_stride=2, w_stride=256, out_stride=200, x=GOOD, x_scale=GOOD,
             w=GOOD, w_scale=GOOD, bias=GOOD, out=GOOD)
    a.update(kw)
    return B.lq_matmul(**a)


ADD = [
    (dict(tokens=-1), EINVAL), (dict(tokens=1 << 31), EUNSUP), (dict(channels=0), EINVAL), (dict(channels=-8), EINVAL),
    (dict(channels=252), EUNSUP), (dict(channels=16392, x_stride=20000), EUNSUP), (dict(norm=B.LQ_NORM_L2), EINVAL),
    (dict(norm=3), EINVAL), (dict(norm=B.LQ_NORM_NONE), EINVAL), (dict(dtype=2), EINVAL), (dict(residual_dtype=2), EINVAL),
    (dict(out_dtype=3), EINVAL), (dict(out_dtype=-1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(scale=None), EINVAL),
    (dict(x=GOOD + 8), EALIGN), (dict(residual=GOOD + 4), EALIGN), (dict(residual_out=GOOD + 4), EALIGN), (dict(out=GOOD + 8), EALIGN),
    (dict(weight=GOOD + 4), EALIGN), (dict(scale=GOOD + 2), EALIGN), (dict(x_stride=248), EINVAL), (dict(x_stride=260), EALIGN),
    (dict(residual_stride=255), EINVAL), (dict(residual_out_stride=258), EALIGN), (dict(out_stride=264), EALIGN),
    (dict(scale_stride=1), EINVAL), (dict(out_stride=1 << 41), EINVAL),
]
GATED = [
    (dict(tokens=-1), EINVAL), (dict(heads=0), EINVAL), (dict(d=0), EINVAL), (dict(d=32), EUNSUP), (dict(d=192), EUNSUP),
    (dict(d=16512, x_stride=1 << 17), EUNSUP), (dict(act=2), EINVAL), (dict(gate_first=2), EINVAL), (dict(weight_heads=-1), EINVAL),
    (dict(dtype=2), EINVAL), (dict(gate_dtype=2), EINVAL), (dict(out_dtype=5), EINVAL), (dict(eps=-1.0), EINVAL), (dict(x=None), EINVAL),
    (dict(gate=None), EINVAL), (dict(out=None), EINVAL), (dict(scale=None), EINVAL), (dict(gate=GOOD + 8), EALIGN),
    (dict(weight=GOOD + 8), EALIGN), (dict(x_stride=380), EINVAL), (dict(gate_stride=388), EALIGN), (dict(out_stride=392), EALIGN),
    (dict(scale_stride=2), EINVAL), (dict(tokens=1 << 31), EUNSUP), (dict(heads=(1 << 20) + 1, x_stride=1 << 28), EUNSUP),
]
WEIGHT = [
    (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(k=264, w_stride=272), EUNSUP), (dict(dtype=2), EINVAL), (dict(w=None), EINVAL),
    (dict(out=None), EINVAL), (dict(scale=None), EINVAL), (dict(w=GOOD + 8), EALIGN), (dict(out=GOOD + 8), EALIGN),
    (dict(scale=GOOD + 2), EALIGN), (dict(w_stride=252), EINVAL), (dict(w_stride=260), EALIGN), (dict(out_stride=264), EALIGN),
    (dict(n=(1 << 31) - 1, k=1 << 20, w_stride=1 << 20, out_stride=1 << 20), EUNSUP),
]
PRODUCT = [
    (dict(tokens=-1), EINVAL), (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(k=264, x_stride=272), EUNSUP),
    (dict(out_dtype=2), EINVAL), (dict(x=None), EINVAL), (dict(x_scale=None), EINVAL), (dict(w=None), EINVAL), (dict(w_scale=None), EINVAL),
    (dict(out=None), EINVAL), (dict(x=GOOD + 8), EALIGN), (dict(x_scale=GOOD + 2), EALIGN), (dict(w=GOOD + 8), EALIGN),
    (dict(w_scale=GOOD + 2), EALIGN), (dict(bias=GOOD + 2), EALIGN), (dict(out=GOOD + 8), EALIGN), (dict(x_stride=240), EINVAL),
    (dict(x_stride=264), EALIGN), (dict(w_stride=255), EINVAL), (dict(w_stride=264), EALIGN), (dict(out_stride=199), EINVAL),
    (dict(out_stride=204), EALIGN), (dict(x_scale_stride=1), EINVAL), (dict(x_stride=(1 << 23) + 16), EUNSUP),
    (dict(w_stride=(1 << 23) + 16), EUNSUP), (dict(x_scale_stride=(1 << 20) + 1), EUNSUP),
    (dict(tokens=(1 << 31) - 1, n=1 << 20, out_stride=1 << 20), EUNSUP), (dict(n=(1 << 26) + 1, out_stride=1 << 27), EUNSUP),
    (dict(n=1 << 26, k=1 << 22, w_stride=1 << 22, x_stride=1 << 22, out_stride=1 << 26, x_scale_stride=1 << 15), EUNSUP),
]


@pytest.mark.parametrize("kw,status", ADD)
def test_add_norm_refusals(kw, status):
    assert B.lib().leapquant_add_norm(C.byref(add(**kw)), None) == status


@pytest.mark.parametrize("kw,status", GATED)
def test_gate_norm_refusals(kw, status):
    assert B.lib().leapquant_gate_norm(C.byref(gated(**kw)), None) == status


@pytest.mark.parametrize("kw,status", WEIGHT)
def test_quantize_weight_refusals(kw, status):
    assert B.lib().leapquant_quantize_weight(C.byref(weight(**kw)), None) == status


@pytest.mark.parametrize("kw,status", PRODUCT)
def test_matmul_refusals(kw, status):
    assert B.lib().leapquant_matmul(C.byref(product(**kw)), None) == status


def test_null_structs():
    L = B.lib()
    assert L.leapquant_add_norm(None, None) == EINVAL and L.leapquant_gate_norm(None, None) == EINVAL
    assert L.leapquant_quantize_weight(None, None) == EINVAL and L.leapquant_matmul(None, None) == EINVAL


def test_no_tokens_need_no_arrays():
    L = B.lib()
    none = dict(tokens=0, x=None, out=None, scale=None, residual=None, residual_out=None)
    assert L.leapquant_add_norm(C.byref(add(**none)), None) == 0
    assert L.leapquant_gate_norm(C.byref(gated(tokens=0, x=None, gate=None, out=None, scale=None)), None) == 0
    assert L.leapquant_matmul(C.byref(product(tokens=0, x=None, x_scale=None, out=None)), None) == 0


def e(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype)


def test_the_binding_refuses_what_is_not_a_device_tensor_or_has_other_shapes():
    for call in (lambda: B.leapquant_add_norm(e(2, 128), e(2, 128)), lambda: B.leapquant_gate_norm(e(2, 1, 128), e(2, 1, 128), e(2, 1, 128)),
                 lambda: B.leapquant_quantize_weight(e(2, 128), e(2, 128, dtype=E4), e(1, 1)),
                 lambda: B.leapquant_matmul(e(2, 128, dtype=E4), e(2, 1), e(4, 128, dtype=E4), e(1, 1), e(2, 4))):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()
    with pytest.raises(ValueError, match=r"x must be \[tokens, channels\]"):
        B.leapquant_add_norm(e(2, 1, 128), e(2, 128))
    with pytest.raises(ValueError, match=r"x must be \[tokens, heads, d\]"):
        B.leapquant_gate_norm(e(2, 128), e(2, 128), e(2, 128))
    with pytest.raises(ValueError, match=r"weight must be \[n, k\]"):
        B.leapquant_quantize_weight(e(128), e(128, dtype=E4), e(1, 1))
    with pytest.raises(ValueError, match="x must be"):
        B.leapquant_matmul(e(128, dtype=E4), e(2, 1), e(4, 128, dtype=E4), e(1, 1), e(2, 4))


G = dict(device="cuda")


def _calls():
    """Calls of each operator that differ from a regular one in one argument, and what refuses it."""
    def t(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, **G)
    x, r, o8, s = t(3, 256), t(3, 256), t(3, 256, dtype=E4), t(3, 2)
    yield "add_norm", (x, o8), dict(residual=r, residual_out=t(3, 256), weight=t(256), scale=s), [
        (dict(scale=None), "scale is required"), (dict(scale=t(3, 3)), "scale must have shape"), (dict(scale=s.double()), "scale must be"),
        (dict(residual=t(3, 248)), "residual must have shape"), (dict(residual_out=t(3, 256).bfloat16()), "residual_out must be"),
        (dict(weight=t(255)), "weight must have shape"), (dict(weight=t(256).bfloat16()), "weight must be"),
        (dict(residual=r.half(), residual_out=None), "residual must be float32 or bfloat16"), (dict(norm=B.LQ_NORM_L2), "LQ_EINVAL|invalid"),
        (dict(residual=r.cpu()), "device tensor")]
    yield "add_norm", (x, t(3, 256)), {}, [(dict(scale=s), "scale belongs to")]
    yield "add_norm", (x, t(3, 256).half()), {}, [({}, "out must be float32, bfloat16 or float8_e4m3fn")]
    x3 = t(3, 2, 128)
    yield "gate_norm", (x3, t(3, 2, 128), t(3, 2, 128, dtype=E4)), dict(weight=t(128), scale=s), [
        (dict(scale=None), "scale is required"), (dict(weight=t(2, 64)), "weight must have shape"), (dict(weight=t(3, 128)), "weight must have shape"),
        (dict(weight=t(1, 2, 128)), "weight must have shape")]
    yield "gate_norm", (x3, t(3, 2, 64), t(3, 2, 128)), {}, [({}, "gate must have shape")]
    w, w8, ws = t(200, 256), t(200, 256, dtype=E4), t(2, 2)
    yield "quantize_weight", (w, w8, t(2, 3)), {}, [({}, "scale must have shape")]
    yield "quantize_weight", (w, w, ws), {}, [({}, "out must be")]
    xq, wq, out = t(3, 256, dtype=E4), t(200, 256, dtype=E4), t(3, 200)
    yield "matmul", (xq, s, wq, ws, out), {}, [
        (dict(bias=t(199)), "bias must have shape"), (dict(bias=t(200).bfloat16()), "bias must be")]
    yield "matmul", (xq, s, wq, ws, t(3, 200, dtype=E4)), {}, [({}, "out must be float32 or bfloat16")]
    yield "matmul", (xq.float(), s, wq, ws, out), {}, [({}, "x must be torch.float8")]
    yield "matmul", (xq, s, wq, t(200, 2), out), {}, [({}, "weight_scale must have shape")]
    yield "matmul", (xq, t(3, 1), wq, ws, out), {}, [({}, "x_scale must have shape")]
    yield "matmul", (xq, s, t(200, 512, dtype=E4)[:, ::2], ws, out), {}, [({}, "weight must be dense within")]


@pytest.mark.gpu
def test_irregular_calls_are_refused_by_the_python_checks_and_enqueue_nothing():
    for name, args, good, bad in _calls():
        for kw, says in bad:
            whole = dict(good, **kw)
            with pytest.raises((ValueError, B.LeapQuantError), match=says):
                getattr(B, "leapquant_" + name)(*args, **whole)


@pytest.mark.gpu
def test_regular_calls_take_the_native_path_and_give_the_same():
    torch.manual_seed(1)
    x, r, w = torch.randn(5, 256, **G).bfloat16(), torch.randn(5, 256, **G), torch.rand(256, **G)
    got = {}
    for path in ("native", "python"):
        kw = {} if path == "native" else {"stream": torch.cuda.current_stream()}
        o8, s, ro = torch.zeros(5, 256, dtype=E4, **G), torch.zeros(5, 2, **G), torch.zeros(5, 256, **G)
        g8, gs = torch.zeros(5, 2, 128, dtype=E4, **G), torch.zeros(5, 2, **G)
        w8, ws, out = torch.zeros(40, 256, dtype=E4, **G), torch.zeros(1, 2, **G), torch.zeros(5, 40, **G)
        gate, weight, bias = r.view(5, 2, 128), torch.cat([r] * 8), w[:40].contiguous()
        if path == "native":
            M, F = B._M, B._FN
            B.lib()
            M = B._M
            assert M.add_norm(F["leapquant_add_norm"], x, o8, r, ro, w, B.LQ_NORM_RMS, 1e-6, s) == 0
            assert M.gate_norm(F["leapquant_gate_norm"], x.view(5, 2, 128), gate, g8, w[:128].contiguous(), 0, False, 1e-6, gs) == 0
            assert M.gate_norm(F["leapquant_gate_norm"], x.view(5, 2, 128), gate, g8, w.view(2, 128), 0, True, 1e-6, gs) == 0
            assert M.quantize_weight(F["leapquant_quantize_weight"], weight, w8, ws) == 0
            assert M.matmul(F["leapquant_matmul"], o8, s, w8, ws, out, bias) == 0
        else:
            B.leapquant_add_norm(x, o8, residual=r, residual_out=ro, weight=w, scale=s, **kw)
            B.leapquant_gate_norm(x.view(5, 2, 128), gate, g8, weight=w[:128].contiguous(), scale=gs, **kw)
            B.leapquant_gate_norm(x.view(5, 2, 128), gate, g8, weight=w.view(2, 128), gate_first=True, scale=gs, **kw)
            B.leapquant_quantize_weight(weight, w8, ws, **kw)
            B.leapquant_matmul(o8, s, w8, ws, out, bias=bias, **kw)
        got[path] = [t.float().clone() for t in (o8, s, ro, g8, gs, w8, ws, out)]
    for a, b in zip(got["native"], got["python"]):
        assert torch.equal(a, b)
