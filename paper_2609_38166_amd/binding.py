"""Thin ctypes binding of libleapquant.so (the C ABI in include/leapquant.h).

Argument marshalling only: torch tensors are passed as raw device pointers and
the current HIP stream; every step runs in the library's HIP kernels.  Loading
fails loudly if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import warnings
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# The library; LEAPQUANT_LIB may name another build of it (a measurement
# variant made by build.py), which must export the same symbols.
LIB_PATH = os.environ.get("LEAPQUANT_LIB") or os.path.join(_PKG, "libleapquant.so")

LQ_OK, LQ_EINVAL, LQ_EALIGN, LQ_EUNSUPPORTED, LQ_EHIP, LQ_EDEVICE = 0, -1, -2, -3, -4, -5
LQ_GATE_SCALAR, LQ_GATE_DIAG = 0, 1
LQ_CODE_INT8, LQ_CODE_E4M3, LQ_CODE_INT4, LQ_CODE_INT6, LQ_CODE_BF16 = 0, 1, 2, 3, 4
CODE_BITS = {LQ_CODE_INT8: 8, LQ_CODE_E4M3: 8, LQ_CODE_INT4: 4, LQ_CODE_INT6: 6, LQ_CODE_BF16: 16}
LQ_STATE_F32, LQ_STATE_BF16 = 0, 1
LQ_RULE_DELTA, LQ_RULE_ADD, LQ_RULE_GENERAL = 0, 1, 2
LQ_DEVERR_WINDOW_FULL = 1
LQ_DEVERR_BAD_REC_LEN = 2
LQ_DEVERR_BAD_SEQLENS, LQ_DEVERR_BAD_SLOT, LQ_DEVERR_BAD_POSITION = 4, 8, 16
LQ_TOKEN_F32, LQ_TOKEN_BF16 = 0, 1
LQ_NORM_NONE, LQ_NORM_L2, LQ_NORM_RMS = 0, 1, 2
LQ_TOKEN_E4M3 = 2
LQ_ACT_SILU, LQ_ACT_SIGMOID = 0, 1
LQ_SCALE_BLOCK = 128

EXPORTS = ("leapquant_state_bytes", "leapquant_quantize_state", "leapquant_decode_step",
           "leapquant_decode_step_general", "leapquant_decode_step_commit", "leapquant_window_commit",
           "leapquant_baseline_step",
           "leapquant_baseline_step_general", "leapquant_dequantize_state",
           "leapquant_check_error", "leapquant_strerror", "leapquant_last_hip_error",
           "leapquant_conv_prompt", "leapquant_conv_step", "leapquant_qk_norm", "leapquant_scan_workspace_bytes",
           "leapquant_scan_prompt", "leapquant_scan_step", "leapquant_scan_gates",
           "leapquant_add_norm", "leapquant_gate_norm", "leapquant_quantize_weight", "leapquant_matmul")


class LeapQuantError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = f"{where}: {strerror(status)} (status {status})"
        if status == LQ_EHIP:
            msg += f": {_lib().leapquant_last_hip_error().decode()}"
        super().__init__(msg)
        self.status = status


class lq_dims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "batch", "heads_v", "heads_k", "d_k", "d_v", "window", "n_comp", "power_iters", "gate",
        "code", "smooth", "rule")]


class lq_state(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "codes", "scale", "smooth", "comp_k", "comp_u", "rec_k", "rec_u", "rec_a", "rec_len", "err")]


def _struct(name, fields):
    kinds = {"p": C.c_void_p, "i": C.c_int32, "l": C.c_int64, "f": C.c_float, "z": C.c_size_t}
    return type(name, (C.Structure,), {"_fields_": [(n, kinds[k]) for k, names in fields for n in names.split()]})


# the layer operators' arguments, field by field as in leapquant.h
lq_conv = _struct("lq_conv", (("i", "seqs channels width dtype out_dtype silu carry n_slots"),
                              ("l", "tokens x_stride out_stride"),
                              ("p", "x weight bias out state cu_seqlens slots err")))
lq_qk = _struct("lq_qk", (("l", "tokens"), ("i", "heads_q heads_k d norm rot interleaved dtype out_dtype"),
                          ("f", "eps q_scale"), ("l", "q_stride k_stride q_out_stride k_out_stride"),
                          ("p", "q k q_out k_out q_weight k_weight cos sin positions"), ("i", "n_positions"),
                          ("p", "err")))
lq_scan = _struct("lq_scan", (("l", "tokens"), ("i", "dtype state_dtype softplus carry n_slots max_len"),
                              ("l", "q_stride k_stride v_stride dt_stride o_stride"),
                              ("p", "q k v dt A skip dt_bias o state cu_seqlens slots err workspace"),
                              ("z", "workspace_bytes")))
# ... and the projection operators'
lq_add = _struct("lq_add", (("l", "tokens"), ("i", "channels norm dtype residual_dtype out_dtype"), ("f", "eps"),
                            ("l", "x_stride residual_stride residual_out_stride out_stride scale_stride"),
                            ("p", "x residual weight residual_out out scale")))
lq_gated = _struct("lq_gated", (("l", "tokens"), ("i", "heads d act gate_first weight_heads dtype gate_dtype out_dtype"),
                                ("f", "eps"), ("l", "x_stride gate_stride out_stride scale_stride"),
                                ("p", "x gate weight out scale")))
lq_weight = _struct("lq_weight", (("i", "n k dtype"), ("l", "w_stride out_stride"), ("p", "w out scale")))
lq_matmul = _struct("lq_matmul", (("l", "tokens"), ("i", "n k out_dtype"),
                                  ("l", "x_stride x_scale_stride w_stride out_stride"),
                                  ("p", "x x_scale w w_scale bias out")))


_L = None
# the native marshalling of regular calls (py_csrc/marshal.cpp; once the library is
# loaded, it or what stands in for it) and the addresses of the entry points it calls
_M = None
_FN = {"leapquant_decode_step": 0, "leapquant_decode_step_general": 0, "leapquant_decode_step_commit": 0,
       "leapquant_window_commit": 0, "leapquant_conv_prompt": 0, "leapquant_conv_step": 0, "leapquant_qk_norm": 0,
       "leapquant_scan_prompt": 0, "leapquant_scan_step": 0, "leapquant_scan_workspace_bytes": 0, "leapquant_add_norm": 0,
       "leapquant_gate_norm": 0, "leapquant_quantize_weight": 0, "leapquant_matmul": 0}


class _NoMarshal:
    """Stands in for the native marshalling where it cannot be loaded: every call is
    left to the Python checks (about 16 us a call, the same results)."""

    @staticmethod
    def step(*args):
        return None

    step_general = commit = conv = qk_norm = scan = step
    add_norm = gate_norm = quantize_weight = matmul = step


def _load_marshal(addr):
    """The native marshalling, set up, or its stand-in: the extension is tied to one
    build of torch and takes no call that the Python path does not."""
    try:
        from . import _marshal as native
        built = getattr(native, "torch_version", None)
        if built != torch.__version__:
            raise ImportError(f"_marshal.so was built against torch {built}, this is {torch.__version__}")
    except ImportError as e:
        warnings.warn(f"calls are checked and unpacked in Python, about 16 us each ({e}); "
                      "paper_2609_38166_amd/build.py builds _marshal.so", RuntimeWarning, stacklevel=3)
        return _NoMarshal
    native.setup(lq_dims, State, FIELDS, addr["leapquant_state_bytes"])
    return native


def _lib():
    global _L, _M
    if _L is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2609_38166_amd/build.py "
                              "(or __graft_entry__.build()); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, i32 = C.c_void_p, C.c_int32
        L.leapquant_state_bytes.argtypes = [vp, vp]
        L.leapquant_quantize_state.argtypes = [vp, vp, vp, vp]
        L.leapquant_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.leapquant_decode_step_general.argtypes = [vp] * 10
        L.leapquant_decode_step_commit.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.leapquant_window_commit.argtypes = [vp, vp, vp, vp]
        L.leapquant_baseline_step.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
        L.leapquant_baseline_step_general.argtypes = [vp, vp, i32] + [vp] * 8
        L.leapquant_dequantize_state.argtypes = [vp, vp, vp, vp]
        L.leapquant_check_error.argtypes = [vp, vp, vp]
        L.leapquant_conv_prompt.argtypes = [vp, vp]
        L.leapquant_conv_step.argtypes = [vp, vp]
        L.leapquant_qk_norm.argtypes = [vp, vp]
        L.leapquant_scan_workspace_bytes.argtypes = [vp, vp, vp]
        L.leapquant_scan_prompt.argtypes = [vp, vp, vp]
        L.leapquant_scan_step.argtypes = [vp, vp, vp]
        L.leapquant_scan_gates.argtypes = [vp, vp, vp, vp, vp]
        L.leapquant_add_norm.argtypes = [vp, vp]
        L.leapquant_gate_norm.argtypes = [vp, vp]
        L.leapquant_quantize_weight.argtypes = [vp, vp]
        L.leapquant_matmul.argtypes = [vp, vp]
        L.leapquant_strerror.argtypes = [i32]
        L.leapquant_strerror.restype = C.c_char_p
        L.leapquant_last_hip_error.argtypes = []
        L.leapquant_last_hip_error.restype = C.c_char_p
        for n in EXPORTS:
            if n not in ("leapquant_strerror", "leapquant_last_hip_error"):
                getattr(L, n).restype = C.c_int32
        addr = {n: C.cast(getattr(L, n), vp).value for n in EXPORTS}
        for n in _FN:
            _FN[n] = addr[n]
        _M, _L = _load_marshal(addr), L
    return _L


def lib():
    return _lib()


def strerror(status: int) -> str:
    return _lib().leapquant_strerror(status).decode()


def _check(status: int, where: str):
    if status != LQ_OK:
        raise LeapQuantError(status, where)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _need(t, nbytes: int, name: str, dtype=None):
    """Marshalling check: a contiguous device tensor (of `dtype`, if given)
    holding at least nbytes.  Raw integer addresses are passed through."""
    if t is None:
        raise ValueError(f"{name} is required")
    if isinstance(t, int):
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes, the call needs {nbytes}")


def _check_state(dims, st):
    for f, nb in zip(FIELDS, leapquant_state_bytes(dims)):
        if f in ("comp_k", "comp_u") and dims.n_comp == 0:
            continue
        _need(getattr(st, f), nb, f"state.{f}")


def _check_tokens(dims, q, k, v, alpha, beta, o):
    t, tk = dims.batch * dims.heads_v, dims.batch * dims.heads_k
    g = dims.d_k if dims.gate == LQ_GATE_DIAG else 1
    f32 = torch.float32
    _need(q, tk * dims.d_k * 4, "q", f32)
    _need(k, tk * dims.d_k * 4, "k", f32)
    _need(v, t * dims.d_v * 4, "v", f32)
    _need(alpha, t * g * 4, "alpha", f32)
    _need(beta, t * 4, "beta", f32)
    _need(o, t * dims.d_v * 4, "o", f32)


def _check_read(dims, b):
    _need(b, dims.batch * dims.heads_v * dims.d_k * 4, "b", torch.float32)


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_dims(batch, heads_v, heads_k=None, window=16, n_comp=4, power_iters=4,
              gate=LQ_GATE_SCALAR, code=LQ_CODE_INT8, smooth=1, d_k=128, d_v=128,
              rule=LQ_RULE_DELTA) -> lq_dims:
    return lq_dims(batch, heads_v, heads_k or heads_v, d_k, d_v, window, n_comp, power_iters, gate,
                   code, smooth, rule)


FIELDS = ("codes", "scale", "smooth", "comp_k", "comp_u", "rec_k", "rec_u", "rec_a", "rec_len", "err")


def leapquant_state_bytes(dims: lq_dims) -> list[int]:
    out = (C.c_size_t * 10)()
    _check(_lib().leapquant_state_bytes(C.byref(dims), out), "leapquant_state_bytes")
    return list(out)


@dataclass
class State:
    """Device buffers of the quantized state, allocated by torch (caller-owned).
    The FP16 buffers are float16 tensors (the C ABI sees their bits as uint16)."""
    dims: lq_dims
    codes: torch.Tensor
    scale: torch.Tensor
    smooth: torch.Tensor
    comp_k: torch.Tensor
    comp_u: torch.Tensor
    rec_k: torch.Tensor
    rec_u: torch.Tensor
    rec_a: torch.Tensor
    rec_len: torch.Tensor
    err: torch.Tensor

    @classmethod
    def empty(cls, dims: lq_dims, device="cuda") -> "State":
        B, Hv, dk, dv = dims.batch, dims.heads_v, dims.d_k, dims.d_v
        r, W = dims.n_comp, dims.window
        g = dk if dims.gate == LQ_GATE_DIAG else 1
        kw = {"device": device}
        return cls(
            dims,
            torch.zeros((B, Hv, dv, dk * CODE_BITS[dims.code] // 8), dtype=torch.uint8, **kw),
            torch.zeros((B, Hv, dv), dtype=torch.float32, **kw),
            torch.zeros((B, Hv, dk), dtype=torch.float32, **kw),
            torch.zeros((B, Hv, max(r, 1), dk), dtype=torch.float16, **kw),
            torch.zeros((B, Hv, max(r, 1), dv), dtype=torch.float16, **kw),
            torch.zeros((B, Hv, W, dk), dtype=torch.float16, **kw),
            torch.zeros((B, Hv, W, dv), dtype=torch.float16, **kw),
            torch.zeros((B, Hv, W, g), dtype=torch.float16, **kw),
            torch.zeros((B, Hv), dtype=torch.int32, **kw),
            torch.zeros((4,), dtype=torch.int32, **kw),
        )

    def struct(self) -> lq_state:
        return lq_state(*[getattr(self, f).data_ptr() for f in FIELDS])

    def requests(self, b0: int, b1: int) -> "State":
        """Requests b0 .. b1-1 as views into this state (every array starts at
        tile b0 * heads_v; the error word is shared), with dims for b1 - b0
        requests: a group that runs on its own schedule or stream."""
        if not 0 <= b0 < b1 <= self.dims.batch:
            raise ValueError(f"request range [{b0}, {b1}) outside [0, {self.dims.batch})")
        d = lq_dims.from_buffer_copy(self.dims)
        d.batch = b1 - b0
        return State(d, *[self.err if f == "err" else getattr(self, f)[b0:b1] for f in FIELDS])

    def nbytes(self) -> int:
        return sum(getattr(self, f).numel() * getattr(self, f).element_size() for f in FIELDS)


def leapquant_quantize_state(dims: lq_dims, S: torch.Tensor, st: State, stream=None):
    _check_state(dims, st)
    _need(S, dims.batch * dims.heads_v * dims.d_v * dims.d_k * 4, "S", torch.float32)
    s = st.struct()
    _check(_lib().leapquant_quantize_state(C.byref(dims), _ptr(S), C.byref(s), _stream(stream)),
           "leapquant_quantize_state")


def leapquant_decode_step(dims: lq_dims, st: State, q, k, v, alpha, beta, o, stream=None):
    if stream is None and (_M or _lib()):
        status = _M.step(_FN["leapquant_decode_step"], dims, st, q, k, v, alpha, beta, o)
        if status is not None:
            return _check(status, "leapquant_decode_step")
    _check_state(dims, st)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    s = st.struct()
    _check(_lib().leapquant_decode_step(C.byref(dims), C.byref(s), _ptr(q), _ptr(k), _ptr(v),
                                        _ptr(alpha), _ptr(beta), _ptr(o), _stream(stream)),
           "leapquant_decode_step")


def leapquant_decode_step_commit(dims: lq_dims, st: State, q, k, v, alpha, beta, o, stream=None):
    """Decode step, then the commit of every tile whose window it filled, in one
    launch."""
    if stream is None and (_M or _lib()):
        status = _M.step(_FN["leapquant_decode_step_commit"], dims, st, q, k, v, alpha, beta, o)
        if status is not None:
            return _check(status, "leapquant_decode_step_commit")
    _check_state(dims, st)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    s = st.struct()
    _check(_lib().leapquant_decode_step_commit(C.byref(dims), C.byref(s), _ptr(q), _ptr(k), _ptr(v),
                                               _ptr(alpha), _ptr(beta), _ptr(o), _stream(stream)),
           "leapquant_decode_step_commit")


def leapquant_decode_step_general(dims: lq_dims, st: State, q, k, b, v, alpha, beta, o,
                                  stream=None):
    """Decode step with the read vectors b [B][heads_v][d_k] given (dims.rule
    must be LQ_RULE_GENERAL)."""
    if stream is None and (_M or _lib()):
        status = _M.step_general(_FN["leapquant_decode_step_general"], dims, st, q, k, b, v, alpha, beta, o)
        if status is not None:
            return _check(status, "leapquant_decode_step_general")
    _check_state(dims, st)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    _check_read(dims, b)
    s = st.struct()
    _check(_lib().leapquant_decode_step_general(C.byref(dims), C.byref(s), _ptr(q), _ptr(k), _ptr(b),
                                                _ptr(v), _ptr(alpha), _ptr(beta), _ptr(o),
                                                _stream(stream)),
           "leapquant_decode_step_general")


def leapquant_window_commit(dims: lq_dims, st: State, mask=None, stream=None):
    if stream is None and (_M or _lib()):
        status = _M.commit(_FN["leapquant_window_commit"], dims, st, mask)
        if status is not None:
            return _check(status, "leapquant_window_commit")
    _check_state(dims, st)
    if mask is not None:
        _need(mask, dims.batch * 4, "mask")
    s = st.struct()
    _check(_lib().leapquant_window_commit(C.byref(dims), C.byref(s), _ptr(mask), _stream(stream)),
           "leapquant_window_commit")


def leapquant_baseline_step(dims: lq_dims, S, state_dtype: int, q, k, v, alpha, beta, o,
                            stream=None):
    width = 2 if state_dtype == LQ_STATE_BF16 else 4
    _need(S, dims.batch * dims.heads_v * dims.d_v * dims.d_k * width, "S",
          torch.bfloat16 if state_dtype == LQ_STATE_BF16 else torch.float32)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    _check(_lib().leapquant_baseline_step(C.byref(dims), _ptr(S), state_dtype, _ptr(q), _ptr(k),
                                          _ptr(v), _ptr(alpha), _ptr(beta), _ptr(o),
                                          _stream(stream)),
           "leapquant_baseline_step")


def leapquant_baseline_step_general(dims: lq_dims, S, state_dtype: int, q, k, b, v, alpha, beta, o,
                                    stream=None):
    width = 2 if state_dtype == LQ_STATE_BF16 else 4
    _need(S, dims.batch * dims.heads_v * dims.d_v * dims.d_k * width, "S",
          torch.bfloat16 if state_dtype == LQ_STATE_BF16 else torch.float32)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    _check_read(dims, b)
    _check(_lib().leapquant_baseline_step_general(C.byref(dims), _ptr(S), state_dtype, _ptr(q),
                                                  _ptr(k), _ptr(b), _ptr(v), _ptr(alpha), _ptr(beta),
                                                  _ptr(o), _stream(stream)),
           "leapquant_baseline_step_general")


def leapquant_dequantize_state(dims: lq_dims, st: State, S_out, stream=None):
    _check_state(dims, st)
    _need(S_out, dims.batch * dims.heads_v * dims.d_v * dims.d_k * 4, "S_out", torch.float32)
    s = st.struct()
    _check(_lib().leapquant_dequantize_state(C.byref(dims), C.byref(s), _ptr(S_out),
                                             _stream(stream)),
           "leapquant_dequantize_state")


def leapquant_check_error(st: State, stream=None) -> int:
    """Synchronise, return the sticky device error bits and clear them."""
    s = st.struct()
    bits = C.c_int32(0)
    status = _lib().leapquant_check_error(C.byref(s), _stream(stream), C.byref(bits))
    if status not in (LQ_OK, LQ_EDEVICE):
        raise LeapQuantError(status, "leapquant_check_error")
    return bits.value


class Prepared:
    """A call with its ctypes arguments built once, for tight timing loops."""

    def __init__(self, fn, *args):
        self.fn, self.args = fn, args

    def __call__(self):
        status = self.fn(*self.args)
        if status != LQ_OK:
            raise LeapQuantError(status, self.fn.__name__)


def prepare_decode(dims, st: State, q, k, v, alpha, beta, o, stream=None) -> Prepared:
    _check_state(dims, st)
    _check_tokens(dims, q, k, v, alpha, beta, o)
    s = st.struct()
    st._keep = s
    return Prepared(_lib().leapquant_decode_step, C.byref(dims), C.byref(s), _ptr(q), _ptr(k),
                    _ptr(v), _ptr(alpha), _ptr(beta), _ptr(o), _stream(stream))


def prepare_commit(dims, st: State, mask=None, stream=None) -> Prepared:
    _check_state(dims, st)
    if mask is not None:
        _need(mask, dims.batch * 4, "mask")
    s = st.struct()
    st._keep_c = s
    return Prepared(_lib().leapquant_window_commit, C.byref(dims), C.byref(s), _ptr(mask),
                    _stream(stream))


# ---- layer operators around the decode step: convolution, query/key norm, selective scan ----

_TOKEN = {torch.float32: LQ_TOKEN_F32, torch.bfloat16: LQ_TOKEN_BF16}


def _token(t, name):
    if t.dtype not in _TOKEN:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return _TOKEN[t.dtype]


def _device(t, name, dtype=None, optional=False):
    """Address of a device tensor (None: NULL if it is optional)."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _rows(t, name, shape, dtype=None):
    """Address and row stride (elements) of a token array of this shape: dense within a
    row, rows at any distance."""
    p = _device(t, name, dtype)
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    row = 1
    for n, stride in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if n != 1 and stride != row:
            raise ValueError(f"{name} must be dense within a token's row")
        row *= n
    return p, t.stride(0) if shape[0] > 1 else row


def _dense(t, name, shape, dtype=torch.float32, optional=False):
    p = _device(t, name, dtype, optional)
    if t is not None:
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    return p


def _slots(slots, seqs):
    return _dense(slots, "slots", (seqs,), torch.int32, True)


def _err(err):
    return _device(err, "err", torch.int32, True)


def _conv(fn, x, weight, out, seqs, cu_seqlens, bias, silu, state, carry, slots, err, stream):
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be [tokens, channels] and weight [channels, width]")
    (tokens, channels), width = x.shape, weight.shape[1]
    px, xs = _rows(x, "x", (tokens, channels))
    po, os_ = _rows(out, "out", (tokens, channels))
    n_slots = 0
    if state is not None:
        n_slots = state.shape[0]
        _dense(state, "state", (n_slots, width - 1, channels), x.dtype)
    a = lq_conv(seqs, channels, width, _token(x, "x"), _token(out, "out"), int(silu), int(carry), n_slots, tokens, xs, os_,
                px, _dense(weight, "weight", (channels, width)), _dense(bias, "bias", (channels,), optional=True), po,
                _ptr(state), _ptr(cu_seqlens), _slots(slots, seqs), _err(err))
    _check(getattr(_lib(), fn)(C.byref(a), _stream(stream)), fn)


def leapquant_conv_prompt(x, weight, out, cu_seqlens, bias=None, silu=True, state=None, carry=False, slots=None, err=None,
                          stream=None):
    """Short causal convolution of packed sequences: x, out [tokens, channels], weight
    [channels, width], cu_seqlens int32 [sequences + 1]; state [slots, width-1, channels]
    of x's type, read if `carry`, holds the last inputs afterwards."""
    if stream is None and cu_seqlens is not None and (_M or _lib()):
        status = _M.conv(_FN["leapquant_conv_prompt"], x, weight, out, cu_seqlens, bias, silu, state, carry, slots, err)
        if status is not None:
            return _check(status, "leapquant_conv_prompt")
    seqs = _seqs(cu_seqlens)
    _conv("leapquant_conv_prompt", x, weight, out, seqs, cu_seqlens, bias, silu, state, carry, slots, err, stream)


def leapquant_conv_step(x, weight, out, state, bias=None, silu=True, slots=None, err=None, stream=None):
    """The convolution for one token of every request (row b of x), state in place."""
    if state is None:
        raise ValueError("state is required")
    if stream is None and (_M or _lib()):
        status = _M.conv(_FN["leapquant_conv_step"], x, weight, out, None, bias, silu, state, True, slots, err)
        if status is not None:
            return _check(status, "leapquant_conv_step")
    _conv("leapquant_conv_step", x, weight, out, x.shape[0], None, bias, silu, state, True, slots, err, stream)


def _seqs(cu_seqlens):
    _device(cu_seqlens, "cu_seqlens", torch.int32)
    if cu_seqlens.dim() != 1 or not cu_seqlens.is_contiguous() or cu_seqlens.shape[0] < 2:
        raise ValueError("cu_seqlens must be a contiguous vector of sequences + 1 entries")
    return cu_seqlens.shape[0] - 1


def leapquant_qk_norm(q, k, q_out, k_out, norm=LQ_NORM_L2, eps=1e-6, q_weight=None, k_weight=None, q_scale=1.0, cos=None,
                      sin=None, positions=None, interleaved=False, err=None, stream=None):
    """Norm of every query and key head [tokens, heads, d] and the rotation of the first
    2 * cos.shape[1] channels by the token's position (cos, sin [positions, rot/2]); k and
    k_out may be None."""
    if stream is None and (_M or _lib()):
        status = _M.qk_norm(_FN["leapquant_qk_norm"], q, k, q_out, k_out, norm, eps, q_weight, k_weight, q_scale, cos, sin,
                            positions, interleaved, err)
        if status is not None:
            return _check(status, "leapquant_qk_norm")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, d]")
    tokens, hq, d = q.shape
    pq, qs = _rows(q, "q", (tokens, hq, d))
    pqo, qos = _rows(q_out, "q_out", (tokens, hq, d))
    hk, pk, ks, pko, kos = 0, None, 0, None, 0
    if k is not None:
        hk = k.shape[1] if k.dim() == 3 else 0
        pk, ks = _rows(k, "k", (tokens, hk, d), q.dtype)
        pko, kos = _rows(k_out, "k_out", (tokens, hk, d), q_out.dtype)
    rot = n_pos = 0
    pc = ps = pp = None
    if cos is not None:
        n_pos, half = cos.shape
        rot = 2 * half
        pc, ps = _dense(cos, "cos", (n_pos, half)), _dense(sin, "sin", (n_pos, half))
        pp = _dense(positions, "positions", (tokens,), torch.int32)
    a = lq_qk(tokens, hq, hk, d, norm, rot, int(interleaved), _token(q, "q"), _token(q_out, "q_out"), eps, q_scale, qs, ks,
              qos, kos, pq, pk, pqo, pko, _dense(q_weight, "q_weight", (d,), optional=True),
              _dense(k_weight, "k_weight", (d,), optional=True), pc, ps, pp, n_pos, _err(err))
    _check(_lib().leapquant_qk_norm(C.byref(a), _stream(stream)), "leapquant_qk_norm")


def _scan_args(dims, q, k, v, dt, A, o, state, cu_seqlens, D, dt_bias, softplus, carry, slots, max_len, err):
    tokens, dtype = v.shape[0], v.dtype
    hv, hk, dk, dv = dims.heads_v, dims.heads_k, dims.d_k, dims.d_v
    pq, qs = _rows(q, "q", (tokens, hk, dk), dtype)
    pk, ks = _rows(k, "k", (tokens, hk, dk), dtype)
    pv, vs = _rows(v, "v", (tokens, hv, dv))
    pd, ds = _rows(dt, "dt", (tokens, hv), dtype)
    po, os_ = _rows(o, "o", (tokens, hv, dv), dtype)
    n_slots, sdt = 0, LQ_STATE_F32
    if state is not None:
        n_slots, sdt = state.shape[0], LQ_STATE_BF16 if state.dtype == torch.bfloat16 else LQ_STATE_F32
        _dense(state, "state", (n_slots, hv, dv, dk), torch.bfloat16 if sdt == LQ_STATE_BF16 else torch.float32)
    return lq_scan(tokens, _token(v, "v"), sdt, int(softplus), int(carry), n_slots, max_len, qs, ks, vs, ds, os_, pq, pk, pv, pd,
                   _dense(A, "A", (hv,)), _dense(D, "D", (hv,), optional=True),
                   _dense(dt_bias, "dt_bias", (hv,), optional=True), po, _ptr(state), _ptr(cu_seqlens),
                   _slots(slots, dims.batch), _err(err), None, 0)


def leapquant_scan_prompt(dims: lq_dims, q, k, v, dt, A, o, cu_seqlens, D=None, dt_bias=None, softplus=True, state=None,
                          carry=False, slots=None, max_len=0, workspace=None, err=None, stream=None):
    """Selective scan of packed sequences: q, k [tokens, heads_k, 128], v, o [tokens,
    heads_v, 128], dt [tokens, heads_v] of one type, A, D, dt_bias fp32 [heads_v]; state
    fp32 [slots, heads_v, d_v, d_k] (S^T), read if `carry`, is the final state afterwards.
    max_len, the longest sequence, lets the work be split better where it is known.  The
    workspace is allocated here unless a uint8 tensor is given; a stream of the caller's
    needs one."""
    if stream is None and cu_seqlens is not None and (_M or _lib()):
        status = _M.scan(_FN["leapquant_scan_prompt"], _FN["leapquant_scan_workspace_bytes"], dims, q, k, v, dt, A, o, D, dt_bias,
                         softplus, state, cu_seqlens, carry, slots, max_len, workspace, err)
        if status is not None:
            return _check(status, "leapquant_scan_prompt")
    if _seqs(cu_seqlens) != dims.batch:
        raise ValueError(f"cu_seqlens holds {_seqs(cu_seqlens)} sequences, dims.batch is {dims.batch}")
    a = _scan_args(dims, q, k, v, dt, A, o, state, cu_seqlens, D, dt_bias, softplus, carry, slots,
                   min(v.shape[0], 2**31 - 1) if max_len == 0 else max_len, err)
    need = C.c_size_t(0)
    _check(_lib().leapquant_scan_workspace_bytes(C.byref(dims), C.byref(a), C.byref(need)), "leapquant_scan_workspace_bytes")
    if need.value:
        if workspace is None:
            if stream is not None:
                raise ValueError(f"a call on a stream of the caller's needs a workspace of {need.value} bytes")
            workspace = torch.empty(need.value, dtype=torch.uint8, device=v.device)
        a.workspace, a.workspace_bytes = _device(workspace, "workspace", torch.uint8), workspace.numel()
        _need(workspace, need.value, "workspace")
    _check(_lib().leapquant_scan_prompt(C.byref(dims), C.byref(a), _stream(stream)), "leapquant_scan_prompt")


def leapquant_scan_workspace_bytes(dims: lq_dims, tokens, dtype=torch.bfloat16, max_len=0) -> int:
    """Workspace that leapquant_scan_prompt needs: for a call of these tokens and max_len, or, with
    max_len = 0, for every call with at most so many tokens."""
    need = C.c_size_t(0)
    a = lq_scan(tokens=tokens, dtype=_TOKEN[dtype], max_len=max_len)
    _check(_lib().leapquant_scan_workspace_bytes(C.byref(dims), C.byref(a), C.byref(need)), "leapquant_scan_workspace_bytes")
    return need.value


def leapquant_scan_step(dims: lq_dims, state, q, k, v, dt, A, o, D=None, dt_bias=None, softplus=True, slots=None, err=None,
                        stream=None):
    """The scan for one token of every request (row b), its dense state (fp32 or bf16) in place."""
    if state is None:
        raise ValueError("state is required")
    if stream is None and (_M or _lib()):
        status = _M.scan(_FN["leapquant_scan_step"], 0, dims, q, k, v, dt, A, o, D, dt_bias, softplus, state, None, True, slots,
                         0, None, err)
        if status is not None:
            return _check(status, "leapquant_scan_step")
    a = _scan_args(dims, q, k, v, dt, A, o, state, None, D, dt_bias, softplus, True, slots, 0, err)
    _check(_lib().leapquant_scan_step(C.byref(dims), C.byref(a), _stream(stream)), "leapquant_scan_step")


def leapquant_scan_gates(dims: lq_dims, dt, A, alpha, beta, dt_bias=None, softplus=True, stream=None):
    """alpha = exp(delta A), beta = delta, fp32 [tokens, heads_v]: what leapquant_decode_step takes under LQ_RULE_ADD."""
    tokens, hv = dt.shape[0], dims.heads_v
    pd, ds = _rows(dt, "dt", (tokens, hv))
    a = lq_scan(tokens=tokens, dtype=_token(dt, "dt"), softplus=int(softplus), dt_stride=ds, dt=pd, A=_dense(A, "A", (hv,)),
                dt_bias=_dense(dt_bias, "dt_bias", (hv,), optional=True))
    _check(_lib().leapquant_scan_gates(C.byref(dims), C.byref(a), _dense(alpha, "alpha", (tokens, hv)),
                                       _dense(beta, "beta", (tokens, hv)), _stream(stream)), "leapquant_scan_gates")


def leapquant_check_error_word(err, stream=None) -> int:
    """leapquant_check_error for a layer operator's error word (int32 device tensor)."""
    s = lq_state(err=_device(err, "err", torch.int32))
    bits = C.c_int32(0)
    status = _lib().leapquant_check_error(C.byref(s), _stream(stream), C.byref(bits))
    if status not in (LQ_OK, LQ_EDEVICE):
        raise LeapQuantError(status, "leapquant_check_error")
    return bits.value


# ---- projection operators: residual and norm, gated norm, weights and products in E4M3 ----

_OUT = {**_TOKEN, torch.float8_e4m3fn: LQ_TOKEN_E4M3}
E4M3 = torch.float8_e4m3fn


def _out(t, name):
    if t.dtype not in _OUT:
        raise ValueError(f"{name} must be float32, bfloat16 or float8_e4m3fn, got {t.dtype}")
    return _OUT[t.dtype]


def _blocks(channels):
    return -(-channels // LQ_SCALE_BLOCK)


def _here(first, *others):
    """All tensors on the current device, whose stream the call goes to."""
    for t in (first, *others):
        if t is not None and t.is_cuda and t.device.index != torch.cuda.current_device():
            raise ValueError(f"a tensor is on {t.device}, the current device is {torch.cuda.current_device()}")


def _scales(scale, out, tokens, channels):
    """Address and stride of an E4M3 output's scales (None for the other types)."""
    if out.dtype != E4M3:
        if scale is not None:
            raise ValueError("scale belongs to a float8_e4m3fn output")
        return None, 0
    if scale is None:
        raise ValueError("scale is required for a float8_e4m3fn output")
    return _rows(scale, "scale", (tokens, _blocks(channels)), torch.float32)


def leapquant_add_norm(x, out, residual=None, residual_out=None, weight=None, norm=LQ_NORM_RMS, eps=1e-6, scale=None,
                       stream=None):
    """h = x + residual (kept in residual_out) and its RMS norm times weight (or h itself, LQ_NORM_NONE), rows [tokens,
    channels]; out fp32, bf16, or float8_e4m3fn with scale fp32 [tokens, ceil(channels / 128)].  residual_out may be
    residual, in place."""
    if stream is None and (_M or _lib()):
        status = _M.add_norm(_FN["leapquant_add_norm"], x, out, residual, residual_out, weight, norm, eps, scale)
        if status is not None:
            return _check(status, "leapquant_add_norm")
    if x.dim() != 2:
        raise ValueError("x must be [tokens, channels]")
    _here(x, out, residual, residual_out, weight, scale)
    shape = tokens, channels = tuple(x.shape)
    px, xs = _rows(x, "x", shape)
    po, os_ = _rows(out, "out", shape)
    pr = ps = None
    rs = ss = 0
    kind = x
    if residual is not None:
        pr, rs = _rows(residual, "residual", shape)
        kind = residual
    if residual_out is not None:
        ps, ss = _rows(residual_out, "residual_out", shape, residual.dtype if residual is not None else None)
        kind = residual_out
    pc, cs = _scales(scale, out, tokens, channels)
    a = lq_add(tokens, channels, norm, _token(x, "x"), _token(kind, "residual"), _out(out, "out"), eps, xs, rs, ss, os_, cs, px, pr,
               _dense(weight, "weight", (channels,), optional=True), ps, po, pc)
    _check(_lib().leapquant_add_norm(C.byref(a), _stream(stream)), "leapquant_add_norm")


def leapquant_gate_norm(x, gate, out, weight=None, act=LQ_ACT_SILU, gate_first=False, eps=1e-6, scale=None, stream=None):
    """RMS norm of every head of x [tokens, heads, d] times weight ([d] or [heads, d]) and act(gate) (gate_first: the norm of
    x * act(gate) times weight); out fp32, bf16, or float8_e4m3fn with scale fp32 [tokens, ceil(heads * d / 128)]."""
    if stream is None and (_M or _lib()):
        status = _M.gate_norm(_FN["leapquant_gate_norm"], x, gate, out, weight, act, gate_first, eps, scale)
        if status is not None:
            return _check(status, "leapquant_gate_norm")
    if x.dim() != 3:
        raise ValueError("x must be [tokens, heads, d]")
    _here(x, gate, out, weight, scale)
    shape = tokens, heads, d = tuple(x.shape)
    px, xs = _rows(x, "x", shape)
    pg, gs = _rows(gate, "gate", shape)
    po, os_ = _rows(out, "out", shape)
    pc, cs = _scales(scale, out, tokens, heads * d)
    each = weight is not None and weight.dim() == 2
    pw = _dense(weight, "weight", (heads, d) if each else (d,), optional=True)
    a = lq_gated(tokens, heads, d, act, int(gate_first), int(each), _token(x, "x"), _token(gate, "gate"), _out(out, "out"), eps, xs,
                 gs, os_, cs, px, pg, pw, po, pc)
    _check(_lib().leapquant_gate_norm(C.byref(a), _stream(stream)), "leapquant_gate_norm")


def leapquant_quantize_weight(weight, out, scale, stream=None):
    """A weight [n, k] (fp32 or bf16) in float8_e4m3fn, out [n, k], with scale fp32 [ceil(n / 128), ceil(k / 128)]."""
    if stream is None and (_M or _lib()):
        status = _M.quantize_weight(_FN["leapquant_quantize_weight"], weight, out, scale)
        if status is not None:
            return _check(status, "leapquant_quantize_weight")
    if weight.dim() != 2:
        raise ValueError("weight must be [n, k]")
    _here(weight, out, scale)
    shape = n, k = tuple(weight.shape)
    pw, ws = _rows(weight, "weight", shape)
    po, os_ = _rows(out, "out", shape, E4M3)
    a = lq_weight(n, k, _token(weight, "weight"), ws, os_, pw, po, _dense(scale, "scale", (_blocks(n), _blocks(k))))
    _check(_lib().leapquant_quantize_weight(C.byref(a), _stream(stream)), "leapquant_quantize_weight")


def leapquant_matmul(x, x_scale, weight, weight_scale, out, bias=None, stream=None):
    """out [tokens, n] (fp32 or bf16) = x [tokens, k] times weight [n, k] transposed, plus bias [n]: x float8_e4m3fn with x_scale
    [tokens, ceil(k / 128)], weight float8_e4m3fn with weight_scale [ceil(n / 128), ceil(k / 128)]."""
    if stream is None and (_M or _lib()):
        status = _M.matmul(_FN["leapquant_matmul"], x, x_scale, weight, weight_scale, out, bias)
        if status is not None:
            return _check(status, "leapquant_matmul")
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be [tokens, k] and weight [n, k]")
    _here(x, x_scale, weight, weight_scale, out, bias)
    (tokens, k), n = x.shape, weight.shape[0]
    px, xs = _rows(x, "x", (tokens, k), E4M3)
    pxs, xss = _rows(x_scale, "x_scale", (tokens, _blocks(k)), torch.float32)
    pw, ws = _rows(weight, "weight", (n, k), E4M3)
    pws = _dense(weight_scale, "weight_scale", (_blocks(n), _blocks(k)))
    po, os_ = _rows(out, "out", (tokens, n))
    a = lq_matmul(tokens, n, k, _token(out, "out"), xs, xss, ws, os_, px, pxs, pw, pws, _dense(bias, "bias", (n,), optional=True), po)
    _check(_lib().leapquant_matmul(C.byref(a), _stream(stream)), "leapquant_matmul")
