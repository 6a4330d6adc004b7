// Argument marshalling of the Python binding's per-token calls.
//
// A call made of regular arguments (an lq_dims, a binding.State, contiguous
// device tensors of the right type and size, the current stream) takes 15.7 us of
// host time when its 16 tensors are checked and unpacked from Python (7.7 us of
// it the checks), against 3 to 6 us for the kernel it launches on a small batch.
// The same checks here take 0.3 us, the call 4.0 (the C entry with its launch
// 3.9).  Anything else -- another type, raw addresses, a stream of the
// caller's, an argument that fails a check -- returns None before anything is
// enqueued, and the Python path takes the call: it accepts what it accepts and
// words what it refuses.  Nothing is kept from one call for the next.
#include <Python.h>

#include <algorithm>

#include <c10/hip/HIPStream.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "leapquant.h"

namespace {

PyTypeObject *g_dims_type = nullptr, *g_state_type = nullptr;
PyObject *g_names[10];      // attribute names of the state buffers, in lq_state's order
int32_t (*g_state_bytes)(const lq_dims *, size_t *) = nullptr;

enum { ANY = -1 };

// The address of a contiguous device tensor of scalar type `type` (ANY: any)
// with at least `bytes` bytes; false for anything else.
bool tensor_ptr(PyObject *o, size_t bytes, int type, void **p) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) return false;
    if (type != ANY && t.scalar_type() != static_cast<at::ScalarType>(type)) return false;
    if (t.nbytes() < bytes) return false;
    *p = t.data_ptr();
    return true;
}

struct Call {
    lq_dims dims;
    lq_state st;
    size_t tiles, ktiles, gate;
};

bool unpack(PyObject *dims, PyObject *state, Call &c) {
    if (Py_TYPE(dims) != g_dims_type || Py_TYPE(state) != g_state_type) return false;
    Py_buffer v;
    if (PyObject_GetBuffer(dims, &v, PyBUF_SIMPLE) != 0) return false;
    const bool whole = v.len == (Py_ssize_t)sizeof(lq_dims);
    if (whole) memcpy(&c.dims, v.buf, sizeof(lq_dims));
    PyBuffer_Release(&v);
    if (!whole) return false;
    size_t need[10];
    if (g_state_bytes(&c.dims, need) != LQ_OK) return false;
    void **field[10] = {&c.st.codes, (void **)&c.st.scale, (void **)&c.st.smooth, (void **)&c.st.comp_k,
                        (void **)&c.st.comp_u, (void **)&c.st.rec_k, (void **)&c.st.rec_u, (void **)&c.st.rec_a,
                        (void **)&c.st.rec_len, (void **)&c.st.err};
    for (int i = 0; i < 10; ++i) {
        PyObject *o = PyObject_GetAttr(state, g_names[i]);
        if (!o) return false;
        bool ok;
        if ((i == 3 || i == 4) && c.dims.n_comp == 0) {     // the tokens of a state without any: only addressed
            ok = THPVariable_CheckExact(o);
            if (ok) *field[i] = THPVariable_Unpack(o).data_ptr();
        } else {
            ok = tensor_ptr(o, need[i], ANY, field[i]);
        }
        Py_DECREF(o);                                       // (the state holds it)
        if (!ok) return false;
    }
    c.tiles = (size_t)c.dims.batch * c.dims.heads_v;
    c.ktiles = (size_t)c.dims.batch * c.dims.heads_k;
    c.gate = c.dims.gate == LQ_GATE_DIAG ? c.dims.d_k : 1;
    return true;
}

// Runs body, which enqueues on the current stream and sets `status`; None where
// it returns false or throws.
template <typename F>
PyObject *guarded(F body) {
    int32_t status = 0;
    bool ok = false;
    try {
        ok = body(status);
    } catch (...) {
    }
    if (!ok) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

void *current_stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

constexpr int F32 = (int)at::ScalarType::Float;

// step(fn, dims, state, q, k, v, alpha, beta, o)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        Call c;
        if (!unpack(a[1], a[2], c)) return false;
        const size_t vec = c.tiles * c.dims.d_v * 4, key = c.ktiles * c.dims.d_k * 4;
        const size_t need[6] = {key, key, vec, c.tiles * c.gate * 4, c.tiles * 4, vec};
        void *p[6];
        for (int i = 0; i < 6; ++i)
            if (!tensor_ptr(a[3 + i], need[i], F32, &p[i])) return false;
        using Fn = int32_t (*)(const lq_dims *, lq_state *, void *, void *, void *, void *, void *, void *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&c.dims, &c.st, p[0], p[1], p[2], p[3], p[4], p[5], s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// step_general(fn, dims, state, q, k, b, v, alpha, beta, o)
PyObject *step_general(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 10) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        Call c;
        if (!unpack(a[1], a[2], c)) return false;
        const size_t vec = c.tiles * c.dims.d_v * 4, key = c.ktiles * c.dims.d_k * 4;
        const size_t need[7] = {key, key, c.tiles * c.dims.d_k * 4, vec, c.tiles * c.gate * 4, c.tiles * 4, vec};
        void *p[7];
        for (int i = 0; i < 7; ++i)
            if (!tensor_ptr(a[3 + i], need[i], F32, &p[i])) return false;
        using Fn = int32_t (*)(const lq_dims *, lq_state *, void *, void *, void *, void *, void *, void *, void *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&c.dims, &c.st, p[0], p[1], p[2], p[3], p[4], p[5], p[6], s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// commit(fn, dims, state, mask or None)
PyObject *commit(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        Call c;
        if (!unpack(a[1], a[2], c)) return false;
        void *mask = nullptr;
        if (a[3] != Py_None && !tensor_ptr(a[3], (size_t)c.dims.batch * 4, ANY, &mask)) return false;
        using Fn = int32_t (*)(const lq_dims *, lq_state *, void *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&c.dims, &c.st, mask, s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// ---- layer operators: the checks of the binding's _conv, leapquant_qk_norm and _scan_args ----

// A device tensor, or None where it may be missing (*p is then NULL); t: the tensor or nullptr.
bool device(PyObject *o, bool optional, const at::Tensor **t, void **p) {
    *t = nullptr;
    *p = nullptr;
    if (o == Py_None) return optional;
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &x = THPVariable_Unpack(o);
    if (!x.is_cuda()) return false;
    *t = &x;
    *p = x.data_ptr();
    return true;
}

bool token_type(const at::Tensor &t, int32_t *type) {
    if (t.scalar_type() == at::ScalarType::BFloat16) *type = LQ_TOKEN_BF16;
    else if (t.scalar_type() == at::ScalarType::Float) *type = LQ_TOKEN_F32;
    else return false;
    return true;
}

// A token array of n dimensions and these sizes, dense within a row.
bool token_rows(PyObject *o, int n, const int64_t *size, const void **p, int64_t *stride, const at::Tensor **t) {
    void *q;
    if (!device(o, false, t, &q) || (*t)->dim() != n) return false;
    *p = q;
    int64_t row = 1;
    for (int i = n - 1; i >= 0; --i) {
        if ((*t)->size(i) != size[i]) return false;
        if (i == 0) break;
        if (size[i] != 1 && (*t)->stride(i) != row) return false;
        row *= size[i];
    }
    *stride = size[0] > 1 ? (*t)->stride(0) : row;
    return true;
}

// A contiguous tensor of these sizes and type (or None).
bool dense(PyObject *o, int n, const int64_t *size, at::ScalarType type, bool optional, void **p) {
    const at::Tensor *t;
    if (!device(o, optional, &t, p)) return false;
    if (!t) return true;
    if (t->dim() != n || t->scalar_type() != type || !t->is_contiguous()) return false;
    for (int i = 0; i < n; ++i)
        if (t->size(i) != size[i]) return false;
    return true;
}
template <typename T>
bool vec(PyObject *o, int64_t n, at::ScalarType type, bool optional, T **p) {
    void *q;
    if (!dense(o, 1, &n, type, optional, &q)) return false;
    *p = (T *)q;
    return true;
}

// Sequences of cu_seqlens (its entries less one; 0: not regular).
int64_t sequences(PyObject *o, const int32_t **p) {
    const at::Tensor *t;
    void *q;
    if (!device(o, false, &t, &q)) return 0;
    *p = (const int32_t *)q;
    if (t->dim() != 1 || t->scalar_type() != at::ScalarType::Int || !t->is_contiguous()) return 0;
    return t->size(0) - 1;
}

bool error_word(PyObject *o, int32_t **p) {
    const at::Tensor *t;
    void *q;
    if (!device(o, true, &t, &q)) return false;
    if (t && t->scalar_type() != at::ScalarType::Int) return false;
    *p = (int32_t *)q;
    return true;
}

// False, True, 0 or 1; what else int() makes of a flag, or refuses, is the Python path's.
bool flag(PyObject *o, int32_t *p) {
    if (o == Py_True || o == Py_False) {
        *p = o == Py_True;
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    const long x = PyLong_AsLong(o);
    *p = (int32_t)x;
    return x == 0 || x == 1;
}

constexpr at::ScalarType F = at::ScalarType::Float, I32 = at::ScalarType::Int;

// conv(fn, x, weight, out, cu_seqlens or None (the step), bias, silu, state, carry, slots, err)
PyObject *conv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        lq_conv c = {};
        const at::Tensor *x, *w, *o, *st;
        void *p;
        if (!device(a[1], false, &x, &p) || x->dim() != 2 || !device(a[2], false, &w, &p) || w->dim() != 2) return false;
        const int64_t size[2] = {x->size(0), x->size(1)}, width = w->size(1), wsize[2] = {size[1], width};
        const void *out;
        if (size[1] > INT32_MAX || width > INT32_MAX) return false;
        if (!token_rows(a[1], 2, size, &c.x, &c.x_stride, &x) || !token_type(*x, &c.dtype)) return false;
        if (!token_rows(a[3], 2, size, &out, &c.out_stride, &o) || !token_type(*o, &c.out_dtype)) return false;
        if (!dense(a[2], 2, wsize, F, false, &p)) return false;
        c.weight = (const float *)p;
        c.out = (void *)out;
        const bool step = a[4] == Py_None;
        const int64_t seqs = step ? size[0] : sequences(a[4], &c.cu_seqlens);
        if (seqs < 1 || seqs > INT32_MAX) return false;
        if (!vec(a[5], size[1], F, true, &c.bias)) return false;
        if (!device(a[7], !step, &st, &c.state)) return false;
        if (st) {
            const int64_t ssize[3] = {st->dim() ? st->size(0) : 0, width - 1, size[1]};
            if (ssize[0] > INT32_MAX || !dense(a[7], 3, ssize, x->scalar_type(), false, &c.state)) return false;
            c.n_slots = (int32_t)ssize[0];
        }
        if (!vec(a[9], seqs, I32, true, &c.slots) || !error_word(a[10], &c.err)) return false;
        c.seqs = (int32_t)seqs;
        c.channels = (int32_t)size[1];
        c.width = (int32_t)width;
        if (!flag(a[6], &c.silu) || !flag(a[8], &c.carry)) return false;
        c.tokens = size[0];
        using Fn = int32_t (*)(const lq_conv *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&c, s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// qk_norm(fn, q, k, q_out, k_out, norm, eps, q_weight, k_weight, q_scale, cos, sin, positions, interleaved, err)
PyObject *qk_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 15) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        lq_qk c = {};
        const at::Tensor *q, *k, *t;
        const void *p;
        void *v;
        if (!device(a[1], false, &q, &v) || q->dim() != 3) return false;
        const int64_t qs[3] = {q->size(0), q->size(1), q->size(2)};
        if (!token_rows(a[1], 3, qs, &c.q, &c.q_stride, &q) || !token_type(*q, &c.dtype)) return false;
        if (!token_rows(a[3], 3, qs, &p, &c.q_out_stride, &t) || !token_type(*t, &c.out_dtype)) return false;
        c.q_out = (void *)p;
        const at::ScalarType out_type = t->scalar_type();
        if (!device(a[2], true, &k, &v)) return false;
        int64_t hk = 0;
        if (k) {
            if (k->dim() != 3) return false;
            hk = k->size(1);
            const int64_t ks[3] = {qs[0], hk, qs[2]};
            if (!token_rows(a[2], 3, ks, &c.k, &c.k_stride, &k) || k->scalar_type() != q->scalar_type()) return false;
            if (!token_rows(a[4], 3, ks, &p, &c.k_out_stride, &t) || t->scalar_type() != out_type) return false;
            c.k_out = (void *)p;
        }
        if (qs[1] > INT32_MAX || qs[2] > INT32_MAX || hk > INT32_MAX) return false;
        if (!vec(a[7], qs[2], F, true, &c.q_weight) || !vec(a[8], qs[2], F, true, &c.k_weight)) return false;
        if (!device(a[10], true, &t, &v)) return false;
        if (t) {
            if (t->dim() != 2 || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX / 2) return false;
            const int64_t size[2] = {t->size(0), t->size(1)};
            if (!dense(a[10], 2, size, F, false, &v)) return false;
            c.cos = (const float *)v;
            if (!dense(a[11], 2, size, F, false, &v)) return false;
            c.sin = (const float *)v;
            if (!vec(a[12], qs[0], I32, false, &c.positions)) return false;
            c.rot = (int32_t)(2 * size[1]);
            c.n_positions = (int32_t)size[0];
        }
        if (!error_word(a[14], &c.err)) return false;
        const long norm = PyLong_AsLong(a[5]);
        c.eps = (float)PyFloat_AsDouble(a[6]);
        c.q_scale = (float)PyFloat_AsDouble(a[9]);
        if (PyErr_Occurred() || norm < INT32_MIN || norm > INT32_MAX) return false;
        c.norm = (int32_t)norm;
        if (!flag(a[13], &c.interleaved)) return false;
        c.tokens = qs[0];
        c.heads_q = (int32_t)qs[1];
        c.heads_k = (int32_t)hk;
        c.d = (int32_t)qs[2];
        using Fn = int32_t (*)(const lq_qk *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&c, s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// scan(fn, workspace_bytes fn, dims, q, k, v, dt, A, o, D, dt_bias, softplus, state, cu_seqlens or None (the step),
//      carry, slots, max_len, workspace or None, err)
PyObject *scan(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 19) Py_RETURN_NONE;
    return guarded([&](int32_t &status) {
        lq_scan c = {};
        lq_dims d;
        if (Py_TYPE(a[2]) != g_dims_type) return false;
        Py_buffer b;
        if (PyObject_GetBuffer(a[2], &b, PyBUF_SIMPLE) != 0) return false;
        const bool whole = b.len == (Py_ssize_t)sizeof(lq_dims);
        if (whole) memcpy(&d, b.buf, sizeof(lq_dims));
        PyBuffer_Release(&b);
        if (!whole) return false;
        const at::Tensor *v, *t, *st;
        const void *p;
        void *w;
        if (!device(a[5], false, &v, &w) || v->dim() != 3) return false;
        const int64_t T = v->size(0), ks[3] = {T, d.heads_k, d.d_k}, vs[3] = {T, d.heads_v, d.d_v};
        if (!token_rows(a[5], 3, vs, &c.v, &c.v_stride, &v) || !token_type(*v, &c.dtype)) return false;
        const at::ScalarType type = v->scalar_type();
        if (!token_rows(a[3], 3, ks, &c.q, &c.q_stride, &t) || t->scalar_type() != type) return false;
        if (!token_rows(a[4], 3, ks, &c.k, &c.k_stride, &t) || t->scalar_type() != type) return false;
        if (!token_rows(a[6], 2, vs, &c.dt, &c.dt_stride, &t) || t->scalar_type() != type) return false;
        if (!token_rows(a[8], 3, vs, &p, &c.o_stride, &t) || t->scalar_type() != type) return false;
        c.o = (void *)p;
        if (!vec(a[7], d.heads_v, F, false, &c.A) || !vec(a[9], d.heads_v, F, true, &c.skip) ||
            !vec(a[10], d.heads_v, F, true, &c.dt_bias))
            return false;
        const bool step = a[13] == Py_None;
        if (!device(a[12], !step, &st, &c.state)) return false;
        if (st) {
            if (st->dim() != 4 || st->size(0) > INT32_MAX) return false;
            const bool bf = st->scalar_type() == at::ScalarType::BFloat16;
            const int64_t ss[4] = {st->size(0), d.heads_v, d.d_v, d.d_k};
            if (!dense(a[12], 4, ss, bf ? at::ScalarType::BFloat16 : F, false, &c.state)) return false;
            c.state_dtype = bf ? LQ_STATE_BF16 : LQ_STATE_F32;
            c.n_slots = (int32_t)ss[0];
        }
        if (!step && sequences(a[13], &c.cu_seqlens) != d.batch) return false;
        if (!vec(a[15], d.batch, I32, true, &c.slots) || !error_word(a[18], &c.err)) return false;
        const long max_len = PyLong_AsLong(a[16]);
        if (PyErr_Occurred() || max_len < INT32_MIN || max_len > INT32_MAX) return false;
        c.max_len = (int32_t)(max_len ? max_len : std::min<int64_t>(T, INT32_MAX));     // (the need of this call alone)
        if (!flag(a[11], &c.softplus) || !flag(a[14], &c.carry)) return false;
        c.tokens = T;
        at::Tensor own;                 // freed into the allocator's pool of this stream after the launch
        if (!step) {
            size_t need = 0;
            using Size = int32_t (*)(const lq_dims *, const lq_scan *, size_t *);
            if (((Size)PyLong_AsVoidPtr(a[1]))(&d, &c, &need) != LQ_OK) return false;
            if (need) {
                if (a[17] == Py_None) {
                    own = at::empty({(int64_t)need}, v->options().dtype(at::ScalarType::Byte));
                    c.workspace = own.data_ptr();
                } else if (!tensor_ptr(a[17], need, (int)at::ScalarType::Byte, &c.workspace)) {
                    return false;
                }
                c.workspace_bytes = need;
            }
        }
        using Fn = int32_t (*)(const lq_dims *, const lq_scan *, void *);
        const Fn fn = (Fn)PyLong_AsVoidPtr(a[0]);
        void *s = current_stream();
        Py_BEGIN_ALLOW_THREADS
        status = fn(&d, &c, s);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// setup(lq_dims type, State type, field names, address of leapquant_state_bytes)
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *dims, *state, *names, *fn;
    if (!PyArg_ParseTuple(args, "OOOO", &dims, &state, &names, &fn)) return nullptr;
    if (!PyType_Check(dims) || !PyType_Check(state) || !PyTuple_Check(names) || PyTuple_Size(names) != 10) {
        PyErr_SetString(PyExc_TypeError, "setup(type, type, ten names, address)");
        return nullptr;
    }
    void *addr = PyLong_AsVoidPtr(fn);
    if (!addr) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_ValueError, "no address"), nullptr);
    for (int i = 0; i < 10; ++i) {
        PyObject *s = PyTuple_GetItem(names, i);
        Py_INCREF(s);
        PyUnicode_InternInPlace(&s);
        Py_XSETREF(g_names[i], s);
    }
    Py_INCREF(dims);
    Py_XSETREF(g_dims_type, (PyTypeObject *)dims);
    Py_INCREF(state);
    Py_XSETREF(g_state_type, (PyTypeObject *)state);
    g_state_bytes = (int32_t(*)(const lq_dims *, size_t *))addr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"setup", setup, METH_VARARGS, "types, field names and leapquant_state_bytes of the binding"},
    {"step", (PyCFunction)(void (*)(void))step, METH_FASTCALL, "decode step: status, or None for the Python path"},
    {"step_general", (PyCFunction)(void (*)(void))step_general, METH_FASTCALL, "decode step with read vectors"},
    {"commit", (PyCFunction)(void (*)(void))commit, METH_FASTCALL, "window commit"},
    {"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, "convolution, prompt or step"},
    {"qk_norm", (PyCFunction)(void (*)(void))qk_norm, METH_FASTCALL, "query and key norm"},
    {"scan", (PyCFunction)(void (*)(void))scan, METH_FASTCALL, "selective scan, prompt or step"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (the binding uses the extension with the torch that it was built against only)
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", LQ_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
