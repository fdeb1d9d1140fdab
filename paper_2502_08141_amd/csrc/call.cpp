// The binding's calls that a training step or a decoding loop makes once per layer, without Python between the caller and
// the library: argument checks, the output's allocation and the library call in one C function.
//
// Why: a linear call spent 5.7 us in Python (1.8 of them in torch.empty) beside 2.6 us per kernel launch, more than many of
// these calls take on the GPU; here it spends about 2.  Only the plain case is handled -- exact torch.Tensor arguments that
// pass every check, and no torch mode that wants to see the allocations.  For anything else (a subclass, a wrong type, shape or
// device, an exception from torch) the functions return None with nothing launched, and lowra.py goes through its own checks,
// which raise what they always raised.  So every object that a call returns exists before the library is called.  The interpreter's
// lock is given up for the allocations too, as torch.empty does (one may wait for the GPU).  Nothing is kept between calls but
// the library's entry points.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

typedef int (*linear_fn)(const void*, const void*, const void*, const void*, const void*, int, const void*, const void*, int, float, void*,
                         void*, size_t, void*);
typedef const void* (*side_fn)(const void*, int, int, int, const void*);
typedef int (*grads_fn)(const void*, const void*, const void*, int, const void*, const void*, int, float, void*, void*, void*, size_t, void*);
typedef int (*grads_side_fn)(const void*, const void*, const void*, int, int, const void*, const void*, void*, void*, void*, size_t, void*);
typedef int (*dequant_fn)(const void*, const void*, const void*, const void*, int, void*, void*);
linear_fn lib_linear[2];
side_fn lib_side;
grads_fn lib_grads;
grads_side_fn lib_grads_side;
dequant_fn lib_dequant;

// what a call needs of a layout, in the order of Layout.native (lowra.py)
struct Lay { const void* handle; int64_t N, K, C, packed_bytes; bool bf16_scales; };

bool layout_of(PyObject* o, Lay& l) {
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 6) return false;
    l.handle = PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0));
    l.N = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 1));
    l.K = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
    l.C = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 3));
    l.packed_bytes = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 4));
    l.bf16_scales = PyTuple_GET_ITEM(o, 5) == Py_True;
    return l.handle != nullptr && !PyErr_Occurred();
}

// a plain, contiguous device tensor of this type, or null
const at::Tensor* plain(PyObject* o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.scalar_type() == type && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}
bool shape2(const at::Tensor& t, int64_t a, int64_t b) { return t.dim() == 2 && t.size(0) == a && t.size(1) == b; }

bool state_ok(const Lay& l, const at::Tensor* packed, const at::Tensor* absmax, const at::Tensor* mappings) {
    return packed && absmax && mappings && packed->numel() == l.packed_bytes && absmax->numel() == l.N * (l.K / 64) && shape2(*mappings, l.C, 16);
}
bool modes() { return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled(); }
void* current_stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

PyObject* none() {
    PyErr_Clear();
    Py_RETURN_NONE;
}
// the interpreter's lock, given up for a scope
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
at::Tensor empty(at::IntArrayRef sizes, const at::TensorOptions& options) {
    Unlocked u;
    return at::empty(sizes, options);
}
// what the caller returns: the result, or the library's status when that is not zero
PyObject* done(int status, PyObject* result) {
    if (status == 0) return result;
    Py_DECREF(result);
    return PyLong_FromLong(status);
}

// linear(which, layout, packed, absmax, mappings, act, A, B, s, workspace): which = 0 forward, 1 input gradient
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return none();
    try {
        if (modes()) return none();
        const long which = PyLong_AsLong(a[0]);
        Lay l;
        if ((which != 0 && which != 1) || !layout_of(a[1], l)) return none();
        const at::Tensor* packed = plain(a[2], at::kByte);
        const at::Tensor* absmax = plain(a[3], l.bf16_scales ? at::kBFloat16 : at::kFloat);
        const at::Tensor* mappings = plain(a[4], at::kFloat);
        const at::Tensor* act = plain(a[5], at::kBFloat16);
        const int64_t in = which ? l.N : l.K, cols = which ? l.K : l.N;
        if (!state_ok(l, packed, absmax, mappings) || !act || act->dim() != 2 || act->size(1) != in || !PyFloat_Check(a[8])) return none();
        const int64_t M = act->size(0);
        if (M > INT32_MAX) return none();
        const at::Tensor *A = nullptr, *B = nullptr;
        int64_t r = 0;
        if (a[6] != Py_None && a[7] != Py_None) {
            A = plain(a[6], at::kBFloat16); B = plain(a[7], at::kBFloat16);
            if (!A || !B || A->dim() != 2 || A->size(0) < 1) return none();
            r = A->size(0);
            if (r > INT32_MAX || A->size(1) != l.K || !shape2(*B, l.N, r)) return none();
        }
        if (!THPVariable_CheckExact(a[9])) return none();             // the caller's own workspace; the library checks its size
        const at::Tensor& ws = THPVariable_Unpack(a[9]);
        void* const wp = ws.data_ptr();
        const size_t ws_bytes = (size_t)ws.numel() * ws.element_size();
        const float s = (float)PyFloat_AS_DOUBLE(a[8]);
        at::Tensor out = empty({M, cols}, act->options());
        void *po = out.data_ptr(), *st = current_stream();
        const void *pp = packed->data_ptr(), *pa = absmax->data_ptr(), *pm = mappings->data_ptr(), *px = act->data_ptr();
        const void *pA = A ? A->data_ptr() : nullptr, *pB = B ? B->data_ptr() : nullptr;
        PyObject* res = THPVariable_Wrap(std::move(out));
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_linear[which](l.handle, pp, pa, pm, px, (int)M, pA, pB, (int)r, s, po, wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// the operands of a linear call's epilogue, as include/lowra.h lays them out
struct FwdEpilogue { int act; const void *bias, *mul, *residual; void* z; };
struct BwdEpilogue { int act; const void *z, *mul, *residual; void* dmul; };
typedef int (*linear_act_fn)(const void*, const void*, const void*, const void*, const void*, int, const void*, const void*, int, float, const void*,
                             void*, void*, size_t, void*);
typedef int (*act_bwd_fn)(int, int, int, const void*, const void*, const void*, void*, void*, void*, void*, size_t, void*);
linear_act_fn lib_linear_act[2];
act_bwd_fn lib_act_bwd;

// (first, second or None)
PyObject* pair_or_none(at::Tensor first, at::Tensor second, bool has_second) {
    PyObject* x = THPVariable_Wrap(std::move(first));
    PyObject* y = x && has_second ? THPVariable_Wrap(std::move(second)) : nullptr;
    PyObject* t = x && (y || !has_second) ? PyTuple_Pack(2, x, y ? y : Py_None) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}
// an operand that may be None: false if it is neither that nor a plain bf16 tensor of this shape on `device`
bool operand(PyObject* o, int64_t rows, int64_t cols, const at::Tensor& like, const void*& p) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o, at::kBFloat16);
    if (!t || t->device() != like.device() || !(rows < 0 ? t->dim() == 1 && t->size(0) == cols : shape2(*t, rows, cols))) return false;
    p = t->data_ptr();
    return true;
}

// linear_act(which, layout, packed, absmax, mappings, act, A, B, s, activation, bias or z, mul, residual, second, workspace) ->
// (y, z or None) or (dX, dmul or None); `second`: whether z is kept (forward; the input gradient returns dmul where there is mul)
PyObject* linear_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 15) return none();
    try {
        if (modes()) return none();
        const long which = PyLong_AsLong(a[0]);
        Lay l;
        if ((which != 0 && which != 1) || !layout_of(a[1], l)) return none();
        const at::Tensor* packed = plain(a[2], at::kByte);
        const at::Tensor* absmax = plain(a[3], l.bf16_scales ? at::kBFloat16 : at::kFloat);
        const at::Tensor* mappings = plain(a[4], at::kFloat);
        const at::Tensor* act = plain(a[5], at::kBFloat16);
        const int64_t in = which ? l.N : l.K, cols = which ? l.K : l.N;
        if (!state_ok(l, packed, absmax, mappings) || !act || act->dim() != 2 || act->size(1) != in || !PyFloat_Check(a[8]) || !PyLong_CheckExact(a[9]) ||
            !PyBool_Check(a[13])) return none();
        const int64_t M = act->size(0);
        if (M > INT32_MAX) return none();
        const at::Tensor *A = nullptr, *B = nullptr;
        int64_t r = 0;
        if (a[6] != Py_None && a[7] != Py_None) {
            A = plain(a[6], at::kBFloat16); B = plain(a[7], at::kBFloat16);
            if (!A || !B || A->dim() != 2 || A->size(0) < 1) return none();
            r = A->size(0);
            if (r > INT32_MAX || A->size(1) != l.K || !shape2(*B, l.N, r)) return none();
        }
        const void *first, *mul, *residual;
        if (!operand(a[10], which ? M : -1, cols, *act, first) || !operand(a[11], M, cols, *act, mul) || !operand(a[12], M, cols, *act, residual)) return none();
        const long activation = PyLong_AsLong(a[9]);
        if (PyErr_Occurred() || activation != (int)activation) return none();
        const at::Tensor* ws = plain(a[14], at::kByte);
        if (!ws || act->get_device() != c10::hip::current_device()) return none();
        for (const at::Tensor* t : {ws, packed, absmax, mappings, A, B})
            if (t && t->device() != act->device()) return none();
        void* const wp = ws->data_ptr();
        const size_t ws_bytes = (size_t)ws->numel();
        const float s = (float)PyFloat_AS_DOUBLE(a[8]);
        const bool two = which ? mul != nullptr : a[13] == Py_True;
        at::Tensor out = empty({M, cols}, act->options()), second;
        if (two) second = empty({M, cols}, act->options());
        void *po = out.data_ptr(), *p2 = two ? second.data_ptr() : nullptr, *st = current_stream();
        const void *pp = packed->data_ptr(), *pa = absmax->data_ptr(), *pm = mappings->data_ptr(), *px = act->data_ptr();
        const void *pA = A ? A->data_ptr() : nullptr, *pB = B ? B->data_ptr() : nullptr;
        const FwdEpilogue fe{(int)activation, first, mul, residual, p2};
        const BwdEpilogue be{(int)activation, first, mul, residual, p2};
        PyObject* res = pair_or_none(std::move(out), std::move(second), two);
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_linear_act[which](l.handle, pp, pa, pm, px, (int)M, pA, pB, (int)r, s, which ? (const void*)&be : (const void*)&fe, po, wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// act_bwd(dY, activation, z, mul, bias_grad, workspace) -> (dZ or None, dmul or None, db or None)
PyObject* act_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return none();
    try {
        if (modes()) return none();
        const at::Tensor* dY = plain(a[0], at::kBFloat16);
        if (!dY || dY->dim() != 2 || !PyLong_CheckExact(a[1]) || !PyBool_Check(a[4])) return none();
        const int64_t M = dY->size(0), N = dY->size(1);
        const long activation = PyLong_AsLong(a[1]);
        const void *z, *mul;
        if (PyErr_Occurred() || activation != (int)activation || M > INT32_MAX || N > INT32_MAX || !operand(a[2], M, N, *dY, z) || !operand(a[3], M, N, *dY, mul))
            return none();
        const at::Tensor* ws = plain(a[5], at::kByte);
        const bool want[3] = {activation != 0 || mul, mul != nullptr, a[4] == Py_True};
        if (!ws || ws->device() != dY->device() || dY->get_device() != c10::hip::current_device() || !(want[0] || want[2])) return none();
        at::Tensor out[3];
        void* p[3] = {nullptr, nullptr, nullptr};
        if (want[0]) out[0] = empty({M, N}, dY->options());
        if (want[1]) out[1] = empty({M, N}, dY->options());
        if (want[2]) out[2] = empty({N}, dY->options().dtype(at::kFloat));
        for (int i = 0; i < 3; ++i) if (want[i]) p[i] = out[i].data_ptr();
        const void* py = dY->data_ptr();
        void *wp = ws->data_ptr(), *st = current_stream();
        const size_t ws_bytes = (size_t)ws->numel();
        PyObject* v[3] = {nullptr, nullptr, nullptr};
        bool fine = true;
        for (int i = 0; i < 3 && fine; ++i) {
            if (want[i]) { v[i] = THPVariable_Wrap(std::move(out[i])); fine = v[i] != nullptr; }
            else { Py_INCREF(Py_None); v[i] = Py_None; }
        }
        PyObject* res = fine ? PyTuple_Pack(3, v[0], v[1], v[2]) : nullptr;
        for (PyObject* o : v) Py_XDECREF(o);
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_act_bwd((int)M, (int)N, (int)activation, py, z, mul, p[0], p[1], p[2], wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// side_product(layout, op, M, r, workspace) -> (view,) or (None,)
PyObject* side_product(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return none();
    try {
        if (modes()) return none();
        Lay l;
        if (!layout_of(a[0], l) || !PyLong_CheckExact(a[1]) || !PyLong_CheckExact(a[2]) || !PyLong_CheckExact(a[3])) return none();
        const long op = PyLong_AsLong(a[1]), M = PyLong_AsLong(a[2]), r = PyLong_AsLong(a[3]);
        const at::Tensor* ws = plain(a[4], at::kByte);
        if (PyErr_Occurred() || !ws || op != (int)op || M != (int)M || r != (int)r || ws->dim() != 1) return none();
        const uint8_t* base = static_cast<const uint8_t*>(ws->data_ptr());
        const uint8_t* p = static_cast<const uint8_t*>(lib_side(l.handle, (int)op, (int)M, (int)r, base));
        if (!p) return PyTuple_Pack(1, Py_None);
        const int64_t off = p - base, bytes = (int64_t)M * 128;
        if (off < 0 || off + bytes > ws->numel()) return none();
        PyObject* v = THPVariable_Wrap(ws->narrow(0, off, bytes).view(at::kBFloat16).view({M, 64}));
        if (!v) return none();
        PyObject* t = PyTuple_Pack(1, v);
        Py_DECREF(v);
        return t;
    } catch (...) {
        return none();
    }
}

PyObject* pair(at::Tensor dA, at::Tensor dB) {
    PyObject* x = THPVariable_Wrap(std::move(dA));
    PyObject* y = x ? THPVariable_Wrap(std::move(dB)) : nullptr;
    PyObject* t = y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}

// grads(layout, x, dY, A, B, s, workspace)
PyObject* grads(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return none();
    try {
        if (modes()) return none();
        Lay l;
        if (!layout_of(a[0], l) || !PyFloat_Check(a[5])) return none();
        const at::Tensor *x = plain(a[1], at::kBFloat16), *dY = plain(a[2], at::kBFloat16), *A = plain(a[3], at::kBFloat16), *B = plain(a[4], at::kBFloat16);
        const at::Tensor* ws = plain(a[6], at::kByte);
        if (!x || !dY || !A || !B || !ws || x->dim() != 2 || A->dim() != 2) return none();
        const int64_t M = x->size(0), r = A->size(0);
        if (M > INT32_MAX || r > INT32_MAX || !shape2(*x, M, l.K) || !shape2(*dY, M, l.N) || !shape2(*A, r, l.K) || !shape2(*B, l.N, r)) return none();
        const auto opt = x->options().dtype(at::kFloat);
        at::Tensor dA = empty({r, l.K}, opt), dB = empty({l.N, r}, opt);
        const void *px = x->data_ptr(), *py = dY->data_ptr(), *pA = A->data_ptr(), *pB = B->data_ptr();
        void *qa = dA.data_ptr(), *qb = dB.data_ptr(), *wp = ws->data_ptr(), *st = current_stream();
        const size_t ws_bytes = (size_t)ws->numel();
        const float s = (float)PyFloat_AS_DOUBLE(a[5]);
        PyObject* res = pair(std::move(dA), std::move(dB));
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_grads(l.handle, px, py, (int)M, pA, pB, (int)r, s, qa, qb, wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// grads_from_side(layout, x, dY, r, st, su, workspace)
PyObject* grads_from_side(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return none();
    try {
        if (modes()) return none();
        Lay l;
        if (!layout_of(a[0], l) || !PyLong_CheckExact(a[3])) return none();
        const int64_t r = PyLong_AsLongLong(a[3]);
        const at::Tensor *x = plain(a[1], at::kBFloat16), *dY = plain(a[2], at::kBFloat16), *ts = plain(a[4], at::kBFloat16), *us = plain(a[5], at::kBFloat16);
        const at::Tensor* ws = plain(a[6], at::kByte);
        if (PyErr_Occurred() || !x || !dY || !ts || !us || !ws || x->dim() != 2 || r < 0 || r > INT32_MAX) return none();
        const int64_t M = x->size(0);
        if (M > INT32_MAX || !shape2(*x, M, l.K) || !shape2(*dY, M, l.N) || !shape2(*ts, M, 64) || !shape2(*us, M, 64)) return none();
        const auto opt = x->options().dtype(at::kFloat);
        at::Tensor dA = empty({r, l.K}, opt), dB = empty({l.N, r}, opt);
        const void *px = x->data_ptr(), *py = dY->data_ptr(), *pt = ts->data_ptr(), *pu = us->data_ptr();
        void *qa = dA.data_ptr(), *qb = dB.data_ptr(), *wp = ws->data_ptr(), *st = current_stream();
        const size_t ws_bytes = (size_t)ws->numel();
        PyObject* res = pair(std::move(dA), std::move(dB));
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_grads_side(l.handle, px, py, (int)M, (int)r, pt, pu, qa, qb, wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// dequantize(layout, packed, absmax, mappings): bf16
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) return none();
    try {
        if (modes()) return none();
        Lay l;
        if (!layout_of(a[0], l)) return none();
        const at::Tensor* packed = plain(a[1], at::kByte);
        const at::Tensor* absmax = plain(a[2], l.bf16_scales ? at::kBFloat16 : at::kFloat);
        const at::Tensor* mappings = plain(a[3], at::kFloat);
        if (!state_ok(l, packed, absmax, mappings)) return none();
        at::Tensor out = empty({l.N, l.K}, packed->options().dtype(at::kBFloat16));
        const void *pp = packed->data_ptr(), *pa = absmax->data_ptr(), *pm = mappings->data_ptr();
        void *po = out.data_ptr(), *st = current_stream();
        PyObject* res = THPVariable_Wrap(std::move(out));
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_dequant(l.handle, pp, pa, pm, 0, po, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// init(addresses): the library's entry points, in the order of lowra.py
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "init: six addresses"); return nullptr; }
    void* f[6];
    for (int i = 0; i < 6; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    lib_linear[0] = (linear_fn)f[0]; lib_linear[1] = (linear_fn)f[1]; lib_side = (side_fn)f[2];
    lib_grads = (grads_fn)f[3]; lib_grads_side = (grads_side_fn)f[4]; lib_dequant = (dequant_fn)f[5];
    Py_RETURN_NONE;
}

// init_act(addresses): those of the calls with an activation
PyObject* init_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "init_act: three addresses"); return nullptr; }
    void* f[3];
    for (int i = 0; i < 3; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    lib_linear_act[0] = (linear_act_fn)f[0]; lib_linear_act[1] = (linear_act_fn)f[1]; lib_act_bwd = (act_bwd_fn)f[2];
    Py_RETURN_NONE;
}

// ---- the operators of a training step beside the linear
typedef int (*norm_fwd_fn)(int, int, int, const void*, const void*, const void*, float, void*, void*);
typedef int (*norm_bwd_fn)(int, int, int, const void*, const void*, const void*, float, const void*, void*, void*, void*, void*, size_t, void*);
struct RopeTensor { const void* x; void* y; int heads; int64_t x_token, x_head, y_token, y_head; };      // as include/lowra.h lays it out
typedef int (*rope_fn)(int, const RopeTensor*, int, int, int, int, const void*, const void*, float, int, void*);
typedef int (*vocab_loss_fn)(int, int, int, const void*, const void*, const void*, const void*, void*, void*, void*, void*, size_t, void*);
norm_fwd_fn lib_norm_fwd;
norm_bwd_fn lib_norm_bwd;
rope_fn lib_rope;
vocab_loss_fn lib_vocab_loss;

bool here(const at::Tensor& t) { return t.get_device() == c10::hip::current_device(); }
bool small_int(PyObject* o, int& v) {
    if (!PyLong_CheckExact(o)) return false;
    const long x = PyLong_AsLong(o);
    v = (int)x;
    return !PyErr_Occurred() && x == v;
}
// a tuple of the tensors that are wanted, None for the others
template <size_t N>
PyObject* tuple_of(at::Tensor (&out)[N], const bool (&want)[N]) {
    PyObject* res = PyTuple_New(N);
    for (size_t i = 0; i < N && res; ++i) {
        PyObject* v = Py_None;
        if (want[i]) {
            try {
                v = THPVariable_Wrap(std::move(out[i]));
            } catch (...) {
                Py_DECREF(res);
                throw;
            }
        } else {
            Py_INCREF(v);
        }
        if (v) PyTuple_SET_ITEM(res, i, v);
        else Py_CLEAR(res);
    }
    return res;
}

// norm_fwd(x, weight, bias, kind, eps) -> y
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return none();
    try {
        if (modes()) return none();
        const at::Tensor* x = plain(a[0], at::kBFloat16);
        int kind;
        const void *weight, *bias;
        if (!x || x->dim() != 2 || !here(*x) || !small_int(a[3], kind) || !PyFloat_CheckExact(a[4])) return none();
        const int64_t M = x->size(0), N = x->size(1);
        if (M > INT32_MAX || N > INT32_MAX || !operand(a[1], -1, N, *x, weight) || !operand(a[2], -1, N, *x, bias)) return none();
        at::Tensor y = empty({M, N}, x->options());
        const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
        const void* px = x->data_ptr();
        void *py = y.data_ptr(), *st = current_stream();
        PyObject* res = THPVariable_Wrap(std::move(y));
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_norm_fwd((int)M, (int)N, kind, px, weight, bias, eps, py, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// norm_bwd(dY, x, weight, kind, eps, residual, input_grad, weight_grad, bias_grad, workspace) -> (dX or None, dweight or None, dbias or None)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return none();
    try {
        if (modes()) return none();
        const at::Tensor *dY = plain(a[0], at::kBFloat16), *ws = plain(a[9], at::kByte);
        int kind;
        if (!dY || !ws || dY->dim() != 2 || !here(*dY) || ws->device() != dY->device() || !small_int(a[3], kind) || !PyFloat_CheckExact(a[4])) return none();
        for (int i = 6; i < 9; ++i)
            if (!PyBool_Check(a[i])) return none();
        const int64_t M = dY->size(0), N = dY->size(1);
        const void *x, *weight, *residual;
        if (M > INT32_MAX || N > INT32_MAX || a[1] == Py_None || !operand(a[1], M, N, *dY, x) || !operand(a[2], -1, N, *dY, weight) || !operand(a[5], M, N, *dY, residual))
            return none();
        const bool want[3] = {a[6] == Py_True, a[7] == Py_True, a[8] == Py_True};
        at::Tensor out[3];
        void* p[3] = {nullptr, nullptr, nullptr};
        for (int i = 0; i < 3; ++i) {
            if (!want[i]) continue;
            out[i] = i == 0 ? empty({M, N}, dY->options()) : empty({N}, dY->options().dtype(at::kFloat));
            p[i] = out[i].data_ptr();
        }
        const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
        const void* py = dY->data_ptr();
        void *wp = ws->data_ptr(), *st = current_stream();
        const size_t ws_bytes = (size_t)ws->numel();
        PyObject* res = tuple_of(out, want);
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_norm_bwd((int)M, (int)N, kind, py, x, weight, eps, residual, p[0], p[1], p[2], wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// rope(x or list of x, positions, turns, layout, inverse, magnitude) -> y or list of y
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return none();
    PyObject* res = nullptr;
    try {
        if (modes()) return none();
        const bool many = PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0]);
        const Py_ssize_t count = many ? PySequence_Fast_GET_SIZE(a[0]) : 1;
        const at::Tensor *positions = plain(a[1], at::kInt), *turns = plain(a[2], at::kLong);
        int layout;
        if (count < 1 || count > 4 || !positions || !turns || positions->dim() != 1 || turns->dim() != 1 || !small_int(a[3], layout) || !PyBool_Check(a[4]) ||
            !PyFloat_CheckExact(a[5]))
            return none();
        RopeTensor t[4];
        at::Tensor in[4], out[4];                                     // in: a list may lose its tensors while others have the interpreter's lock
        const int64_t M = positions->size(0);
        int64_t D = -1;
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* o = many ? PySequence_Fast_GET_ITEM(a[0], i) : a[0];
            if (!THPVariable_CheckExact(o)) return none();
            const at::Tensor& x = THPVariable_Unpack(o);
            if (x.scalar_type() != at::kBFloat16 || !x.is_cuda() || x.dim() != 3 || (x.stride(2) != 1 && x.size(2) != 1) || x.size(0) != M || !here(x)) return none();
            if (D < 0) D = x.size(2);
            if (x.size(2) != D || x.size(1) > INT32_MAX) return none();
            in[i] = x;
            t[i] = RopeTensor{x.data_ptr(), nullptr, (int)x.size(1), x.stride(0), x.stride(1), x.size(1) * D, D};
        }
        if (M > INT32_MAX || D > INT32_MAX || turns->size(0) > INT32_MAX / 2 || !here(*positions) || !here(*turns)) return none();
        for (Py_ssize_t i = 0; i < count; ++i) {
            out[i] = empty({M, t[i].heads, D}, turns->options().dtype(at::kBFloat16));
            t[i].y = out[i].data_ptr();
        }
        const float magnitude = (float)PyFloat_AS_DOUBLE(a[5]);
        const int inverse = a[4] == Py_True, rot = 2 * (int)turns->size(0);
        const void *pp = positions->data_ptr(), *pt = turns->data_ptr();
        void* st = current_stream();
        if (many) {
            res = PyList_New(count);
            for (Py_ssize_t i = 0; i < count && res; ++i) {
                PyObject* v = THPVariable_Wrap(std::move(out[i]));
                if (v) PyList_SET_ITEM(res, i, v);
                else Py_CLEAR(res);
            }
        } else {
            res = THPVariable_Wrap(std::move(out[0]));
        }
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_rope((int)count, t, (int)M, (int)D, rot, layout, pp, pt, magnitude, inverse, st);
        }
        return done(status, res);
    } catch (...) {
        Py_XDECREF(res);
        return none();
    }
}

// vocab_loss(h, W, targets, weights, grad, workspace) -> (loss, lse, dH or None)
PyObject* vocab_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return none();
    try {
        if (modes()) return none();
        const at::Tensor *h = plain(a[0], at::kBFloat16), *W = plain(a[1], at::kBFloat16), *targets = plain(a[2], at::kInt), *ws = plain(a[5], at::kByte);
        const at::Tensor* weights = a[3] == Py_None ? nullptr : plain(a[3], at::kFloat);
        if (!h || !W || !targets || !ws || (!weights && a[3] != Py_None) || !PyBool_Check(a[4]) || h->dim() != 2 || W->dim() != 2 || !here(*h)) return none();
        const int64_t M = h->size(0), K = h->size(1), V = W->size(0);
        if (M > INT32_MAX || K > INT32_MAX || V > INT32_MAX || W->size(1) != K || targets->dim() != 1 || targets->size(0) != M) return none();
        if (weights && (weights->dim() != 1 || weights->size(0) != M)) return none();
        for (const at::Tensor* t : {targets, weights})
            if (t && (reinterpret_cast<uintptr_t>(t->data_ptr()) & 15u)) return none();      // lowra.py copies it
        for (const at::Tensor* t : {W, targets, ws, weights})
            if (t && t->device() != h->device()) return none();
        const bool want[3] = {true, true, a[4] == Py_True};
        at::Tensor out[3];
        out[0] = empty({M}, h->options().dtype(at::kFloat));
        out[1] = empty({M}, h->options().dtype(at::kFloat));
        if (want[2]) out[2] = empty({M, K}, h->options());
        const void *ph = h->data_ptr(), *pw = W->data_ptr(), *pt = targets->data_ptr(), *pf = weights ? weights->data_ptr() : nullptr;
        void *p0 = out[0].data_ptr(), *p1 = out[1].data_ptr(), *p2 = want[2] ? out[2].data_ptr() : nullptr, *wp = ws->data_ptr(), *st = current_stream();
        const size_t ws_bytes = (size_t)ws->numel();
        PyObject* res = tuple_of(out, want);
        if (!res) return none();
        int status;
        {
            Unlocked u;
            status = lib_vocab_loss((int)M, (int)V, (int)K, ph, pw, pt, pf, p0, p1, p2, wp, ws_bytes, st);
        }
        return done(status, res);
    } catch (...) {
        return none();
    }
}

// init_step(addresses): those of the operators beside the linear
PyObject* init_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "init_step: four addresses"); return nullptr; }
    void* f[4];
    for (int i = 0; i < 4; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    lib_norm_fwd = (norm_fwd_fn)f[0]; lib_norm_bwd = (norm_bwd_fn)f[1]; lib_rope = (rope_fn)f[2]; lib_vocab_loss = (vocab_loss_fn)f[3];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)())init, METH_FASTCALL, nullptr},
                         {"init_act", (PyCFunction)(void (*)())init_act, METH_FASTCALL, nullptr},
                         {"linear_act", (PyCFunction)(void (*)())linear_act, METH_FASTCALL, nullptr},
                         {"act_bwd", (PyCFunction)(void (*)())act_bwd, METH_FASTCALL, nullptr},
                         {"init_step", (PyCFunction)(void (*)())init_step, METH_FASTCALL, nullptr},
                         {"norm_fwd", (PyCFunction)(void (*)())norm_fwd, METH_FASTCALL, nullptr},
                         {"norm_bwd", (PyCFunction)(void (*)())norm_bwd, METH_FASTCALL, nullptr},
                         {"rope", (PyCFunction)(void (*)())rope, METH_FASTCALL, nullptr},
                         {"vocab_loss", (PyCFunction)(void (*)())vocab_loss, METH_FASTCALL, nullptr},
                         {"linear", (PyCFunction)(void (*)())linear, METH_FASTCALL, nullptr},
                         {"side_product", (PyCFunction)(void (*)())side_product, METH_FASTCALL, nullptr},
                         {"grads", (PyCFunction)(void (*)())grads, METH_FASTCALL, nullptr},
                         {"grads_from_side", (PyCFunction)(void (*)())grads_from_side, METH_FASTCALL, nullptr},
                         {"dequantize", (PyCFunction)(void (*)())dequantize, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lowra_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lowra_call() { return PyModule_Create(&module); }
