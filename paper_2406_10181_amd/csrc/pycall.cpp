// CPython module `_call`: argument marshalling for the entry points a training program calls in every step.
//
// The binding's general path (ctypes) converts a dozen arguments at about 0.1 us each besides the Python code that
// collects them: 2.2 us for lsp_compress_planned and 2.6 us for lsp_decompress_apply, a fifth of what enqueuing a small
// problem's kernels costs.  Here it is 0.7 and 1.1 us.  Nothing else happens in this file; the functions called are those of the
// C ABI, whose addresses the binding hands over once (bind), so this module links against nothing but Python.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "lsp.h"

namespace {

PyObject* g_data_ptr;      // interned names
PyObject* g_cuda_stream;
PyObject* g_ctypes;
PyObject* g_data;
PyObject* g_argument_error;   // ctypes.ArgumentError

decltype(&lsp_compress_planned) g_compress_planned;
decltype(&lsp_decompress_apply) g_decompress_apply;
decltype(&lsp_compress_planned_grouped) g_compress_grouped;
decltype(&lsp_decompress_apply_grouped) g_apply_grouped;
decltype(&lsp_dropout) g_dropout;
decltype(&lsp_attention_forward) g_attention_forward;
decltype(&lsp_attention_backward) g_attention_backward;
decltype(&lsp_residual_norm_forward) g_norm_forward;
decltype(&lsp_residual_norm_backward) g_norm_backward;

PyObject* g_shape;
PyObject* g_stride;
PyObject* g_dtype;
PyObject* g_get_device;
PyObject* g_types[3];         // torch's types, in the order of lsp_dtype; from the first descriptor on

// Converts one argument after another, to what ctypes makes of it; the first failure leaves a Python exception and ok = false.
struct Args {
    PyObject* const* first;
    PyObject* const* a = first;
    bool ok = true;

    explicit Args(PyObject* const* args) : first(args) {}
    void refuse() {                                    // the argument before `a`
        PyErr_Format(g_argument_error, "argument %zd: TypeError: wrong type", (Py_ssize_t)(a - first));
        ok = false;
    }
    // the low bits of an integer, however large: a value that makes no sense is the library's to refuse
    uint64_t integer() {
        PyObject* x = *a++;
        if (!ok) return 0;
        const uint64_t v = PyLong_AsUnsignedLongLongMask(x);
        if (v == (uint64_t)-1 && PyErr_Occurred()) { PyErr_Clear(); refuse(); }
        return v;
    }
    int64_t int64() { return (int64_t)integer(); }
    int32_t int32() { return (int32_t)integer(); }
    // address held by a Python int (None: NULL), and gives the reference up
    void* taken(PyObject* i) {
        if (!i) { ok = false; return nullptr; }
        void* p = nullptr;
        if (PyLong_Check(i)) p = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLongMask(i));
        else if (i != Py_None) refuse();
        Py_DECREF(i);
        return p;
    }
    // a tensor, a numpy array, an address or None
    void* pointer() {
        PyObject* x = *a++;
        if (!ok || x == Py_None) return nullptr;
        if (PyLong_Check(x)) { Py_INCREF(x); return taken(x); }
        PyObject* i = PyObject_CallMethodNoArgs(x, g_data_ptr);
        if (!i && PyErr_ExceptionMatches(PyExc_AttributeError)) {
            PyErr_Clear();
            if (PyObject* c = PyObject_GetAttr(x, g_ctypes)) {
                i = PyObject_GetAttr(c, g_data);
                Py_DECREF(c);
            } else if (PyErr_ExceptionMatches(PyExc_AttributeError)) {
                PyErr_Format(PyExc_TypeError, "cannot take the address of %R", (PyObject*)Py_TYPE(x));
            }
        }
        return taken(i);
    }
    // a torch stream, an address or None
    void* stream() {
        PyObject* x = *a++;
        if (!ok || x == Py_None) return nullptr;
        if (PyLong_Check(x)) { Py_INCREF(x); return taken(x); }
        return taken(PyObject_GetAttr(x, g_cuda_stream));
    }
};

bool count_is(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", have, want);
    return false;
}

template <typename F> PyObject* without_gil(F&& call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (G, plan, m, n, r, d, S, dtype, workspace, workspace_bytes, stream)
PyObject* compress_planned(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 11)) return nullptr;
    Args a(args);
    const void* G = a.pointer(); const void* plan = a.pointer();
    const int64_t m = a.int64(), n = a.int64();
    const int32_t r = a.int32(), d = a.int32();
    float* S = static_cast<float*>(a.pointer());
    const int32_t dtype = a.int32();
    void* ws = a.pointer();
    const size_t bytes = a.integer();
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return g_compress_planned(G, plan, m, n, r, d, S, static_cast<lsp_dtype>(dtype), ws, bytes, st); });
}

// (W, S, P_idx, P_val, Q_idx, Q_val, m, n, r, d, dtype, stream)
PyObject* decompress_apply(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 12)) return nullptr;
    Args a(args);
    void* W = a.pointer();
    const float* S = static_cast<const float*>(a.pointer());
    const int32_t* P_idx = static_cast<const int32_t*>(a.pointer());
    const float* P_val = static_cast<const float*>(a.pointer());
    const int32_t* Q_idx = static_cast<const int32_t*>(a.pointer());
    const float* Q_val = static_cast<const float*>(a.pointer());
    const int64_t m = a.int64(), n = a.int64();
    const int32_t r = a.int32(), d = a.int32(), dtype = a.int32();
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return g_decompress_apply(W, S, P_idx, P_val, Q_idx, Q_val, m, n, r, d, static_cast<lsp_dtype>(dtype), st); });
}

// (address of the items, count, r, d, dtype, stream)
template <typename Item, typename Entry> PyObject* grouped(Entry entry, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 6)) return nullptr;
    Args a(args);
    const Item* items = static_cast<const Item*>(a.pointer());
    const int32_t count = a.int32(), r = a.int32(), d = a.int32(), dtype = a.int32();
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return entry(items, count, r, d, static_cast<lsp_dtype>(dtype), st); });
}
PyObject* compress_planned_grouped(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return grouped<lsp_compress_item>(g_compress_grouped, args, nargs); }
PyObject* decompress_apply_grouped(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return grouped<lsp_apply_item>(g_apply_grouped, args, nargs); }

// (addresses of the four functions, in the order of the methods)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 4)) return nullptr;
    Args a(args);
    void* p[4];
    for (void*& x : p) x = a.pointer();
    if (!a.ok) return nullptr;
    g_compress_planned = reinterpret_cast<decltype(g_compress_planned)>(p[0]);
    g_decompress_apply = reinterpret_cast<decltype(g_decompress_apply)>(p[1]);
    g_compress_grouped = reinterpret_cast<decltype(g_compress_grouped)>(p[2]);
    g_apply_grouped = reinterpret_cast<decltype(g_apply_grouped)>(p[3]);
    Py_RETURN_NONE;
}

// The training operators.  Their descriptors are C structures that the binding has as ctypes objects; here they are filled from torch tensors (7.7 us for the
// residual norm's in Python, 3.7 here with three vectors; attention's 4.2, with lengths 4.5), with the checks that only the tensors allow: shapes, types and devices that belong
// together, contiguous last axes.

// What a tensor says of itself; false with a Python exception set
struct Tensor {
    void* data = nullptr;
    int64_t shape[4] = {}, stride[4] = {};
    PyObject* dtype = nullptr;                         // borrowed: torch's types live as long as torch

    bool numbers(PyObject* tuple, int dims, int64_t* to, const char* what) {
        const bool ok = tuple && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == dims;
        for (int k = 0; ok && k < dims; ++k) to[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, k));
        Py_XDECREF(tuple);
        if (!ok && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: tensors of %d axes are wanted", what, dims);
        return ok && !PyErr_Occurred();
    }
    bool read(PyObject* t, int dims, const char* what) {
        if (!numbers(PyObject_GetAttr(t, g_shape), dims, shape, what)) return false;
        if (!numbers(PyObject_CallMethodNoArgs(t, g_stride), dims, stride, what)) return false;
        PyObject* type = PyObject_GetAttr(t, g_dtype);
        PyObject* at = type ? PyObject_CallMethodNoArgs(t, g_data_ptr) : nullptr;
        if (!at) { Py_XDECREF(type); return false; }
        dtype = type;
        Py_DECREF(type);
        data = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLongMask(at));
        Py_DECREF(at);
        if (PyErr_Occurred()) return false;
        if (stride[dims - 1] != 1 && shape[dims - 1] != 1) { PyErr_Format(PyExc_ValueError, "%s: the last axis must be contiguous", what); return false; }
        return true;
    }
    bool same_shape(const Tensor& o) const { return shape[0] == o.shape[0] && shape[1] == o.shape[1] && shape[2] == o.shape[2] && shape[3] == o.shape[3]; }
};

// The device that a tensor is on, -1: the host; false with a Python exception set
bool device_of(PyObject* t, long& device) {
    PyObject* where = PyObject_CallMethodNoArgs(t, g_get_device);
    if (!where) return false;
    device = PyLong_AsLong(where);
    Py_DECREF(where);
    return !PyErr_Occurred();
}

PyObject* refuse(const char* text) {
    PyErr_SetString(PyExc_ValueError, text);
    return nullptr;
}

bool know_types() {
    if (g_types[0]) return true;
    PyObject* torch = PyImport_ImportModule("torch");
    if (!torch) return false;
    const char* names[3] = {"float32", "float16", "bfloat16"};
    for (int i = 2; i >= 0; --i) if (!(g_types[i] = PyObject_GetAttrString(torch, names[i]))) break;
    Py_DECREF(torch);
    return g_types[0] != nullptr;
}
// An lsp_dtype, or -1
int type_code(const PyObject* dtype) {
    for (int i = 0; i < 3; ++i) if (dtype == g_types[i]) return i;
    return -1;
}

// A size as the C structures have it; 0, which the library refuses, where it has no room there
int32_t size32(int64_t n) { return n > INT32_MAX ? 0 : (int32_t)n; }

float number(PyObject* x, bool& ok) {
    const double v = PyFloat_AsDouble(x);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return (float)v;
}

// What a descriptor made here remembers beside the C structure, so that the call can compare it with its other arguments: the binding's objects have these
// fields behind the structure's own.
struct AttentionOfTensors { lsp_attention_problem p; int32_t dtype; };
struct AttentionGradientsOfTensors { lsp_attention_gradients g; int64_t q_shape[4], k_shape[4]; int32_t dtype; };
struct ResidualNormOfTensors { lsp_residual_norm_problem p; int32_t dtype; };
struct ResidualNormGradientsOfTensors { lsp_residual_norm_gradients g; int64_t rows, width; int32_t dtype; };

bool matches(const AttentionOfTensors& a, const AttentionGradientsOfTensors& b) {
    const int64_t q[4] = {a.p.batch, a.p.q_len, a.p.heads, a.p.head_dim}, k[4] = {a.p.batch, a.p.k_len, a.p.kv_heads, a.p.head_dim};
    for (int i = 0; i < 4; ++i) if (q[i] != b.q_shape[i] || k[i] != b.k_shape[i]) return false;
    return true;
}
bool matches(const ResidualNormOfTensors& a, const ResidualNormGradientsOfTensors& b) { return a.p.rows == b.rows && a.p.width == b.width; }

// (address of the binding's attention_problem, Q, K, V, O, L, q_lens, k_lens, scale, causal, dropout, seed, offset)
PyObject* attention_problem(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 13)) return nullptr;
    const char* what = "attention_problem";
    Args head(args);
    auto* d = static_cast<AttentionOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor q, k, v, o, l;
    if (!q.read(args[1], 4, what) || !k.read(args[2], 4, what) || !v.read(args[3], 4, what) || !o.read(args[4], 4, what) || !l.read(args[5], 3, what)) return nullptr;
    if (!k.same_shape(v) || !q.same_shape(o) || k.shape[0] != q.shape[0] || k.shape[3] != q.shape[3] || l.shape[0] != q.shape[0] || l.shape[1] != q.shape[2] ||
        l.shape[2] != q.shape[1] || (l.shape[1] != 1 && l.stride[1] != l.shape[2]) || (l.shape[0] != 1 && l.stride[0] != l.shape[1] * l.shape[2]))
        return refuse("attention_problem: Q, O [batch][q_len][heads][head_dim], K, V [batch][k_len][kv_heads][head_dim] and a contiguous L [batch][heads][q_len] are wanted");
    if (type_code(q.dtype) < 0 || k.dtype != q.dtype || v.dtype != q.dtype || o.dtype != q.dtype) return refuse("attention_problem: Q, K, V and O are of one type, float32, float16 or bfloat16");
    if (type_code(l.dtype) != LSP_F32) return refuse("attention_problem: L is float32");
    void* lens[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
        if (args[6 + i] == Py_None) continue;
        Tensor n;
        if (!n.read(args[6 + i], 1, what)) return nullptr;
        if (n.shape[0] != q.shape[0]) return refuse("attention_problem: lengths are [batch]");
        long there, here;                              // (the one operand that a program may well have on the host, where the kernels must not read it)
        if (!device_of(args[6 + i], there) || !device_of(args[1], here)) return nullptr;
        if (there != here) return refuse("attention_problem: lengths are on the device of the other tensors");
        lens[i] = n.data;
    }
    Args tail(args + 9);
    bool ok = true;
    const float scale = number(args[8], ok), dropout = number(args[10], ok);
    if (!ok) return nullptr;
    const int32_t causal = PyObject_IsTrue(*tail.a++);
    ++tail.a;                                          // (dropout)
    const uint64_t seed = tail.integer();
    const uint32_t offset = (uint32_t)tail.integer();
    if (!tail.ok || PyErr_Occurred()) return nullptr;
    d->dtype = type_code(q.dtype);
    d->p = lsp_attention_problem{q.data, k.data, v.data, o.data, static_cast<float*>(l.data), static_cast<const int32_t*>(lens[0]), static_cast<const int32_t*>(lens[1]),
                               {q.stride[0], q.stride[1], q.stride[2]}, {k.stride[0], k.stride[1], k.stride[2]}, {v.stride[0], v.stride[1], v.stride[2]}, {o.stride[0], o.stride[1], o.stride[2]},
                               size32(q.shape[0]), size32(q.shape[2]), size32(k.shape[2]), size32(q.shape[1]), size32(k.shape[1]), size32(q.shape[3]), causal, scale, dropout, offset, seed};
    Py_RETURN_NONE;
}

// (address of the binding's attention_gradients, dO, dQ, dK, dV)
PyObject* attention_gradients(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    Args head(args);
    auto* d = static_cast<AttentionGradientsOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor t[4];
    for (int i = 0; i < 4; ++i) if (!t[i].read(args[1 + i], 4, "attention_gradients")) return nullptr;
    if (!t[0].same_shape(t[1]) || !t[2].same_shape(t[3])) return refuse("attention_gradients: dO and dQ, and dK and dV, are of one shape");
    for (const Tensor& x : t) if (type_code(x.dtype) < 0 || x.dtype != t[0].dtype) return refuse("attention_gradients: dO, dQ, dK and dV are of one type, float32, float16 or bfloat16");
    for (int i = 0; i < 4; ++i) { d->q_shape[i] = t[1].shape[i]; d->k_shape[i] = t[2].shape[i]; }
    d->dtype = type_code(t[0].dtype);
    d->g = lsp_attention_gradients{t[0].data, t[1].data, t[2].data, t[3].data, {t[0].stride[0], t[0].stride[1], t[0].stride[2]}, {t[1].stride[0], t[1].stride[1], t[1].stride[2]},
                                 {t[2].stride[0], t[2].stride[1], t[2].stride[2]}, {t[3].stride[0], t[3].stride[1], t[3].stride[2]}};
    Py_RETURN_NONE;
}

// A [width] vector of type `dtype`, or None
bool vector(PyObject* t, int64_t width, const PyObject* dtype, void*& to, const char* what) {
    to = nullptr;
    if (t == Py_None) return true;
    Tensor v;
    if (!v.read(t, 1, what)) return false;
    if (v.shape[0] != width || v.dtype != dtype) { PyErr_Format(PyExc_ValueError, "%s: weights, biases and gate are [width], of the type of x, and their gradients float32", what); return false; }
    to = v.data;
    return true;
}

// (address of the binding's residual_norm_problem, x, f, y, h, stats, post_weight, post_bias, gate, pre_weight, pre_bias, post, pre, eps, residual_scale, branch_scale, dropout, seed, offset)
PyObject* residual_norm_problem(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 19)) return nullptr;
    const char* what = "residual_norm_problem";
    Args head(args);
    auto* d = static_cast<ResidualNormOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor x, f, y, h, stats;
    if (!x.read(args[1], 2, what) || !f.read(args[2], 2, what) || !y.read(args[3], 2, what) || (args[4] != Py_None && !h.read(args[4], 2, what)) || !stats.read(args[5], 2, what)) return nullptr;
    if (type_code(x.dtype) < 0 || !f.same_shape(x) || !y.same_shape(x) || f.dtype != x.dtype || y.dtype != x.dtype || (h.dtype && (!h.same_shape(x) || h.dtype != x.dtype)))
        return refuse("residual_norm_problem: x, f, y and h are of one shape and type, float32, float16 or bfloat16");
    if (type_code(stats.dtype) != LSP_F32 || stats.shape[0] != 4 || stats.shape[1] != x.shape[0] || stats.stride[0] != stats.shape[1])
        return refuse("residual_norm_problem: stats are [4][rows], float32");
    void* v[5];
    for (int i = 0; i < 5; ++i) if (!vector(args[6 + i], x.shape[1], x.dtype, v[i], what)) return nullptr;
    Args kinds(args + 11), tail(args + 17);
    const int32_t post = kinds.int32(), pre = kinds.int32();
    bool ok = kinds.ok;
    float n[4];
    for (int i = 0; ok && i < 4; ++i) n[i] = number(args[13 + i], ok);
    const uint64_t seed = tail.integer();
    const uint32_t offset = (uint32_t)tail.integer();
    if (!ok || !tail.ok) return nullptr;
    d->dtype = type_code(x.dtype);
    d->p = lsp_residual_norm_problem{x.data, f.data, y.data, h.data, static_cast<float*>(stats.data), v[0], v[1], v[2], v[3], v[4], x.stride[0], f.stride[0], y.stride[0], h.stride[0],
                                   x.shape[0], size32(x.shape[1]), post, pre, n[0], n[1], n[2], n[3], offset, seed};
    Py_RETURN_NONE;
}

// (address of the binding's residual_norm_gradients, dy, dh, dx, df, post_weight, post_bias, gate, pre_weight, pre_bias)
PyObject* residual_norm_gradients(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 10)) return nullptr;
    const char* what = "residual_norm_gradients";
    Args head(args);
    auto* d = static_cast<ResidualNormGradientsOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor t[4];
    for (int i = 0; i < 4; ++i) if ((i != 1 || args[2] != Py_None) && !t[i].read(args[1 + i], 2, what)) return nullptr;
    for (int i = 0; i < 4; ++i)
        if (t[i].dtype && (!t[i].same_shape(t[0]) || t[i].dtype != t[0].dtype || type_code(t[i].dtype) < 0))
            return refuse("residual_norm_gradients: dy, dh, dx and df are of one shape and type, float32, float16 or bfloat16");
    void* v[5];
    for (int i = 0; i < 5; ++i) if (!vector(args[5 + i], t[0].shape[1], g_types[LSP_F32], v[i], what)) return nullptr;
    d->rows = t[0].shape[0]; d->width = t[0].shape[1]; d->dtype = type_code(t[0].dtype);
    d->g = lsp_residual_norm_gradients{t[0].data, t[1].data, t[2].data, t[3].data, static_cast<float*>(v[0]), static_cast<float*>(v[1]), static_cast<float*>(v[2]), static_cast<float*>(v[3]),
                                     static_cast<float*>(v[4]), t[0].stride[0], t[1].stride[0], t[2].stride[0], t[3].stride[0]};
    Py_RETURN_NONE;
}

// (x, y, rows, width, dropout, seed, offset, dtype, stream)
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a(args);
    const void* x = a.pointer(); void* y = a.pointer();
    const int64_t rows = a.int64(), width = a.int64();
    bool ok = a.ok;
    const float p = ok ? number(*a.a++, ok) : 0.0f;
    if (!ok) return nullptr;
    const uint64_t seed = a.integer();
    const uint32_t offset = (uint32_t)a.integer();
    const int32_t dtype = a.int32();
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return g_dropout(x, y, rows, width, p, seed, offset, static_cast<lsp_dtype>(dtype), st); });
}

// The binding's classes of descriptors: those of the C structures and, derived from these, those that are made of tensors
enum Kind { ATTENTION, ATTENTION_GRADIENTS, RESIDUAL_NORM, RESIDUAL_NORM_GRADIENTS };
PyTypeObject* g_base[4];
PyTypeObject* g_of_tensors[4];

// A descriptor as it is given, made by hand or of tensors; None: NULL
template <Kind KIND, typename Base, typename OfTensors> struct Given {
    const Base* p = nullptr;
    const OfTensors* of_tensors = nullptr;
    bool take(PyObject* x) {
        if (x == Py_None) return true;
        if (!PyObject_TypeCheck(x, g_base[KIND])) { PyErr_Format(PyExc_TypeError, "a descriptor of class %s is wanted", g_base[KIND]->tp_name); return false; }
        Py_buffer v;
        if (PyObject_GetBuffer(x, &v, PyBUF_SIMPLE) < 0) return false;
        p = static_cast<const Base*>(v.buf);
        if (PyObject_TypeCheck(x, g_of_tensors[KIND])) of_tensors = static_cast<const OfTensors*>(v.buf);
        PyBuffer_Release(&v);                          // (the object stays the caller's during the call)
        return true;
    }
    bool is_of(int32_t dtype) const {
        if (!of_tensors || of_tensors->dtype == dtype) return true;
        refuse("the descriptor's tensors are of another type than the call's");
        return false;
    }
};
using GivenAttention = Given<ATTENTION, lsp_attention_problem, AttentionOfTensors>;
using GivenAttentionGradients = Given<ATTENTION_GRADIENTS, lsp_attention_gradients, AttentionGradientsOfTensors>;
using GivenResidualNorm = Given<RESIDUAL_NORM, lsp_residual_norm_problem, ResidualNormOfTensors>;
using GivenResidualNormGradients = Given<RESIDUAL_NORM_GRADIENTS, lsp_residual_norm_gradients, ResidualNormGradientsOfTensors>;

// (problem, dtype, ...)
template <typename P> bool problem_of(Args& a, P& p, int32_t& dtype) {
    if (!p.take(*a.a++)) return false;
    dtype = a.int32();
    return a.ok && p.is_of(dtype);
}

// (problem, dtype, workspace, workspace_bytes, stream)
PyObject* attention_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    Args a(args);
    GivenAttention p;
    int32_t dtype;
    if (!problem_of(a, p, dtype)) return nullptr;
    void* ws = a.pointer();
    const size_t bytes = a.integer();
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return g_attention_forward(p.p, static_cast<lsp_dtype>(dtype), ws, bytes, st); });
}
// (problem, gradients, dtype, workspace, workspace_bytes, stream)
template <typename Problem, typename Gradients, typename Entry> PyObject* backward(Entry entry, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 6)) return nullptr;
    Args a(args);
    Problem p;
    Gradients g;
    if (!p.take(*a.a++) || !g.take(*a.a++)) return nullptr;
    const int32_t dtype = a.int32();
    void* ws = a.pointer();
    const size_t bytes = a.integer();
    void* st = a.stream();
    if (!a.ok || !p.is_of(dtype) || !g.is_of(dtype)) return nullptr;
    if (p.of_tensors && g.of_tensors && !matches(*p.of_tensors, *g.of_tensors)) return refuse("the gradients are of other shapes than the problem's tensors");
    return without_gil([&] { return entry(p.p, g.p, static_cast<lsp_dtype>(dtype), ws, bytes, st); });
}
PyObject* attention_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return backward<GivenAttention, GivenAttentionGradients>(g_attention_backward, args, nargs);
}
PyObject* residual_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return backward<GivenResidualNorm, GivenResidualNormGradients>(g_norm_backward, args, nargs);
}
// (problem, dtype, stream)
PyObject* residual_norm_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 3)) return nullptr;
    Args a(args);
    GivenResidualNorm p;
    int32_t dtype;
    if (!problem_of(a, p, dtype)) return nullptr;
    void* st = a.stream();
    if (!a.ok) return nullptr;
    return without_gil([&] { return g_norm_forward(p.p, static_cast<lsp_dtype>(dtype), st); });
}

// (addresses of lsp_dropout, lsp_attention_forward, lsp_attention_backward, lsp_residual_norm_forward, lsp_residual_norm_backward; the classes of the four C structures, in
// the order of Kind, and those of descriptors made of tensors)
PyObject* bind_operators(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 13)) return nullptr;
    Args a(args);
    void* p[5];
    for (void*& x : p) x = a.pointer();
    if (!a.ok) return nullptr;
    for (int i = 5; i < 13; ++i) if (!PyType_Check(args[i])) return refuse("bind_operators: classes are wanted");
    for (int i = 0; i < 4; ++i) {
        Py_INCREF(args[5 + i]); Py_INCREF(args[9 + i]);                    // (kept as long as the module is)
        g_base[i] = reinterpret_cast<PyTypeObject*>(args[5 + i]);
        g_of_tensors[i] = reinterpret_cast<PyTypeObject*>(args[9 + i]);
    }
    g_dropout = reinterpret_cast<decltype(g_dropout)>(p[0]);
    g_attention_forward = reinterpret_cast<decltype(g_attention_forward)>(p[1]);
    g_attention_backward = reinterpret_cast<decltype(g_attention_backward)>(p[2]);
    g_norm_forward = reinterpret_cast<decltype(g_norm_forward)>(p[3]);
    g_norm_backward = reinterpret_cast<decltype(g_norm_backward)>(p[4]);
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {
    method<compress_planned>("compress_planned"), method<decompress_apply>("decompress_apply"),
    method<compress_planned_grouped>("compress_planned_grouped"), method<decompress_apply_grouped>("decompress_apply_grouped"),
    method<bind>("bind"),
    method<attention_problem>("attention_problem"), method<attention_gradients>("attention_gradients"),
    method<residual_norm_problem>("residual_norm_problem"), method<residual_norm_gradients>("residual_norm_gradients"),
    method<dropout>("dropout"), method<attention_forward>("attention_forward"), method<attention_backward>("attention_backward"),
    method<residual_norm_forward>("residual_norm_forward"), method<residual_norm_backward>("residual_norm_backward"),
    method<bind_operators>("bind_operators"), {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_call", "Argument marshalling of the per-step entry points.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) {
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    g_ctypes = PyUnicode_InternFromString("ctypes");
    g_data = PyUnicode_InternFromString("data");
    g_shape = PyUnicode_InternFromString("shape");
    g_stride = PyUnicode_InternFromString("stride");
    g_dtype = PyUnicode_InternFromString("dtype");
    g_get_device = PyUnicode_InternFromString("get_device");
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    if (!ctypes) return nullptr;
    g_argument_error = PyObject_GetAttrString(ctypes, "ArgumentError");
    Py_DECREF(ctypes);
    if (!g_argument_error) return nullptr;
    return PyModule_Create(&g_module);
}
