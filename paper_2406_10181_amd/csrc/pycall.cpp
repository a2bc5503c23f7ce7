// CPython module `_call`: argument marshalling for the entry points a training program calls in every step.
//
// The binding's general path (ctypes) converts a dozen arguments at about 0.1 us each besides the Python code that
// collects them: 2.2 us for lsp_compress_planned and 2.6 us for lsp_decompress_apply, a fifth of what enqueuing a small
// problem's kernels costs.  Here it is 0.7 and 1.1 us.  Nothing else happens in this file; the functions called are those of the
// C ABI, whose addresses the binding hands over once (bind), so this module links against nothing but Python.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <new>
#include <vector>

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
decltype(&lsp_rotary_forward) g_rotary_forward;
decltype(&lsp_rotary_backward) g_rotary_backward;
decltype(&lsp_cross_entropy_forward) g_loss_forward;
decltype(&lsp_cross_entropy_backward) g_loss_backward;
decltype(&lsp_attention_forward_workspace_bytes) g_attention_forward_bytes, g_attention_backward_bytes;
decltype(&lsp_residual_norm_backward_workspace_bytes) g_norm_backward_bytes;
decltype(&lsp_rotary_backward_workspace_bytes) g_rotary_backward_bytes;
decltype(&lsp_cross_entropy_forward_workspace_bytes) g_loss_forward_bytes, g_loss_backward_bytes;

PyObject* g_shape;
PyObject* g_stride;
PyObject* g_dtype;
PyObject* g_get_device;
PyObject* g_numel;
PyObject* g_is_contiguous;
PyObject* g_element_size;
PyObject* g_item_names[9];
PyObject* g_types[3];         // torch's types, in the order of lsp_dtype; from the first descriptor on
PyObject* g_int32;
PyObject* g_int64;

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

// The device that a tensor is on, -1: the host; false with a Python exception set
bool device_of(PyObject* t, long& device) {
    PyObject* where = PyObject_CallMethodNoArgs(t, g_get_device);
    if (!where) return false;
    device = PyLong_AsLong(where);
    Py_DECREF(where);
    return !PyErr_Occurred();
}

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

PyObject* refuse(const char* text) {
    PyErr_SetString(PyExc_ValueError, text);
    return nullptr;
}

bool know_types() {
    if (g_types[0]) return true;
    PyObject* torch = PyImport_ImportModule("torch");
    if (!torch) return false;
    const char* names[3] = {"float32", "float16", "bfloat16"};
    if (!g_int32) g_int32 = PyObject_GetAttrString(torch, "int32");
    if (!g_int64) g_int64 = PyObject_GetAttrString(torch, "int64");
    if (g_int32 && g_int64)
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

// Whether all tensors of a descriptor (None: passed over) are on one device, and on which: a kernel that follows an address of the host, where caches and lists of lengths may well be, faults.
// False with a Python exception set.  (0.08 us a tensor.)
bool on_one_device(PyObject* const* t, int count, int32_t& device, const char* what) {
    bool any = false;
    for (int i = 0; i < count; ++i) {
        if (t[i] == Py_None) continue;
        long d;
        if (!device_of(t[i], d)) return false;
        if (any && d != device) { PyErr_Format(PyExc_ValueError, "%s: the tensors are on one device", what); return false; }
        device = (int32_t)d;
        any = true;
    }
    return true;
}

// What a descriptor made here remembers beside the C structure, so that the call can compare it with its other arguments: the binding's objects have these
// fields behind the structure's own.
struct AttentionOfTensors { lsp_attention_problem p; int32_t dtype, device; };
struct AttentionGradientsOfTensors { lsp_attention_gradients g; int64_t q_shape[4], k_shape[4]; int32_t dtype, device; };
struct ResidualNormOfTensors { lsp_residual_norm_problem p; int32_t dtype, device; };
struct ResidualNormGradientsOfTensors { lsp_residual_norm_gradients g; int64_t rows, width; int32_t dtype, device; };
struct RotaryOfTensors { lsp_rotary_problem p; int32_t dtype, device; };
struct RotaryGradientsOfTensors { lsp_rotary_gradients g; int64_t q_shape[4], k_shape[4], kr_shape[4]; int32_t dtype, device; };
struct CrossEntropyOfTensors { lsp_cross_entropy_problem p; int32_t dtype, device; };
struct CrossEntropyGradientsOfTensors { lsp_cross_entropy_gradients g; int64_t h_shape[2], w_shape[2], weights; int32_t dtype, device; };

bool matches(const AttentionOfTensors& a, const AttentionGradientsOfTensors& b) {
    const int64_t q[4] = {a.p.batch, a.p.q_len, a.p.heads, a.p.head_dim}, k[4] = {a.p.batch, a.p.k_len, a.p.kv_heads, a.p.head_dim};
    for (int i = 0; i < 4; ++i) if (q[i] != b.q_shape[i] || k[i] != b.k_shape[i]) return false;
    return true;
}
bool matches(const ResidualNormOfTensors& a, const ResidualNormGradientsOfTensors& b) { return a.p.rows == b.rows && a.p.width == b.width; }
bool matches(const RotaryOfTensors& a, const RotaryGradientsOfTensors& b) {
    const int64_t q[4] = {a.p.batch, a.p.length, a.p.heads, a.p.head_dim}, k[4] = {a.p.batch, a.p.length, a.p.kv_heads, a.p.head_dim}, kr[4] = {a.p.batch, a.p.cache, a.p.kv_heads, a.p.head_dim};
    for (int i = 0; i < 4; ++i) if (q[i] != b.q_shape[i] || k[i] != b.k_shape[i] || kr[i] != b.kr_shape[i]) return false;
    return true;
}
bool matches(const CrossEntropyOfTensors& a, const CrossEntropyGradientsOfTensors& b) {      // (-1: not there)
    const bool h = b.h_shape[0] < 0 || (b.h_shape[0] == a.p.rows && b.h_shape[1] == a.p.width), w = b.w_shape[0] < 0 || (b.w_shape[0] == a.p.vocab && b.w_shape[1] == a.p.width);
    return h && w && (b.weights < 0 || b.weights == a.p.rows);
}

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
        lens[i] = n.data;
    }
    if (!on_one_device(args + 1, 7, d->device, what)) return nullptr;
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
    if (!on_one_device(args + 1, 4, d->device, "attention_gradients")) return nullptr;
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
    if (!on_one_device(args + 1, 10, d->device, what)) return nullptr;
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
    if (!on_one_device(args + 1, 9, d->device, what)) return nullptr;
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

// A contiguous tensor of integers of one type, or None
bool whole_numbers(PyObject* t, int dims, const int64_t* shape, const PyObject* dtype, void*& to, const char* what) {
    to = nullptr;
    if (t == Py_None) return true;
    Tensor x;
    if (!x.read(t, dims, what)) return false;
    bool ok = x.dtype == dtype;
    for (int i = 0; ok && i < dims; ++i) ok = x.shape[i] == shape[i];
    if (ok && dims == 2) ok = x.shape[0] == 1 || x.stride[0] == x.shape[1];
    if (!ok) { PyErr_Format(PyExc_ValueError, "%s: positions [batch][length], starts and lens [batch] are int32, targets [rows] int64, all contiguous", what); return false; }
    to = x.data;
    return true;
}

// (address of the binding's rotary_problem, Q, K, V, Qr, Kr, Vr, q_weight, k_weight, q_bias, k_bias, frequencies, positions, starts, lens, neighbours, norm, eps)
PyObject* rotary_problem(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 18)) return nullptr;
    const char* what = "rotary_problem";
    Args head(args);
    auto* d = static_cast<RotaryOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor t[6];                                       // Q, K, V, Qr, Kr, Vr
    for (int i = 0; i < 6; ++i) if ((args[1 + i] != Py_None || i % 3 != 2) && !t[i].read(args[1 + i], 4, what)) return nullptr;
    const Tensor &q = t[0], &k = t[1], &v = t[2], &qr = t[3], &kr = t[4], &vr = t[5];
    if (!qr.same_shape(q) || k.shape[0] != q.shape[0] || k.shape[1] != q.shape[1] || k.shape[3] != q.shape[3] || kr.shape[0] != k.shape[0] || kr.shape[2] != k.shape[2] ||
        kr.shape[3] != k.shape[3] || !v.dtype != !vr.dtype || (v.dtype && (!v.same_shape(k) || !vr.same_shape(kr))))
        return refuse("rotary_problem: Q, Qr [batch][length][heads][head_dim], K [batch][length][kv_heads][head_dim], Kr [batch][cache][kv_heads][head_dim] and, both or neither, V like K and Vr like Kr are wanted");
    for (const Tensor& x : t) if (x.dtype && (x.dtype != q.dtype || type_code(x.dtype) < 0)) return refuse("rotary_problem: all of Q, K, V, Qr, Kr and Vr are of one type, float32, float16 or bfloat16");
    void* w[4];
    for (int i = 0; i < 4; ++i) if (!vector(args[7 + i], q.shape[3], q.dtype, w[i], what)) return nullptr;
    Tensor f;
    if (args[11] != Py_None) {
        if (!f.read(args[11], 1, what)) return nullptr;
        if (type_code(f.dtype) != LSP_F32) return refuse("rotary_problem: frequencies are [rotated / 2], float32");
    }
    void* n[3];
    const int64_t tokens[2] = {q.shape[0], q.shape[1]};
    for (int i = 0; i < 3; ++i) if (!whole_numbers(args[12 + i], i == 0 ? 2 : 1, tokens, g_int32, n[i], what)) return nullptr;
    if (!on_one_device(args + 1, 14, d->device, what)) return nullptr;
    Args tail(args + 15);
    const int32_t neighbours = PyObject_IsTrue(*tail.a++), norm = tail.int32();
    bool ok = tail.ok;
    const float eps = number(args[17], ok);
    if (!ok || PyErr_Occurred()) return nullptr;
    d->dtype = type_code(q.dtype);
    d->p = lsp_rotary_problem{q.data, k.data, v.data, qr.data, kr.data, vr.data, w[0], w[1], w[2], w[3], static_cast<const float*>(f.data), static_cast<const int32_t*>(n[0]),
                              static_cast<const int32_t*>(n[1]), static_cast<const int32_t*>(n[2]),
                              {q.stride[0], q.stride[1], q.stride[2]}, {k.stride[0], k.stride[1], k.stride[2]}, {v.stride[0], v.stride[1], v.stride[2]},
                              {qr.stride[0], qr.stride[1], qr.stride[2]}, {kr.stride[0], kr.stride[1], kr.stride[2]}, {vr.stride[0], vr.stride[1], vr.stride[2]},
                              size32(q.shape[0]), size32(q.shape[1]), size32(kr.shape[1]), size32(q.shape[2]), size32(k.shape[2]), size32(q.shape[3]),
                              f.shape[0] > INT32_MAX / 2 ? -1 : 2 * (int32_t)f.shape[0], neighbours, norm, eps};
    Py_RETURN_NONE;
}

// (address of the binding's rotary_gradients, dQr, dKr, dQ, dK, q_weight, k_weight, q_bias, k_bias)
PyObject* rotary_gradients(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    const char* what = "rotary_gradients";
    Args head(args);
    auto* d = static_cast<RotaryGradientsOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor t[4];
    for (int i = 0; i < 4; ++i) if (!t[i].read(args[1 + i], 4, what)) return nullptr;
    if (!t[0].same_shape(t[2])) return refuse("rotary_gradients: dQr and dQ are of one shape");
    for (const Tensor& x : t) if (type_code(x.dtype) < 0 || x.dtype != t[0].dtype) return refuse("rotary_gradients: dQr, dKr, dQ and dK are of one type, float32, float16 or bfloat16");
    void* w[4];
    for (int i = 0; i < 4; ++i) if (!vector(args[5 + i], t[0].shape[3], g_types[LSP_F32], w[i], what)) return nullptr;
    if (!on_one_device(args + 1, 8, d->device, what)) return nullptr;
    for (int i = 0; i < 4; ++i) { d->q_shape[i] = t[2].shape[i]; d->k_shape[i] = t[3].shape[i]; d->kr_shape[i] = t[1].shape[i]; }
    d->dtype = type_code(t[0].dtype);
    d->g = lsp_rotary_gradients{t[0].data, t[1].data, t[2].data, t[3].data, static_cast<float*>(w[0]), static_cast<float*>(w[1]), static_cast<float*>(w[2]), static_cast<float*>(w[3]),
                                {t[0].stride[0], t[0].stride[1], t[0].stride[2]}, {t[1].stride[0], t[1].stride[1], t[1].stride[2]},
                                {t[2].stride[0], t[2].stride[1], t[2].stride[2]}, {t[3].stride[0], t[3].stride[1], t[3].stride[2]}};
    Py_RETURN_NONE;
}

// A contiguous [count] vector in float32, or None
bool floats(PyObject* t, int64_t count, float*& to, const char* what) {
    to = nullptr;
    if (t == Py_None) return true;
    Tensor x;
    if (!x.read(t, 1, what)) return false;
    if (type_code(x.dtype) != LSP_F32 || (count >= 0 && x.shape[0] != count)) { PyErr_Format(PyExc_ValueError, "%s: losses, logs and weights are [rows], float32", what); return false; }
    to = static_cast<float*>(x.data);
    return true;
}

// (address of the binding's cross_entropy_problem, H, W, targets, losses, logs, smoothing, z_loss)
PyObject* cross_entropy_problem(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 8)) return nullptr;
    const char* what = "cross_entropy_problem";
    Args head(args);
    auto* d = static_cast<CrossEntropyOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor h, w;
    if (!h.read(args[1], 2, what) || !w.read(args[2], 2, what)) return nullptr;
    if (h.shape[1] != w.shape[1] || h.dtype != w.dtype || type_code(h.dtype) < 0) return refuse("cross_entropy_problem: H [rows][width] and W [vocab][width] of one type, float32, float16 or bfloat16, are wanted");
    void* targets;
    float *losses, *logs;
    if (args[3] == Py_None || args[4] == Py_None) return refuse("cross_entropy_problem: targets and losses are wanted");
    if (!whole_numbers(args[3], 1, h.shape, g_int64, targets, what) || !floats(args[4], h.shape[0], losses, what) || !floats(args[5], h.shape[0], logs, what)) return nullptr;
    if (!on_one_device(args + 1, 5, d->device, what)) return nullptr;
    bool ok = true;
    const float smoothing = number(args[6], ok), z_loss = number(args[7], ok);
    if (!ok) return nullptr;
    d->dtype = type_code(h.dtype);
    d->p = lsp_cross_entropy_problem{h.data, w.data, static_cast<const int64_t*>(targets), losses, logs, h.stride[0], w.stride[0], h.shape[0], size32(h.shape[1]), size32(w.shape[0]), smoothing, z_loss};
    Py_RETURN_NONE;
}

// (address of the binding's cross_entropy_gradients, dH, dW, weights, scale)
PyObject* cross_entropy_gradients(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    const char* what = "cross_entropy_gradients";
    Args head(args);
    auto* d = static_cast<CrossEntropyGradientsOfTensors*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    Tensor t[2];
    for (int i = 0; i < 2; ++i) if (args[1 + i] != Py_None && !t[i].read(args[1 + i], 2, what)) return nullptr;
    const PyObject* dtype = t[0].dtype ? t[0].dtype : t[1].dtype;
    if (!dtype) return refuse("cross_entropy_gradients: dH, dW or both are wanted");
    for (const Tensor& x : t) if (x.dtype && (x.dtype != dtype || type_code(x.dtype) < 0)) return refuse("cross_entropy_gradients: dH and dW are of one type, float32, float16 or bfloat16");
    float* weights;
    Tensor n;
    if (args[3] != Py_None && !n.read(args[3], 1, what)) return nullptr;
    if (!floats(args[3], -1, weights, what) || !on_one_device(args + 1, 3, d->device, what)) return nullptr;
    bool ok = true;
    const float scale = number(args[4], ok);
    if (!ok) return nullptr;
    for (int i = 0; i < 2; ++i) { d->h_shape[i] = t[0].dtype ? t[0].shape[i] : -1; d->w_shape[i] = t[1].dtype ? t[1].shape[i] : -1; }
    d->weights = weights ? n.shape[0] : -1;
    d->dtype = type_code(dtype);
    d->g = lsp_cross_entropy_gradients{t[0].data, t[1].data, weights, t[0].stride[0], t[1].stride[0], scale};
    Py_RETURN_NONE;
}

// What a tensor of any shape says of itself; false with a Python exception set
struct Flat {
    PyObject* t = nullptr;                             // borrowed; NULL: None
    uintptr_t data = 0;
    int64_t   count = 0, element = 0;
    PyObject* dtype = nullptr;
    long      device = 0;
    static bool number(PyObject* t, PyObject* name, int64_t& to) {
        PyObject* x = PyObject_CallMethodNoArgs(t, name);
        if (!x) return false;
        to = PyLong_AsLongLong(x);
        Py_DECREF(x);
        return !PyErr_Occurred();
    }
    bool read(PyObject* x) {
        if (!x || x == Py_None) return true;
        t = x;
        PyObject* type = PyObject_GetAttr(x, g_dtype);
        PyObject* at = type ? PyObject_CallMethodNoArgs(x, g_data_ptr) : nullptr;
        if (!at) { Py_XDECREF(type); return false; }
        dtype = type;
        Py_DECREF(type);
        data = (uintptr_t)PyLong_AsUnsignedLongLongMask(at);
        Py_DECREF(at);
        int64_t whole = 0;
        if (PyErr_Occurred() || !number(x, g_numel, count) || !number(x, g_is_contiguous, whole) || !device_of(x, device)) return false;
        const int code = type_code(dtype);
        if (code >= 0) element = code == LSP_F32 ? 4 : 2;
        else if (!number(x, g_element_size, element)) return false;
        if (!whole) { refuse("adamw_items: tensors are contiguous"); return false; }
        return true;
    }
};

PyObject* fill_adamw_items(PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 2)) return nullptr;
    Args head(args);
    auto* to = static_cast<lsp_adamw_item*>(head.pointer());
    if (!head.ok || !know_types()) return nullptr;
    if (!PyList_Check(args[1]) || PyList_GET_SIZE(args[1]) == 0) return refuse("adamw_items: tensors are wanted");
    struct Range { uintptr_t begin, end; bool written; };
    std::vector<Range> ranges;
    int states = -1;
    long device = 0;
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(args[1]); ++i) {
        PyObject* d = PyList_GET_ITEM(args[1], i);
        if (!PyDict_Check(d)) return refuse("adamw_items: a dict for each tensor is wanted");
        PyObject* x[9];
        Py_ssize_t known = 0;
        for (int k = 0; k < 9; ++k) { x[k] = PyDict_GetItem(d, g_item_names[k]); known += x[k] != nullptr; }
        if (known != PyDict_GET_SIZE(d)) return refuse("adamw_items: unknown names");
        Flat f[7];
        for (int k = 0; k < 7; ++k) if (!f[k].read(x[k])) return nullptr;
        const Flat &param = f[0], &grad = f[1], &m = f[2], &v = f[3], &ms = f[4], &vs = f[5], &master = f[6];
        if (!param.t || !grad.t || !m.t || !v.t) return refuse("adamw_items: param, grad, m and v are wanted");
        if (type_code(param.dtype) < 0 || type_code(grad.dtype) < 0) return refuse("adamw_items: param and grad are float32, float16 or bfloat16");
        const bool f32 = m.dtype == g_types[LSP_F32] && v.dtype == g_types[LSP_F32], bits8 = m.element == 1 && v.element == 1;
        if (!f32 && !bits8) return refuse("adamw_items: m and v are both float32 or both of one byte an element");
        if (master.t && master.dtype != g_types[LSP_F32]) return refuse("adamw_items: master is float32");
        if (param.count <= 0 || grad.count != param.count || m.count != param.count || v.count != param.count || (master.t && master.count != param.count))
            return refuse("adamw_items: param, grad, m, v and master are of one size, and not empty");
        const int64_t blocks = (param.count + 255) / 256;
        if (bits8 && (!ms.t || !vs.t || ms.dtype != g_types[LSP_F32] || vs.dtype != g_types[LSP_F32] || ms.count != blocks || vs.count != blocks))
            return refuse("adamw_items: m_scale and v_scale are float32, one for 256 elements");
        if (f32 && (ms.t || vs.t)) return refuse("adamw_items: scales belong to states in 8 bits");
        if (states >= 0 && states != (int)bits8) return refuse("adamw_items: states are all in fp32 or all in 8 bits");
        states = bits8;
        if (i == 0) device = param.device;
        for (int k = 0; k < 7; ++k) {
            if (!f[k].t) continue;
            if (f[k].device != device) return refuse("adamw_items: the tensors are on one device");
            ranges.push_back({f[k].data, f[k].data + (uintptr_t)(f[k].count * f[k].element), k != 1});
        }
        bool ok = true;
        const float factor = x[7] ? number(x[7], ok) : 1.0f, decay = x[8] && ok ? number(x[8], ok) : 0.0f;
        if (!ok) return nullptr;
        to[i] = lsp_adamw_item{(void*)param.data, (const void*)grad.data, (void*)m.data, (void*)v.data, (float*)ms.data, (float*)vs.data, (float*)master.data, param.count, factor, decay,
                               type_code(param.dtype), type_code(grad.dtype)};
    }
    // what is written overlaps nothing (gradients may overlap one another)
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t written = 0, any = 0;
    for (const Range& r : ranges) {
        if (r.begin < (r.written ? any : written)) return refuse("adamw_items: tensors overlap, or one appears twice");
        any = std::max(any, r.end);
        if (r.written) written = std::max(written, r.end);
    }
    return PyLong_FromLong(states);
}
// (address of an array of lsp_adamw_item, list of as many dicts): fills the array, and says which states they are
PyObject* adamw_items(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    try { return fill_adamw_items(args, nargs); }
    catch (const std::bad_alloc&) { return PyErr_NoMemory(); }
}

// The binding's classes of descriptors: those of the C structures and, derived from these, those that are made of tensors
enum Kind { ATTENTION, ATTENTION_GRADIENTS, RESIDUAL_NORM, RESIDUAL_NORM_GRADIENTS, ROTARY, ROTARY_GRADIENTS, CROSS_ENTROPY, CROSS_ENTROPY_GRADIENTS, KINDS };
PyTypeObject* g_base[KINDS];
PyTypeObject* g_of_tensors[KINDS];

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
    bool on_host() const { return of_tensors && of_tensors->device < 0; }
    bool is_of(int32_t dtype) const {
        if (!of_tensors || of_tensors->dtype == dtype) return true;
        refuse("the descriptor's tensors are of another type than the call's");
        return false;
    }
};
// Whether all sizes are there: the library refuses a problem without
bool sizes_are_there(const lsp_attention_problem& p) { return p.batch && p.q_len && p.k_len && p.heads && p.kv_heads && p.head_dim; }
bool sizes_are_there(const lsp_residual_norm_problem& p) { return p.rows && p.width; }
bool sizes_are_there(const lsp_rotary_problem& p) { return p.batch && p.length && p.cache && p.heads && p.kv_heads && p.head_dim; }
bool sizes_are_there(const lsp_cross_entropy_problem& p) { return p.rows && p.width && p.vocab; }
// Whether a call may go to the library as far as devices go: a workspace that is a tensor is where the problem's tensors are, and those are not on the host, but for a call that the library refuses for
// its sizes or its workspace (`need`: bytes of it), with the code that it has for that.  False with a Python exception set.
template <typename Problem> bool may_run(const Problem& p, PyObject* workspace, const void* ws, size_t bytes, size_t need) {
    if (!p.of_tensors) return true;
    const int32_t device = p.of_tensors->device;
    if (device < 0) {
        if (!sizes_are_there(*p.p) || (need && (!ws || bytes < need))) return true;
        refuse("the descriptor's tensors are on the host");
        return false;
    }
    if (!ws || PyLong_Check(workspace)) return true;
    long there;
    if (!device_of(workspace, there)) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
        PyErr_Clear();
        there = -1;                                    // (numpy's)
    }
    if (there != device) { refuse("the workspace is on another device than the descriptor's tensors"); return false; }
    return true;
}
using GivenAttention = Given<ATTENTION, lsp_attention_problem, AttentionOfTensors>;
using GivenAttentionGradients = Given<ATTENTION_GRADIENTS, lsp_attention_gradients, AttentionGradientsOfTensors>;
using GivenResidualNorm = Given<RESIDUAL_NORM, lsp_residual_norm_problem, ResidualNormOfTensors>;
using GivenResidualNormGradients = Given<RESIDUAL_NORM_GRADIENTS, lsp_residual_norm_gradients, ResidualNormGradientsOfTensors>;
using GivenRotary = Given<ROTARY, lsp_rotary_problem, RotaryOfTensors>;
using GivenRotaryGradients = Given<ROTARY_GRADIENTS, lsp_rotary_gradients, RotaryGradientsOfTensors>;
using GivenCrossEntropy = Given<CROSS_ENTROPY, lsp_cross_entropy_problem, CrossEntropyOfTensors>;
using GivenCrossEntropyGradients = Given<CROSS_ENTROPY_GRADIENTS, lsp_cross_entropy_gradients, CrossEntropyGradientsOfTensors>;

// (problem, dtype, ...)
template <typename P> bool problem_of(Args& a, P& p, int32_t& dtype) {
    if (!p.take(*a.a++)) return false;
    dtype = a.int32();
    return a.ok && p.is_of(dtype);
}

// (problem, dtype, workspace, workspace_bytes, stream)
template <typename Problem, typename Entry, typename Query> PyObject* forward(Entry entry, Query query, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    Args a(args);
    Problem p;
    int32_t dtype;
    if (!problem_of(a, p, dtype)) return nullptr;
    void* ws = a.pointer();
    const size_t bytes = a.integer();
    void* st = a.stream();
    if (!a.ok || !may_run(p, args[2], ws, bytes, p.on_host() ? query(p.p, static_cast<lsp_dtype>(dtype)) : 0)) return nullptr;
    return without_gil([&] { return entry(p.p, static_cast<lsp_dtype>(dtype), ws, bytes, st); });
}
PyObject* attention_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return forward<GivenAttention>(g_attention_forward, g_attention_forward_bytes, args, nargs); }
PyObject* cross_entropy_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return forward<GivenCrossEntropy>(g_loss_forward, g_loss_forward_bytes, args, nargs); }
// (problem, gradients, dtype, workspace, workspace_bytes, stream)
template <typename Problem, typename Gradients, typename Entry, typename Query> PyObject* backward(Entry entry, Query query, PyObject* const* args, Py_ssize_t nargs) {
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
    if (p.of_tensors && g.of_tensors && p.of_tensors->device != g.of_tensors->device) return refuse("the gradients are on another device than the problem's tensors");
    if (!may_run(p, args[3], ws, bytes, p.on_host() ? query(p.p, static_cast<lsp_dtype>(dtype)) : 0)) return nullptr;
    return without_gil([&] { return entry(p.p, g.p, static_cast<lsp_dtype>(dtype), ws, bytes, st); });
}
PyObject* attention_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return backward<GivenAttention, GivenAttentionGradients>(g_attention_backward, g_attention_backward_bytes, args, nargs);
}
PyObject* residual_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return backward<GivenResidualNorm, GivenResidualNormGradients>(g_norm_backward, g_norm_backward_bytes, args, nargs);
}
PyObject* rotary_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return backward<GivenRotary, GivenRotaryGradients>(g_rotary_backward, g_rotary_backward_bytes, args, nargs); }
PyObject* cross_entropy_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return backward<GivenCrossEntropy, GivenCrossEntropyGradients>(g_loss_backward, g_loss_backward_bytes, args, nargs);
}
// (problem, dtype, stream)
template <typename Problem, typename Entry> PyObject* forward_alone(Entry entry, PyObject* const* args, Py_ssize_t nargs) {
    if (!count_is(nargs, 3)) return nullptr;
    Args a(args);
    Problem p;
    int32_t dtype;
    if (!problem_of(a, p, dtype)) return nullptr;
    void* st = a.stream();
    if (!a.ok || !may_run(p, Py_None, nullptr, 0, 0)) return nullptr;
    return without_gil([&] { return entry(p.p, static_cast<lsp_dtype>(dtype), st); });
}
PyObject* residual_norm_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return forward_alone<GivenResidualNorm>(g_norm_forward, args, nargs); }
PyObject* rotary_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return forward_alone<GivenRotary>(g_rotary_forward, args, nargs); }

// (addresses of lsp_dropout, lsp_attention_forward, lsp_attention_backward, lsp_residual_norm_forward, lsp_residual_norm_backward, lsp_rotary_forward, lsp_rotary_backward,
// lsp_cross_entropy_forward, lsp_cross_entropy_backward, and of the workspace queries of those that have one, in the same order; the classes of the C structures, in the order of Kind, and those of descriptors made of tensors)
PyObject* bind_operators(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    constexpr int kCalls = 15;
    if (!count_is(nargs, kCalls + 2 * KINDS)) return nullptr;
    Args a(args);
    void* p[kCalls];
    for (void*& x : p) x = a.pointer();
    if (!a.ok) return nullptr;
    for (int i = kCalls; i < kCalls + 2 * KINDS; ++i) if (!PyType_Check(args[i])) return refuse("bind_operators: classes are wanted");
    for (int i = 0; i < KINDS; ++i) {
        Py_INCREF(args[kCalls + i]); Py_INCREF(args[kCalls + KINDS + i]);  // (kept as long as the module is)
        g_base[i] = reinterpret_cast<PyTypeObject*>(args[kCalls + i]);
        g_of_tensors[i] = reinterpret_cast<PyTypeObject*>(args[kCalls + KINDS + i]);
    }
    g_dropout = reinterpret_cast<decltype(g_dropout)>(p[0]);
    g_attention_forward = reinterpret_cast<decltype(g_attention_forward)>(p[1]);
    g_attention_backward = reinterpret_cast<decltype(g_attention_backward)>(p[2]);
    g_norm_forward = reinterpret_cast<decltype(g_norm_forward)>(p[3]);
    g_norm_backward = reinterpret_cast<decltype(g_norm_backward)>(p[4]);
    g_rotary_forward = reinterpret_cast<decltype(g_rotary_forward)>(p[5]);
    g_rotary_backward = reinterpret_cast<decltype(g_rotary_backward)>(p[6]);
    g_loss_forward = reinterpret_cast<decltype(g_loss_forward)>(p[7]);
    g_loss_backward = reinterpret_cast<decltype(g_loss_backward)>(p[8]);
    g_attention_forward_bytes = reinterpret_cast<decltype(g_attention_forward_bytes)>(p[9]);
    g_attention_backward_bytes = reinterpret_cast<decltype(g_attention_backward_bytes)>(p[10]);
    g_norm_backward_bytes = reinterpret_cast<decltype(g_norm_backward_bytes)>(p[11]);
    g_rotary_backward_bytes = reinterpret_cast<decltype(g_rotary_backward_bytes)>(p[12]);
    g_loss_forward_bytes = reinterpret_cast<decltype(g_loss_forward_bytes)>(p[13]);
    g_loss_backward_bytes = reinterpret_cast<decltype(g_loss_backward_bytes)>(p[14]);
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
    method<rotary_problem>("rotary_problem"), method<rotary_gradients>("rotary_gradients"), method<rotary_forward>("rotary_forward"), method<rotary_backward>("rotary_backward"),
    method<cross_entropy_problem>("cross_entropy_problem"), method<cross_entropy_gradients>("cross_entropy_gradients"),
    method<cross_entropy_forward>("cross_entropy_forward"), method<cross_entropy_backward>("cross_entropy_backward"), method<adamw_items>("adamw_items"),
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
    g_numel = PyUnicode_InternFromString("numel");
    g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    g_element_size = PyUnicode_InternFromString("element_size");
    const char* const names[9] = {"param", "grad", "m", "v", "m_scale", "v_scale", "master", "rate_factor", "decay"};
    for (int k = 0; k < 9; ++k) g_item_names[k] = PyUnicode_InternFromString(names[k]);
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    if (!ctypes) return nullptr;
    g_argument_error = PyObject_GetAttrString(ctypes, "ArgumentError");
    Py_DECREF(ctypes);
    if (!g_argument_error) return nullptr;
    return PyModule_Create(&g_module);
}
