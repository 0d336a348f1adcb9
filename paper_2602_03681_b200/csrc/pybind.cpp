// Python entry points of the calls a program makes per token, layer or step: the same names and argument
// order as binding.py's, marshalled natively.  A generation step is a 7-12 us kernel; marshalling its
// twelve tensors through ctypes and asking torch for the current stream in Python took 13-16 us per call and
// set the pace of small batches.  Here a tensor argument is checked (device-resident, contiguous; in the calls of
// speculative generation and of a bounded cache, whose tensors share dimensions, large enough too: NATSL_ERR_SHAPE),
// unwrapped and passed on without an intermediate Python object.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <initializer_list>

#include "../../include/natsl.h"

namespace {

// Arguments of one call, in order; `ok` goes false with a Python error set.
struct Args {
    PyObject *const *v;
    bool ok = true;

    const at::Tensor *tensor(int i) {
        if (!ok) return nullptr;
        if (v[i] == Py_None) return nullptr;
        if (!THPVariable_Check(v[i])) {
            PyErr_Format(PyExc_TypeError, "argument %d: a tensor or None is expected", i);
            ok = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_AssertionError, "device-resident contiguous tensors only");
            ok = false;
            return nullptr;
        }
        return &t;
    }
    template <typename T> T *ptr(int i) {
        const at::Tensor *t = tensor(i);
        return t ? static_cast<T *>(t->data_ptr()) : nullptr;
    }
    size_t numel(int i) {
        const at::Tensor *t = tensor(i);
        return t ? static_cast<size_t>(t->numel()) : 0;
    }
    int64_t size(int i, int dim) {
        const at::Tensor *t = tensor(i);
        if (t && (dim < 0 ? t->dim() < -dim : t->dim() <= dim)) {
            PyErr_Format(PyExc_IndexError, "argument %d: too few dimensions", i);
            ok = false;
        }
        return t && ok ? t->size(dim) : 0;
    }
    long integer(int i) {
        if (!ok) return 0;
        const long x = PyLong_AsLong(v[i]);
        if (x == -1 && PyErr_Occurred()) ok = false;
        return x;
    }
    const natsl_params *params(int i) {      // a ctypes natsl_params, through the buffer protocol
        if (!ok) return nullptr;
        Py_buffer b;
        if (PyObject_GetBuffer(v[i], &b, PyBUF_SIMPLE) != 0) { ok = false; return nullptr; }
        const void *p = b.buf;
        if (b.len != (Py_ssize_t)sizeof(natsl_params)) {
            PyErr_SetString(PyExc_TypeError, "natsl_params expected");
            ok = false;
        }
        PyBuffer_Release(&b);                // (the caller's argument keeps the structure alive)
        return ok ? static_cast<const natsl_params *>(p) : nullptr;
    }
};

// The tensors of a call against its parameters: whether each has room for what the call reads or writes of it, and whether
// those that share a capacity agree on it.  The C call sees addresses alone and would run past their ends.  What is None, or no
// tensor at all, is somebody else's to judge, and so are parameters that the call refuses itself.
struct Room {
    PyObject *const *v;
    const natsl_params *p;
    const size_t esz = p->dtype == NATSL_BF16 ? 2 : 4;
    bool ok = true;

    const at::Tensor *at(int i) const { return THPVariable_Check(v[i]) ? &THPVariable_Unpack(v[i]) : nullptr; }
    Room &has(int i, size_t size, std::initializer_list<int64_t> dims) {
        const at::Tensor *t = at(i);
        double bytes = (double)size;          // (exact up to 2^53; a tensor is far smaller)
        for (int64_t n : dims) bytes *= (double)std::max<int64_t>(n, 0);
        ok = ok && (!t || (double)t->numel() * (double)t->element_size() >= bytes);
        return *this;
    }
    Room &tokens(std::initializer_list<int> list, size_t size) {                  // [B,L,H,d]
        for (int i : list) has(i, size, {p->B, p->L, p->H, p->d});
        return *this;
    }
    Room &heads(std::initializer_list<int> list, size_t size) {                   // [B,L,H]
        for (int i : list) has(i, size, {p->B, p->L, p->H});
        return *this;
    }
    int64_t capacity(int i) const {           // of a cache [B,H,cap,d]; -1: none, and nothing is held against it
        const at::Tensor *t = at(i);
        return t && t->dim() > 2 ? t->size(2) : -1;
    }
    Room &caches(std::initializer_list<int> list, int64_t cap) {
        for (int i : list) {
            const at::Tensor *t = at(i);
            ok = ok && (!t || cap < 0 || (t->dim() == 4 && t->size(2) == cap && t->size(3) == p->d)) && cap <= INT32_MAX;
            has(i, esz, {p->B, p->H, cap, p->d});
        }
        return *this;
    }
    Room &per_entry(int i, int64_t n) {       // [B,H,n] of four bytes
        const at::Tensor *t = at(i);
        ok = ok && (!t || n < 0 || (t->dim() > 0 && t->size(-1) == n));
        return has(i, 4, {p->B, p->H, n});
    }
};

bool current_stream(void **st) {
    try {
        *st = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return false;
    }
}

bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return false;
}

// (the call itself only enqueues work, but may wait for the library's enqueue mutex: without the GIL)
#define NATSL_CALL(expr)                          \
    void *st;                                     \
    if (!a.ok || !current_stream(&st)) return nullptr; \
    int rc;                                       \
    Py_BEGIN_ALLOW_THREADS rc = (expr);           \
    Py_END_ALLOW_THREADS                          \
    return PyLong_FromLong(rc)

PyObject *hybrid_fwd(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 9)) return nullptr;
    Args a{v};
    const void *q = a.ptr<void>(0), *k = a.ptr<void>(1), *vv = a.ptr<void>(2);
    const float *g = a.ptr<float>(3), *beta = a.ptr<float>(4);
    const uint8_t *route = a.ptr<uint8_t>(5);
    void *out = a.ptr<void>(6), *ws = a.ptr<void>(8);
    const natsl_params *p = a.params(7);
    const size_t wb = a.numel(8);
    NATSL_CALL(natsl_hybrid_fwd(q, k, vv, g, beta, route, out, p, ws, wb, st));
}

PyObject *hybrid_fwd_static(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 8)) return nullptr;
    Args a{v};
    const void *q = a.ptr<void>(0), *k = a.ptr<void>(1), *vv = a.ptr<void>(2);
    const float *g = a.ptr<float>(3), *beta = a.ptr<float>(4);
    const uint8_t *route = a.ptr<uint8_t>(5);
    void *out = a.ptr<void>(6);
    const natsl_params *p = a.params(7);
    NATSL_CALL(natsl_hybrid_fwd_static(q, k, vv, g, beta, route, out, p, st));
}

PyObject *hybrid_bwd(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 15)) return nullptr;
    Args a{v};
    const void *q = a.ptr<void>(0), *k = a.ptr<void>(1), *vv = a.ptr<void>(2);
    const float *g = a.ptr<float>(3), *beta = a.ptr<float>(4);
    const uint8_t *route = a.ptr<uint8_t>(5);
    const void *dout = a.ptr<void>(6);
    void *dq = a.ptr<void>(7), *dk = a.ptr<void>(8), *dv = a.ptr<void>(9), *ws = a.ptr<void>(14);
    float *dg = a.ptr<float>(10), *dbeta = a.ptr<float>(11), *dw = a.ptr<float>(12);
    const natsl_params *p = a.params(13);
    const size_t wb = a.numel(14);
    NATSL_CALL(natsl_hybrid_bwd(q, k, vv, g, beta, route, dout, dq, dk, dv, dg, dbeta, dw, p, ws, wb, st));
}

PyObject *decode_step(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 13)) return nullptr;
    Args a{v};
    const void *q = a.ptr<void>(0), *k = a.ptr<void>(1), *vv = a.ptr<void>(2);
    const float *g = a.ptr<float>(3), *beta = a.ptr<float>(4);
    const uint8_t *route = a.ptr<uint8_t>(5);
    float *state = a.ptr<float>(6);
    void *kc = a.ptr<void>(7), *vc = a.ptr<void>(8), *out = a.ptr<void>(10), *ws = a.ptr<void>(12);
    int32_t *len = a.ptr<int32_t>(9);
    const int32_t cap = (int32_t)a.size(7, 2);
    const natsl_params *p = a.params(11);
    const size_t wb = a.numel(12);
    NATSL_CALL(natsl_decode_step(q, k, vv, g, beta, route, state, kc, vc, len, cap, out, p, ws, wb, st));
}

PyObject *decode_block_end(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 8)) return nullptr;
    Args a{v};
    const uint8_t *route = a.ptr<uint8_t>(0);
    const float *g = a.ptr<float>(1);
    float *state = a.ptr<float>(2), *start = a.ptr<float>(3);
    int32_t *len = a.ptr<int32_t>(4);
    const int32_t block_len = (int32_t)a.integer(5);
    const natsl_params *p = a.params(6);
    void *ws = a.ptr<void>(7);
    const size_t wb = a.numel(7);
    NATSL_CALL(natsl_decode_block_end(route, g, state, start, len, block_len, p, ws, wb, st));
}

PyObject *score_layer(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 5)) return nullptr;
    Args a{v};
    const void *x = a.ptr<void>(0);
    const float *w = a.ptr<float>(1);
    float *scores = a.ptr<float>(2);
    uint8_t *route = a.ptr<uint8_t>(3);
    const int32_t d_model = (int32_t)a.size(0, -1);
    const natsl_params *p = a.params(4);
    NATSL_CALL(natsl_score_layer(x, w, scores, route, d_model, p, st));
}

PyObject *tree_step(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 16)) return nullptr;
    Args a{v};
    const natsl_params *p = a.params(14);
    if (!p) return nullptr;
    Room r{v, p};
    r.tokens({0, 1, 2, 12}, r.esz).tokens({13}, 4).heads({3, 4}, 4).heads({5}, 1).has(6, 4, {p->B, p->L}).has(7, 4, {p->B});
    r.has(8, 4, {p->B, p->H, p->d, p->d}).caches({9, 10}, r.capacity(9)).has(11, 4, {p->B, p->H});
    if (!r.ok) return PyLong_FromLong(NATSL_ERR_SHAPE);
    const void *q = a.ptr<void>(0), *k = a.ptr<void>(1), *vv = a.ptr<void>(2);
    const float *g = a.ptr<float>(3), *beta = a.ptr<float>(4);
    const uint8_t *route = a.ptr<uint8_t>(5);
    const int32_t *parent = a.ptr<int32_t>(6), *nodes = a.ptr<int32_t>(7);
    const float *state = a.ptr<float>(8);
    const void *kc = a.ptr<void>(9), *vc = a.ptr<void>(10);
    const int32_t *len = a.ptr<int32_t>(11);
    const int32_t cap = (int32_t)a.size(9, 2);
    void *out = a.ptr<void>(12), *ws = a.ptr<void>(15);
    float *u = a.ptr<float>(13);
    const size_t wb = a.numel(15);
    NATSL_CALL(natsl_tree_step(q, k, vv, g, beta, route, parent, nodes, state, kc, vc, len, cap, out, u, p, ws, wb, st));
}

PyObject *tree_commit(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 13)) return nullptr;
    Args a{v};
    const natsl_params *p = a.params(11);
    if (!p) return nullptr;
    Room r{v, p};
    r.tokens({0, 1}, r.esz).tokens({4}, 4).heads({2}, 4).heads({3}, 1).has(5, 4, {p->B, p->L}).has(6, 4, {p->B});
    r.has(7, 4, {p->B, p->H, p->d, p->d}).caches({8, 9}, r.capacity(8)).has(10, 4, {p->B, p->H});
    if (!r.ok) return PyLong_FromLong(NATSL_ERR_SHAPE);
    const void *k = a.ptr<void>(0), *vv = a.ptr<void>(1);
    const float *g = a.ptr<float>(2);
    const uint8_t *route = a.ptr<uint8_t>(3);
    const float *u = a.ptr<float>(4);
    const int32_t *path = a.ptr<int32_t>(5), *n_path = a.ptr<int32_t>(6);
    float *state = a.ptr<float>(7);
    void *kc = a.ptr<void>(8), *vc = a.ptr<void>(9), *ws = a.ptr<void>(12);
    int32_t *len = a.ptr<int32_t>(10);
    const int32_t cap = (int32_t)a.size(8, 2);
    const size_t wb = a.numel(12);
    NATSL_CALL(natsl_tree_commit(k, vv, g, route, u, path, n_path, state, kc, vc, len, cap, p, ws, wb, st));
}

PyObject *cache_weights(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 7)) return nullptr;
    Args a{v};
    const natsl_params *p = a.params(6);
    if (!p) return nullptr;
    Room r{v, p};
    r.tokens({0}, r.esz).heads({2}, 4).has(1, 4, {p->B, p->H, std::max(p->G, 1), p->L}).caches({3}, r.capacity(3));
    r.has(4, 4, {p->B, p->H}).per_entry(5, r.capacity(3));
    if (!r.ok) return PyLong_FromLong(NATSL_ERR_SHAPE);
    const void *q = a.ptr<void>(0);
    const float *lse = a.ptr<float>(1);
    const int32_t *visible = a.ptr<int32_t>(2);
    const void *kc = a.ptr<void>(3);
    const int32_t *len = a.ptr<int32_t>(4);
    float *weight = a.ptr<float>(5);
    const int32_t cap = (int32_t)a.size(3, 2);
    NATSL_CALL(natsl_cache_weights(q, lse, visible, kc, len, cap, weight, p, st));
}

PyObject *cache_evict(PyObject *, PyObject *const *v, Py_ssize_t n) {
    if (!count_is(n, 9)) return nullptr;
    Args a{v};
    const natsl_params *p = a.params(8);
    if (!p) return nullptr;
    const long keep_as = a.integer(4), first_as = a.integer(5), recent_as = a.integer(6);
    if (!a.ok) return nullptr;
    Room r{v, p};
    r.caches({0, 1}, r.capacity(0)).per_entry(2, r.capacity(0)).has(3, 4, {p->B, p->H}).per_entry(7, keep_as);
    for (long x : {keep_as, first_as, recent_as}) r.ok = r.ok && x >= 0 && x <= INT32_MAX;
    if (!r.ok) return PyLong_FromLong(NATSL_ERR_SHAPE);
    void *kc = a.ptr<void>(0), *vc = a.ptr<void>(1);
    float *weight = a.ptr<float>(2);
    int32_t *len = a.ptr<int32_t>(3);
    const int32_t cap = (int32_t)a.size(0, 2);
    const int32_t keep = (int32_t)keep_as, first = (int32_t)first_as, recent = (int32_t)recent_as;
    int32_t *kept = a.ptr<int32_t>(7);
    NATSL_CALL(natsl_cache_evict(kc, vc, weight, len, cap, keep, first, recent, kept, p, st));
}

PyMethodDef kMethods[] = {
#define NATSL_DEF(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
    NATSL_DEF(hybrid_fwd), NATSL_DEF(hybrid_fwd_static), NATSL_DEF(hybrid_bwd), NATSL_DEF(decode_step),
    NATSL_DEF(decode_block_end), NATSL_DEF(score_layer), NATSL_DEF(tree_step), NATSL_DEF(tree_commit),
    NATSL_DEF(cache_weights), NATSL_DEF(cache_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_natsl_py", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__natsl_py(void) { return PyModule_Create(&kModule); }
