// CPython side of the binding: takes tensors apart and calls the C entry points (ss_msa.h) of the library that api.py has
// loaded, whose addresses it is given: it is not linked to one.
//
// A decode step of a small model is a handful of calls of 3 to 8 us of GPU time each, so the host has to spend less than that
// on a call.  Through ctypes, with the pointers collected in Python, a verification call took 5.6 us, of which the launch is
// 2.6; here it takes 3.5 us.  Only the CPython API is used: a tensor is any object with `data_ptr()`, `shape` and
// `nbytes` (and, for the cache in 4 bits, `stride()`, `dtype`, `is_contiguous()` and `get_device()`).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "ss_msa.h"

namespace {

// interned attribute names
PyObject *s_data_ptr, *s_shape, *s_stride, *s_nbytes, *s_cuda_stream, *s_dtype, *s_is_contiguous, *s_get_device;
PyObject *g_error, *g_raw_stream, *g_device;                    // SsError; torch's raw current stream and current device
PyObject *g_attn_params, *g_cache_layout;                       // the ctypes structures of ss_attn_params and ss_cache_layout,
PyObject *g_kvq_params, *g_kvq_cache;                           // of ss_kvq_attn_params and ss_kvq_cache
PyObject *g_int32, *g_int64, *g_bfloat16;                       // torch's types
// the entry points, in the order in which setup() takes them
#define SS_FUNCTIONS(F)                                                                                                 \
    F(ss_msa_attention) F(ss_tree_verify) F(ss_tree_verify_soft) F(ss_tree_verify_sampled) F(ss_tree_prune)             \
    F(ss_next_draft) F(ss_kv_compact) F(ss_stream_insert) F(ss_value_rotate)                                            \
    F(ss_msa_attention_kvq) F(ss_kvq_write) F(ss_kvq_read)
struct Functions {
#define SS_MEMBER(name) decltype(&::name) name;
    SS_FUNCTIONS(SS_MEMBER)
} g_lib;
PyObject *g_byref, *g_argument_error;                           // ctypes.byref and ctypes.ArgumentError

// One call's arguments.  After the first Python error everything reads as zero and `ok` stays false.
struct Args {
    PyObject* const* a;
    bool ok;
    void* ptr(int i) {
        if (!ok || a[i] == Py_None) return nullptr;
        PyObject* r = PyObject_CallMethodNoArgs(a[i], s_data_ptr);
        void* p = r ? reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(r)) : nullptr;
        if (!r || PyErr_Occurred()) ok = false;
        Py_XDECREF(r);
        return p;
    }
    template <typename T>
    T* as(int i) { return static_cast<T*>(ptr(i)); }
    // the first n sizes of argument i, which has to have exactly (or at least) n dimensions
    void sizes(int i, int n, long long* out, bool exact = true) {
        for (int k = 0; k < n; ++k) out[k] = 0;
        if (!ok) return;
        PyObject* s = PyObject_GetAttr(a[i], s_shape);
        if (!s || !PyTuple_Check(s) || PyTuple_GET_SIZE(s) < n || (exact && PyTuple_GET_SIZE(s) != n)) {
            if (s && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions", n);
            ok = false;
        } else {
            for (int k = 0; k < n; ++k) out[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, k));
        }
        Py_XDECREF(s);
    }
    // the first n strides of argument i, in elements (after sizes(): the dimensions are known to be n)
    void strides(int i, int n, long long* out) {
        for (int k = 0; k < n; ++k) out[k] = 0;
        if (!ok) return;
        PyObject* s = PyObject_CallMethodNoArgs(a[i], s_stride);
        ok = s && PyTuple_Check(s) && PyTuple_GET_SIZE(s) == n;
        for (int k = 0; ok && k < n; ++k) out[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, k));
        if (!ok && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions", n);
        Py_XDECREF(s);
    }
    // K and V rows [n_layers][batch][rows][n_heads][head_dim] of a cache in 4 bits
    ss_kvq_rows rows(int k, int v, const ss_kvq_cache* cache) {
        long long n[5], m[5], x[5], y[5];
        ss_kvq_rows r = {};
        sizes(k, 5, n);
        sizes(v, 5, m);
        strides(k, 5, x);
        strides(v, 5, y);
        r.k = ptr(k), r.v = ptr(v);
        if (!ok) return r;
        if (!is_of(k, g_bfloat16) || !is_of(v, g_bfloat16) || !on_device(k, cache) || !on_device(v, cache)) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "rows are bf16 tensors on the cache's device");
            ok = false;
            return r;
        }
        bool same = x[4] == 1 || n[4] <= 1;
        for (int i = 0; i < 5; ++i) same = same && n[i] == m[i] && (x[i] == y[i] || n[i] <= 1);
        if (!same || n[0] != cache->n_layers || n[3] != cache->n_heads || n[4] != cache->head_dim || n[1] > INT32_MAX || n[2] > INT32_MAX) {
            PyErr_SetString(PyExc_ValueError, "expected rows [n_layers][batch][rows][n_heads][head_dim] of the cache's sizes, K and V laid out alike, "
                                              "the last dimension contiguous");
            ok = false;
        }
        // (a stride that is never used may have any value)
        r.layer_stride = n[0] > 1 ? x[0] : 0, r.batch_stride = n[1] > 1 ? x[1] : 0, r.row_stride = n[2] > 1 ? x[2] : 0, r.head_stride = n[3] > 1 ? x[3] : 0;
        r.batch = static_cast<int32_t>(n[1]), r.max_rows = static_cast<int32_t>(n[2]);
        return r;
    }
    // `count` whole numbers of type T next to each other on the cache's device, or None (which the library refuses where it has to)
    template <typename T>
    T* numbers(int i, long long count, const ss_kvq_cache* cache, const char* what) {
        if (!ok || a[i] == Py_None) return nullptr;
        if (!is_of(i, sizeof(T) == 8 ? g_int64 : g_int32) || static_cast<long long>(nbytes(i)) < count * static_cast<long long>(sizeof(T)) ||
            (count > 1 && !truth(i, s_is_contiguous)) || !on_device(i, cache)) {
            if (!PyErr_Occurred())
                PyErr_Format(PyExc_ValueError, "%s: expected %lld contiguous int%d numbers on the cache's device", what, count, static_cast<int>(8 * sizeof(T)));
            ok = false;
        }
        return as<T>(i);
    }
    bool is_of(int i, PyObject* type) {
        PyObject* const dtype = PyObject_GetAttr(a[i], s_dtype);
        Py_XDECREF(dtype);                           // (the type itself is kept by torch)
        return dtype == type;
    }
    bool truth(int i, PyObject* method) {
        PyObject* const r = PyObject_CallMethodNoArgs(a[i], method);
        const bool yes = r == Py_True;
        Py_XDECREF(r);
        return yes;
    }
    bool on_device(int i, const ss_kvq_cache* cache) {
        PyObject* const r = PyObject_CallMethodNoArgs(a[i], s_get_device);
        const long d = r ? PyLong_AsLong(r) : -1;
        Py_XDECREF(r);
        return cache->device >= 0 ? d == cache->device : d >= 0;
    }
    size_t nbytes(int i) {
        if (!ok) return 0;
        PyObject* r = PyObject_GetAttr(a[i], s_nbytes);
        const size_t n = r ? static_cast<size_t>(PyLong_AsUnsignedLongLong(r)) : 0;
        if (!r || PyErr_Occurred()) ok = false;
        Py_XDECREF(r);
        return n;
    }
    int32_t i32(int i) {
        const long v = ok ? PyLong_AsLong(a[i]) : 0;
        if (v == -1 && PyErr_Occurred()) ok = false;
        return static_cast<int32_t>(v);
    }
    float f32(int i) {
        const double v = ok ? PyFloat_AsDouble(a[i]) : 0.0;
        if (v == -1.0 && PyErr_Occurred()) ok = false;
        return static_cast<float>(v);
    }
    // a torch.cuda.Stream, or None for the current stream of the current device
    void* stream(int i) {
        if (!ok) return nullptr;
        PyObject* r;
        if (a[i] != Py_None) {
            r = PyObject_GetAttr(a[i], s_cuda_stream);
        } else {
            PyObject* dev = PyObject_CallNoArgs(g_device);
            r = dev ? PyObject_CallOneArg(g_raw_stream, dev) : nullptr;
            Py_XDECREF(dev);
        }
        void* p = r ? reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(r)) : nullptr;
        if (!r || PyErr_Occurred()) ok = false;
        Py_XDECREF(r);
        return p;
    }
    // The memory of a ctypes structure of class `type`.  Anything else is refused as ctypes refuses it: a TypeError for what is
    // no ctypes object, an ArgumentError for another one.
    template <typename T>
    const T* structure(int i, PyObject* type, Py_buffer* view) {
        view->obj = nullptr;
        if (!ok) return nullptr;
        ok = false;
        const int is = PyObject_IsInstance(a[i], type);
        if (is < 0) return nullptr;
        if (!is) {
            PyObject* r = PyObject_CallOneArg(g_byref, a[i]);
            if (r) PyErr_Format(g_argument_error, "expected an instance of %R instead of %R", type, reinterpret_cast<PyObject*>(Py_TYPE(a[i])));
            Py_XDECREF(r);
            return nullptr;
        }
        if (PyObject_GetBuffer(a[i], view, PyBUF_SIMPLE) != 0) return nullptr;
        ok = view->len >= static_cast<Py_ssize_t>(sizeof(T));
        if (ok) return static_cast<const T*>(view->buf);
        PyBuffer_Release(view);
        PyErr_Format(g_argument_error, "%R is smaller than the structure", type);
        return nullptr;
    }
};

PyObject* done(const char* what, int32_t status) {
    if (status == SS_OK) Py_RETURN_NONE;
    PyObject* e = PyObject_CallFunction(g_error, "si", what, static_cast<int>(status));
    if (e) PyErr_SetObject(g_error, e);
    Py_XDECREF(e);
    return nullptr;
}

#define SS_ENTRY(name, count)                                                                    \
    PyObject* name(PyObject*, PyObject* const* argv, Py_ssize_t argc) {                          \
        if (argc != count) return PyErr_Format(PyExc_TypeError, #name ": %d arguments", count);  \
        Args a{argv, true};                                                                      \
        int32_t st = SS_OK;
// (the GIL is free while the call runs, as under ctypes)
#define SS_CALL(expr)                                                                            \
        if (!a.ok) return nullptr;                                                               \
        Py_BEGIN_ALLOW_THREADS st = expr;                                                        \
        Py_END_ALLOW_THREADS

SS_ENTRY(msa_attention, 2)
    Py_buffer view;
    void* const s = a.stream(1);
    const ss_attn_params* const p = a.structure<ss_attn_params>(0, g_attn_params, &view);
    SS_CALL(g_lib.ss_msa_attention(p, s))
    PyBuffer_Release(&view);
    return done("ss_msa_attention", st);
}

SS_ENTRY(tree_verify, 10)
    long long n[3];
    a.sizes(0, 3, n);
    const float* lg = a.as<float>(0);
    const int32_t* tok = a.as<int32_t>(1);
    const ss_tree_desc* tr = a.as<ss_tree_desc>(2);
    int32_t *al = a.as<int32_t>(3), *ap = a.as<int32_t>(4), *ln = a.as<int32_t>(5), *bt = a.as<int32_t>(6), *am = a.as<int32_t>(7);
    void* const ws = a.ptr(8);
    const size_t wb = a.nbytes(8);
    void* const s = a.stream(9);
    SS_CALL(g_lib.ss_tree_verify(lg, tok, tr, static_cast<int32_t>(n[0]), static_cast<int32_t>(n[1]), static_cast<int32_t>(n[2]), al, ap, ln, bt, am, ws, wb, s))
    return done("ss_tree_verify", st);
}

SS_ENTRY(tree_verify_soft, 13)
    long long n[3];
    a.sizes(0, 3, n);
    const float* lg = a.as<float>(0);
    const int32_t* tok = a.as<int32_t>(1);
    const ss_tree_desc* tr = a.as<ss_tree_desc>(2);
    const float eps = a.f32(3), delta = a.f32(4);
    int32_t *al = a.as<int32_t>(5), *ap = a.as<int32_t>(6), *ln = a.as<int32_t>(7), *bt = a.as<int32_t>(8);
    float *ep = a.as<float>(9), *en = a.as<float>(10);
    void* const ws = a.ptr(11);
    const size_t wb = a.nbytes(11);
    void* const s = a.stream(12);
    SS_CALL(g_lib.ss_tree_verify_soft(lg, tok, tr, static_cast<int32_t>(n[0]), static_cast<int32_t>(n[1]), static_cast<int32_t>(n[2]), eps, delta, al, ap, ln, bt,
                                ep, en, ws, wb, s))
    return done("ss_tree_verify_soft", st);
}

SS_ENTRY(tree_verify_sampled, 12)
    long long n[3];
    a.sizes(0, 3, n);
    const float* lg = a.as<float>(0);
    const int32_t* tok = a.as<int32_t>(1);
    const ss_tree_desc* tr = a.as<ss_tree_desc>(2);
    const float* un = a.as<float>(3);
    const int32_t k = a.i32(4);
    int32_t *al = a.as<int32_t>(5), *ap = a.as<int32_t>(6), *ln = a.as<int32_t>(7), *bt = a.as<int32_t>(8), *nt = a.as<int32_t>(9);
    void* const ws = a.ptr(10);
    const size_t wb = a.nbytes(10);
    void* const s = a.stream(11);
    SS_CALL(g_lib.ss_tree_verify_sampled(lg, tok, tr, un, static_cast<int32_t>(n[0]), static_cast<int32_t>(n[1]), static_cast<int32_t>(n[2]), k, al, ap, ln, bt, nt,
                                   ws, wb, s))
    return done("ss_tree_verify_sampled", st);
}

SS_ENTRY(tree_prune, 11)
    long long n[3];
    a.sizes(0, 3, n);
    const float* lg = a.as<float>(0);
    const int32_t* tok = a.as<int32_t>(1);
    const ss_tree_desc* tr = a.as<ss_tree_desc>(2);
    const float threshold = a.f32(3);
    float* ep = a.as<float>(4);
    int32_t *ni = a.as<int32_t>(5), *kn = a.as<int32_t>(6), *kt = a.as<int32_t>(7);
    ss_tree_desc* pt = a.as<ss_tree_desc>(8);
    void* const ws = a.ptr(9);
    const size_t wb = a.nbytes(9);
    void* const s = a.stream(10);
    SS_CALL(g_lib.ss_tree_prune(lg, tok, tr, static_cast<int32_t>(n[0]), static_cast<int32_t>(n[1]), static_cast<int32_t>(n[2]), threshold, ep, ni, kn, kt, pt, ws, wb, s))
    return done("ss_tree_prune", st);
}

SS_ENTRY(next_draft, 9)
    long long n[4];
    a.sizes(0, 4, n);
    const float* lg = a.as<float>(0);
    const int32_t *ri = a.as<int32_t>(1), *bt = a.as<int32_t>(2);
    const int32_t k = a.i32(3), nodes = a.i32(4);
    int32_t* tok = a.as<int32_t>(5);
    ss_tree_desc* tr = a.as<ss_tree_desc>(6);
    void* const ws = a.ptr(7);
    const size_t wb = a.nbytes(7);
    void* const s = a.stream(8);
    SS_CALL(g_lib.ss_next_draft(lg, static_cast<int32_t>(n[1]), ri, bt, static_cast<int32_t>(n[0]), static_cast<int32_t>(n[2]), static_cast<int32_t>(n[3]), k, nodes, tok,
                          tr, ws, wb, s))
    return done("ss_next_draft", st);
}

SS_ENTRY(kv_compact, 9)
    long long n[1];
    Py_buffer view;
    void *k = a.ptr(0), *v = a.ptr(1);
    a.sizes(3, 1, n, false);
    const int64_t* ks = a.as<int64_t>(3);
    const int32_t *kl = a.as<int32_t>(4), *al = a.as<int32_t>(5), *ap = a.as<int32_t>(6);
    int32_t* ko = a.as<int32_t>(7);
    void* const s = a.stream(8);
    const ss_cache_layout* const lo = a.structure<ss_cache_layout>(2, g_cache_layout, &view);
    SS_CALL(g_lib.ss_kv_compact(k, v, lo, static_cast<int32_t>(n[0]), ks, kl, al, ap, ko, s))
    PyBuffer_Release(&view);
    return done("ss_kv_compact", st);
}

SS_ENTRY(stream_insert, 4)
    long long n[2], g[1];
    a.sizes(0, 2, n);
    a.sizes(1, 1, g, false);
    void *m = a.ptr(0), *e = a.ptr(1), *o = a.ptr(2);
    void* const s = a.stream(3);
    SS_CALL(g_lib.ss_stream_insert(m, e, o, n[0], static_cast<int32_t>(g[0]), static_cast<int32_t>(n[1]), s))
    return done("ss_stream_insert", st);
}

SS_ENTRY(value_rotate, 4)
    long long n[2], g[2];
    a.sizes(0, 2, n);
    a.sizes(1, 2, g, false);
    void *v = a.ptr(0), *o = a.ptr(1);
    const float epsilon = a.f32(2);
    void* const s = a.stream(3);
    SS_CALL(g_lib.ss_value_rotate(v, o, n[0], static_cast<int32_t>(g[1]), static_cast<int32_t>(n[1]), epsilon, s))
    return done("ss_value_rotate", st);
}

SS_ENTRY(msa_attention_kvq, 2)
    Py_buffer view;
    void* const s = a.stream(1);
    const ss_kvq_attn_params* const p = a.structure<ss_kvq_attn_params>(0, g_kvq_params, &view);
    SS_CALL(g_lib.ss_msa_attention_kvq(p, s))
    PyBuffer_Release(&view);
    return done("ss_msa_attention_kvq", st);
}

SS_ENTRY(kvq_write, 11)
    Py_buffer view;
    void* const s = a.stream(10);
    const ss_kvq_cache* const ca = a.structure<ss_kvq_cache>(2, g_kvq_cache, &view);
    const ss_kvq_rows r = a.rows(0, 1, ca);
    const int64_t* ks = a.numbers<int64_t>(3, r.batch, ca, "kv_start");
    const int32_t *kl = a.numbers<int32_t>(4, r.batch, ca, "kv_len_in"), *nr = a.numbers<int32_t>(5, r.batch, ca, "n_rows");
    const int32_t *pa = a.numbers<int32_t>(6, static_cast<long long>(r.batch) * SS_PATH_STRIDE, ca, "path"), *kc = a.numbers<int32_t>(7, r.batch, ca, "kv_capacity");
    int32_t* ko = a.numbers<int32_t>(8, r.batch, ca, "kv_len_out");
    void* const status = a.ptr(9);
    if (a.ok && status && (a.nbytes(9) < sizeof(int32_t) || !a.on_device(9, ca))) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "status: expected a workspace on the cache's device");
        a.ok = false;
    }
    if (!a.ok && view.obj) PyBuffer_Release(&view);
    SS_CALL(g_lib.ss_kvq_write(&r, ca, ks, kl, nr, pa, kc, ko, status, s))
    PyBuffer_Release(&view);
    return done("ss_kvq_write", st);
}

SS_ENTRY(kvq_read, 7)
    Py_buffer view;
    void* const s = a.stream(6);
    const ss_kvq_cache* const ca = a.structure<ss_kvq_cache>(0, g_kvq_cache, &view);
    const ss_kvq_rows r = a.rows(1, 2, ca);
    const int64_t* ks = a.numbers<int64_t>(3, r.batch, ca, "kv_start");
    const int32_t *fi = a.numbers<int32_t>(4, r.batch, ca, "first"), *nr = a.numbers<int32_t>(5, r.batch, ca, "n_rows");
    if (!a.ok && view.obj) PyBuffer_Release(&view);
    SS_CALL(g_lib.ss_kvq_read(ca, &r, ks, fi, nr, s))
    PyBuffer_Release(&view);
    return done("ss_kvq_read", st);
}

// setup(SsError, raw_stream(device) -> int, device() -> int, AttnParams, CacheLayout, ctypes.byref, ctypes.ArgumentError,
//       addresses of SS_FUNCTIONS: a tuple of int, KvqAttnParams, KvqCache, torch.int32, torch.int64, torch.bfloat16)
SS_ENTRY(setup, 13)
    (void)a; (void)st;
    PyObject* const at = argv[7];
    Py_ssize_t n = 0;
    Functions lib = {};
#define SS_TAKE(name)                                                                                                   \
    if (PyTuple_Check(at) && n < PyTuple_GET_SIZE(at)) lib.name = reinterpret_cast<decltype(lib.name)>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, n))); \
    if (!lib.name) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "setup: no address of %s", #name);  \
    ++n;
    SS_FUNCTIONS(SS_TAKE)
    g_lib = lib;
    PyObject** const kept[13] = {&g_error, &g_raw_stream, &g_device, &g_attn_params, &g_cache_layout, &g_byref, &g_argument_error, nullptr, &g_kvq_params,
                                 &g_kvq_cache, &g_int32, &g_int64, &g_bfloat16};
    for (int i = 0; i < 13; ++i)
        if (kept[i]) Py_XSETREF(*kept[i], Py_NewRef(argv[i]));
    Py_RETURN_NONE;
}

#define SS_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SS_METHOD(setup), SS_METHOD(msa_attention), SS_METHOD(tree_verify), SS_METHOD(tree_verify_soft),
                         SS_METHOD(tree_verify_sampled), SS_METHOD(tree_prune), SS_METHOD(next_draft), SS_METHOD(kv_compact),
                         SS_METHOD(stream_insert), SS_METHOD(value_rotate), SS_METHOD(msa_attention_kvq), SS_METHOD(kvq_write),
                         SS_METHOD(kvq_read), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pycall() {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    return PyModule_Create(&module);
}
