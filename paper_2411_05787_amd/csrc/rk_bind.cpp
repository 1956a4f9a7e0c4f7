// Argument marshalling of the short calls, in C++: what binding.py does for them one attribute at a time.
//
// Every function takes the binding's arguments in order, asks of every tensor what _dev() and _kv() ask
// (the plain class, device, type, contiguous or rows contiguous, shape) on every call, and returns the library's status; None if some
// argument is not as the common case has it, and nothing has been called then: binding.py goes through its own checks, for the message
// or the rarer form.  The interpreter lock is given up during the library's call, as ctypes does.
//
// A partial step of one layer over 256 rows takes the GPU 4.6 us; marshalled by Python and ctypes the host took 9.0.  An H2O step of 4 sequences of
// 2048 rows 22.2 -> 20.0.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/refreshkv.h"

namespace {

// binding.py's _stream, and the two functions of torch that give the current stream's handle (None where torch lacks them).
PyObject *g_stream, *g_raw_stream, *g_device;
// The ctypes classes of rk_geom, rk_h2o_state, rk_rope, rk_kv8 and rk_pages: what is of another class is binding.py's to refuse.
PyObject *g_geom, *g_h2o_state, *g_rope, *g_kv8, *g_pages;

// One call's arguments: `ok` until one of them is not the common case's.
struct Args {
    PyObject* const* a;
    bool ok = true;
    rk_geom geom{};
    int device = -1;                          // of the tensors asked for so far; -2: of more than one

    void on(int64_t d) { device = device == -1 || device == d ? (int)d : -2; }
    const at::Tensor* tensor(int i) {
        if (!ok || !THPVariable_CheckExact(a[i])) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda()) { ok = false; return nullptr; }
        on(t.get_device());
        return &t;
    }
    void* dev(int i, at::ScalarType type, std::initializer_list<int64_t> shape) {
        const at::Tensor* t = tensor(i);
        if (!t) return nullptr;
        ok = t->scalar_type() == type && t->is_contiguous() && t->sizes() == at::IntArrayRef(shape);
        return ok ? t->data_ptr() : nullptr;
    }
    void* dev_or_null(int i, at::ScalarType type, std::initializer_list<int64_t> shape) {
        return a[i] == Py_None ? nullptr : dev(i, type, shape);
    }
    int64_t number(int i) {
        if (!ok || !PyLong_CheckExact(a[i])) { ok = false; return 0; }
        const long long v = PyLong_AsLongLong(a[i]);
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }
    int32_t i32(int i) {
        const int64_t v = number(i);
        if (v < INT32_MIN || v > INT32_MAX) ok = false;
        return (int32_t)v;
    }
    // A ctypes structure by value.
    template <class T> T structure(PyObject* o, PyObject* type) {
        T s{};
        Py_buffer b;
        if (!ok || (PyObject*)Py_TYPE(o) != type || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); ok = false; return s; }
        ok = b.len == (Py_ssize_t)sizeof(T);
        if (ok) s = *(const T*)b.buf;
        PyBuffer_Release(&b);
        return s;
    }
    void geometry(int i) {                    // (Geom keeps its C structure once it has been asked for it)
        static PyObject* const name = PyUnicode_InternFromString("_c");
        PyObject* c = PyObject_GetAttr(a[i], name);
        if (!c) { PyErr_Clear(); ok = false; return; }
        geom = structure<rk_geom>(c, g_geom);
        Py_DECREF(c);
    }
    rk_kv kv(int k, int v, int64_t min_rows) {
        rk_kv r{};
        const at::Tensor *K = tensor(k), *V = tensor(v);
        if (!K || !V) return r;
        ok = K->scalar_type() == at::kBFloat16 && V->scalar_type() == at::kBFloat16 && K->dim() == 4 && V->sizes() == K->sizes() &&
             V->strides() == K->strides() && K->size(0) == geom.batch && K->size(1) == geom.n_kv_heads && K->size(3) == geom.head_dim &&
             K->stride(3) == 1 && K->stride(2) == geom.head_dim && K->size(2) >= min_rows;
        if (!ok) return r;
        return rk_kv{K->data_ptr(), V->data_ptr(), K->stride(0), K->stride(1), K->size(2)};
    }
    // [B, T, heads, head_dim] whose heads lie side by side: pointer and strides.
    struct Rows { void* ptr; int64_t b, t; };
    Rows rows(int i, int64_t T, int64_t heads) {
        const at::Tensor* t = tensor(i);
        if (!t) return {};
        ok = t->scalar_type() == at::kBFloat16 && t->sizes() == at::IntArrayRef({geom.batch, T, heads, geom.head_dim}) &&
             t->stride(3) == 1 && (t->stride(2) == geom.head_dim || heads == 1);
        if (!ok) return {};
        return {t->data_ptr(), geom.batch > 1 ? t->stride(0) : 0, T > 1 ? t->stride(1) : 0};
    }
    // The C structure that an object of binding.py (Rope, Kv8, Pages) keeps, and the device of what it points at.
    template <class T> T held(int i, PyObject* type) {
        static PyObject *const name = PyUnicode_InternFromString("_c"), *const dev = PyUnicode_InternFromString("device_index");
        PyObject* c = ok ? PyObject_GetAttr(a[i], name) : nullptr;
        if (!c) { PyErr_Clear(); ok = false; return T{}; }
        const T s = structure<T>(c, type);
        Py_DECREF(c);
        on((int64_t)attribute(a[i], dev));
        return s;
    }
    rk_kv8 cache8(int i) {                    // (one of another geometry, or of an equal one: binding.py's question)
        static PyObject* const name = PyUnicode_InternFromString("geom");
        const rk_kv8 s = held<rk_kv8>(i, g_kv8);
        PyObject* g = ok ? PyObject_GetAttr(a[i], name) : nullptr;
        if (g != a[0]) ok = false;
        if (!g) PyErr_Clear();
        Py_XDECREF(g);
        return s;
    }
    rk_pages pool(int i) {                    // (of this geometry's heads)
        static PyObject *const heads = PyUnicode_InternFromString("n_kv_heads"), *const dim = PyUnicode_InternFromString("head_dim");
        const rk_pages s = held<rk_pages>(i, g_pages);
        if ((int64_t)attribute(a[i], heads) != geom.n_kv_heads || (int64_t)attribute(a[i], dim) != geom.head_dim) ok = false;
        return s;
    }
    // int32 [batch, width].
    struct Table { const int32_t* ptr; int32_t width; };
    Table table(int i) {
        const at::Tensor* t = tensor(i);
        if (!t || t->dim() != 2 || t->size(1) > INT32_MAX) { ok = false; return {}; }
        const int64_t width = t->size(1);
        return {(const int32_t*)dev(i, at::kInt, {geom.batch, width}), (int32_t)width};
    }
    // first, end, cap, slopes of an attention of T new tokens
    rk_prompt_scores scores(int first, int end, int cap, int slopes, int64_t T) {
        rk_prompt_scores s{};
        if (!ok || !PyFloat_CheckExact(a[cap])) { ok = false; return s; }
        s.cap = (float)PyFloat_AS_DOUBLE(a[cap]);
        s.first = (const int32_t*)dev_or_null(first, at::kInt, {geom.batch, T});
        s.end = (const int32_t*)dev_or_null(end, at::kInt, {geom.batch, T});
        s.slopes = (const float*)dev_or_null(slopes, at::kFloat, {geom.n_q_heads});
        return s;
    }
    int64_t tokens(int i) {                   // of q [B, T, Hq, D]
        const at::Tensor* t = tensor(i);
        if (!t || t->dim() != 4 || t->size(1) > INT32_MAX) { ok = false; return 0; }
        return t->size(1);
    }
    struct Scratch { void* ptr; size_t bytes; };
    Scratch workspace(int i) {
        static PyObject *const ptr = PyUnicode_InternFromString("ptr"), *const bytes = PyUnicode_InternFromString("nbytes");
        Scratch s{(void*)attribute(a[i], ptr), (size_t)attribute(a[i], bytes)};
        return s;
    }
    Scratch workspace_here(int i) {           // ... that has to be in the memory of the other arguments' device
        static PyObject* const dev = PyUnicode_InternFromString("device_index");
        const Scratch s = workspace(i);
        on((int64_t)attribute(a[i], dev));
        return s;
    }
    void* stream(int i) {                     // (asked for last, once every tensor is known to be in GPU memory)
        if (!ok || !g_stream) { ok = false; return nullptr; }
        PyObject *d = nullptr, *h = nullptr;
        if (a[i] != Py_None || g_raw_stream == Py_None || g_device == Py_None) {
            h = PyObject_CallFunctionObjArgs(g_stream, a[i], nullptr);
        } else if ((d = PyObject_CallNoArgs(g_device)) != nullptr) {
            h = PyObject_CallFunctionObjArgs(g_raw_stream, d, nullptr);
            Py_DECREF(d);
        }
        unsigned long long x = h && PyLong_Check(h) ? PyLong_AsUnsignedLongLong(h) : 0;
        if (!h || !PyLong_Check(h) || PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        Py_XDECREF(h);
        return (void*)x;
    }

    // ... where the call's tensors are all on the current device.
    void* stream_here(int i) {
        PyObject* d = ok && g_device && g_device != Py_None ? PyObject_CallNoArgs(g_device) : nullptr;
        if (!d || !PyLong_Check(d) || PyLong_AsLong(d) != device) ok = false;
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        Py_XDECREF(d);
        return stream(i);
    }

private:
    unsigned long long attribute(PyObject* o, PyObject* name) {
        PyObject* v = ok ? PyObject_GetAttr(o, name) : nullptr;
        unsigned long long x = 0;
        if (v && PyLong_CheckExact(v)) x = PyLong_AsUnsignedLongLong(v);
        if (!v || !PyLong_CheckExact(v) || PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        Py_XDECREF(v);
        return x;
    }
};

template <class Call>
PyObject* status_of(Call&& call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// Runs `body` on the arguments; None for a wrong number of them, or where a tensor has no memory to point at.
template <class Body>
PyObject* with_args(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, Body&& body) {
    if (n != want) Py_RETURN_NONE;
    Args x{a};
    PyObject* r = nullptr;
    try {
        x.geometry(0);
        if (x.ok) r = body(x);
    } catch (...) {
        r = nullptr;
    }
    if (r) return r;
    PyErr_Clear();
    Py_RETURN_NONE;
}

constexpr auto bf16 = at::kBFloat16;
constexpr auto i32t = at::kInt;
constexpr auto f32 = at::kFloat;

// geom, q, small_K, small_V, n_sel, K, V, tail_start, seq_lens, max_recent, out, pred, pred_val, workspace, stream
template <int (*FN)(const rk_geom*, const void*, rk_kv, int32_t, rk_kv, const int32_t*, const int32_t*, int32_t, void*, const int32_t*, int32_t,
                    void*, size_t, void*)>
PyObject* partial(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 15, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        void* q = x.dev(1, bf16, {g.batch, g.n_q_heads, g.head_dim});
        const int32_t n_sel = x.i32(4), recent = x.i32(9), pred_val = x.i32(12);
        const rk_kv small = x.kv(2, 3, n_sel), full = x.kv(5, 6, 0);
        auto* tail = (const int32_t*)x.dev(7, i32t, {g.batch});
        auto* lens = (const int32_t*)x.dev(8, i32t, {g.batch});
        void* out = x.dev(10, bf16, {g.batch, g.n_q_heads, g.head_dim});
        auto* pred = (const int32_t*)x.dev_or_null(11, i32t, {g.batch});
        const Args::Scratch ws = x.workspace(13);
        void* st = x.stream(14);
        if (!x.ok) return nullptr;
        return status_of([&] { return FN(&g, q, small, n_sel, full, tail, lens, recent, out, pred, pred_val, ws.ptr, ws.bytes, st); });
    });
}

// geom, K, V, idx, k, small_K, small_V, seq_lens, tail_start, pred, pred_val, stream
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 12, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int32_t k = x.i32(4), pred_val = x.i32(10);
        const rk_kv full = x.kv(1, 2, 0), small = x.kv(5, 6, k);
        auto* idx = (const int32_t*)x.dev(3, i32t, {g.batch, g.n_kv_heads, k});
        auto* lens = (const int32_t*)x.dev_or_null(7, i32t, {g.batch});
        auto* tail = (int32_t*)x.dev_or_null(8, i32t, {g.batch});
        auto* pred = (const int32_t*)x.dev_or_null(9, i32t, {g.batch});
        void* st = x.stream(11);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_gather_small_kv(&g, full, idx, k, small, lens, tail, pred, pred_val, st); });
    });
}

// geom, state, q, k_new, v_new, seq_lens, budget, recent, out, agg, dropped, workspace, stream
PyObject* h2o_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 13, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const rk_h2o_state state = x.structure<rk_h2o_state>(x.a[1], g_h2o_state);
        void* q = x.dev(2, bf16, {g.batch, g.n_q_heads, g.head_dim});
        void* k_new = x.dev(3, bf16, {g.batch, g.n_kv_heads, g.head_dim});
        void* v_new = x.dev(4, bf16, {g.batch, g.n_kv_heads, g.head_dim});
        auto* lens = (const int32_t*)x.dev(5, i32t, {g.batch});
        const int32_t budget = x.i32(6), recent = x.i32(7), agg = x.i32(9);
        void* out = x.dev(8, bf16, {g.batch, g.n_q_heads, g.head_dim});
        auto* dropped = (int32_t*)x.dev_or_null(10, i32t, {g.batch, g.n_kv_heads});
        const Args::Scratch ws = x.workspace(11);
        void* st = x.stream(12);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_h2o_step(&g, state, q, k_new, v_new, lens, budget, recent, agg, out, dropped, ws.ptr, ws.bytes, st); });
    });
}

// geom, q, K, V, seq_lens, max_len, out, lse, pred, pred_val, workspace, stream (no weights returned)
PyObject* full_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 12, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        void* q = x.dev(1, bf16, {g.batch, g.n_q_heads, g.head_dim});
        const int32_t max_len = x.i32(5), pred_val = x.i32(9);
        const rk_kv full = x.kv(2, 3, max_len);
        auto* lens = (const int32_t*)x.dev(4, i32t, {g.batch});
        void* out = x.dev(6, bf16, {g.batch, g.n_q_heads, g.head_dim});
        auto* lse = (float*)x.dev_or_null(7, f32, {g.batch, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(8, i32t, {g.batch});
        const Args::Scratch ws = x.workspace(10);
        void* st = x.stream(11);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_full_attn(&g, q, full, lens, max_len, out, nullptr, 0, lse, pred, pred_val, ws.ptr, ws.bytes, st); });
    });
}

// geom, q, k, v, rope, K, V, seq_lens, q_out, new_lens, positions, pred, pred_val, stream; with one cache of 8 bits for K and V: 1; with
// pages and their table: 2
template <int INTO>
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, INTO == 1 ? 13 : 14, [](Args& x) -> PyObject* {
        constexpr bool Q8 = INTO == 1;
        constexpr int o = Q8 ? 6 : 7;         // seq_lens
        const rk_geom& g = x.geom;
        const at::Tensor* k = x.tensor(2);
        if (!k || k->dim() != 4 || k->size(1) > INT32_MAX) return nullptr;
        const int64_t T = k->size(1);
        const bool none = x.a[1] == Py_None;
        const Args::Rows q = none ? Args::Rows{} : x.rows(1, T, g.n_q_heads), kr = x.rows(2, T, g.n_kv_heads), v = x.rows(3, T, g.n_kv_heads);
        if (none != (x.a[o + 1] == Py_None) || (!none && x.a[4] == Py_None)) return nullptr;
        const rk_new_rows rows{q.ptr, kr.ptr, v.ptr, q.b, q.t, kr.b, kr.t, v.b, v.t, (int32_t)T};
        const bool turned = x.a[4] != Py_None;
        const rk_rope rope = turned ? x.held<rk_rope>(4, g_rope) : rk_rope{};
        rk_kv kv{};
        rk_kv8 c8{};
        rk_pages pages{};
        Args::Table table{};
        if (INTO == 2) { pages = x.pool(5); table = x.table(6); }
        else if (Q8) c8 = x.cache8(5);
        else kv = x.kv(5, 6, 0);
        auto* lens = (const int32_t*)x.dev(o, i32t, {g.batch});
        void* q_out = x.dev_or_null(o + 1, bf16, {g.batch, T, g.n_q_heads, g.head_dim});
        auto* new_lens = (const int32_t*)x.dev_or_null(o + 2, i32t, {g.batch});
        auto* pos = (const int32_t*)x.dev_or_null(o + 3, i32t, {g.batch, T});
        auto* pred = (const int32_t*)x.dev_or_null(o + 4, i32t, {g.batch});
        const int32_t pred_val = x.i32(o + 5);
        void* st = x.stream_here(o + 6);
        if (!x.ok) return nullptr;
        return status_of([&] {
            if (INTO == 2) return rk_rope_append_paged(&g, &rows, turned ? &rope : nullptr, pos, &pages, table.ptr, table.width, lens, new_lens, q_out, pred, pred_val, st);
            return Q8 ? rk_rope_append_q8(&g, &rows, turned ? &rope : nullptr, pos, &c8, lens, new_lens, q_out, pred, pred_val, st)
                      : rk_rope_append(&g, &rows, turned ? &rope : nullptr, pos, kv, lens, new_lens, q_out, pred, pred_val, st);
        });
    });
}

// geom, q, cache, seq_lens, max_len, out, weights, lse, pred, pred_val, workspace, stream
PyObject* full_attn_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 12, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        void* q = x.dev(1, bf16, {g.batch, g.n_q_heads, g.head_dim});
        const rk_kv8 c8 = x.cache8(2);
        auto* lens = (const int32_t*)x.dev(3, i32t, {g.batch});
        const int32_t max_len = x.i32(4), pred_val = x.i32(9);
        void* out = x.dev(5, bf16, {g.batch, g.n_q_heads, g.head_dim});
        int64_t width = 0;
        float* weights = nullptr;
        if (x.a[6] != Py_None) {
            const at::Tensor* w = x.tensor(6);
            if (!w || w->dim() != 3) return nullptr;
            width = w->size(2);
            weights = (float*)x.dev(6, f32, {g.batch, g.n_q_heads, width});
            if (width < max_len) return nullptr;
        }
        auto* lse = (float*)x.dev_or_null(7, f32, {g.batch, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(8, i32t, {g.batch});
        const Args::Scratch ws = x.workspace_here(10);
        void* st = x.stream_here(11);
        if (!x.ok || max_len > c8.capacity) return nullptr;
        return status_of([&] { return rk_full_attn_q8(&g, q, &c8, lens, max_len, out, weights, width, lse, pred, pred_val, ws.ptr, ws.bytes, st); });
    });
}

// geom, cache, idx, k, small_K, small_V, seq_lens, tail_start, pred, pred_val, stream
PyObject* gather_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 11, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const rk_kv8 c8 = x.cache8(1);
        const int32_t k = x.i32(3), pred_val = x.i32(9);
        auto* idx = (const int32_t*)x.dev(2, i32t, {g.batch, g.n_kv_heads, k});
        const rk_kv small = x.kv(4, 5, k);
        auto* lens = (const int32_t*)x.dev(6, i32t, {g.batch});
        auto* tail = (int32_t*)x.dev_or_null(7, i32t, {g.batch});
        auto* pred = (const int32_t*)x.dev_or_null(8, i32t, {g.batch});
        void* st = x.stream_here(10);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_gather_small_kv_q8(&g, &c8, idx, k, small, lens, tail, pred, pred_val, st); });
    });
}

// geom, q, K, V, seq_lens, max_len, out, new_lens, first, end, cap, slopes, lse, pred, pred_val, workspace, stream
PyObject* prompt_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 17, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const at::Tensor* qt = x.tensor(1);
        if (!qt || qt->dim() != 4 || qt->size(1) > INT32_MAX || !PyFloat_CheckExact(x.a[10])) return nullptr;
        const int64_t T = qt->size(1);
        const Args::Rows q = x.rows(1, T, g.n_q_heads);
        const int32_t max_len = x.i32(5), pred_val = x.i32(14);
        const rk_kv kv = x.kv(2, 3, max_len);
        auto* lens = (const int32_t*)x.dev(4, i32t, {g.batch});
        void* out = x.dev(6, bf16, {g.batch, T, g.n_q_heads, g.head_dim});
        auto* new_lens = (const int32_t*)x.dev_or_null(7, i32t, {g.batch});
        rk_prompt_scores s{(float)PyFloat_AS_DOUBLE(x.a[10]), nullptr, nullptr, nullptr};
        s.first = (const int32_t*)x.dev_or_null(8, i32t, {g.batch, T});
        s.end = (const int32_t*)x.dev_or_null(9, i32t, {g.batch, T});
        s.slopes = (const float*)x.dev_or_null(11, f32, {g.n_q_heads});
        auto* lse = (float*)x.dev_or_null(12, f32, {g.batch, T, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(13, i32t, {g.batch});
        const Args::Scratch ws = x.a[15] == Py_None ? Args::Scratch{nullptr, 0} : x.workspace_here(15);
        void* st = x.stream_here(16);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_prompt_attn(&g, q.ptr, q.b, q.t, (int32_t)T, kv, lens, new_lens, max_len, &s, out, lse, pred, pred_val, ws.ptr, ws.bytes, st); });
    });
}

// geom, q, pages, table, seq_lens, max_len, out, new_lens, first, end, cap, slopes, lse, pred, pred_val, workspace, stream
PyObject* paged_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 17, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int64_t T = x.tokens(1);
        if (!x.ok) return nullptr;
        const Args::Rows q = x.rows(1, T, g.n_q_heads);
        const rk_pages pages = x.pool(2);
        const Args::Table table = x.table(3);
        auto* lens = (const int32_t*)x.dev(4, i32t, {g.batch});
        const int32_t max_len = x.i32(5), pred_val = x.i32(14);
        void* out = x.dev(6, bf16, {g.batch, T, g.n_q_heads, g.head_dim});
        auto* new_lens = (const int32_t*)x.dev_or_null(7, i32t, {g.batch});
        const rk_prompt_scores s = x.scores(8, 9, 10, 11, T);
        auto* lse = (float*)x.dev_or_null(12, f32, {g.batch, T, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(13, i32t, {g.batch});
        const Args::Scratch ws = x.a[15] == Py_None ? Args::Scratch{nullptr, 0} : x.workspace_here(15);
        void* st = x.stream_here(16);
        if (!x.ok || max_len > (int64_t)table.width * pages.page) return nullptr;
        return status_of([&] {
            return rk_paged_attn(&g, q.ptr, q.b, q.t, (int32_t)T, &pages, table.ptr, table.width, lens, new_lens, max_len, &s, out, lse, pred, pred_val,
                                 ws.ptr, ws.bytes, st);
        });
    });
}

// geom, q, pages, prefix_table, prefix_len, max_prefix, table, seq_lens, max_own, out, new_lens, first, end, cap, slopes, lse, pred, pred_val,
// workspace, stream
PyObject* prefix_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 20, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int64_t T = x.tokens(1);
        const at::Tensor* pt = x.tensor(3);
        if (!x.ok || pt->dim() != 1 || pt->size(0) > INT32_MAX) return nullptr;
        const Args::Rows q = x.rows(1, T, g.n_q_heads);
        const rk_pages pages = x.pool(2);
        const int64_t width = pt->size(0);
        auto* prefix = (const int32_t*)x.dev(3, i32t, {width});
        auto* prefix_len = (const int32_t*)x.dev(4, i32t, {1});
        const int32_t max_prefix = x.i32(5), max_own = x.i32(8), pred_val = x.i32(17);
        const Args::Table table = x.table(6);
        auto* lens = (const int32_t*)x.dev(7, i32t, {g.batch});
        void* out = x.dev(9, bf16, {g.batch, T, g.n_q_heads, g.head_dim});
        auto* new_lens = (const int32_t*)x.dev_or_null(10, i32t, {g.batch});
        const rk_prompt_scores s = x.scores(11, 12, 13, 14, T);
        auto* lse = (float*)x.dev_or_null(15, f32, {g.batch, T, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(16, i32t, {g.batch});
        const Args::Scratch ws = x.workspace_here(18);
        void* st = x.stream_here(19);
        if (!x.ok || max_prefix > width * pages.page) return nullptr;
        return status_of([&] {
            return rk_prefix_attn(&g, q.ptr, q.b, q.t, (int32_t)T, &pages, prefix, (int32_t)width, prefix_len, max_prefix, table.ptr, table.width, lens,
                                  new_lens, max_own, &s, out, lse, pred, pred_val, ws.ptr, ws.bytes, st);
        });
    });
}

// geom, q, pages, table, seq_lens, scores, new_lens, agg, pred, pred_val, stream
PyObject* page_scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 11, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int64_t T = x.tokens(1);
        const at::Tensor* sc = x.tensor(5);
        if (!x.ok || sc->dim() != 4) return nullptr;
        const Args::Rows q = x.rows(1, T, g.n_q_heads);
        const rk_pages pages = x.pool(2);
        const Args::Table table = x.table(3);
        auto* lens = (const int32_t*)x.dev(4, i32t, {g.batch});
        const int64_t width = sc->size(3);
        auto* scores = (float*)x.dev(5, f32, {g.batch, T, g.n_kv_heads, width});
        auto* new_lens = (const int32_t*)x.dev_or_null(6, i32t, {g.batch});
        const int32_t agg = x.i32(7), pred_val = x.i32(9);
        auto* pred = (const int32_t*)x.dev_or_null(8, i32t, {g.batch});
        void* st = x.stream_here(10);
        if (!x.ok || !pages.k_min) return nullptr;
        return status_of([&] {
            return rk_page_scores(&g, q.ptr, q.b, q.t, (int32_t)T, &pages, table.ptr, table.width, lens, new_lens, agg, scores, width, pred, pred_val, st);
        });
    });
}

// geom, scores, page, seq_lens, k, idx, new_lens, keep_first, keep_last, pred, pred_val, stream
PyObject* page_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 12, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int64_t T = x.tokens(1);
        if (!x.ok) return nullptr;
        const int64_t width = x.tensor(1)->size(3);
        auto* scores = (const float*)x.dev(1, f32, {g.batch, T, g.n_kv_heads, width});
        const int32_t page = x.i32(2), k = x.i32(4), first = x.i32(7), last = x.i32(8), pred_val = x.i32(10);
        auto* lens = (const int32_t*)x.dev(3, i32t, {g.batch});
        auto* idx = (int32_t*)x.dev(5, i32t, {g.batch, T, g.n_kv_heads, k});
        auto* new_lens = (const int32_t*)x.dev_or_null(6, i32t, {g.batch});
        auto* pred = (const int32_t*)x.dev_or_null(9, i32t, {g.batch});
        void* st = x.stream_here(11);
        if (!x.ok) return nullptr;
        return status_of([&] { return rk_page_select(&g, scores, width, (int32_t)T, page, lens, new_lens, k, first, last, idx, pred, pred_val, st); });
    });
}

// geom, q, pages, table, idx, seq_lens, out, new_lens, first, end, cap, slopes, lse, pred, pred_val, workspace, stream
PyObject* sparse_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return with_args(a, n, 17, [](Args& x) -> PyObject* {
        const rk_geom& g = x.geom;
        const int64_t T = x.tokens(1);
        const at::Tensor* it = x.tensor(4);
        if (!x.ok || it->dim() != 4 || it->size(3) > INT32_MAX) return nullptr;
        const Args::Rows q = x.rows(1, T, g.n_q_heads);
        const rk_pages pages = x.pool(2);
        const Args::Table table = x.table(3);
        const int64_t k = it->size(3);
        auto* idx = (const int32_t*)x.dev(4, i32t, {g.batch, T, g.n_kv_heads, k});
        auto* lens = (const int32_t*)x.dev(5, i32t, {g.batch});
        void* out = x.dev(6, bf16, {g.batch, T, g.n_q_heads, g.head_dim});
        auto* new_lens = (const int32_t*)x.dev_or_null(7, i32t, {g.batch});
        const rk_prompt_scores s = x.scores(8, 9, 10, 11, T);
        auto* lse = (float*)x.dev_or_null(12, f32, {g.batch, T, g.n_q_heads});
        auto* pred = (const int32_t*)x.dev_or_null(13, i32t, {g.batch});
        const int32_t pred_val = x.i32(14);
        const Args::Scratch ws = x.a[15] == Py_None ? Args::Scratch{nullptr, 0} : x.workspace_here(15);
        void* st = x.stream_here(16);
        if (!x.ok) return nullptr;
        return status_of([&] {
            return rk_sparse_attn(&g, q.ptr, q.b, q.t, (int32_t)T, &pages, table.ptr, table.width, idx, (int32_t)k, lens, new_lens, &s, out, lse, pred, pred_val,
                                  ws.ptr, ws.bytes, st);
        });
    });
}

PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 8) { PyErr_SetString(PyExc_TypeError, "setup(stream, raw_stream, device, geom, h2o_state, rope, kv8, pages)"); return nullptr; }
    for (int i = 0; i < 8; ++i) Py_INCREF(a[i]);
    g_stream = a[0]; g_raw_stream = a[1]; g_device = a[2]; g_geom = a[3]; g_h2o_state = a[4]; g_rope = a[5]; g_kv8 = a[6]; g_pages = a[7];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, nullptr},
    {"rk_partial_attn", (PyCFunction)(void (*)(void))partial<rk_partial_attn>, METH_FASTCALL, nullptr},
    {"rk_partial_attn_fixed", (PyCFunction)(void (*)(void))partial<rk_partial_attn_fixed>, METH_FASTCALL, nullptr},
    {"rk_gather_small_kv", (PyCFunction)(void (*)(void))gather, METH_FASTCALL, nullptr},
    {"rk_h2o_step", (PyCFunction)(void (*)(void))h2o_step, METH_FASTCALL, nullptr},
    {"rk_full_attn", (PyCFunction)(void (*)(void))full_attn, METH_FASTCALL, nullptr},
    {"rk_rope_append", (PyCFunction)(void (*)(void))rope_append<0>, METH_FASTCALL, nullptr},
    {"rk_rope_append_q8", (PyCFunction)(void (*)(void))rope_append<1>, METH_FASTCALL, nullptr},
    {"rk_full_attn_q8", (PyCFunction)(void (*)(void))full_attn_q8, METH_FASTCALL, nullptr},
    {"rk_gather_small_kv_q8", (PyCFunction)(void (*)(void))gather_q8, METH_FASTCALL, nullptr},
    {"rk_prompt_attn", (PyCFunction)(void (*)(void))prompt_attn, METH_FASTCALL, nullptr},
    {"rk_rope_append_paged", (PyCFunction)(void (*)(void))rope_append<2>, METH_FASTCALL, nullptr},
    {"rk_paged_attn", (PyCFunction)(void (*)(void))paged_attn, METH_FASTCALL, nullptr},
    {"rk_prefix_attn", (PyCFunction)(void (*)(void))prefix_attn, METH_FASTCALL, nullptr},
    {"rk_page_scores", (PyCFunction)(void (*)(void))page_scores, METH_FASTCALL, nullptr},
    {"rk_page_select", (PyCFunction)(void (*)(void))page_select, METH_FASTCALL, nullptr},
    {"rk_sparse_attn", (PyCFunction)(void (*)(void))sparse_attn, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rkbind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rkbind() { return PyModule_Create(&module); }
