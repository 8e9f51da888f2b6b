// The marshalling of binding.py's calls, as a CPython module: a call of the C ABI from Python spent 5 us on its arguments (two
// method calls per tensor from bytecode, ctypes' conversions, the current stream through two layers of Python) next to some 2 us
// for the launch itself, which is what a decode step of one layer, whose kernel takes 4 us, or a frame's dozen small calls
// then waited for.  The same steps here take about 1 us.
//
// Each function takes the positional arguments of the Python function of its name, asks tensors for is_contiguous() and
// data_ptr() (as Python code does, so whatever overrides them still does) and calls the library with the GIL released.  It
// returns the status, or None if some argument is not of the plain kind (an exact Shape, a tensor, a RowsFrom, an int that fits,
// None): then, and before torch has initialised the GPU or the library is loaded, binding.py marshals through ctypes, which
// says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stddef.h>
#include <stdint.h>

#include "../../include/kvev.h"

namespace {

// bound once by binding.py: types, what the current stream is asked of, and the library's entry points
PyObject *g_shape_type, *g_rows_type, *g_tensor_type, *g_initialized, *g_get_device, *g_raw_stream;
PyObject *g_pages_type, *g_axes_type, *g_f32, *g_bf16, *g_i32, *g_u8;       // (bind_pages)
PyObject *s_is_contiguous, *s_data_ptr, *s_numel, *s_ptr, *s_dtype, *s_get_device;

enum Entry { kPool, kGate, kGatePrepared, kSelect, kGated, kDense, kRetain, kCompact, kPoolBytes, kAppend, kRead, kPageAttn, kReserve, kFork, kTrim, kCopy, kCompactPages, kRotary, kEntries };
const char *const kNames[kEntries] = {"kvev_chunk_pool", "kvev_lstm_gate", "kvev_lstm_gate_prepared", "kvev_select",
                                      "kvev_gated_attention", "kvev_dense_attention", "kvev_retain", "kvev_compact_attention",
                                      "kvev_page_pool_bytes", "kvev_page_append", "kvev_page_read", "kvev_page_attention",
                                      "kvev_pages_reserve", "kvev_pages_fork", "kvev_pages_trim", "kvev_pages_copy", "kvev_pages_compact",
                                      "kvev_rotary"};
void *g_entry[kEntries];

// Arguments are read one after the other; the first that is not plain leaves `plain` false, an exception leaves `error` true,
// and either turns the rest into no-ops.
struct Reader {
    PyObject *const *args;
    Py_ssize_t n, at = 0;
    bool plain = true, error = false;
    Py_buffer shape_view{}, more_view[2]{};
    bool has_view = false;
    int more_views = 0;
    long device = -1;                      // current device, once stream() was asked

    Reader(PyObject *const *a, Py_ssize_t count, Py_ssize_t want) : args(a), n(count) { plain = g_shape_type && count == want; }
    Reader(const Reader &) = delete;
    ~Reader()
    {
        if (has_view) PyBuffer_Release(&shape_view);
        while (more_views > 0) PyBuffer_Release(&more_view[--more_views]);
    }
    bool ok() const { return plain && !error; }
    PyObject *next() { return args[at++]; }

    const kvev_shape *shape()
    {
        if (!ok()) return nullptr;
        PyObject *o = next();
        if ((PyObject *)Py_TYPE(o) != g_shape_type) { plain = false; return nullptr; }
        if (PyObject_GetBuffer(o, &shape_view, PyBUF_SIMPLE) != 0) { error = true; return nullptr; }
        has_view = true;
        if ((size_t)shape_view.len < sizeof(kvev_shape)) { plain = false; return nullptr; }
        return static_cast<const kvev_shape *>(shape_view.buf);
    }
    // a struct that goes with the shape (kvev_pages, kvev_rotary_axes; two at most)
    template <class S> const S *more(PyObject *type)
    {
        if (!ok()) return nullptr;
        PyObject *o = next();
        if (!type || (PyObject *)Py_TYPE(o) != type) { plain = false; return nullptr; }
        Py_buffer &view = more_view[more_views];
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) { error = true; return nullptr; }
        ++more_views;
        if ((size_t)view.len < sizeof(S)) { plain = false; return nullptr; }
        return static_cast<const S *>(view.buf);
    }
    // a contiguous tensor of at least `least` elements of `dtype` on the current device (after stream()); what is not is left to
    // binding.py, which says so
    void *array(PyObject *dtype, size_t least, bool optional = false)
    {
        if (!ok()) return nullptr;
        PyObject *o = next();
        if (o == Py_None && optional) return nullptr;
        if (!dtype || !PyObject_TypeCheck(o, (PyTypeObject *)g_tensor_type)) { plain = false; return nullptr; }
        PyObject *t = PyObject_GetAttr(o, s_dtype);
        if (!t) { error = true; return nullptr; }
        const bool same = t == dtype;
        Py_DECREF(t);
        if (!same) { plain = false; return nullptr; }
        if (ask(o, s_numel) < least && ok()) plain = false;
        if (!ok()) return nullptr;
        PyObject *d = PyObject_VectorcallMethod(s_get_device, &o, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!d) { error = true; return nullptr; }
        const long at = PyLong_Check(d) ? PyLong_AsLong(d) : -1;
        Py_DECREF(d);
        if (at == -1 && PyErr_Occurred()) PyErr_Clear();
        if (at < 0 || at != device) { plain = false; return nullptr; }
        return address(o, true);
    }
    int integer()
    {
        if (!ok()) return 0;
        PyObject *o = next();
        if (!PyLong_Check(o)) { plain = false; return 0; }
        int over = 0;
        const long v = PyLong_AsLongAndOverflow(o, &over);
        if (over || v > INT32_MAX || v < INT32_MIN) { plain = false; return 0; }
        return (int)v;
    }
    float real()
    {
        if (!ok()) return 0.f;
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); plain = false; return 0.f; }
        return (float)v;
    }
    // o.name() as a non-negative integer
    size_t ask(PyObject *o, PyObject *name)
    {
        PyObject *r = PyObject_VectorcallMethod(name, &o, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { error = true; return 0; }
        size_t v = 0;
        if (PyLong_Check(r)) {
            v = PyLong_AsSize_t(r);
            if (v == (size_t)-1 && PyErr_Occurred()) { PyErr_Clear(); plain = false; }
        } else {
            plain = false;
        }
        Py_DECREF(r);
        return v;
    }
    void *address(PyObject *o, bool check)
    {
        if (!ok() || o == Py_None) return nullptr;
        if (!PyObject_TypeCheck(o, (PyTypeObject *)g_tensor_type)) {
            if ((PyObject *)Py_TYPE(o) != g_rows_type || !check) { plain = false; return nullptr; }
            PyObject *p = PyObject_GetAttr(o, s_ptr);
            if (!p) { error = true; return nullptr; }
            void *v = PyLong_Check(p) ? (void *)PyLong_AsSize_t(p) : nullptr;
            if (!PyLong_Check(p) || PyErr_Occurred()) { PyErr_Clear(); plain = false; }
            Py_DECREF(p);
            return v;
        }
        if (check) {
            PyObject *c = PyObject_VectorcallMethod(s_is_contiguous, &o, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
            if (!c) { error = true; return nullptr; }
            const int yes = PyObject_IsTrue(c);
            Py_DECREF(c);
            if (yes < 0) { error = true; return nullptr; }
            if (!yes) {
                PyErr_SetString(PyExc_AssertionError, "kvev takes contiguous tensors");
                error = true;
                return nullptr;
            }
        }
        return (void *)ask(o, s_data_ptr);
    }
    void *tensor() { return ok() ? address(next(), true) : nullptr; }
    // a scratch tensor (or None) and its size
    void *scratch(size_t &bytes)
    {
        bytes = 0;
        if (!ok()) return nullptr;
        PyObject *o = next();
        if (o == Py_None) return nullptr;
        if (!PyObject_TypeCheck(o, (PyTypeObject *)g_tensor_type)) { plain = false; return nullptr; }
        void *p = address(o, true);
        if (ok()) bytes = ask(o, s_numel);
        return p;
    }
    // a tuple of `count` tensors, whose addresses go to consecutive fields of `out` (false: None stood in its place)
    bool weights(const void **out, Py_ssize_t count, bool may_be_none)
    {
        if (!ok()) return false;
        PyObject *o = next();
        if (o == Py_None && may_be_none) return false;
        if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != count) { plain = false; return false; }
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject *t = PyTuple_GET_ITEM(o, i);
            if (t == Py_None) { plain = false; return false; }
            out[i] = address(t, false);
        }
        return true;
    }
    // torch's current stream
    void *stream()
    {
        if (!ok()) return nullptr;
        PyObject *up = PyObject_CallNoArgs(g_initialized);      // (asked of torch: the flag behind it stays set in a forked child)
        if (!up) { error = true; return nullptr; }
        const bool is_up = up == Py_True;
        Py_DECREF(up);
        if (!is_up) { plain = false; return nullptr; }
        PyObject *dev = PyObject_CallNoArgs(g_get_device);
        if (!dev) { error = true; return nullptr; }
        device = PyLong_Check(dev) ? PyLong_AsLong(dev) : -1;
        if (device == -1 && PyErr_Occurred()) PyErr_Clear();
        PyObject *r = PyObject_CallOneArg(g_raw_stream, dev);
        Py_DECREF(dev);
        if (!r) { error = true; return nullptr; }
        void *v = (void *)PyLong_AsSize_t(r);
        if (PyErr_Occurred()) { PyErr_Clear(); plain = false; }
        Py_DECREF(r);
        return v;
    }
    template <class F> PyObject *run(F &&call)
    {
        if (error) return nullptr;
        if (!plain) Py_RETURN_NONE;
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    }
};

template <class F> F entry(Entry e, F) { return reinterpret_cast<F>(g_entry[e]); }
#define ENTRY(e, fn) entry(e, static_cast<decltype(&fn)>(nullptr))

PyObject *chunk_pool(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 11);
    const kvev_shape *sh = r.shape();
    void *K = r.tensor(), *V = r.tensor();
    const int mode = r.integer();
    kvev_mlp_w wK{}, wV{};
    static_assert(sizeof(kvev_mlp_w) == 4 * sizeof(void *) && sizeof(kvev_lstm_w) == 6 * sizeof(void *), "addresses in a row");
    const bool hasK = r.weights(reinterpret_cast<const void **>(&wK), 4, true), hasV = r.weights(reinterpret_cast<const void **>(&wV), 4, true);
    const int c0 = r.integer(), c1 = r.integer();
    void *Kb = r.tensor(), *Vb = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes), *st = r.stream();
    return r.run([&] { return ENTRY(kPool, kvev_chunk_pool)(sh, K, V, mode, hasK ? &wK : nullptr, hasV ? &wV : nullptr, c0, c1, Kb, Vb, ws, bytes, st); });
}

PyObject *lstm_gate(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 11);
    const kvev_shape *sh = r.shape();
    void *Kb = r.tensor(), *Vb = r.tensor();
    kvev_lstm_w w{};
    r.weights(reinterpret_cast<const void **>(&w), 6, false);
    const int c0 = r.integer(), c1 = r.integer();
    void *h = r.tensor(), *c = r.tensor(), *util = r.tensor(), *gate = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes), *st = r.stream();
    return r.run([&] { return ENTRY(kGate, kvev_lstm_gate)(sh, Kb, Vb, &w, c0, c1, (float *)h, (float *)c, (float *)util, (float *)gate, ws, bytes, st); });
}

PyObject *lstm_gate_prepared(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 12);
    const kvev_shape *sh = r.shape();
    void *Kb = r.tensor(), *Vb = r.tensor();
    kvev_lstm_w w{};
    r.weights(reinterpret_cast<const void **>(&w), 6, false);
    size_t pbytes;
    void *packed = r.scratch(pbytes);
    const int c0 = r.integer(), c1 = r.integer();
    void *h = r.tensor(), *c = r.tensor(), *util = r.tensor(), *gate = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes), *st = r.stream();
    return r.run([&] {
        return ENTRY(kGatePrepared, kvev_lstm_gate_prepared)(sh, Kb, Vb, &w, packed, pbytes, c0, c1, (float *)h, (float *)c, (float *)util, (float *)gate, ws, bytes, st);
    });
}

PyObject *select_(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 9);
    const kvev_shape *sh = r.shape();
    void *util = r.tensor(), *gate = r.tensor();
    const int mode = r.integer(), k = r.integer();
    const float tau = r.real();
    const int k_cap = r.integer();
    void *idx = r.tensor(), *count = r.tensor(), *st = r.stream();
    return r.run([&] { return ENTRY(kSelect, kvev_select)(sh, (float *)util, (float *)gate, mode, k, tau, k_cap, (int32_t *)idx, (int32_t *)count, st); });
}

PyObject *gated_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 13);
    const kvev_shape *sh = r.shape();
    void *Q = r.tensor();
    const int Tq = r.integer();
    void *K = r.tensor(), *V = r.tensor(), *Kb = r.tensor(), *Vb = r.tensor(), *idx = r.tensor(), *count = r.tensor();
    const int k_cap = r.integer();
    void *O = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes);
    const int causal = r.integer();
    void *st = r.stream();
    return r.run([&] { return ENTRY(kGated, kvev_gated_attention)(sh, Q, Tq, K, V, Kb, Vb, (int32_t *)idx, (int32_t *)count, k_cap, causal, O, ws, bytes, st); });
}

PyObject *dense_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 8);
    const kvev_shape *sh = r.shape();
    void *Q = r.tensor();
    const int Tq = r.integer();
    void *K = r.tensor(), *V = r.tensor(), *O = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes);
    const int causal = r.integer();
    void *st = r.stream();
    return r.run([&] { return ENTRY(kDense, kvev_dense_attention)(sh, Q, Tq, K, V, causal, O, ws, bytes, st); });
}

PyObject *retain(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 14);
    const kvev_shape *sh = r.shape();
    const int k = r.integer(), k_cap = r.integer();
    void *Kn = r.tensor(), *Vn = r.tensor(), *un = r.tensor();
    const int cap = r.integer(), first = r.integer(), m = r.integer();
    void *Kc = r.tensor(), *Vc = r.tensor(), *ids = r.tensor(), *uc = r.tensor(), *count = r.tensor(), *st = r.stream();
    return r.run([&] {
        return ENTRY(kRetain, kvev_retain)(sh, k, k_cap, Kn, Vn, (float *)un, cap, first, m, Kc, Vc, (int32_t *)ids, (float *)uc, (int32_t *)count, st);
    });
}

PyObject *compact_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Reader r(args, n, 13);
    const kvev_shape *sh = r.shape();
    void *Q = r.tensor();
    const int Tq = r.integer();
    void *Kw = r.tensor(), *Vw = r.tensor(), *Kc = r.tensor(), *Vc = r.tensor(), *count = r.tensor();
    const int k_cap = r.integer();
    void *O = r.tensor();
    size_t bytes;
    void *ws = r.scratch(bytes);
    const int causal = r.integer(), first = r.integer();
    void *st = r.stream();
    return r.run([&] { return ENTRY(kCompact, kvev_compact_attention)(sh, Q, Tq, Kw, Vw, first, Kc, Vc, (int32_t *)count, k_cap, causal, O, ws, bytes, st); });
}

// ---- the paged cache: its calls check sizes, element types and device as well ----
struct PageReader : Reader {
    void *st;
    const kvev_shape *sh;
    const kvev_pages *pg = nullptr;

    PageReader(PyObject *const *a, Py_ssize_t n, Py_ssize_t want) : Reader(a, n, want)
    {
        st = stream();
        sh = shape();
    }
    const kvev_pages *pages() { return pg = more<kvev_pages>(g_pages_type); }
    int heads() { return sh->H_kv > 0 ? sh->H_kv : sh->H; }
    // a product of counts; what no tensor has if one is negative (the library then says what is wrong) or it is too large
    static size_t product(const long long (&v)[5])
    {
        unsigned __int128 p = 1;
        for (long long x : v) {
            if (x < 0) return SIZE_MAX;
            p *= (unsigned long long)x;
            if (p > SIZE_MAX / 4) return SIZE_MAX;
        }
        return (size_t)p;
    }
    void *ints(long long n, bool optional = false) { return array(g_i32, n < 0 ? SIZE_MAX : (size_t)n, optional); }
    void *rows(int h, int n, bool optional = false)
    {
        if (!ok()) return nullptr;
        return array(sh->dtype == KVEV_F32 ? g_f32 : sh->dtype == KVEV_BF16 ? g_bf16 : nullptr, product({sh->L, sh->B, h, n, sh->d}), optional);
    }
    void *table() { return ok() ? ints((long long)sh->B * pg->max_pages) : nullptr; }
    void *batch(bool optional = false) { return ok() ? ints(sh->B, optional) : nullptr; }
    void *refs() { return ok() ? ints(pg->n_pages) : nullptr; }
    void *pool() { return ok() ? array(g_u8, ENTRY(kPoolBytes, kvev_page_pool_bytes)(sh, pg)) : nullptr; }
    void *bytes(size_t &n)
    {
        n = 0;
        if (!ok()) return nullptr;
        PyObject *o = args[at];
        void *p = array(g_u8, 0, true);
        if (ok() && p) n = ask(o, s_numel);
        return p;
    }
};

PyObject *page_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 9);
    if (!r.pages()) return r.run([] { return 0; });
    const Py_ssize_t tensors = r.at;         // (their size is known once Tn is)
    r.at += 2;
    const int Tn = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = tensors;
    void *K = r.ok() ? r.rows(r.heads(), Tn) : nullptr, *V = r.ok() ? r.rows(r.heads(), Tn) : nullptr;
    r.at = rest;
    void *start = r.batch(), *n_new = r.batch(true), *table = r.table(), *pool = r.pool();
    return r.run([&] { return ENTRY(kAppend, kvev_page_append)(r.sh, r.pg, K, V, Tn, (int32_t *)start, (int32_t *)n_new, (int32_t *)table, pool, r.st); });
}

PyObject *page_read(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 9);
    if (!r.pages()) return r.run([] { return 0; });
    void *pool = r.pool(), *table = r.table(), *first = r.batch(), *count = r.batch(true);
    const int Tn = r.integer();
    void *K = r.ok() ? r.rows(r.heads(), Tn) : nullptr, *V = r.ok() ? r.rows(r.heads(), Tn) : nullptr;
    return r.run([&] { return ENTRY(kRead, kvev_page_read)(r.sh, r.pg, pool, (int32_t *)table, (int32_t *)first, (int32_t *)count, Tn, K, V, r.st); });
}

PyObject *page_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 15);
    if (!r.pages()) return r.run([] { return 0; });
    const Py_ssize_t q_at = r.at++;
    const int Tq = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = q_at;
    void *Q = r.ok() ? r.rows(r.sh->H, Tq) : nullptr;
    r.at = n - 1;
    const int k_cap = r.integer();
    r.at = rest;
    void *pool = r.pool(), *table = r.table(), *length = r.batch(), *O = r.ok() ? r.rows(r.sh->H, Tq) : nullptr;
    size_t bytes;
    void *ws = r.bytes(bytes), *first = r.batch(true), *q_start = r.batch(true);
    const bool none = k_cap == 0;
    void *Kc = r.ok() ? r.rows(r.heads(), k_cap, none) : nullptr, *Vc = r.ok() ? r.rows(r.heads(), k_cap, none) : nullptr;
    void *count = r.ok() ? r.ints((long long)r.sh->L * r.sh->B * r.heads(), none) : nullptr;
    return r.run([&] {
        return ENTRY(kPageAttn, kvev_page_attention)(r.sh, r.pg, Q, Tq, pool, (int32_t *)table, (int32_t *)length, (int32_t *)first, (int32_t *)q_start, Kc, Vc,
                                                     (int32_t *)count, k_cap, O, ws, bytes, r.st);
    });
}

PyObject *pages_reserve(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 10);
    if (!r.pages()) return r.run([] { return 0; });
    void *n_new = r.batch(), *table = r.table(), *length = r.batch(), *refs = r.refs(), *pool = r.pool(), *start = r.batch(), *status = r.ints(1);
    size_t bytes;
    void *ws = r.bytes(bytes);
    return r.run([&] {
        return ENTRY(kReserve, kvev_pages_reserve)(r.sh, r.pg, (int32_t *)n_new, (int32_t *)table, (int32_t *)length, (int32_t *)refs, pool, (int32_t *)start,
                                                   (int32_t *)status, ws, bytes, r.st);
    });
}

PyObject *pages_fork(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 9);
    if (!r.pages()) return r.run([] { return 0; });
    const Py_ssize_t lists = r.at;
    r.at += 2;
    const int count = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = lists;
    void *src = r.ints(count), *dst = r.ints(count);
    r.at = rest;
    void *table = r.table(), *length = r.batch(), *refs = r.refs(), *status = r.ints(1);
    return r.run([&] {
        return ENTRY(kFork, kvev_pages_fork)(r.sh, r.pg, (int32_t *)src, (int32_t *)dst, count, (int32_t *)table, (int32_t *)length, (int32_t *)refs, (int32_t *)status, r.st);
    });
}

PyObject *pages_trim(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 9);
    if (!r.pages()) return r.run([] { return 0; });
    const Py_ssize_t list = r.at++;
    const int count = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = list;
    void *rows = r.ints(count, true);
    r.at = rest;
    void *first = r.ints(count, true), *keep = r.ints(count, true), *table = r.table(), *length = r.batch(), *refs = r.refs();
    return r.run([&] {
        return ENTRY(kTrim, kvev_pages_trim)(r.sh, r.pg, (int32_t *)rows, count, (int32_t *)first, (int32_t *)keep, (int32_t *)table, (int32_t *)length, (int32_t *)refs, r.st);
    });
}

PyObject *pages_copy(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 7);
    if (!r.pages()) return r.run([] { return 0; });
    void *pool = r.pool();
    const Py_ssize_t lists = r.at;
    r.at += 2;
    const int count = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = lists;
    void *src = r.ints(count), *dst = r.ints(count);
    r.at = rest;
    void *status = r.ints(1);
    return r.run([&] { return ENTRY(kCopy, kvev_pages_copy)(r.sh, r.pg, pool, (int32_t *)src, (int32_t *)dst, count, (int32_t *)status, r.st); });
}

PyObject *pages_compact(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 11);
    if (!r.pages()) return r.run([] { return 0; });
    const kvev_pages *from = r.pg;
    void *pool = r.pool(), *table = r.table(), *refs = r.refs();
    const kvev_pages *to = r.more<kvev_pages>(g_pages_type);
    if (!to) return r.run([] { return 0; });
    r.pg = to;
    void *to_pool = r.pool();
    r.pg = from;
    void *to_table = r.table(), *to_refs = r.ints(to->n_pages), *status = r.ints(1);
    size_t bytes;
    void *ws = r.bytes(bytes);
    return r.run([&] {
        return ENTRY(kCompactPages, kvev_pages_compact)(r.sh, from, pool, (int32_t *)table, (int32_t *)refs, to, to_pool, (int32_t *)to_table, (int32_t *)to_refs,
                                                        (int32_t *)status, ws, bytes, r.st);
    });
}

PyObject *rotary(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    PageReader r(args, n, 10);
    const kvev_rotary_axes *ax = r.more<kvev_rotary_axes>(g_axes_type);
    if (!ax) return r.run([] { return 0; });
    long long pairs = 0;
    for (int i = 0; i < ax->n_axes && i < 4; ++i) pairs += ax->section[i];
    const Py_ssize_t front = r.at;
    r.at += 2;
    const int Tq = r.integer();
    const Py_ssize_t rest = r.at;
    r.at = front;
    void *freq = r.array(g_f32, pairs < 0 ? SIZE_MAX : (size_t)pairs);
    void *pos = r.ok() ? r.array(g_i32, PageReader::product({ax->n_axes, r.sh->B, Tq, 1, 1})) : nullptr;
    r.at = rest;
    void *Q = r.ok() ? r.rows(r.sh->H, Tq, true) : nullptr, *K = r.ok() ? r.rows(r.heads(), Tq, true) : nullptr;
    void *Qo = r.ok() ? r.rows(r.sh->H, Tq, true) : nullptr, *Ko = r.ok() ? r.rows(r.heads(), Tq, true) : nullptr;
    const int inverse = r.integer();
    return r.run([&] { return ENTRY(kRotary, kvev_rotary)(r.sh, ax, (float *)freq, (int32_t *)pos, Tq, Q, K, Qo, Ko, inverse, r.st); });
}

// bind_pages(Pages, RotaryAxes, float32, bfloat16, int32, uint8), before bind
PyObject *bind_pages(PyObject *, PyObject *args)
{
    PyObject *pages, *axes, *f32, *bf16, *i32, *u8;
    if (!PyArg_ParseTuple(args, "O!O!OOOO", &PyType_Type, &pages, &PyType_Type, &axes, &f32, &bf16, &i32, &u8)) return nullptr;
    Py_INCREF(pages); Py_INCREF(axes); Py_INCREF(f32); Py_INCREF(bf16); Py_INCREF(i32); Py_INCREF(u8);
    g_pages_type = pages; g_axes_type = axes; g_f32 = f32; g_bf16 = bf16; g_i32 = i32; g_u8 = u8;
    Py_RETURN_NONE;
}

// bind(Shape, RowsFrom, Tensor, is_initialized, get_device, raw_stream, {name: address})
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *shape, *rows, *tensor, *up, *dev, *raw, *entries;
    if (!PyArg_ParseTuple(args, "O!O!O!OOOO!", &PyType_Type, &shape, &PyType_Type, &rows, &PyType_Type, &tensor, &up, &dev, &raw, &PyDict_Type, &entries))
        return nullptr;
    void *found[kEntries];
    for (int e = 0; e < kEntries; ++e) {
        PyObject *a = PyDict_GetItemString(entries, kNames[e]);
        if (!a) return PyErr_Format(PyExc_KeyError, "%s", kNames[e]);
        found[e] = PyLong_AsVoidPtr(a);
        if (PyErr_Occurred()) return nullptr;
    }
    for (int e = 0; e < kEntries; ++e) g_entry[e] = found[e];
    Py_INCREF(rows); Py_INCREF(tensor); Py_INCREF(up); Py_INCREF(dev); Py_INCREF(raw); Py_INCREF(shape);
    g_rows_type = rows; g_tensor_type = tensor; g_initialized = up; g_get_device = dev; g_raw_stream = raw;
    g_shape_type = shape;           // (the last one: its presence says that all are there)
    Py_RETURN_NONE;
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    FAST("chunk_pool", chunk_pool), FAST("lstm_gate", lstm_gate), FAST("lstm_gate_prepared", lstm_gate_prepared), FAST("select", select_),
    FAST("gated_attention", gated_attention), FAST("dense_attention", dense_attention), FAST("retain", retain),
    FAST("compact_attention", compact_attention), FAST("page_append", page_append), FAST("page_read", page_read),
    FAST("page_attention", page_attention), FAST("pages_reserve", pages_reserve), FAST("pages_fork", pages_fork), FAST("pages_trim", pages_trim),
    FAST("pages_copy", pages_copy), FAST("pages_compact", pages_compact), FAST("rotary", rotary), {"bind_pages", bind_pages, METH_VARARGS, nullptr}, {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", "Marshalling of calls into libkvev.so.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_ptr = PyUnicode_InternFromString("ptr");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    if (!s_is_contiguous || !s_data_ptr || !s_numel || !s_ptr || !s_dtype || !s_get_device) return nullptr;
    return PyModule_Create(&g_module);
}
