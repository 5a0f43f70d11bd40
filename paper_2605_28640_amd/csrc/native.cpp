// The per-token calls of the binding (append, decode, replayable step, those around a pool of pages, a 4-bit cache and eviction) with their arguments taken apart in C++: ctypes and a
// Python function per tensor cost the host more than the launch itself.  Only arguments of exactly the types that a program
// ordinarily passes are taken here: rs_shape, contiguous device tensors (torch.Tensor or Parameter) or None, int, float, Workspace.
// Anything else leaves the call unmade and the function answers False: binding.py then makes it through ctypes, which
// accepts, converts or refuses the argument as for every other function of the library.
// The library's functions come in as addresses (setup), so this module links against Python and torch only.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <initializer_list>

#include "../../include/ratsparse.h"

namespace {

decltype(&rat_scan) f_scan;
decltype(&sparse_attn_decode) f_decode;
decltype(&rat_decode_step) f_step;
decltype(&page_pool_reserve) f_reserve;
decltype(&page_pool_fork) f_fork;
decltype(&page_pool_free) f_free;
decltype(&page_pool_compact) f_compact;
decltype(&page_pool_share) f_share;
decltype(&page_copy) f_copy;
decltype(&rat_state_copy) f_state;
decltype(&rat_append_paged) f_append;
decltype(&attn_paged) f_attn;
decltype(&kv4_append) f_kv4_append;
decltype(&kv4_page_meta) f_kv4_meta;
decltype(&kv4_fetch) f_kv4_fetch;
decltype(&kv4_attn_decode) f_kv4_attn;
decltype(&attn_decode_tally) f_tally;
decltype(&cache_evict) f_evict;
decltype(&kv4_evict) f_kv4_evict;
PyObject *g_check, *g_stream_of, *g_device, *g_shape, *g_workspace;  // binding._check, torch's two, binding.rs_shape, .Workspace
PyObject *g_pool;                                                    // binding.rs_pool
PyObject *s_buf;

// One call's arguments.  A getter that meets something else than its plain type clears `plain` and raises nothing.
struct Args {
    PyObject *const *a;
    bool plain = true;

    void *refuse()
    {
        plain = false;
        return nullptr;
    }
    // a device tensor's address; None: null
    void *tensor(int i)
    {
        PyObject *o = a[i];
        if (o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) return refuse();
        try {
            const at::Tensor &t = THPVariable_Unpack(o);
            return t.is_cuda() && t.is_contiguous() ? t.data_ptr() : refuse();
        } catch (const std::exception &) {
            return refuse();
        }
    }
    // the low bits of an int, as ctypes takes them
    int64_t integer(int i)
    {
        if (PyLong_Check(a[i])) return (int64_t)PyLong_AsUnsignedLongLongMask(a[i]);
        refuse();
        return 0;
    }
    float real(int i)
    {
        if (PyFloat_Check(a[i])) return (float)PyFloat_AS_DOUBLE(a[i]);
        refuse();
        return 0.f;
    }
    // a device tensor of this type and shape, all of a call's on one device; None: null
    int device = -1;
    void *typed(int i, at::ScalarType type, std::initializer_list<int64_t> sizes)
    {
        if (a[i] == Py_None) return nullptr;
        void *p = tensor(i);
        if (!plain) return nullptr;
        try {
            const at::Tensor &t = THPVariable_Unpack(a[i]);
            const int d = (int)t.get_device();
            if (t.scalar_type() != type || t.sizes() != at::IntArrayRef(sizes) || (device >= 0 && d != device)) return refuse();
            device = d;
        } catch (const std::exception &) {
            return refuse();
        }
        return p;
    }
    int32_t *ints(int i, std::initializer_list<int64_t> sizes) { return (int32_t *)typed(i, at::kInt, sizes); }
    // a dimension of a tensor; -1: no tensor
    int64_t size(int i, int d)
    {
        if (!THPVariable_CheckExact(a[i])) return refuse(), -1;
        try {
            const at::Tensor &t = THPVariable_Unpack(a[i]);
            return t.dim() > d ? t.size(d) : (refuse(), -1);
        } catch (const std::exception &) {
            return refuse(), -1;
        }
    }
    // a ctypes structure: it exports its memory
    template <typename S>
    S structure(int i, PyObject *type)
    {
        S s = {};
        Py_buffer b;
        if ((PyObject *)Py_TYPE(a[i]) != type) {
            refuse();
        } else if (PyObject_GetBuffer(a[i], &b, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            refuse();
        } else {
            if (b.len == (Py_ssize_t)sizeof(s)) memcpy(&s, b.buf, sizeof(s));
            else refuse();
            PyBuffer_Release(&b);
        }
        return s;
    }
    rs_shape shape(int i) { return structure<rs_shape>(i, g_shape); }
    rs_pool pool(int i) { return structure<rs_pool>(i, g_pool); }
    // a workspace's buffer, on the device of the typed tensors before it
    void *workspace(int i, size_t &bytes)
    {
        bytes = 0;
        if ((PyObject *)Py_TYPE(a[i]) != g_workspace) return refuse();
        PyObject *buf = PyObject_GetAttr(a[i], s_buf);
        void *p = nullptr;
        if (buf && THPVariable_CheckExact(buf)) {
            try {
                const at::Tensor &t = THPVariable_Unpack(buf);
                const int d = (int)t.get_device();
                if (!t.is_cuda() || (device >= 0 && d != device)) {
                    refuse();
                } else {
                    p = t.data_ptr();
                    bytes = (size_t)t.numel();
                }
            } catch (const std::exception &) {
                refuse();
            }
        } else {
            PyErr_Clear();
            refuse();
        }
        Py_XDECREF(buf);
        return p;
    }
};

// the current stream of the current device (on: its number); false: a Python exception
bool stream(void *&s, int *on = nullptr)
{
    PyObject *dev = PyObject_CallNoArgs(g_device);
    if (dev && on) *on = (int)PyLong_AsLong(dev);
    PyObject *r = dev ? PyObject_CallOneArg(g_stream_of, dev) : nullptr;
    Py_XDECREF(dev);
    if (!r) return false;
    s = (void *)PyLong_AsUnsignedLongLongMask(r);
    Py_DECREF(r);
    return !PyErr_Occurred();
}

// True; or the exception that binding._check raises for a status
PyObject *done(int status)
{
    if (status != 0) {
        PyObject *code = PyLong_FromLong(status);
        PyObject *r = code ? PyObject_CallOneArg(g_check, code) : nullptr;
        Py_XDECREF(code);
        if (!r) return nullptr;
        Py_DECREF(r);
    }
    Py_RETURN_TRUE;
}

bool expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
    return false;
}

PyObject *py_rat_scan(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 12)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    void *k = x.tensor(1), *v = x.tensor(2), *g = x.tensor(3), *sk = x.tensor(4), *sv = x.tensor(5), *kc = x.tensor(6),
         *vc = x.tensor(7), *meta = x.tensor(11);
    const int64_t t0 = x.integer(8), T = x.integer(9);
    size_t nb = 0;
    void *ws = a[10] == Py_None ? nullptr : x.workspace(10, nb), *st = nullptr;  // (a run may do without)
    if (!x.plain) Py_RETURN_FALSE;
    if (!stream(st)) return nullptr;
    int r;
    Py_BEGIN_ALLOW_THREADS
    r = f_scan(&s, k, v, (const float *)g, (float *)sk, (float *)sv, kc, vc, meta, t0, T, ws, nb, st);
    Py_END_ALLOW_THREADS
    return done(r);
}

PyObject *py_sparse_attn_decode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 15)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    void *q = x.tensor(1), *kc = x.tensor(2), *vc = x.tensor(3), *idx = x.tensor(6), *meta = x.tensor(8), *out = x.tensor(11),
         *lse = x.tensor(12), *idx_out = x.tensor(13);
    const int64_t T = x.integer(4);
    const float scale = x.real(5);
    const int K = (int)x.integer(7), n_first = (int)x.integer(9), n_local = (int)x.integer(10);
    size_t nb = 0;
    void *ws = x.workspace(14, nb), *st = nullptr;
    if (!x.plain) Py_RETURN_FALSE;
    if (!stream(st)) return nullptr;
    int r;
    Py_BEGIN_ALLOW_THREADS
    r = f_decode(&s, q, kc, vc, T, scale, (const int32_t *)idx, K, meta, n_first, n_local, out, (float *)lse, (int32_t *)idx_out, ws, nb, st);
    Py_END_ALLOW_THREADS
    return done(r);
}

PyObject *py_rat_decode_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 19)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    void *k = x.tensor(1), *v = x.tensor(2), *g = x.tensor(3), *sk = x.tensor(4), *sv = x.tensor(5), *kc = x.tensor(6),
         *vc = x.tensor(7), *meta = x.tensor(8), *q = x.tensor(9), *out = x.tensor(15), *lse = x.tensor(16), *idx_out = x.tensor(17);
    const float scale = x.real(10);
    const int K = (int)x.integer(11), n_first = (int)x.integer(12), n_local = (int)x.integer(13);
    const int64_t T_max = x.integer(14);
    size_t nb = 0;
    void *ws = x.workspace(18, nb), *st = nullptr;
    if (!x.plain) Py_RETURN_FALSE;
    if (!stream(st)) return nullptr;
    int r;
    Py_BEGIN_ALLOW_THREADS
    r = f_step(&s, k, v, (const float *)g, (float *)sk, (float *)sv, kc, vc, meta, q, scale, K, n_first, n_local, T_max, out, (float *)lse,
               (int32_t *)idx_out, ws, nb, st);
    Py_END_ALLOW_THREADS
    return done(r);
}

// ---- the calls around a pool of pages: also the shapes and types are looked at here, anything unexpected being left to binding.py ----
at::ScalarType type_of(const rs_shape &s) { return s.dtype == RS_BF16 ? at::kBFloat16 : at::kFloat; }

// runs f(stream) where everything is plain and on the current device
template <typename F>
PyObject *run(const Args &x, F f)
{
    void *st = nullptr;
    int on = -1;
    if (!x.plain) Py_RETURN_FALSE;
    if (!stream(st, &on)) return nullptr;
    if (x.device >= 0 && x.device != on) Py_RETURN_FALSE;
    int r;
    Py_BEGIN_ALLOW_THREADS
    r = f(st);
    Py_END_ALLOW_THREADS
    return done(r);
}
struct Sequences {
    int32_t *table, *len, *refs;
};
Sequences sequences(Args &x, const rs_pool &p, int i) { return Sequences{x.ints(i, {p.S, p.M}), x.ints(i + 1, {p.S}), x.ints(i + 2, {p.N})}; }
struct Rows {
    void *k, *v, *meta;
};
Rows rows(Args &x, const rs_shape &s, int i)
{
    const at::ScalarType dt = type_of(s);
    const int64_t P = s.P > 0 ? s.P : 1;
    return Rows{x.typed(i, dt, {s.Hkv, s.Tcap, s.D}), x.typed(i + 1, dt, {s.Hkv, s.Tcap, s.D}), x.typed(i + 2, dt, {s.Hkv, s.Tcap / P, 2, s.D})};
}

PyObject *py_page_pool_reserve(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 9)) return nullptr;
    Args x{a};
    const rs_pool p = x.pool(0);
    const Sequences q = sequences(x, p, 1);
    const int64_t n = x.size(4, 0);
    const int32_t *seq = x.ints(4, {n}), *want = x.ints(5, {n});
    const int T = (int)x.integer(6);
    int32_t *granted = x.ints(7, {n});
    size_t nb = 0;
    void *ws = x.workspace(8, nb);
    return run(x, [&](void *st) { return f_reserve(&p, q.table, q.len, q.refs, seq, (int)n, want, T, granted, ws, nb, st); });
}

PyObject *py_page_pool_fork(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 9)) return nullptr;
    Args x{a};
    const rs_pool p = x.pool(0);
    const Sequences q = sequences(x, p, 1);
    const int64_t n = x.size(4, 0);
    const int32_t *src = x.ints(4, {n}), *dst = x.ints(5, {n});
    int32_t *pairs = x.ints(6, {n, 2}), *carry = x.ints(7, {n, 2});
    size_t nb = 0;
    void *ws = x.workspace(8, nb);
    return run(x, [&](void *st) { return f_fork(&p, q.table, q.len, q.refs, src, dst, (int)n, pairs, carry, ws, nb, st); });
}

PyObject *py_page_pool_free(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 6)) return nullptr;
    Args x{a};
    const rs_pool p = x.pool(0);
    const Sequences q = sequences(x, p, 1);
    const int64_t n = x.size(4, 0);
    const int32_t *seq = x.ints(4, {n});
    size_t nb = 0;
    void *ws = x.workspace(5, nb);
    return run(x, [&](void *st) { return f_free(&p, q.table, q.len, q.refs, seq, (int)n, ws, nb, st); });
}

PyObject *py_page_pool_compact(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 7)) return nullptr;
    Args x{a};
    const rs_pool p = x.pool(0);
    const Sequences q = sequences(x, p, 1);
    int32_t *pairs = x.ints(4, {p.N / 2 > 1 ? p.N / 2 : 1, 2}), *n_pairs = x.ints(5, {1});
    size_t nb = 0;
    void *ws = x.workspace(6, nb);
    return run(x, [&](void *st) { return f_compact(&p, q.table, q.len, q.refs, pairs, n_pairs, ws, nb, st); });
}

PyObject *py_page_pool_share(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 6)) return nullptr;
    Args x{a};
    const rs_pool p = x.pool(0);
    const int32_t *table = x.ints(1, {p.S, p.M}), *len = x.ints(2, {p.S});
    const int64_t n = x.size(3, 0);
    const int32_t *seq = x.ints(3, {n});
    const int least = (int)x.integer(4);
    int32_t *share = x.ints(5, {n, 3});
    return run(x, [&](void *st) { return f_share(&p, table, len, seq, (int)n, least, share, st); });
}

PyObject *py_page_copy(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 10)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0), d = x.shape(4);
    const Rows from = rows(x, s, 1), to = rows(x, d, 5);
    const int64_t n = x.size(8, 0);
    const int32_t *pairs = x.ints(8, {n, 2}), *n_pairs = x.ints(9, {1});
    return run(x, [&](void *st) { return f_copy(&s, from.k, from.v, from.meta, &d, to.k, to.v, to.meta, pairs, (int)n, n_pairs, st); });
}

PyObject *py_rat_state_copy(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 4)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const int64_t S = x.size(1, 0), n = x.size(3, 0);
    float *k = (float *)x.typed(1, at::kFloat, {S, s.Hkv, s.D}), *v = (float *)x.typed(2, at::kFloat, {S, s.Hkv, s.D});
    const int32_t *pairs = x.ints(3, {n, 2});
    return run(x, [&](void *st) { return f_state(&s, k, v, (int)S, pairs, (int)n, st); });
}

PyObject *py_rat_append_paged(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 15)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const rs_pool p = x.pool(1);
    const at::ScalarType dt = type_of(s);
    const int T = (int)x.integer(14);
    void *k = x.typed(2, dt, {s.B, s.Hkv, T, s.D}), *v = x.typed(3, dt, {s.B, s.Hkv, T, s.D});
    float *g = (float *)x.typed(4, at::kFloat, {s.B, s.Hkv, T, s.D});
    float *sk = (float *)x.typed(5, at::kFloat, {p.S, s.Hkv, s.D}), *sv = (float *)x.typed(6, at::kFloat, {p.S, s.Hkv, s.D});
    const Rows to = rows(x, s, 7);
    const int32_t *table = x.ints(10, {p.S, p.M}), *len = x.ints(11, {p.S}), *seq = x.ints(12, {s.B}), *n_new = x.ints(13, {s.B});
    return run(x, [&](void *st) { return f_append(&s, &p, k, v, g, sk, sv, to.k, to.v, to.meta, table, len, seq, n_new, T, st); });
}

PyObject *py_attn_paged(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 15)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const rs_pool p = x.pool(1);
    const at::ScalarType dt = type_of(s);
    const int T = (int)x.integer(9);
    void *q = x.typed(2, dt, {s.B, s.Hq, T, s.D}), *k = x.typed(3, dt, {s.Hkv, s.Tcap, s.D}), *v = x.typed(4, dt, {s.Hkv, s.Tcap, s.D});
    const int32_t *table = x.ints(5, {p.S, p.M}), *len = x.ints(6, {p.S}), *seq = x.ints(7, {s.B}), *n_new = x.ints(8, {s.B}), *share = x.ints(10, {s.B, 3});
    const float scale = x.real(11);
    void *out = x.typed(12, dt, {s.B, s.Hq, T, s.D});
    float *lse = (float *)x.typed(13, at::kFloat, {s.B, s.Hq, T});
    size_t nb = 0;
    void *ws = x.workspace(14, nb);
    return run(x, [&](void *st) { return f_attn(&s, &p, q, k, v, table, len, seq, n_new, T, share, scale, out, lse, ws, nb, st); });
}

// setup_pool(the nine functions' addresses in the order of their definitions above, rs_pool)
PyObject *py_setup_pool(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 10)) return nullptr;
    Args x{a};
    f_reserve = (decltype(f_reserve))x.integer(0);
    f_fork = (decltype(f_fork))x.integer(1);
    f_free = (decltype(f_free))x.integer(2);
    f_compact = (decltype(f_compact))x.integer(3);
    f_share = (decltype(f_share))x.integer(4);
    f_copy = (decltype(f_copy))x.integer(5);
    f_state = (decltype(f_state))x.integer(6);
    f_append = (decltype(f_append))x.integer(7);
    f_attn = (decltype(f_attn))x.integer(8);
    if (!x.plain) {
        PyErr_SetString(PyExc_TypeError, "setup_pool: nine addresses expected");
        return nullptr;
    }
    Py_INCREF(a[9]);
    Py_XDECREF(g_pool);
    g_pool = a[9];
    Py_RETURN_NONE;
}

// ---- a cache in 4 bits, and caches that give up rows ----
struct Four {
    uint8_t *k, *ks, *v, *vs;
};
uint8_t *bytes(Args &x, const rs_shape &s, int i, int channels) { return (uint8_t *)x.typed(i, at::kByte, {s.B, s.Hkv, s.Tcap, s.D / channels}); }
Four four(Args &x, const rs_shape &s, int i) { return Four{bytes(x, s, i, 2), bytes(x, s, i + 1, 32), bytes(x, s, i + 2, 2), bytes(x, s, i + 3, 32)}; }
void *bounds(Args &x, const rs_shape &s, int i)
{
    void *p = x.typed(i, type_of(s), {s.B, s.Hkv, s.P > 0 ? s.Tcap / s.P : 0, 2, s.D});
    return p || x.a[i] == Py_None ? p : x.refuse();  // (an empty tensor's address: not to be taken for no bounds)
}
float *per_row(Args &x, const rs_shape &s, int i) { return (float *)x.typed(i, at::kFloat, {s.B, s.Hkv, s.Tcap}); }

PyObject *py_kv4_append(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 12)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const int64_t T_src = x.size(1, 2), t_src = x.integer(3);
    const void *k = x.typed(1, type_of(s), {s.B, s.Hkv, T_src, s.D}), *v = x.typed(2, type_of(s), {s.B, s.Hkv, T_src, s.D});
    const int32_t *len = x.ints(4, {s.B}), *n_new = x.ints(5, {s.B});
    const int T = (int)x.integer(6);
    const Four c = four(x, s, 7);
    void *meta = bounds(x, s, 11);
    return run(x, [&](void *st) { return f_kv4_append(&s, k, v, T_src, t_src, len, n_new, T, c.k, c.ks, c.v, c.vs, meta, st); });
}

PyObject *py_kv4_page_meta(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 7)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const uint8_t *k = bytes(x, s, 1, 2), *ks = bytes(x, s, 2, 32);
    const int32_t *len = x.ints(3, {s.B}), *n_new = x.ints(4, {s.B});
    const int T = (int)x.integer(5);
    void *meta = bounds(x, s, 6);
    return run(x, [&](void *st) { return f_kv4_meta(&s, k, ks, len, n_new, T, meta, st); });
}

PyObject *py_kv4_fetch(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 10)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const Four c = four(x, s, 1);
    const int32_t *len = x.ints(5, {s.B});
    const int64_t t0 = x.integer(6);
    const int T = (int)x.integer(7);
    void *k = x.typed(8, type_of(s), {s.B, s.Hkv, T, s.D}), *v = x.typed(9, type_of(s), {s.B, s.Hkv, T, s.D});
    return run(x, [&](void *st) { return f_kv4_fetch(&s, c.k, c.ks, c.v, c.vs, len, t0, T, k, v, st); });
}

PyObject *py_kv4_attn_decode(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 14)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const void *q = x.typed(1, type_of(s), {s.B, s.Hq, s.D});
    const Four c = four(x, s, 2);
    const int32_t *len = x.ints(6, {s.B});
    const float scale = x.real(7);
    const int64_t H = a[8] == Py_None ? 0 : x.size(8, 1), K = a[8] == Py_None ? 0 : x.size(8, 2);
    const int32_t *idx = x.ints(8, {s.B, H, K});
    if (a[8] != Py_None && !idx) x.refuse();  // (an empty tensor's address: not to be taken for no list)
    float *tally = per_row(x, s, 9);
    const int fresh = (int)x.integer(10);
    void *out = x.typed(11, type_of(s), {s.B, s.Hq, s.D});
    float *lse = (float *)x.typed(12, at::kFloat, {s.B, s.Hq});
    size_t nb = 0;
    void *ws = x.workspace(13, nb);
    return run(x, [&](void *st) {
        return f_kv4_attn(&s, q, c.k, c.ks, c.v, c.vs, len, scale, idx, (int)H, (int)K, tally, fresh, out, lse, ws, nb, st);
    });
}

PyObject *py_attn_decode_tally(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 11)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const at::ScalarType dt = type_of(s);
    const void *q = x.typed(1, dt, {s.B, s.Hq, s.D}), *k = x.typed(2, dt, {s.B, s.Hkv, s.Tcap, s.D}), *v = x.typed(3, dt, {s.B, s.Hkv, s.Tcap, s.D});
    const int32_t *len = x.ints(4, {s.B});
    const float scale = x.real(5);
    float *tally = per_row(x, s, 6);
    const int fresh = (int)x.integer(7);
    void *out = x.typed(8, dt, {s.B, s.Hq, s.D});
    float *lse = (float *)x.typed(9, at::kFloat, {s.B, s.Hq});
    size_t nb = 0;
    void *ws = x.workspace(10, nb);
    return run(x, [&](void *st) { return f_tally(&s, q, k, v, len, scale, tally, fresh, out, lse, ws, nb, st); });
}

// what both evictions take after the cache: tally, pos, mark, len, the four numbers, the workspace
template <typename F>
PyObject *evict(Args &x, const rs_shape &s, int i, F f)
{
    float *tally = per_row(x, s, i);
    int32_t *pos = x.ints(i + 1, {s.B, s.Hkv, s.Tcap}), *mark = x.ints(i + 2, {s.B, 2}), *len = x.ints(i + 3, {s.B});
    const int keep = (int)x.integer(i + 4), first = (int)x.integer(i + 5), recent = (int)x.integer(i + 6), slack = (int)x.integer(i + 7);
    size_t nb = 0;
    void *ws = x.workspace(i + 8, nb);
    return run(x, [&](void *st) { return f(tally, pos, mark, len, keep, first, recent, slack, ws, nb, st); });
}

PyObject *py_cache_evict(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 12)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    void *k = x.typed(1, type_of(s), {s.B, s.Hkv, s.Tcap, s.D}), *v = x.typed(2, type_of(s), {s.B, s.Hkv, s.Tcap, s.D});
    return evict(x, s, 3, [&](auto... more) { return f_evict(&s, k, v, more...); });
}

PyObject *py_kv4_evict(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    if (!expect(na, 14)) return nullptr;
    Args x{a};
    const rs_shape s = x.shape(0);
    const Four c = four(x, s, 1);
    return evict(x, s, 5, [&](auto... more) { return f_kv4_evict(&s, c.k, c.ks, c.v, c.vs, more...); });
}

// setup_cache(the seven functions' addresses in the order of their definitions above)
PyObject *py_setup_cache(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 7)) return nullptr;
    Args x{a};
    f_kv4_append = (decltype(f_kv4_append))x.integer(0);
    f_kv4_meta = (decltype(f_kv4_meta))x.integer(1);
    f_kv4_fetch = (decltype(f_kv4_fetch))x.integer(2);
    f_kv4_attn = (decltype(f_kv4_attn))x.integer(3);
    f_tally = (decltype(f_tally))x.integer(4);
    f_evict = (decltype(f_evict))x.integer(5);
    f_kv4_evict = (decltype(f_kv4_evict))x.integer(6);
    if (!x.plain) {
        PyErr_SetString(PyExc_TypeError, "setup_cache: seven addresses expected");
        return nullptr;
    }
    Py_RETURN_NONE;
}

// setup(address of rat_scan, of sparse_attn_decode, of rat_decode_step, _check, stream of a device, current device,
// rs_shape, Workspace)
PyObject *py_setup(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 8)) return nullptr;
    Args x{a};
    f_scan = (decltype(f_scan))x.integer(0);
    f_decode = (decltype(f_decode))x.integer(1);
    f_step = (decltype(f_step))x.integer(2);
    if (!x.plain) {
        PyErr_SetString(PyExc_TypeError, "setup: three addresses expected");
        return nullptr;
    }
    PyObject **keep[5] = {&g_check, &g_stream_of, &g_device, &g_shape, &g_workspace};
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(a[3 + i]);
        Py_XDECREF(*keep[i]);
        *keep[i] = a[3 + i];
    }
    Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"setup", FAST(py_setup)},
                         {"rat_scan", FAST(py_rat_scan)},
                         {"sparse_attn_decode", FAST(py_sparse_attn_decode)},
                         {"rat_decode_step", FAST(py_rat_decode_step)},
                         {"setup_pool", FAST(py_setup_pool)},
                         {"page_pool_reserve", FAST(py_page_pool_reserve)},
                         {"page_pool_fork", FAST(py_page_pool_fork)},
                         {"page_pool_free", FAST(py_page_pool_free)},
                         {"page_pool_compact", FAST(py_page_pool_compact)},
                         {"page_pool_share", FAST(py_page_pool_share)},
                         {"page_copy", FAST(py_page_copy)},
                         {"rat_state_copy", FAST(py_rat_state_copy)},
                         {"rat_append_paged", FAST(py_rat_append_paged)},
                         {"attn_paged", FAST(py_attn_paged)},
                         {"setup_cache", FAST(py_setup_cache)},
                         {"kv4_append", FAST(py_kv4_append)},
                         {"kv4_page_meta", FAST(py_kv4_page_meta)},
                         {"kv4_fetch", FAST(py_kv4_fetch)},
                         {"kv4_attn_decode", FAST(py_kv4_attn_decode)},
                         {"attn_decode_tally", FAST(py_attn_decode_tally)},
                         {"cache_evict", FAST(py_cache_evict)},
                         {"kv4_evict", FAST(py_kv4_evict)},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    s_buf = PyUnicode_InternFromString("buf");
    return PyModule_Create(&module);
}
