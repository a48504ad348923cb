// torch_args.cpp -- the layer, group and serving calls of cola.py with their checks in
// native code (CPython extension _torch_args).
//
// cola.py checks every tensor against the descriptor before a call (dtype,
// shape, strides, storage, device).  In Python that and the argument conversion
// cost 10 us of a forward call and 17 us of a backward call, as much as the
// kernels of a small layer take; here about 1 us.  Each function takes the
// arguments of the cola.py function of the same name (with the stream as an
// integer; the serving calls have the current device before it) and returns the
// library's status, or None when any argument is not the plain case (a tensor of
// the expected kind, or None where that is allowed): cola.py then runs its own
// checks, which raise the error or take the call.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/cola.h"

namespace {

// dims a tensor must cover, in elements
struct Need {
    int64_t rows, width, ld;
    at::ScalarType dtype;
};

// Device pointer of a plain tensor on a GPU that holds `need`; false if it is
// anything else.
bool take(PyObject* o, const Need& need, void** out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.has_storage() || !t.is_cuda() || t.scalar_type() != need.dtype || t.dim() != 2) return false;
    if (t.size(0) < need.rows || t.size(1) < need.width) return false;
    if (t.stride(1) != 1 || (need.rows > 1 && t.stride(0) != need.ld)) return false;
    const int64_t es = (int64_t)t.element_size();
    if ((int64_t)t.storage().nbytes() - t.storage_offset() * es < need.rows * need.ld * es) return false;
    *out = t.data_ptr();
    return true;
}

bool take_or_none(PyObject* o, const Need& need, void** out) {
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    return take(o, need, out);
}

bool take_list(PyObject* o, const Need* need, int n, void** out) {
    if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
    if (PySequence_Fast_GET_SIZE(o) != n) return false;
    for (int i = 0; i < n; ++i)
        if (!take(PySequence_Fast_GET_ITEM(o, i), need[i], &out[i])) return false;
    return true;
}

// The workspace and its size (None: the whole tensor).
bool take_ws(PyObject* ws, PyObject* bytes, void** out, size_t* n) {
    *out = nullptr;
    *n = 0;
    if (ws == Py_None) return bytes == Py_None;
    if (!THPVariable_CheckExact(ws)) return false;
    const at::Tensor& t = THPVariable_Unpack(ws);
    if (!t.has_storage() || !t.is_cuda() || !t.is_contiguous()) return false;
    const int64_t have = (int64_t)t.numel() * (int64_t)t.element_size();
    int64_t want = have;
    if (bytes != Py_None) {
        if (!PyLong_CheckExact(bytes)) return false;
        want = PyLong_AsLongLong(bytes);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return false;
        }
    }
    if (want < 0 || want > have) return false;
    *out = t.data_ptr();
    *n = (size_t)want;
    return true;
}

bool take_int(PyObject* o, int64_t* out) {
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsLongLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// A ctypes descriptor's bytes.
template <class Desc>
bool take_desc(PyObject* o, Desc* out) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    const bool ok = b.len == (Py_ssize_t)sizeof(Desc);
    if (ok) memcpy(out, b.buf, sizeof(Desc));
    PyBuffer_Release(&b);
    return ok;
}

constexpr int64_t kMaxDim = int64_t(1) << 31;          // products of two dimensions stay below 2^63
bool dim_ok(int64_t v) { return v >= 1 && v <= kMaxDim; }

struct Layer {
    cola_desc d;
    Need x, y, z, a, b, da, db;

    bool init(PyObject* o) {
        if (!take_desc(o, &d) || (d.dtype != COLA_F32 && d.dtype != COLA_BF16)) return false;
        if (d.ldx < 0 || d.ldy < 0 || d.ldz < 0) return false;
        const int64_t ldx = d.ldx ? d.ldx : d.d_in, ldy = d.ldy ? d.ldy : d.d_out, ldz = d.ldz ? d.ldz : d.r;
        for (int64_t v : {d.T, d.d_in, d.d_out, d.r, ldx, ldy, ldz})
            if (!dim_ok(v)) return false;
        const at::ScalarType t = d.dtype == COLA_BF16 ? at::kBFloat16 : at::kFloat;
        x = Need{d.T, d.d_in, ldx, t};
        y = Need{d.T, d.d_out, ldy, t};
        z = Need{d.T, d.r, ldz, t};
        a = Need{d.r, d.d_in, d.d_in, t};
        b = Need{d.d_out, d.r, d.r, t};
        da = Need{d.r, d.d_in, d.d_in, at::kFloat};
        db = Need{d.d_out, d.r, d.r, at::kFloat};
        return true;
    }
};

struct Group {
    cola_group_desc d;
    Need x, z, a, da, y[COLA_GROUP_MAX], b[COLA_GROUP_MAX], db[COLA_GROUP_MAX];

    bool init(PyObject* o) {
        if (!take_desc(o, &d) || (d.dtype != COLA_F32 && d.dtype != COLA_BF16)) return false;
        if (d.n < 1 || d.n > COLA_GROUP_MAX || d.ldx < 0 || d.ldz < 0) return false;
        const at::ScalarType t = d.dtype == COLA_BF16 ? at::kBFloat16 : at::kFloat;
        int64_t R = 0;
        for (int p = 0; p < d.n; ++p) {
            if (d.ldy[p] < 0 || !dim_ok(d.r[p]) || !dim_ok(d.d_out[p])) return false;
            const int64_t ldy = d.ldy[p] ? d.ldy[p] : d.d_out[p];
            if (!dim_ok(ldy)) return false;
            R += d.r[p];
            y[p] = Need{d.T, d.d_out[p], ldy, t};
            b[p] = Need{d.d_out[p], d.r[p], d.r[p], t};
            db[p] = Need{d.d_out[p], d.r[p], d.r[p], at::kFloat};
        }
        const int64_t ldx = d.ldx ? d.ldx : d.d_in, ldz = d.ldz ? d.ldz : R;
        for (int64_t v : {d.T, d.d_in, R, ldx, ldz})
            if (!dim_ok(v)) return false;
        x = Need{d.T, d.d_in, ldx, t};
        z = Need{d.T, R, ldz, t};
        a = Need{R, d.d_in, d.d_in, t};
        da = Need{R, d.d_in, d.d_in, at::kFloat};
        return true;
    }
};

using Args = PyObject* const*;

// Runs f (false: not the plain case; else *st holds the status).  No C++
// exception leaves.
template <class F>
PyObject* call(F&& f) {
    int st = 0;
    bool plain = false;
    try {
        plain = f(&st);
    } catch (...) {
        plain = false;
    }
    if (!plain) Py_RETURN_NONE;
    return PyLong_FromLong(st);
}

struct Tail {                                            // ws, ws_bytes, stream
    void* ws;
    size_t n;
    int64_t stream;
    bool init(Args v) { return take_ws(v[0], v[1], &ws, &n) && take_int(v[2], &stream); }
    cola_stream_t s() const { return reinterpret_cast<cola_stream_t>(stream); }
};

// The library call itself, without the interpreter lock.
#define COLA_CALL(expr)        \
    Py_BEGIN_ALLOW_THREADS     \
    *st = (expr);              \
    Py_END_ALLOW_THREADS       \
    return true

PyObject* fwd(PyObject*, Args v, Py_ssize_t n) {         // d, X, A, B, Y, Z, H, ws, ws_bytes, stream
    return call([&](int* st) {
        Layer l;
        Tail t;
        void *X, *A, *B, *Y, *Z, *H;
        if (n != 10 || !l.init(v[0]) || !take(v[1], l.x, &X) || !take(v[2], l.a, &A) || !take(v[3], l.b, &B) ||
            !take(v[4], l.y, &Y) || !take(v[5], l.z, &Z) || !take_or_none(v[6], l.z, &H) || !t.init(v + 7))
            return false;
        COLA_CALL(cola_fwd(&l.d, X, A, B, Y, Z, H, t.ws, t.n, t.s()));
    });
}

PyObject* fwd_outer(PyObject*, Args v, Py_ssize_t n) {   // d, outer, X, A, B, Y, P, Z, H, ws, ws_bytes, stream
    return call([&](int* st) {
        Layer l;
        Tail t;
        int64_t outer;
        void *X, *A, *B, *Y, *P, *Z, *H;
        if (n != 12 || !l.init(v[0]) || !take_int(v[1], &outer) || outer < 0 || outer > 1000 || !take(v[2], l.x, &X) ||
            !take(v[3], l.a, &A) || !take(v[4], l.b, &B) || !take(v[5], l.y, &Y) || !take(v[6], l.y, &P) ||
            !take(v[7], l.z, &Z) || !take_or_none(v[8], l.z, &H) || !t.init(v + 9))
            return false;
        COLA_CALL(cola_fwd_outer(&l.d, (int)outer, X, A, B, Y, P, Z, H, t.ws, t.n, t.s()));
    });
}

PyObject* infer(PyObject*, Args v, Py_ssize_t n) {       // d, X, A, B, Y, ws, ws_bytes, stream
    return call([&](int* st) {
        Layer l;
        Tail t;
        void *X, *A, *B, *Y;
        if (n != 8 || !l.init(v[0]) || !take(v[1], l.x, &X) || !take(v[2], l.a, &A) || !take(v[3], l.b, &B) ||
            !take(v[4], l.y, &Y) || !t.init(v + 5))
            return false;
        COLA_CALL(cola_infer(&l.d, X, A, B, Y, t.ws, t.n, t.s()));
    });
}

PyObject* bwd(PyObject*, Args v, Py_ssize_t n) {         // d, dY, X, Z, H, A, B, dX, dA, dB, ws, ws_bytes, stream
    return call([&](int* st) {
        Layer l;
        Tail t;
        void *dY, *X, *Z, *H, *A, *B, *dX, *dA, *dB;
        if (n != 13 || !l.init(v[0]) || !take(v[1], l.y, &dY) || !take(v[2], l.x, &X) || !take(v[3], l.z, &Z) ||
            !take_or_none(v[4], l.z, &H) || !take(v[5], l.a, &A) || !take(v[6], l.b, &B) || !take(v[7], l.x, &dX) ||
            !take(v[8], l.da, &dA) || !take(v[9], l.db, &dB) || !t.init(v + 10))
            return false;
        COLA_CALL(cola_bwd(&l.d, dY, X, Z, H, A, B, dX, static_cast<float*>(dA), static_cast<float*>(dB), t.ws, t.n,
                           t.s()));
    });
}

PyObject* bwd_outer(PyObject*, Args v, Py_ssize_t n) {   // d, outer, dY, P, X, Z, H, A, B, dX, dA, dB, ws, ws_bytes, stream
    return call([&](int* st) {
        Layer l;
        Tail t;
        int64_t outer;
        void *dY, *P, *X, *Z, *H, *A, *B, *dX, *dA, *dB;
        if (n != 15 || !l.init(v[0]) || !take_int(v[1], &outer) || outer < 0 || outer > 1000 || !take(v[2], l.y, &dY) ||
            !take(v[3], l.y, &P) || !take(v[4], l.x, &X) || !take(v[5], l.z, &Z) || !take_or_none(v[6], l.z, &H) ||
            !take(v[7], l.a, &A) || !take(v[8], l.b, &B) || !take(v[9], l.x, &dX) || !take(v[10], l.da, &dA) ||
            !take(v[11], l.db, &dB) || !t.init(v + 12))
            return false;
        COLA_CALL(cola_bwd_outer(&l.d, (int)outer, dY, P, X, Z, H, A, B, dX, static_cast<float*>(dA),
                                 static_cast<float*>(dB), t.ws, t.n, t.s()));
    });
}

PyObject* group_fwd(PyObject*, Args v, Py_ssize_t n) {   // d, X, A_all, B, Y, Z_all, H_all, ws, ws_bytes, stream
    return call([&](int* st) {
        Group g;
        Tail t;
        void *X, *A, *Z, *H, *B[COLA_GROUP_MAX], *Y[COLA_GROUP_MAX];
        if (n != 10 || !g.init(v[0]) || !take(v[1], g.x, &X) || !take(v[2], g.a, &A) || !take_list(v[3], g.b, g.d.n, B) ||
            !take_list(v[4], g.y, g.d.n, Y) || !take(v[5], g.z, &Z) || !take_or_none(v[6], g.z, &H) || !t.init(v + 7))
            return false;
        COLA_CALL(cola_group_fwd(&g.d, X, A, B, Y, Z, H, t.ws, t.n, t.s()));
    });
}

PyObject* group_infer(PyObject*, Args v, Py_ssize_t n) { // d, X, A_all, B, Y, ws, ws_bytes, stream
    return call([&](int* st) {
        Group g;
        Tail t;
        void *X, *A, *B[COLA_GROUP_MAX], *Y[COLA_GROUP_MAX];
        if (n != 8 || !g.init(v[0]) || !take(v[1], g.x, &X) || !take(v[2], g.a, &A) || !take_list(v[3], g.b, g.d.n, B) ||
            !take_list(v[4], g.y, g.d.n, Y) || !t.init(v + 5))
            return false;
        COLA_CALL(cola_group_infer(&g.d, X, A, B, Y, t.ws, t.n, t.s()));
    });
}

PyObject* group_bwd(PyObject*, Args v, Py_ssize_t n) {   // d, dY, X, Z_all, H_all, A_all, B, dX, dA_all, dB, ws, ws_bytes, stream
    return call([&](int* st) {
        Group g;
        Tail t;
        void *X, *Z, *H, *A, *dX, *dA, *dY[COLA_GROUP_MAX], *B[COLA_GROUP_MAX], *dB[COLA_GROUP_MAX];
        if (n != 13 || !g.init(v[0]) || !take_list(v[1], g.y, g.d.n, dY) || !take(v[2], g.x, &X) || !take(v[3], g.z, &Z) ||
            !take_or_none(v[4], g.z, &H) || !take(v[5], g.a, &A) || !take_list(v[6], g.b, g.d.n, B) ||
            !take(v[7], g.x, &dX) || !take(v[8], g.da, &dA) || !take_list(v[9], g.db, g.d.n, dB) || !t.init(v + 10))
            return false;
        float* dBf[COLA_GROUP_MAX];
        for (int p = 0; p < g.d.n; ++p) dBf[p] = static_cast<float*>(dB[p]);
        COLA_CALL(cola_group_bwd(&g.d, dY, X, Z, H, A, B, dX, static_cast<float*>(dA), dBf, t.ws, t.n, t.s()));
    });
}

// ---- serving ----

struct Here {                                            // the current device, stream
    int64_t device, stream;
    bool init(Args v) { return take_int(v[0], &device) && take_int(v[1], &stream); }
    cola_stream_t s() const { return reinterpret_cast<cola_stream_t>(stream); }

    const at::Tensor* mine(PyObject* o, at::ScalarType dtype) const {
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.has_storage() || !t.is_cuda() || t.get_device() != device || t.scalar_type() != dtype) return nullptr;
        return &t;
    }
    // [rows][width] at a row pitch of ld; None where no element is needed
    bool rows(PyObject* o, int64_t rows, int64_t width, int64_t ld, at::ScalarType dtype, void** out) const {
        *out = nullptr;
        if (width == 0) return o == Py_None;
        const at::Tensor* t = mine(o, dtype);
        if (!t || t->dim() != 2 || t->size(0) < rows || t->size(1) < width) return false;
        if (t->stride(1) != 1 || (rows > 1 && t->stride(0) != (ld ? ld : width))) return false;
        *out = t->data_ptr();
        return true;
    }
    // contiguous, at least n0 along the first dimension, the others exactly
    bool flat(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, bool none_ok, void** out) const {
        *out = nullptr;
        if (o == Py_None) return none_ok;
        const at::Tensor* t = mine(o, dtype);
        if (!t || t->dim() != (int64_t)shape.size() || !t->is_contiguous() || t->size(0) < shape[0]) return false;
        for (size_t i = 1; i < shape.size(); ++i)
            if (t->size(i) != shape[i]) return false;
        *out = t->data_ptr();
        return true;
    }
    bool ints(PyObject* o, int64_t n, bool none_ok, const int32_t** out) const {
        void* p;
        if (!flat(o, {n}, at::kInt, none_ok, &p)) return false;
        *out = static_cast<const int32_t*>(p);
        return true;
    }
};

bool count_ok(int64_t v) { return v >= 0 && v <= kMaxDim; }

struct Rope {
    cola_rope_desc d;
    at::ScalarType t;
    int64_t wq, wk;

    bool init(PyObject* o) {
        if (!take_desc(o, &d) || (d.dtype != COLA_F32 && d.dtype != COLA_BF16)) return false;
        if (d.T < 1) return false;
        for (int64_t v : {d.T, d.heads_q, d.heads_k, d.head_dim, d.ldq, d.ldk, d.ldv, d.ldqo, d.ldko})
            if (!count_ok(v)) return false;
        t = d.dtype == COLA_BF16 ? at::kBFloat16 : at::kFloat;
        wq = d.heads_q * d.head_dim;
        wk = d.heads_k * d.head_dim;
        return true;
    }
};

struct Cache {
    cola_cache_desc c;
    bool init(PyObject* o) {
        if (!take_desc(o, &c) || (c.dtype != COLA_F32 && c.dtype != COLA_BF16)) return false;
        return dim_ok(c.n_pages) && dim_ok(c.page_size) && dim_ok(c.heads) && dim_ok(c.head_dim);
    }
    bool pages(const Here& h, PyObject* o, void** out) const {
        return h.flat(o, {c.n_pages, c.heads, c.page_size, c.head_dim},
                      c.dtype == COLA_BF16 ? at::kBFloat16 : at::kFloat, false, out);
    }
};

template <class F>
PyObject* rope(Args v, Py_ssize_t n, F f) {              // d, q, k, positions, q_out, k_out, device, stream
    return call([&](int* st) {
        Rope r;
        Here h;
        void *q, *k, *qo, *ko;
        const int32_t* pos;
        if (n != 8 || !h.init(v + 6) || !r.init(v[0]) || !h.rows(v[1], r.d.T, r.wq, r.d.ldq, r.t, &q) ||
            !h.rows(v[2], r.d.T, r.wk, r.d.ldk, r.t, &k) || !h.ints(v[3], r.d.T, true, &pos) ||
            !h.rows(v[4], r.d.T, r.wq, r.d.ldqo, r.t, &qo) || !h.rows(v[5], r.d.T, r.wk, r.d.ldko, r.t, &ko))
            return false;
        COLA_CALL(f(&r.d, q, k, pos, qo, ko, h.s()));
    });
}
PyObject* rope_fwd(PyObject*, Args v, Py_ssize_t n) { return rope(v, n, cola_rope_fwd); }
PyObject* rope_bwd(PyObject*, Args v, Py_ssize_t n) { return rope(v, n, cola_rope_bwd); }

PyObject* cache_append(PyObject*, Args v, Py_ssize_t n) { // d, c, q, k, v, positions, slots, q_out, K, V, device, stream
    return call([&](int* st) {
        Rope r;
        Cache c;
        Here h;
        void *q, *k, *val, *qo, *K, *V;
        const int32_t *pos, *slots;
        if (n != 12 || !h.init(v + 10) || !r.init(v[0]) || !c.init(v[1]) ||
            !h.rows(v[2], r.d.T, r.wq, r.d.ldq, r.t, &q) || !h.rows(v[3], r.d.T, r.wk, r.d.ldk, r.t, &k) ||
            !h.rows(v[4], r.d.T, r.wk, r.d.ldv, r.t, &val) || !h.ints(v[5], r.d.T, true, &pos) ||
            !h.ints(v[6], r.d.T, false, &slots) || !h.rows(v[7], r.d.T, r.wq, r.d.ldqo, r.t, &qo) ||
            !c.pages(h, v[8], &K) || !c.pages(h, v[9], &V))
            return false;
        COLA_CALL(cola_cache_append(&r.d, &c.c, q, k, val, pos, slots, qo, K, V, h.s()));
    });
}

PyObject* page_map(PyObject*, Args v, Py_ssize_t n) {    // d, kv_len, n_new, free_pages, free_at, table, start, slots, positions, free_next, device, stream
    return call([&](int* st) {
        cola_page_map_desc d;
        Here h;
        void* table;
        const int32_t *kv, *nw, *list, *at, *start, *slots, *pos, *next;
        if (n != 12 || !h.init(v + 10) || !take_desc(v[0], &d) || !dim_ok(d.n_req) || !dim_ok(d.T) || !dim_ok(d.max_pages) ||
            !dim_ok(d.n_free) || !h.ints(v[1], d.n_req, false, &kv) || !h.ints(v[2], d.n_req, false, &nw) ||
            !h.ints(v[3], d.n_free, false, &list) || !h.ints(v[4], 1, true, &at) ||
            !h.flat(v[5], {d.n_req, d.max_pages}, at::kInt, false, &table) || !h.ints(v[6], d.n_req + 1, false, &start) ||
            !h.ints(v[7], d.T, false, &slots) || !h.ints(v[8], d.T, false, &pos) || !h.ints(v[9], 1, false, &next))
            return false;
        auto out = [](const int32_t* p) { return const_cast<int32_t*>(p); };
        COLA_CALL(cola_page_map(&d, kv, nw, list, at, static_cast<int32_t*>(table), out(start), out(slots), out(pos),
                                out(next), h.s()));
    });
}

// The arguments that prefix_attn and tree_attn share: d, c, q, K, V, prefix_table, table, kv_len, start; then
// out, lse, ws, ws_bytes.
struct Attend {
    cola_prefix_attn_desc d;
    Cache c;
    void *q, *K, *V, *table = nullptr, *out, *lse, *ws;
    const int32_t *prefix, *kv = nullptr, *start;
    size_t ws_bytes;

    bool init(const Here& h, Args v, Args o) {
        if (!take_desc(v[0], &d) || !c.init(v[1]) || c.c.dtype != COLA_BF16 || d.n_req < 1 || d.T < 1) return false;
        for (int64_t x : {d.n_req, d.T, d.heads_q, d.prefix_len, d.max_kv, d.max_pages, d.ldq, d.ldo})
            if (!count_ok(x)) return false;
        const int64_t w = d.heads_q * c.c.head_dim, ps = c.c.page_size;
        if (!h.rows(v[2], d.T, w, d.ldq, at::kBFloat16, &q) || !c.pages(h, v[3], &K) || !c.pages(h, v[4], &V) ||
            !h.ints(v[5], (d.prefix_len + ps - 1) / ps, d.prefix_len == 0, &prefix))
            return false;
        if (d.max_kv > 0) {
            const int64_t width = d.max_pages ? d.max_pages : (d.max_kv + ps - 1) / ps;
            if (!h.flat(v[6], {d.n_req, width}, at::kInt, false, &table) || !h.ints(v[7], d.n_req, false, &kv)) return false;
        }
        if (!h.ints(v[8], d.n_req + 1, true, &start) || !h.rows(o[0], d.T, w, d.ldo, at::kBFloat16, &out) ||
            !h.flat(o[1], {d.heads_q, d.T}, at::kFloat, true, &lse) || !take_ws(o[2], o[3], &ws, &ws_bytes))
            return false;
        return !ws || THPVariable_Unpack(o[2]).get_device() == h.device;
    }
};

PyObject* prefix_attn(PyObject*, Args v, Py_ssize_t n) { // d, c, q, K, V, prefix_table, table, kv_len, start, out, lse, ws, ws_bytes, device, stream
    return call([&](int* st) {
        Attend a;
        Here h;
        if (n != 15 || !h.init(v + 13) || !a.init(h, v, v + 9)) return false;
        COLA_CALL(cola_prefix_attn(&a.d, &a.c.c, a.q, a.K, a.V, a.prefix, static_cast<const int32_t*>(a.table), a.kv, a.start,
                                   a.out, static_cast<float*>(a.lse), a.ws, a.ws_bytes, h.s()));
    });
}

PyObject* tree_attn(PyObject*, Args v, Py_ssize_t n) {   // prefix_attn's with mask before out
    return call([&](int* st) {
        Attend a;
        Here h;
        void* mask;
        if (n != 16 || !h.init(v + 14) || !a.init(h, v, v + 10) || !dim_ok(a.d.max_new) ||
            !h.flat(v[9], {a.d.T, (a.d.max_new + 63) / 64}, at::kLong, false, &mask))
            return false;
        COLA_CALL(cola_tree_attn(&a.d, &a.c.c, a.q, a.K, a.V, a.prefix, static_cast<const int32_t*>(a.table), a.kv, a.start,
                                 static_cast<const uint64_t*>(mask), a.out, static_cast<float*>(a.lse), a.ws, a.ws_bytes, h.s()));
    });
}

bool take_real(PyObject* o, double* out) {
    if (!PyFloat_CheckExact(o)) return false;
    *out = PyFloat_AS_DOUBLE(o);
    return true;
}

struct Gains {
    void *q, *k;
    double eps;
    bool init(const Here& h, const Rope& r, PyObject* g_q, PyObject* g_k, PyObject* e) {
        return take_real(e, &eps) && h.flat(g_q, {r.d.head_dim}, r.t, true, &q) && h.flat(g_k, {r.d.head_dim}, r.t, true, &k);
    }
};

PyObject* norm_rope_fwd(PyObject*, Args v, Py_ssize_t n) { // d, q, k, g_q, g_k, positions, q_out, k_out, eps, device, stream
    return call([&](int* st) {
        Rope r;
        Here h;
        Gains g;
        void *q, *k, *qo, *ko;
        const int32_t* pos;
        if (n != 11 || !h.init(v + 9) || !r.init(v[0]) || !g.init(h, r, v[3], v[4], v[8]) ||
            !h.rows(v[1], r.d.T, r.wq, r.d.ldq, r.t, &q) || !h.rows(v[2], r.d.T, r.wk, r.d.ldk, r.t, &k) ||
            !h.ints(v[5], r.d.T, true, &pos) || !h.rows(v[6], r.d.T, r.wq, r.d.ldqo, r.t, &qo) ||
            !h.rows(v[7], r.d.T, r.wk, r.d.ldko, r.t, &ko))
            return false;
        COLA_CALL(cola_norm_rope_fwd(&r.d, g.eps, q, k, g.q, g.k, pos, qo, ko, h.s()));
    });
}

PyObject* norm_rope_bwd(PyObject*, Args v, Py_ssize_t n) { // d, dq_out, dk_out, q, k, g_q, g_k, positions, dq, dk, dg_q, dg_k, ws, ws_bytes, eps, device, stream
    return call([&](int* st) {
        Rope r;
        Here h;
        Gains g;
        void *q, *k, *dqo, *dko, *dq, *dk, *dgq, *dgk, *ws;
        const int32_t* pos;
        size_t ws_bytes;
        if (n != 17 || !h.init(v + 15) || !r.init(v[0]) || !g.init(h, r, v[5], v[6], v[14]) ||
            !h.rows(v[1], r.d.T, r.wq, r.d.ldqo, r.t, &dqo) || !h.rows(v[2], r.d.T, r.wk, r.d.ldko, r.t, &dko) ||
            !h.rows(v[3], r.d.T, r.wq, r.d.ldq, r.t, &q) || !h.rows(v[4], r.d.T, r.wk, r.d.ldk, r.t, &k) ||
            !h.ints(v[7], r.d.T, true, &pos) || !h.rows(v[8], r.d.T, r.wq, r.d.ldq, r.t, &dq) ||
            !h.rows(v[9], r.d.T, r.wk, r.d.ldk, r.t, &dk) || !h.flat(v[10], {r.d.head_dim}, at::kFloat, true, &dgq) ||
            !h.flat(v[11], {r.d.head_dim}, at::kFloat, true, &dgk) || !take_ws(v[12], v[13], &ws, &ws_bytes))
            return false;
        if (ws && THPVariable_Unpack(v[12]).get_device() != h.device) return false;
        COLA_CALL(cola_norm_rope_bwd(&r.d, g.eps, dqo, dko, q, k, g.q, g.k, pos, dq, dk, static_cast<float*>(dgq),
                                     static_cast<float*>(dgk), ws, ws_bytes, h.s()));
    });
}

PyObject* norm_append(PyObject*, Args v, Py_ssize_t n) { // d, c, q, k, v, g_q, g_k, positions, slots, q_out, K, V, eps, device, stream
    return call([&](int* st) {
        Rope r;
        Cache c;
        Here h;
        Gains g;
        void *q, *k, *val, *qo, *K, *V;
        const int32_t *pos, *slots;
        if (n != 15 || !h.init(v + 13) || !r.init(v[0]) || !c.init(v[1]) || !g.init(h, r, v[5], v[6], v[12]) ||
            !h.rows(v[2], r.d.T, r.wq, r.d.ldq, r.t, &q) || !h.rows(v[3], r.d.T, r.wk, r.d.ldk, r.t, &k) ||
            !h.rows(v[4], r.d.T, r.wk, r.d.ldv, r.t, &val) || !h.ints(v[7], r.d.T, true, &pos) ||
            !h.ints(v[8], r.d.T, false, &slots) || !h.rows(v[9], r.d.T, r.wq, r.d.ldqo, r.t, &qo) ||
            !c.pages(h, v[10], &K) || !c.pages(h, v[11], &V))
            return false;
        COLA_CALL(cola_norm_append(&r.d, &c.c, g.eps, q, k, val, g.q, g.k, pos, slots, qo, K, V, h.s()));
    });
}

PyObject* tree_map(PyObject*, Args v, Py_ssize_t n) {    // d, parent, kv_len, start, mask, positions, device, stream
    return call([&](int* st) {
        cola_tree_map_desc d;
        Here h;
        void* mask;
        const int32_t *parent, *kv, *start, *pos;
        if (n != 8 || !h.init(v + 6) || !take_desc(v[0], &d) || !dim_ok(d.n_req) || !dim_ok(d.T) || !dim_ok(d.max_new) ||
            !h.ints(v[1], d.T, false, &parent) || !h.ints(v[2], d.n_req, false, &kv) || !h.ints(v[3], d.n_req + 1, true, &start) ||
            !h.flat(v[4], {d.T, (d.max_new + 63) / 64}, at::kLong, false, &mask) || !h.ints(v[5], d.T, false, &pos))
            return false;
        COLA_CALL(cola_tree_map(&d, parent, kv, start, static_cast<uint64_t*>(mask), const_cast<int32_t*>(pos), h.s()));
    });
}

PyObject* logits_adjust(PyObject*, Args v, Py_ssize_t n) { // d, rules, logits, start, out, device, stream
    return call([&](int* st) {
        cola_logits_desc d;
        cola_logits_rules u;
        Here h;
        void *logits, *out, *mask, *rep, *pres, *freq, *bias, *allowed;
        const int32_t* start;
        if (n != 7 || !h.init(v + 5) || !take_desc(v[0], &d) || !PyTuple_CheckExact(v[1]) || PyTuple_GET_SIZE(v[1]) != 13 ||
            (d.dtype != COLA_F32 && d.dtype != COLA_BF16) || !dim_ok(d.T) || !dim_ok(d.V) || !dim_ok(d.n_req))
            return false;
        for (int64_t x : {d.max_hist, d.max_new, d.n_bias, d.n_allowed, d.ldl, d.ldo, d.lda})
            if (!count_ok(x)) return false;
        const at::ScalarType t = d.dtype == COLA_BF16 ? at::kBFloat16 : at::kFloat;
        auto rule = [&](int i) { return PyTuple_GET_ITEM(v[1], i); };
        void* history;
        if (!h.flat(rule(0), {d.n_req, d.max_hist}, at::kInt, true, &history) || !h.ints(rule(1), d.n_req, true, &u.prompt_len) ||
            !h.ints(rule(2), d.n_req, true, &u.hist_len) || !h.ints(rule(3), d.T, true, &u.draft) ||
            !h.flat(rule(4), {d.T, (d.max_new + 63) / 64}, at::kLong, true, &mask) ||
            !h.flat(rule(5), {d.n_req}, at::kFloat, true, &rep) || !h.flat(rule(6), {d.n_req}, at::kFloat, true, &pres) ||
            !h.flat(rule(7), {d.n_req}, at::kFloat, true, &freq) || !h.ints(rule(8), d.n_req + 1, true, &u.bias_start) ||
            !h.ints(rule(9), d.n_bias, true, &u.bias_token) || !h.flat(rule(10), {d.n_bias}, at::kFloat, true, &bias) ||
            !h.flat(rule(11), {d.n_allowed, d.lda ? d.lda : (d.V + 31) / 32}, at::kInt, true, &allowed) ||
            !h.ints(rule(12), d.T, true, &u.allowed_row) || !h.rows(v[2], d.T, d.V, d.ldl, t, &logits) ||
            !h.ints(v[3], d.n_req + 1, true, &start) || !h.rows(v[4], d.T, d.V, d.ldo, t, &out))
            return false;
        u.history = static_cast<const int32_t*>(history);
        u.mask = static_cast<const uint64_t*>(mask);
        u.repetition = static_cast<const float*>(rep);
        u.presence = static_cast<const float*>(pres);
        u.frequency = static_cast<const float*>(freq);
        u.bias = static_cast<const float*>(bias);
        u.allowed = static_cast<const uint32_t*>(allowed);
        COLA_CALL(cola_logits_adjust(&d, &u, logits, start, out, h.s()));
    });
}

#define COLA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {COLA_METHOD(fwd),       COLA_METHOD(fwd_outer), COLA_METHOD(infer),       COLA_METHOD(bwd),
                         COLA_METHOD(bwd_outer), COLA_METHOD(group_fwd), COLA_METHOD(group_infer), COLA_METHOD(group_bwd),
                         COLA_METHOD(rope_fwd),  COLA_METHOD(rope_bwd),  COLA_METHOD(cache_append), COLA_METHOD(page_map),
                         COLA_METHOD(prefix_attn), COLA_METHOD(norm_rope_fwd), COLA_METHOD(norm_rope_bwd), COLA_METHOD(norm_append),
                         COLA_METHOD(tree_map),  COLA_METHOD(tree_attn), COLA_METHOD(logits_adjust),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_args() { return PyModule_Create(&module); }
