// serve_abi.hip -- the serving entry points of libcola.so (include/cola.h):
// cola_rope_fwd, cola_rope_bwd, cola_cache_append, cola_page_map, cola_prefix_attn,
// cola_norm_rope_fwd, cola_norm_rope_bwd, cola_norm_append, cola_tree_map,
// cola_tree_attn and cola_logits_adjust.  Argument checks, frequencies and launches; the
// kernels are in rope.hip, page_map.hip, prefix_attn.hip, norm_rope.hip, tree_map.hip,
// tree_attn.hip and logits.hip.
#include <float.h>
#include <math.h>

#include "block.hpp"
#include "serve.hpp"

using namespace cola;

namespace {

constexpr int64_t kMaxInt = INT32_MAX;
constexpr int64_t kMaxKeys = int64_t(1) << 30;     // sums of two lengths stay below 2^31

template <class F>
int guarded(F&& f) {
    try {
        return f();
    } catch (...) {
        return set_hip_error(hipErrorUnknown, "unexpected host exception");
    }
}

int chk(hipError_t e, const char* where) { return e == hipSuccess ? COLA_OK : set_hip_error(e, where); }

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool al8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool dtype_ok(int32_t t) { return t == COLA_F32 || t == COLA_BF16; }
bool aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == COLA_F32 ? 3u : 1u)) == 0; }
int log2_of(int64_t n) { return __builtin_ctzll((unsigned long long)n); }
bool page_ok(int64_t n, int64_t least) { return n >= least && n <= 4096 && (n & (n - 1)) == 0; }

// Turns per position of each pair, in 64 bits, and the factor on cosine and sine.
void frequencies(const cola_rope_desc& d, RopeArgs* a) {
    const int half = (int)(d.rot_dim / 2);
    const double two_pi = 6.283185307179586476925286766559;
    double scale = d.mscale;
    if (scale == 0.0) scale = d.scaling == COLA_ROPE_YARN ? 1.0 + 0.1 * log(d.factor) : 1.0;
    a->mscale = (float)scale;
    double base = d.base;
    if (d.scaling == COLA_ROPE_BASE) base *= pow(d.factor, (double)d.rot_dim / (double)(d.rot_dim - 2));
    double first = 0.0, width = 1.0;
    if (d.scaling == COLA_ROPE_YARN && half > 0) {
        auto pair = [&](double turns) {
            return (double)d.rot_dim * log((double)d.orig_len / (two_pi * turns)) / (2.0 * log(base));
        };
        // The ends may lie past the slowest pair, half - 1, up to rot_dim - 1: the bound
        // is part of the rule that checkpoints with this scaling are trained under.
        auto end = [&](double x) { return fmin(fmax(x, 0.0), (double)d.rot_dim - 1.0); };
        first = end(floor(pair(d.high)));
        width = fmax(end(ceil(pair(d.low))) - first, 0.001);
    }
    // f_i = base^(-2i/rot): products of one root, in the long double's 64 bits
    const long double root = half > 0 ? powl((long double)base, -1.0L / half) : 1.0L;
    long double f = 1.0L;
    for (int i = 0; i < half; ++i, f *= root) {
        double x = (double)f;
        switch (d.scaling) {
            case COLA_ROPE_LINEAR: x /= d.factor; break;
            case COLA_ROPE_YARN: {
                const double w = fmin(fmax((i - first) / width, 0.0), 1.0);
                x = x * (1.0 - w) + x / d.factor * w;
                break;
            }
            case COLA_ROPE_WAVELENGTH: {
                const double s = fmin(fmax(((double)d.orig_len * x / two_pi - d.low) / (d.high - d.low), 0.0), 1.0);
                x = s * x + (1.0 - s) * x / d.factor;
                break;
            }
            default: break;
        }
        a->rev[i] = x / two_pi;
    }
}

int check_rope(const cola_rope_desc* d, bool cache, RopeArgs* a) {
    if (!d || !dtype_ok(d->dtype) || d->reserved != 0) return COLA_ERR_INVALID_ARG;
    if (d->layout != COLA_ROPE_HALF && d->layout != COLA_ROPE_INTERLEAVED) return COLA_ERR_INVALID_ARG;
    if (d->scaling < COLA_ROPE_NONE || d->scaling > COLA_ROPE_WAVELENGTH) return COLA_ERR_INVALID_ARG;
    if (!(d->base > 1.0) || !isfinite(d->base) || !(d->mscale >= 0.0) || !(d->mscale <= 1e30)) return COLA_ERR_INVALID_ARG;
    if (d->scaling != COLA_ROPE_NONE && (!(d->factor >= 1.0) || !isfinite(d->factor))) return COLA_ERR_INVALID_ARG;
    if (d->scaling == COLA_ROPE_YARN || d->scaling == COLA_ROPE_WAVELENGTH)
        if (!(d->low > 0.0) || !(d->high > d->low) || !isfinite(d->high) || d->orig_len < 1) return COLA_ERR_INVALID_ARG;
    if (d->T < 0 || d->T > kMaxInt || d->seq_len < 0 || d->heads_q < 0 || d->heads_k < 0) return COLA_ERR_BAD_SHAPE;
    if (d->heads_q + d->heads_k < 1 || d->head_dim < 1 || d->head_dim > kRopeMaxDim) return COLA_ERR_BAD_SHAPE;
    if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 2 != 0) return COLA_ERR_BAD_SHAPE;
    if (d->scaling == COLA_ROPE_BASE && d->rot_dim == 2) return COLA_ERR_BAD_SHAPE;   // its exponent is infinite
    if (d->heads_q > kMaxPitch || d->heads_k > kMaxPitch) return COLA_ERR_BAD_SHAPE;
    const int64_t wq = d->heads_q * d->head_dim, wk = d->heads_k * d->head_dim;
    a->ldq = d->ldq ? d->ldq : wq;
    a->ldqo = d->ldqo ? d->ldqo : wq;
    a->ldk = d->ldk ? d->ldk : wk;
    a->ldko = d->ldko ? d->ldko : wk;
    a->ldv = d->ldv ? d->ldv : wk;
    if (a->ldq < wq || a->ldqo < wq || a->ldk < wk || a->ldko < wk || (cache && a->ldv < wk)) return COLA_ERR_BAD_SHAPE;
    for (int64_t ld : {a->ldq, a->ldqo, a->ldk, a->ldko, a->ldv})
        if (ld > kMaxPitch) return COLA_ERR_BAD_SHAPE;
    a->T = d->T;
    a->seq_len = d->seq_len;
    a->hq = (int)d->heads_q;
    a->hk = (int)d->heads_k;
    a->hd = (int)d->head_dim;
    a->rot = (int)d->rot_dim;
    a->interleaved = d->layout == COLA_ROPE_INTERLEAVED;
    return COLA_OK;
}

int check_cache(const cola_cache_desc* c) {
    if (!c || !dtype_ok(c->dtype) || c->reserved != 0) return COLA_ERR_INVALID_ARG;
    if (c->n_pages < 0 || c->n_pages > kMaxInt || !page_ok(c->page_size, 16) || c->heads < 1 || c->heads > kMaxPitch ||
        c->head_dim < 1 || c->head_dim > kRopeMaxDim)
        return COLA_ERR_BAD_SHAPE;
    if ((double)c->n_pages * (double)c->page_size * (double)c->heads * (double)c->head_dim > 4.0e15)
        return COLA_ERR_BAD_SHAPE;
    return COLA_OK;
}

// An output over its input: the same rows, or none of them (the pitches decide
// what interleaves, so only equal starts are judged).
bool in_place_ok(const void* in, int64_t ld_in, const void* out, int64_t ld_out) { return in != out || ld_in == ld_out; }

int rope(const cola_rope_desc* d, const void* q, const void* k, const int32_t* pos, void* qo, void* ko, float sign,
         cola_stream_t stream) {
    return guarded([&]() -> int {
        RopeArgs a{};
        const int st = check_rope(d, false, &a);
        if (st != COLA_OK) return st;
        if (a.T == 0) return COLA_OK;
        if ((a.hq > 0 && (!q || !qo)) || (a.hk > 0 && (!k || !ko))) return COLA_ERR_INVALID_ARG;
        for (const void* p : {q, k, (const void*)qo, (const void*)ko})
            if (!aligned(p, d->dtype)) return COLA_ERR_INVALID_ARG;
        if (!al4(pos)) return COLA_ERR_INVALID_ARG;
        if ((a.hq > 0 && !in_place_ok(q, a.ldq, qo, a.ldqo)) || (a.hk > 0 && !in_place_ok(k, a.ldk, ko, a.ldko)))
            return COLA_ERR_INVALID_ARG;
        a.q = q; a.k = k; a.qo = qo; a.ko = ko; a.pos = pos;
        a.sign = sign;
        frequencies(*d, &a);
        const double es = d->dtype == COLA_BF16 ? 2.0 : 4.0, n = (double)a.T * (a.hq + a.hk);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_POINTWISE, 3.0 * n * a.rot, 2.0 * es * n * a.hd, s,
                            [&] { return launch_rope(d->dtype == COLA_BF16, false, a, s); }), "rope");
    });
}

// ---- rows into the cache ----
int check_append(const cola_rope_desc* rot, const cola_cache_desc* cache) {
    const int st = check_cache(cache);
    if (st != COLA_OK) return st;
    if (rot->heads_k != cache->heads || rot->head_dim != cache->head_dim) return COLA_ERR_BAD_SHAPE;
    return rot->dtype != cache->dtype ? COLA_ERR_INVALID_ARG : COLA_OK;
}

// The pointers of an append, checked, and its frequencies (T > 0).
int take_append(const cola_rope_desc* rot, const cola_cache_desc* cache, const void* q, const void* k, const void* v,
                const int32_t* positions, const int32_t* slots, void* q_out, void* K, void* V, RopeArgs* a) {
    if ((a->hq > 0 && (!q || !q_out)) || !k || !v || !slots) return COLA_ERR_INVALID_ARG;
    if (cache->n_pages > 0 && (!K || !V || K == V)) return COLA_ERR_INVALID_ARG;
    for (const void* p : {q, k, v, (const void*)q_out})
        if (!aligned(p, rot->dtype)) return COLA_ERR_INVALID_ARG;
    if (!al4(positions) || !al4(slots) || !al16(K) || !al16(V)) return COLA_ERR_INVALID_ARG;
    if (a->hq > 0 && !in_place_ok(q, a->ldq, q_out, a->ldqo)) return COLA_ERR_INVALID_ARG;
    a->q = q; a->k = k; a->v = v; a->qo = q_out; a->K = K; a->V = V; a->pos = positions; a->slots = slots;
    a->lg_page = log2_of(cache->page_size);
    a->n_slots = cache->n_pages * cache->page_size;
    a->sign = 1.0f;
    frequencies(*rot, a);
    return COLA_OK;
}

// ---- norms ----
int check_norm(const cola_rope_desc* d, bool cache, double eps, const void* g_q, const void* g_k, NormRopeArgs* a) {
    const int st = check_rope(d, cache, a);
    if (st != COLA_OK) return st;
    const float e = (float)eps;
    // below the normal numbers the hardware's 1 / sqrt may take it for zero: NaN for a head of zeros
    if (!(e >= FLT_MIN) || !isfinite(e)) return COLA_ERR_INVALID_ARG;
    if (!aligned(g_q, d->dtype) || !aligned(g_k, d->dtype)) return COLA_ERR_INVALID_ARG;
    a->gq = g_q; a->gk = g_k;
    a->eps = e;
    a->inv_hd = 1.0f / (float)a->hd;
    return COLA_OK;
}

// Rows that are there where there are heads, aligned to their elements.
bool rows_ok(const cola_rope_desc* d, const RopeArgs& a, const void* q, const void* k, const void* qo, const void* ko) {
    if ((a.hq > 0 && (!q || !qo)) || (a.hk > 0 && (!k || !ko))) return false;
    for (const void* p : {q, k, qo, ko})
        if (!aligned(p, d->dtype)) return false;
    return true;
}

// ---- attention ----
int check_attn(const cola_prefix_attn_desc* d, const cola_cache_desc* c, bool tree, PrefixAttnShape* out) {
    const int st = check_cache(c);
    if (st != COLA_OK) return st;
    if (!d) return COLA_ERR_INVALID_ARG;
    if (!(d->scale >= 0.0) || !isfinite(d->scale)) return COLA_ERR_INVALID_ARG;
    if (c->dtype != COLA_BF16 || (c->head_dim != 64 && c->head_dim != 128)) return COLA_ERR_UNSUPPORTED;
    if (d->n_req < 0 || d->n_req > 65535 || d->T < 0 || d->T > kMaxInt || d->heads_q < 1 || d->heads_q > kMaxPitch)
        return COLA_ERR_BAD_SHAPE;
    if (d->T * d->heads_q > kMaxInt || d->heads_q % c->heads != 0) return COLA_ERR_BAD_SHAPE;
    // A launch has a tile for every row that a request may have, whether it has or not.
    // These bounds keep it below 2^30 workgroups (a request's tiles are 128 rows where
    // it may have more than 32, and the plan parts the keys of so many tiles no
    // further), 1.4 s if all are empty.
    const int64_t pairs = d->n_req * d->heads_q;
    if (pairs > (int64_t(1) << 28)) return COLA_ERR_BAD_SHAPE;
    if (d->prefix_len < 0 || d->prefix_len > kMaxKeys || d->max_kv < 0 || d->max_kv > kMaxKeys || d->max_new < 1 ||
        d->max_new > (tree ? COLA_TREE_MAX : kMaxKeys) || d->max_pages < 0 || d->max_pages > kMaxInt)
        return COLA_ERR_BAD_SHAPE;
    if (pairs * (d->max_new < d->T ? d->max_new : d->T) > (int64_t(1) << 36)) return COLA_ERR_BAD_SHAPE;
    PrefixAttnShape s{};
    const int64_t need = (d->max_kv + c->page_size - 1) / c->page_size, w = d->heads_q * c->head_dim;
    s.max_pages = d->max_pages ? d->max_pages : need;
    s.ldq = d->ldq ? d->ldq : w;
    s.ldo = d->ldo ? d->ldo : w;
    if (s.max_pages < need || s.ldq < w || s.ldo < w || s.ldq > kMaxPitch || s.ldo > kMaxPitch || s.ldq % 8 != 0 ||
        s.ldo % 8 != 0)
        return COLA_ERR_BAD_SHAPE;
    s.scale = d->scale != 0.0 ? d->scale : 1.0 / sqrt((double)c->head_dim);
    const float f = (float)(s.scale * 1.4426950408889634);
    if (!(f > 1e-30f) || !(f < 1e30f)) return COLA_ERR_INVALID_ARG;       // the exponent's factor in fp32
    s.n_req = d->n_req; s.T = d->T; s.max_new = d->max_new; s.prefix = d->prefix_len; s.max_kv = d->max_kv;
    s.n_pages = c->n_pages; s.page_size = c->page_size;
    s.hq = (int)d->heads_q; s.hk = (int)c->heads; s.hd = (int)c->head_dim;
    *out = s;
    return COLA_OK;
}

size_t attn_workspace(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache, bool tree) {
    PrefixAttnShape sh;
    if (check_attn(desc, cache, tree, &sh) != COLA_OK || sh.n_req == 0 || sh.T == 0) return 0;
    return (tree ? plan_tree_attn(sh) : plan_prefix_attn(sh)).ws_bytes;
}

// cola_prefix_attn, or cola_tree_attn.
int attend(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache, const void* q, const void* K, const void* V,
           const int32_t* prefix_table, const int32_t* table, const int32_t* kv_len, const int32_t* start, bool tree,
           const uint64_t* mask, void* out, float* lse, void* ws, size_t ws_bytes, cola_stream_t stream) {
    return guarded([&]() -> int {
        PrefixAttnShape sh;
        const int st = check_attn(desc, cache, tree, &sh);
        if (st != COLA_OK) return st;
        if (sh.n_req == 0 || sh.T == 0) return COLA_OK;
        if (!q || !out || q == out) return COLA_ERR_INVALID_ARG;
        if (sh.n_pages > 0 && (!K || !V)) return COLA_ERR_INVALID_ARG;
        if ((sh.prefix > 0 && !prefix_table) || (sh.max_kv > 0 && (!table || !kv_len))) return COLA_ERR_INVALID_ARG;
        for (const void* p : {q, K, V, (const void*)out, (const void*)ws})
            if (!al16(p)) return COLA_ERR_INVALID_ARG;
        for (const void* p : {(const void*)prefix_table, (const void*)table, (const void*)kv_len, (const void*)start,
                              (const void*)lse})
            if (!al4(p)) return COLA_ERR_INVALID_ARG;
        if (tree && (!mask || !al8(mask))) return COLA_ERR_INVALID_ARG;
        const PrefixAttnPlan p = tree ? plan_tree_attn(sh) : plan_prefix_attn(sh);
        if (p.ws_bytes > 0 && (!ws || ws_bytes < p.ws_bytes)) return COLA_ERR_WORKSPACE;
        PrefixAttnPtrs t{};
        t.q = static_cast<const uint16_t*>(q);
        t.K = static_cast<const uint16_t*>(K);
        t.V = static_cast<const uint16_t*>(V);
        t.prefix_table = prefix_table; t.table = table; t.kv_len = kv_len; t.start = start;
        t.out = static_cast<uint16_t*>(out);
        t.lse = lse;
        t.ws = ws;
        t.mask = mask;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        // work for the bounds: the lengths themselves are in GPU memory
        const double rows = (double)p.rows, keys = (double)sh.prefix + (double)sh.max_kv;
        const double bytes = 4.0 * rows * sh.hd + 4.0 * ((double)sh.prefix + (double)sh.n_req * sh.max_kv) * sh.hk * sh.hd;
        const int e = chk(timed_fn(COLA_KC_ATTN_FWD, 4.0 * rows * keys * sh.hd, bytes, s,
                                   [&] { return launch_prefix_attn(sh, p, t, s); }), tree ? "tree_attn" : "prefix_attn");
        if (e != COLA_OK || p.direct) return e;
        const double parts = (double)p.splits_p + p.splits_s;
        return chk(timed_fn(COLA_KC_ATTN_FWD, 2.0 * rows * sh.hd * parts, rows * sh.hd * (4.0 * parts + 2.0), s,
                            [&] { return launch_prefix_join(sh, p, t, s); }), "prefix_join");
    });
}

}  // namespace

extern "C" {

int cola_rope_fwd(const cola_rope_desc* desc, const void* q, const void* k, const int32_t* positions, void* q_out,
                  void* k_out, cola_stream_t stream) {
    return rope(desc, q, k, positions, q_out, k_out, 1.0f, stream);
}

int cola_rope_bwd(const cola_rope_desc* desc, const void* dq_out, const void* dk_out, const int32_t* positions,
                  void* dq, void* dk, cola_stream_t stream) {
    return rope(desc, dq_out, dk_out, positions, dq, dk, -1.0f, stream);
}

int cola_cache_append(const cola_rope_desc* rot, const cola_cache_desc* cache, const void* q, const void* k,
                      const void* v, const int32_t* positions, const int32_t* slots, void* q_out, void* K, void* V,
                      cola_stream_t stream) {
    return guarded([&]() -> int {
        RopeArgs a{};
        int st = check_rope(rot, true, &a);
        if (st == COLA_OK) st = check_append(rot, cache);
        if (st != COLA_OK) return st;
        if (a.T == 0) return COLA_OK;
        st = take_append(rot, cache, q, k, v, positions, slots, q_out, K, V, &a);
        if (st != COLA_OK) return st;
        const double es = rot->dtype == COLA_BF16 ? 2.0 : 4.0, n = (double)a.T * a.hd;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_POINTWISE, 3.0 * (double)a.T * (a.hq + a.hk) * a.rot, 2.0 * es * n * (a.hq + 2 * a.hk), s,
                            [&] { return launch_rope(rot->dtype == COLA_BF16, true, a, s); }), "cache_append");
    });
}

int cola_page_map(const cola_page_map_desc* d, const int32_t* kv_len, const int32_t* n_new, const int32_t* free_pages,
                  const int32_t* free_at, int32_t* table, int32_t* start, int32_t* slots, int32_t* positions,
                  int32_t* free_next, cola_stream_t stream) {
    return guarded([&]() -> int {
        if (!d) return COLA_ERR_INVALID_ARG;
        if (d->n_req < 0 || d->n_req > COLA_PAGE_MAP_MAX_REQ || d->T < 0 || d->T > kMaxInt || !page_ok(d->page_size, 1) ||
            d->max_pages < 0 || d->max_pages > kMaxInt || d->n_free < 0 || d->n_free > kMaxInt || d->pos0 < 0 ||
            d->pos0 > kMaxInt || d->n_req * d->max_pages > kMaxInt)
            return COLA_ERR_BAD_SHAPE;
        if (!start || !free_next || free_next == free_at) return COLA_ERR_INVALID_ARG;
        if (d->n_req > 0 && (!kv_len || !n_new || (d->max_pages > 0 && !table))) return COLA_ERR_INVALID_ARG;
        if ((d->T > 0 && (!slots || !positions)) || (d->n_free > 0 && !free_pages)) return COLA_ERR_INVALID_ARG;
        for (const void* p : {(const void*)kv_len, (const void*)n_new, (const void*)free_pages, (const void*)free_at,
                              (const void*)table, (const void*)start, (const void*)slots, (const void*)positions,
                              (const void*)free_next})
            if (!al4(p)) return COLA_ERR_INVALID_ARG;
        PageMapArgs a{};
        a.kv_len = kv_len; a.n_new = n_new; a.free_pages = free_pages; a.free_at = free_at;
        a.table = table; a.start = start; a.slots = slots; a.positions = positions; a.free_next = free_next;
        a.n_req = (int)d->n_req; a.lg_page = log2_of(d->page_size);
        a.T = d->T; a.max_pages = d->max_pages; a.n_free = d->n_free; a.pos0 = d->pos0;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_POINTWISE, 0.0, 4.0 * (3.0 * (double)d->n_req + 2.0 * (double)d->T), s,
                            [&] { return launch_page_map(a, s); }), "page_map");
    });
}

size_t cola_prefix_attn_workspace_bytes(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache) {
    return attn_workspace(desc, cache, false);
}

int cola_prefix_attn(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache, const void* q, const void* K,
                     const void* V, const int32_t* prefix_table, const int32_t* table, const int32_t* kv_len,
                     const int32_t* start, void* out, float* lse, void* ws, size_t ws_bytes, cola_stream_t stream) {
    return attend(desc, cache, q, K, V, prefix_table, table, kv_len, start, false, nullptr, out, lse, ws, ws_bytes, stream);
}

size_t cola_tree_attn_workspace_bytes(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache) {
    return attn_workspace(desc, cache, true);
}

int cola_tree_attn(const cola_prefix_attn_desc* desc, const cola_cache_desc* cache, const void* q, const void* K,
                   const void* V, const int32_t* prefix_table, const int32_t* table, const int32_t* kv_len,
                   const int32_t* start, const uint64_t* mask, void* out, float* lse, void* ws, size_t ws_bytes,
                   cola_stream_t stream) {
    return attend(desc, cache, q, K, V, prefix_table, table, kv_len, start, true, mask, out, lse, ws, ws_bytes, stream);
}

int cola_norm_rope_fwd(const cola_rope_desc* desc, double eps, const void* q, const void* k, const void* g_q,
                       const void* g_k, const int32_t* positions, void* q_out, void* k_out, cola_stream_t stream) {
    return guarded([&]() -> int {
        NormRopeArgs a{};
        const int st = check_norm(desc, false, eps, g_q, g_k, &a);
        if (st != COLA_OK) return st;
        if (a.T == 0) return COLA_OK;
        if (!rows_ok(desc, a, q, k, q_out, k_out) || !al4(positions)) return COLA_ERR_INVALID_ARG;
        if ((a.hq > 0 && !in_place_ok(q, a.ldq, q_out, a.ldqo)) || (a.hk > 0 && !in_place_ok(k, a.ldk, k_out, a.ldko)))
            return COLA_ERR_INVALID_ARG;
        a.q = q; a.k = k; a.qo = q_out; a.ko = k_out; a.pos = positions;
        a.sign = 1.0f;
        frequencies(*desc, &a);
        const double es = desc->dtype == COLA_BF16 ? 2.0 : 4.0, n = (double)a.T * (a.hq + a.hk) * a.hd;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_NORM, 7.0 * n, 2.0 * es * n, s,
                            [&] { return launch_norm_rope(desc->dtype == COLA_BF16, NORM_FWD, a, s); }), "norm_rope");
    });
}

size_t cola_norm_rope_workspace_bytes(const cola_rope_desc* desc) {
    NormRopeArgs a{};
    if (check_norm(desc, false, 1.0, nullptr, nullptr, &a) != COLA_OK || a.T == 0) return 0;
    return norm_rope_parts(desc->dtype == COLA_BF16, a) * 8 * (size_t)a.hd;
}

int cola_norm_rope_bwd(const cola_rope_desc* desc, double eps, const void* dq_out, const void* dk_out, const void* q,
                       const void* k, const void* g_q, const void* g_k, const int32_t* positions, void* dq, void* dk,
                       float* dg_q, float* dg_k, void* ws, size_t ws_bytes, cola_stream_t stream) {
    return guarded([&]() -> int {
        NormRopeArgs a{};
        const int st = check_norm(desc, false, eps, g_q, g_k, &a);
        if (st != COLA_OK) return st;
        if (!al4(dg_q) || !al4(dg_k) || !al4(positions) || !al4(ws) || (dg_q && dg_q == dg_k)) return COLA_ERR_INVALID_ARG;
        if ((a.hq == 0 && dg_q) || (a.hk == 0 && dg_k)) return COLA_ERR_INVALID_ARG;
        const bool bf16 = desc->dtype == COLA_BF16;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        if (a.T == 0) {
            for (float* g : {dg_q, dg_k}) {
                if (!g) continue;
                const int e = chk(timed_fn(COLA_KC_FILL, 0.0, 4.0 * a.hd, s, [&] { return launch_fill_zero(g, a.hd, s); }), "norm_fill");
                if (e != COLA_OK) return e;
            }
            return COLA_OK;
        }
        if (!rows_ok(desc, a, q, k, dq, dk) || !rows_ok(desc, a, dq_out, dk_out, dq, dk)) return COLA_ERR_INVALID_ARG;
        // dq and dk have the pitches of q and k
        if ((a.hq > 0 && !in_place_ok(dq_out, a.ldqo, dq, a.ldq)) || (a.hk > 0 && !in_place_ok(dk_out, a.ldko, dk, a.ldk)))
            return COLA_ERR_INVALID_ARG;
        const size_t parts = norm_rope_parts(bf16, a);
        if (!ws || ws_bytes < parts * 8 * (size_t)a.hd) return COLA_ERR_WORKSPACE;
        a.q = q; a.k = k; a.dqo = dq_out; a.dko = dk_out; a.qo = dq; a.ko = dk; a.pos = positions;
        a.dgq = dg_q; a.dgk = dg_k; a.part = static_cast<float*>(ws);
        a.sign = -1.0f;
        frequencies(*desc, &a);
        const double es = bf16 ? 2.0 : 4.0, n = (double)a.T * (a.hq + a.hk) * a.hd;
        const int e = chk(timed_fn(COLA_KC_NORM_BWD, 20.0 * n, 3.0 * es * n, s,
                                   [&] { return launch_norm_rope(bf16, NORM_BWD, a, s); }), "norm_rope_bwd");
        if (e != COLA_OK || (!dg_q && !dg_k)) return e;
        return chk(timed_fn(COLA_KC_NORM_BWD, 2.0 * (double)parts * a.hd, 8.0 * (double)parts * a.hd, s,
                            [&] { return launch_norm_gain(a, parts, s); }), "norm_gain");
    });
}

int cola_norm_append(const cola_rope_desc* rot, const cola_cache_desc* cache, double eps, const void* q, const void* k,
                     const void* v, const void* g_q, const void* g_k, const int32_t* positions, const int32_t* slots,
                     void* q_out, void* K, void* V, cola_stream_t stream) {
    return guarded([&]() -> int {
        NormRopeArgs a{};
        int st = check_norm(rot, true, eps, g_q, g_k, &a);
        if (st == COLA_OK) st = check_append(rot, cache);
        if (st != COLA_OK) return st;
        if (a.T == 0) return COLA_OK;
        st = take_append(rot, cache, q, k, v, positions, slots, q_out, K, V, &a);
        if (st != COLA_OK) return st;
        const double es = rot->dtype == COLA_BF16 ? 2.0 : 4.0, n = (double)a.T * a.hd;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_NORM, 7.0 * n * (a.hq + a.hk), 2.0 * es * n * (a.hq + 2 * a.hk), s,
                            [&] { return launch_norm_rope(rot->dtype == COLA_BF16, NORM_APPEND, a, s); }), "norm_append");
    });
}

int cola_tree_map(const cola_tree_map_desc* d, const int32_t* parent, const int32_t* kv_len, const int32_t* start,
                  uint64_t* mask, int32_t* positions, cola_stream_t stream) {
    return guarded([&]() -> int {
        if (!d) return COLA_ERR_INVALID_ARG;
        if (d->n_req < 0 || d->n_req > 65535 || d->T < 0 || d->T > kMaxInt || d->max_new < 1 || d->max_new > COLA_TREE_MAX ||
            d->pos0 < 0 || d->pos0 > kMaxInt)
            return COLA_ERR_BAD_SHAPE;
        if (d->T == 0) return COLA_OK;
        if (!mask || !positions || (d->n_req > 0 && (!parent || !kv_len))) return COLA_ERR_INVALID_ARG;
        if ((const void*)positions == parent || (const void*)mask == parent || (const void*)mask == positions) return COLA_ERR_INVALID_ARG;
        for (const void* p : {(const void*)parent, (const void*)kv_len, (const void*)start, (const void*)positions})
            if (!al4(p)) return COLA_ERR_INVALID_ARG;
        if (!al8(mask)) return COLA_ERR_INVALID_ARG;
        TreeMapArgs a{};
        a.parent = parent; a.kv_len = kv_len; a.start = start; a.mask = mask; a.positions = positions;
        a.T = d->T; a.pos0 = d->pos0;
        a.n_req = (int)d->n_req; a.max_new = (int)d->max_new; a.words = (int)((d->max_new + 63) / 64);
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_POINTWISE, 0.0, (double)d->T * (8.0 + 8.0 * a.words), s,
                            [&] { return launch_tree_map(a, s); }), "tree_map");
    });
}

int cola_logits_adjust(const cola_logits_desc* d, const cola_logits_rules* rules, const void* logits,
                       const int32_t* start, void* out, cola_stream_t stream) {
    return guarded([&]() -> int {
        if (!d || !rules || !dtype_ok(d->dtype) || d->reserved != 0) return COLA_ERR_INVALID_ARG;
        if (d->T < 0 || d->T > kMaxInt || d->V < 1 || d->V > kMaxPitch || d->n_req < 0 || d->n_req > 65535 || d->max_hist < 0 ||
            d->max_hist >= kMaxKeys || d->max_new < 0 || d->max_new > COLA_TREE_MAX || d->n_bias < 0 || d->n_bias >= kMaxKeys ||
            d->n_allowed < 0 || d->n_allowed > kMaxInt)
            return COLA_ERR_BAD_SHAPE;
        LogitsArgs a{};
        a.ldl = d->ldl ? d->ldl : d->V;
        a.ldo = d->ldo ? d->ldo : d->V;
        a.lda = d->lda ? d->lda : (d->V + 31) / 32;
        if (a.ldl < d->V || a.ldl > kMaxPitch || a.ldo < d->V || a.ldo > kMaxPitch || a.lda < (d->V + 31) / 32 || a.lda > kMaxPitch)
            return COLA_ERR_BAD_SHAPE;
        if (d->T == 0 || d->n_req == 0) return COLA_OK;
        const cola_logits_rules& u = *rules;
        if (!logits || !out || !in_place_ok(logits, a.ldl, out, a.ldo)) return COLA_ERR_INVALID_ARG;
        if (!aligned(logits, d->dtype) || !aligned(out, d->dtype) || !al8(u.mask)) return COLA_ERR_INVALID_ARG;
        for (const void* p : {(const void*)start, (const void*)u.history, (const void*)u.prompt_len, (const void*)u.hist_len,
                              (const void*)u.draft, (const void*)u.repetition, (const void*)u.presence, (const void*)u.frequency,
                              (const void*)u.bias_start, (const void*)u.bias_token, (const void*)u.bias, (const void*)u.allowed,
                              (const void*)u.allowed_row})
            if (!al4(p)) return COLA_ERR_INVALID_ARG;
        if (u.hist_len && d->max_hist > 0 && !u.history) return COLA_ERR_INVALID_ARG;
        if (u.draft && (!u.mask || d->max_new < 1)) return COLA_ERR_INVALID_ARG;
        if (u.bias_start && d->n_bias > 0 && (!u.bias_token || !u.bias)) return COLA_ERR_INVALID_ARG;
        a.logits = logits; a.out = out; a.start = start;
        a.history = u.history; a.prompt_len = u.prompt_len; a.hist_len = u.hist_len; a.draft = u.draft; a.mask = u.mask;
        if (u.hist_len || u.draft) {
            a.repetition = u.repetition; a.presence = u.presence; a.frequency = u.frequency;
        }
        a.bias_start = d->n_bias > 0 ? u.bias_start : nullptr; a.bias_token = u.bias_token; a.bias = u.bias;
        a.allowed = d->n_allowed > 0 ? u.allowed : nullptr; a.allowed_row = u.allowed_row;
        a.T = d->T; a.V = d->V; a.max_hist = d->max_hist; a.n_bias = d->n_bias; a.n_allowed = d->n_allowed;
        a.n_req = (int)d->n_req; a.max_new = (int)d->max_new; a.words = (int)((d->max_new + 63) / 64);
        const double es = d->dtype == COLA_BF16 ? 2.0 : 4.0, n = (double)d->T * (double)d->V;
        hipStream_t s = reinterpret_cast<hipStream_t>(stream);
        return chk(timed_fn(COLA_KC_POINTWISE, 4.0 * n, 2.0 * es * n, s,
                            [&] { return launch_logits(d->dtype == COLA_BF16, a, s); }), "logits_adjust");
    });
}

}  // extern "C"
