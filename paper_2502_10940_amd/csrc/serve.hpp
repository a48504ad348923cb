// serve.hpp -- declarations of the serving path shared by rope.hip, page_map.hip,
// prefix_attn.hip and serve_abi.hip.  Not part of the public ABI (that is
// include/cola.h).
#pragma once

#include "../../include/cola.h"
#include "internal.hpp"

namespace cola {

// Largest head, and so the most pairs that turn (their frequencies travel in the
// kernel's arguments: 2 KB of the 4 KB a launch may pass).
constexpr int kRopeMaxDim = 512;

struct RopeArgs {
    const void *q, *k, *v;            // v: with a cache only
    void *qo, *ko;                    // ko: without a cache
    void *K, *V;                      // the cache
    const int32_t *pos, *slots;
    int64_t ldq, ldk, ldv, ldqo, ldko;
    int64_t T, seq_len;
    int64_t n_slots;                  // slots of the cache
    int hq, hk, hd, rot;
    int lg_page;
    int interleaved;
    float mscale, sign;               // on cosine and sine; on the sine alone (-1: the way back)
    // filled by the launcher
    int units, turning, lanes, tpw;
    double rev[kRopeMaxDim / 2];      // turns per position of each pair
};
hipError_t launch_rope(bool bf16, bool cache, RopeArgs& a, hipStream_t s);

struct PageMapArgs {
    const int32_t *kv_len, *n_new, *free_pages, *free_at;
    int32_t *table, *start, *slots, *positions, *free_next;
    int n_req, lg_page;
    int64_t T, max_pages, n_free, pos0;
};
hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s);

struct PrefixAttnShape {
    int64_t n_req, T, max_new, prefix, max_kv, max_pages;
    int64_t n_pages, page_size;
    int hq, hk, hd;
    int64_t ldq, ldo;
    double scale;
};
struct PrefixAttnPtrs {
    const uint16_t *q, *K, *V;
    const int32_t *prefix_table, *table, *kv_len, *start;
    uint16_t* out;
    float* lse;
    void* ws;
};
// Launches of one call, and the bytes of its workspace.
struct PrefixAttnPlan {
    int kind_p, kind_s;               // kinds of tiles on the prefix and on the requests' own tokens (Kind in prefix_attn.hip)
    int tiles_p, tiles_s;             // row tiles: of the batch, of one request
    int splits_p, splits_s;           // parts of the keys
    int64_t chunk_p, chunk_s;         // keys per part
    int64_t rows;                     // T * heads_q
    bool direct;                      // one part in all, of the requests' own keys: no join
    size_t ws_bytes;
};
PrefixAttnPlan plan_prefix_attn(const PrefixAttnShape& sh);
hipError_t launch_prefix_attn(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t, hipStream_t s);
hipError_t launch_prefix_join(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t, hipStream_t s);

}  // namespace cola
