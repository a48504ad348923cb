// serve.hpp -- declarations of the serving path shared by rope.hip, norm_rope.hip,
// page_map.hip, tree_map.hip, prefix_attn.hpp, prefix_attn.hip, tree_attn.hip,
// logits.hip and serve_abi.hip.  Not part of the public ABI (that is
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

// The rotation with each head normalised and scaled before it.  Backward: q and k are
// the forward's, dqo and dko the gradients' rows, qo and ko what they become (at the
// pitches ldq, ldk).
struct NormRopeArgs : RopeArgs {
    const void *gq, *gk;              // gains [hd], or NULL
    const void *dqo, *dko;
    float *dgq, *dgk, *part;          // part: [workgroups][2][hd]
    float eps, inv_hd;
    // filled by the launcher: lanes of a head, elements of a vector
    int group, pv;
    bool past;
};
enum NormKind : int { NORM_FWD = 0, NORM_APPEND = 1, NORM_BWD = 2 };
// Most workgroups of the backward's first launch, but where one row needs more: four a
// CU.  Of the bf16 form for halves in vectors of 8 a CU holds two at once (183 registers),
// of the one for neighbours three (142), of fp32 and narrower vectors four to seven, where
// heads have more than 64 units one or two: two rounds, a round and a third, one, and two
// or four.  1536 took 64 us against 70 where neighbours turn (8191 rows of 32 + 8 heads of
// 128) and 205 against 191 where halves do.
constexpr int64_t kParts = 1024;
size_t norm_rope_parts(bool bf16, NormRopeArgs a);
hipError_t launch_norm_rope(bool bf16, NormKind kind, NormRopeArgs& a, hipStream_t s);
hipError_t launch_norm_gain(const NormRopeArgs& a, size_t parts, hipStream_t s);

struct TreeMapArgs {
    const int32_t *parent, *kv_len, *start;
    uint64_t* mask;
    int32_t* positions;
    int64_t T, pos0;
    int n_req, max_new, words;
};
hipError_t launch_tree_map(const TreeMapArgs& a, hipStream_t s);

struct LogitsArgs {
    const void* logits;
    void* out;
    const int32_t *start, *history, *prompt_len, *hist_len, *draft;
    const uint64_t* mask;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_start, *bias_token;
    const float* bias;
    const uint32_t* allowed;
    const int32_t* allowed_row;
    int64_t T, V, ldl, ldo, lda, max_hist, n_bias, n_allowed;
    int n_req, max_new, words;
};
hipError_t launch_logits(bool bf16, const LogitsArgs& a, hipStream_t s);

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
    const uint64_t* mask;             // trees: [T][words of max_new bits]; NULL: new tokens see each other in order
};
// Launches of one call, and the bytes of its workspace.
struct PrefixAttnPlan {
    int kind_p, kind_s;               // kinds of tiles on the prefix and on the requests' own tokens (Kind in prefix_attn.hpp)
    int tiles_p, tiles_s;             // row tiles: of the batch, of one request
    int splits_p, splits_s;           // parts of the keys
    int64_t chunk_p, chunk_s;         // keys per part
    int64_t rows;                     // T * heads_q
    bool direct;                      // one part in all, of the requests' own keys: no join
    size_t ws_bytes;
};
PrefixAttnPlan plan_prefix_attn(const PrefixAttnShape& sh);
PrefixAttnPlan plan_tree_attn(const PrefixAttnShape& sh);
// One launch of the kernels for trees; args: their arguments (Args in prefix_attn.hpp).
hipError_t start_tree_attn(int hd, const PrefixAttnPlan& p, const void* args, unsigned grid, hipStream_t s);
hipError_t launch_prefix_attn(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t, hipStream_t s);
hipError_t launch_prefix_join(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t, hipStream_t s);

}  // namespace cola
