// Attention over an uncompressed cache that grows and shrinks, its blocks and its eviction: what the kernels (cache_attend.hip,
// cache_blocks.hip, evict.hip) and the C ABI (cache_api.hip) share.
#pragma once

#include "xkv_common.h"

namespace xkv {

// What a query attends to.  Its tokens are numbered 0 .. T - 1, T known on the device only:
//   tree     the rows of the cache in use, then the drafted tokens; bits of `tree` say which of those it sees
//   weights  the rows in use; logits are kept
//   blocks   the rows of the blocks listed in sel, ascending; the last one is the query's own and ends with the last visible row
enum class CacheMode { tree, weights, blocks };

struct CacheArgs {
    const void *K, *V, *q;            // [batch][H_kv][L][d_h], [batch][N][H_q][d_h]
    const void *K_draft, *V_draft;    // tree: [batch][H_kv][N][d_h]
    const int32_t *lengths;           // tree, weights: [batch], blocks: [batch][N] visible rows (nullable: L)
    const uint32_t *tree;             // tree: [batch][N][words] (nullable: token i sees the drafted tokens up to i)
    const int32_t *sel;               // blocks: [batch][N][H_kv][k_ch]
    float *part_o, *part_ml, *logits; // partials [batch][N][H_q][splits][d_h], [..][2]; weights: logits [batch][H_q][L]
    void *out;
    int L, H_kv, H_q, d_h, batch, N, words, c, k_ch, splits, chunk;
    int rows;  // rows (query token, head) per workgroup of the matrix-core kernel, 0: the general one
    float scale;
};

// Rows of the cache that sequence (or query) i may read; lengths are clamped to the room that there is.
__device__ __forceinline__ int cache_rows(const CacheArgs &a, int i)
{
    if (!a.lengths) return a.L;
    const int n = a.lengths[i];
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

// Tokens of a query, with n = cache_rows.
__device__ __forceinline__ int cache_tokens(const CacheArgs &a, CacheMode mode, int n)
{
    if (mode == CacheMode::tree) return n + a.N;
    if (mode == CacheMode::weights) return n;
    const int blocks = (n + a.c - 1) / a.c, listed = blocks < a.k_ch ? blocks : a.k_ch;
    return listed > 0 ? (listed - 1) * a.c + n - (blocks - 1) * a.c : 0;
}

struct CachePlan {
    int n_rep, words, n_c, k_ch;
    float scale;
    int chunk, splits, rows;  // tokens per workgroup, partials per query head, and as in CacheArgs
    xkv_shape sel_shape;  // the selection as a problem of launch_topk: rows of blocks, or rows of the cache
    Plan sel_plan;
    size_t off_hist, off_state, off_keys, off_sel, off_n, off_logits, off_part_o, off_part_ml, total;
};

// The plan of one call.  N: query tokens of a sequence; c: rows of a block.
xkv_status plan_cache_attend(const xkv_shape &s, CacheMode mode, int N, int c, CachePlan &p);
xkv_status plan_evict(const xkv_shape &s, CachePlan &p);

hipError_t launch_cache_attend(CacheMode mode, const xkv_shape &s, const CacheArgs &a, hipStream_t st);
// weights += the weights that belong to the logits that launch_cache_attend kept
hipError_t launch_cache_weights(const CacheArgs &a, float *weights, hipStream_t st);
hipError_t launch_block_scores(const xkv_shape &s, const CacheArgs &a, const void *landmarks, int n_c, float *scores, hipStream_t st);
hipError_t launch_landmarks_update(const xkv_shape &s, const void *K, const int32_t *lengths, int N, int c, void *landmarks, hipStream_t st);

struct EvictArgs {
    const void *K, *V;
    const float *weights;
    const int32_t *lengths;
    void *K_out, *V_out;
    float *weights_out;
    int32_t *rows_out, *lengths_out;  // nullable
    float *keys;    // [batch][H_kv][L]
    int32_t *sel;   // [batch][H_kv][k]
    int32_t *n;     // [batch] rows in use before
    int L, L_out, H_kv, d_h, k, sink, recent, batch;
};
hipError_t launch_evict(const xkv_shape &s, const CachePlan &p, const EvictArgs &a, uint32_t *hist, uint32_t *state, hipStream_t st);

}  // namespace xkv
