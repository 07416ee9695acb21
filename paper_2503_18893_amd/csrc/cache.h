// Attention over an uncompressed cache that grows and shrinks, its blocks and its eviction: what the kernels (cache_attend.hip,
// cache_blocks.hip, evict.hip) and the C ABI (cache_api.hip) share.
#pragma once

#include "xkv_common.h"

namespace xkv {

constexpr int kMaxCacheParts = 256;  // parts of a sequence that the merge takes
constexpr int kPartBlocks = 2048;    // blocks of a part (its first and its last one may be shared with its neighbours)

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
    // Partials, [part][N][H_q] rows of d_h numbers and of (maximum, sum); the parts of all sequences stand one after the other.
    float *part_o, *part_ml;
    int32_t *table;                   // [batch + 1]: the first part of every sequence, and behind the last one
    float *logits, *weights;          // weights: [batch][H_q][L], [batch][H_kv][L]
    void *out;
    int L, H_kv, H_q, d_h, batch, N, words, c, k_ch;
    int rows;    // rows (query token, head) per workgroup
    int round;   // tokens that a workgroup takes at a time: parts are multiples of it
    int parts;   // room: parts of all sequences (tree, weights), of one query (blocks)
    bool mfma;
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
    const int blocks = (int)(((unsigned)n + (unsigned)a.c - 1u) / (unsigned)a.c), listed = blocks < a.k_ch ? blocks : a.k_ch;
    return listed > 0 ? (listed - 1) * a.c + n - (blocks - 1) * a.c : 0;
}

// ------------------------------------------------------------------------------------------
// Which workgroup takes what.  How many tokens a sequence has is known on the device only, and a cache may have far more room than
// rows in use: every workgroup reads the lengths and finds for itself the smallest part, a multiple of `round` tokens, with which the
// parts of all sequences are at most a.parts.  One lane per sequence, then one per candidate; about 1 us.
// That is even where a.parts is a few times the number of sequences.  The parts planned include one of every sequence, so towards as many sequences
// as parts they round up badly, and from there on a sequence is one part: with 8 KV heads and 64 drafted tokens (32 parts of 256 rows) 11 equal
// sequences give 176 workgroups to 256 compute units, 17 of them 136; and one of 65536 tokens beside 32 of 1024 takes 1025 rounds where an
// even share is 49.
// ------------------------------------------------------------------------------------------
struct CacheUnit {
    int seq, g, tile;    // sequence (blocks: of batch N queries), KV head, row tile
    int part, first;     // place among all parts, and of the sequence's first one
    int t_begin, t_end;  // its tokens
    int n, n_tok;        // rows in use, tokens of the sequence
    bool some;           // whether there is anything to do
};

// Over the 64 lanes of a wavefront, in all of them, without LDS: neighbours, then rows of 16, halves.
template <int CTRL> __device__ __forceinline__ uint32_t lanes_by(uint32_t x) { return __builtin_amdgcn_update_dpp(0u, x, CTRL, 0xF, 0xF, true); }
template <typename T, typename OP> __device__ __forceinline__ T wave_all(T v, OP op)
{
    static_assert(sizeof(T) == 4, "one register");
    auto with = [&](uint32_t o) { v = op(v, __builtin_bit_cast(T, o)); };
    with(lanes_by<0xB1>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x4E>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x141>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x140>(__builtin_bit_cast(uint32_t, v)));
    const auto r16 = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(T, (uint32_t)r16[0]), __builtin_bit_cast(T, (uint32_t)r16[1]));
    const auto r32 = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return op(__builtin_bit_cast(T, (uint32_t)r32[0]), __builtin_bit_cast(T, (uint32_t)r32[1]));
}
struct AddOp {
    template <typename T> __device__ __forceinline__ T operator()(T x, T y) const { return x + y; }
};
struct MaxOp {
    __device__ __forceinline__ float operator()(float x, float y) const { return fmaxf(x, y); }
    __device__ __forceinline__ int operator()(int x, int y) const { return x > y ? x : y; }
};

struct UMaxOp {
    __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return x > y ? x : y; }
};

__device__ __forceinline__ int ceil_div_dev(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

// Tokens per part.  All lanes of a wavefront call it together; t: tokens of sequence `lane` (of the first 64).
// In rounds: r_i of sequence i, at most 2^24, R altogether.  Parts of m rounds number sum ceil(r_i / m), between R / m and R / m + batch,
// so m is at least R / parts, and R / (parts - batch) is enough.  A lane counts for one m between the two.  Divisions are
// products with a reciprocal, a factor of 1 + 2^-20 upwards: never too few, and exact up to 2^20 rounds of a sequence ((r + m - 1) / m
// is a multiple of 1 / m).
__device__ __forceinline__ int cache_chunk(const CacheArgs &a, CacheMode mode, int t)
{
    const int lane = lane_id(), shift = __builtin_ctz(a.round);  // (a power of two)
    constexpr float UP = 1.0f + 0x1p-20f;
    int r = 0, top = 1;
    long long R = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {
        if (b0 > 0) t = b0 + lane < a.batch ? cache_tokens(a, mode, cache_rows(a, b0 + lane)) : 0;
        r = (t + a.round - 1) >> shift;
        R += wave_all(r, AddOp());
        top = MaxOp()(top, wave_all(r, MaxOp()));
    }
    if (a.parts <= a.batch || R == 0) return top << shift;  // (a part per sequence is always allowed)
    const float enough = (float)R * __builtin_amdgcn_rcpf((float)(a.parts - a.batch)) * UP + 1.0f;
    const float least = (float)R * __builtin_amdgcn_rcpf((float)a.parts) * (1.0f - 0x1p-20f);
    const int most_parts = ceil_div_dev(top, kMaxCacheParts);  // (the others may be empty: one sequence may have all the parts)
    int hi = enough < (float)top ? (int)enough : top, lo = least < (float)hi ? (int)least : hi;
    lo = lo > most_parts ? lo : most_parts;
    hi = hi > lo ? hi : lo;
    const int step = ceil_div_dev(hi - lo, kWave - 1), m = lo + lane * step;
    const float inv = __builtin_amdgcn_rcpf((float)m) * UP;
    float used = 0.0f;
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {
        if (a.batch > kWave) {
            t = b0 + lane < a.batch ? cache_tokens(a, mode, cache_rows(a, b0 + lane)) : 0;
            r = (t + a.round - 1) >> shift;
        }
        for (int i = 0; i < kWave && b0 + i < a.batch; ++i) used += floorf((float)(__builtin_amdgcn_readlane(r, i) + m - 1) * inv);
    }
    const uint64_t fits = __ballot(used <= (float)a.parts);  // (the last candidate is at least hi)
    const int best = lo + (fits ? __builtin_ctzll(fits) : kWave - 1) * step;
    return (best > 0 && best < top ? best : top) << shift;
}

__device__ __forceinline__ CacheUnit cache_unit(const CacheArgs &a, CacheMode mode, int tiles)
{
    CacheUnit u{};
    const int lane = lane_id();
    // workgroups go to the eight XCDs in turn: the row tiles of a part, which share its rows of K and V, to one XCD, one after the other
    const int x = (int)blockIdx.x;
    int id = x / tiles;
    u.tile = x % tiles;
    if ((int)gridDim.x % (8 * tiles) == 0) {
        u.tile = x / 8 % tiles;
        id = x / (8 * tiles) * 8 + x % 8;
    }
    if (mode == CacheMode::blocks) {
        const int p = id % a.parts;
        id /= a.parts;
        u.g = id % a.H_kv;
        u.seq = id / a.H_kv;
        u.n = cache_rows(a, u.seq);
        u.n_tok = cache_tokens(a, mode, u.n);
        const int chunk = ceil_div_dev(ceil_div_dev(u.n_tok > 0 ? u.n_tok : 1, a.parts), a.round) * a.round;
        u.first = u.seq * a.parts;
        u.part = u.first + p;
        u.t_begin = p * chunk;
        u.t_end = u.t_begin + chunk < u.n_tok ? u.t_begin + chunk : u.n_tok;
        u.some = u.t_begin < u.t_end;
        return u;
    }
    u.g = id % a.H_kv;
    u.part = id / a.H_kv;
    if (a.batch == 1) {
        u.n = cache_rows(a, 0);
        u.n_tok = cache_tokens(a, mode, u.n);
        const int chunk = ceil_div_dev(ceil_div_dev(u.n_tok > 0 ? u.n_tok : 1, a.parts), a.round) * a.round;
        u.t_begin = u.part * chunk;
        u.t_end = u.t_begin + chunk < u.n_tok ? u.t_begin + chunk : u.n_tok;
        u.some = u.t_begin < u.t_end;
        if (x == 0 && threadIdx.x == 0) {
            a.table[0] = 0;
            a.table[1] = ceil_div_dev(u.n_tok, chunk);
        }
        return u;
    }
    int n = lane < a.batch ? cache_rows(a, lane) : 0, t = lane < a.batch ? cache_tokens(a, mode, n) : 0;
    const int chunk = __builtin_amdgcn_readfirstlane(cache_chunk(a, mode, t));
    int before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {
        if (b0 > 0) {
            n = b0 + lane < a.batch ? cache_rows(a, b0 + lane) : 0;
            t = b0 + lane < a.batch ? cache_tokens(a, mode, n) : 0;
        }
        const int mine = ceil_div_dev(t, chunk);
        int upto = mine;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            if (off >= a.batch) break;
            const int o = __shfl_up(upto, off, kWave);
            upto += lane >= off ? o : 0;
        }
        if (x == 0 && threadIdx.x < kWave) {  // for the merge
            if (b0 + lane < a.batch) a.table[b0 + lane] = before + upto - mine;
            if (b0 + lane == a.batch - 1) a.table[a.batch] = before + upto;
        }
        const uint64_t in = __ballot(u.part >= before + upto - mine && u.part < before + upto);
        if (in) {
            const int l = __builtin_ctzll(in);
            u.seq = b0 + l;
            u.n = __builtin_amdgcn_readlane(n, l);
            u.n_tok = __builtin_amdgcn_readlane(t, l);
            u.first = before + __builtin_amdgcn_readlane(upto - mine, l);
            u.t_begin = (u.part - u.first) * chunk;
            u.t_end = u.t_begin + chunk < u.n_tok ? u.t_begin + chunk : u.n_tok;
            u.some = true;
        }
        before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return u;
}

// The parts of a sequence (blocks: of a query), for what follows the attention.
__device__ __forceinline__ void cache_parts(const CacheArgs &a, CacheMode mode, int i, int &first, int &count)
{
    if (mode == CacheMode::blocks) {
        const int n_tok = cache_tokens(a, mode, cache_rows(a, i));
        const int chunk = ceil_div_dev(ceil_div_dev(n_tok > 0 ? n_tok : 1, a.parts), a.round) * a.round;
        first = i * a.parts;
        count = ceil_div_dev(n_tok, chunk);
    } else {
        first = a.table[i];
        count = a.table[i + 1] - first;
    }
}

// Row of a partial: blocks have one query token per part.
__device__ __forceinline__ size_t part_row(const CacheArgs &a, CacheMode mode, int part, int token, int head)
{
    return ((size_t)part * (mode == CacheMode::blocks ? 1 : a.N) + (mode == CacheMode::blocks ? 0 : token)) * a.H_q + head;
}


struct CachePlan {
    int n_rep, words, n_c, k_ch;
    float scale;
    int rows, round, parts;  // as in CacheArgs
    bool mfma;
    xkv_shape sel_shape;  // the selection as a problem of launch_topk: rows of blocks, or rows of the cache
    Plan sel_plan;
    size_t off_hist, off_state, off_keys, off_reach, off_sel, off_n, off_logits, off_table, off_part_o, off_part_ml, total;
};

// The plan of one call.  N: query tokens of a sequence; c: rows of a block.
xkv_status plan_cache_attend(const xkv_shape &s, CacheMode mode, int N, int c, CachePlan &p);
xkv_status plan_evict(const xkv_shape &s, CachePlan &p);

hipError_t launch_cache_attend(CacheMode mode, const xkv_shape &s, const CacheArgs &a, hipStream_t st);
hipError_t launch_block_scores(const xkv_shape &s, const CacheArgs &a, const void *landmarks, int n_c, float *scores, hipStream_t st);
// The blocks of every query and KV head, for up to 16384 of them (block_select_ok); reach: room for [batch][N][H_kv][n_c / 16] numbers.
bool block_select_ok(int n_c);
hipError_t launch_block_select(const xkv_shape &s, const CacheArgs &a, const void *landmarks, int n_c, float *scores, float *reach, int32_t *blocks,
                               hipStream_t st);
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
bool evict_select_ok(int L);  // one launch selects; longer rows go through launch_topk
hipError_t launch_evict(const xkv_shape &s, const CachePlan &p, const EvictArgs &a, uint32_t *hist, uint32_t *state, hipStream_t st);

}  // namespace xkv
