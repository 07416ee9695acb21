// A cache held in 8 bits with a scale for every block of rows of a KV head, and rotary positions: what the kernels (cache8_attend.hip,
// cache8_append.hip, rope.hip) and the C ABI (cache8_api.hip) share.
#pragma once

#include "cache.h"

namespace xkv {

// A result in its type: rounded to nearest even, NaN stays NaN.
template <typename T> __device__ __forceinline__ T result(float x);
template <> __device__ __forceinline__ float result<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t result<bf16_t>(float x) { return __builtin_bit_cast(bf16_t, (__bf16)x); }

// Grids of up to 2^31 workgroups of 256 threads: a launch takes less than 2^32 threads in a direction, so more than 2^22 workgroups lie in rows of
// as many, the last of which may reach beyond the end.
constexpr int kLongGrid = 22;
inline dim3 long_grid(unsigned n) { return n <= 1u << kLongGrid ? dim3(n) : dim3(1u << kLongGrid, ((n - 1) >> kLongGrid) + 1); }
__device__ __forceinline__ unsigned long_grid_unit() { return blockIdx.x + (blockIdx.y << kLongGrid); }

struct Cache8Args {
    const uint8_t *K8, *V8;            // [batch][H_kv][L][d_h]
    const float *k_scales, *v_scales;  // [batch][H_kv][n_c]
    const void *q;                     // [batch][N][H_q][d_h]
    const int32_t *visible;            // [batch][N] (nullable: L)
    void *out;
    // Partials, [part][N][H_q] rows of d_h numbers and of (maximum, sum); NULL: there is one part of everything, whose results go to out.
    float *part_o, *part_ml;
    int32_t *table;                    // by_length: as in CacheArgs
    int L, H_kv, H_q, d_h, batch, N, n_c;
    int shift;      // a block has 2^shift rows
    int rows;       // rows (query, head) per workgroup
    int round;      // rows of the cache that a workgroup takes at a time: parts are multiples of it
    int parts;      // by_length: of all sequences, else of every row tile
    bool by_length; // the parts of all sequences are cut as cache_unit does
    float scale;
};

__device__ __forceinline__ int visible8(const Cache8Args &a, int seq, int i)
{
    const int n = a.visible ? a.visible[(size_t)seq * a.N + i] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

// What cache_unit needs to cut by length: `rows` (LDS, [batch]) are the rows that any query of a sequence sees; NULL: one query of each, or all.
struct Cache8Cut {
    const int *rows;
    const int32_t *visible;
    int32_t *table;
    int L, H_kv, batch, round, parts;
};
__device__ __forceinline__ int cache_rows(const Cache8Cut &a, int seq)
{
    const int n = a.rows ? a.rows[seq] : a.visible ? a.visible[seq] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}
__device__ __forceinline__ int cache_tokens(const Cache8Cut &, CacheMode, int n) { return n; }

constexpr int kCutBatch = 1024, kCutQueries = 16384;  // sequences, and queries of all of them, up to which parts are cut by length

struct Cache8Plan {
    int n_rep, n_c, shift;
    int rows, round, parts;
    bool mfma, by_length, direct;
    float scale;
    size_t off_table, off_part_o, off_part_ml, total;
};
hipError_t launch_cache8_attend(const xkv_shape &s, const Cache8Args &a, int code, bool mfma, hipStream_t st);

struct Cache8Append {
    const void *K, *V;
    xkv_rows K_at, V_at;
    const int32_t *lengths, *counts;
    uint8_t *K8, *V8;
    float *k_scales, *v_scales;
    int N, L, H_kv, d_h, batch, n_c, shift;
    int blocks;  // of a sequence and head, that its new rows can lie in
};
hipError_t launch_cache8_append(const xkv_shape &s, const Cache8Append &a, int code, hipStream_t st);

struct RotateArgs {
    const void *x[2];  // queries, keys (either may be absent: no heads)
    void *y[2];
    xkv_rows x_at[2], y_at[2];
    int heads[2];
    const int32_t *positions;
    const double *frequencies;
    int batch, N, d_h, d_rot;
    float amplitude, sign;  // what multiplies cosines and sines, and the angles
};
hipError_t launch_rotate(const xkv_shape &s, const RotateArgs &a, bool interleaved, hipStream_t st);
hipError_t launch_rope_frequencies(int d_rot, double theta, int scaling, double factor, double low, double high, double context, double *out,
                                   hipStream_t st);

}  // namespace xkv
