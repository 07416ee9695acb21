// Blocks of an uncompressed cache: how well their means agree with a query, and the means themselves (cache.h).
#include "cache.h"

namespace xkv {
namespace {

// S[j] = max over the query heads of a KV head of <q_h, mean_j>; +inf for the block that ends with the query's last visible row,
// -inf for those behind it.  The sums decide which block is read, so they are taken in double precision and rounded once to
// single: then the order of addition does not show in the selection.  A wavefront per block, lanes over the channels.
template <typename T>
__global__ __launch_bounds__(256) void block_scores_kernel(CacheArgs a, const T *__restrict__ landmarks, float *__restrict__ scores,
                                                           int n_c)
{
    const int lane = lane_id(), w = wave_id(), g = blockIdx.y, z = blockIdx.z, b = z / a.N, d = a.d_h, n_rep = a.H_q / a.H_kv;
    const int v = cache_rows(a, z), last = v > 0 ? (v - 1) / a.c : -1;
    const T *q = (const T *)a.q + ((size_t)z * a.H_q + g * n_rep) * d;
    for (int j = blockIdx.x * 4 + w; j < n_c; j += gridDim.x * 4) {
        float best = j == last ? INFINITY : -INFINITY;
        if (j < last) {
            const T *m = landmarks + (((size_t)b * a.H_kv + g) * n_c + j) * d;
            for (int h = 0; h < n_rep; ++h) {
                double sum = 0.0;
                for (int e = lane; e < d; e += kWave) sum = fma((double)to_f32(m[e]), (double)to_f32(q[h * d + e]), sum);
#pragma unroll
                for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
                best = fmaxf(best, (float)sum);
            }
        }
        if (lane == 0) scores[((size_t)z * a.H_kv + g) * n_c + j] = best;
    }
}

// The same on the double-precision matrix cores, for 4 ROUNDS channels (ROUNDS a multiple of 8 in bf16, of 4 in fp32): a wavefront multiplies 16 means with the rows of as many whole
// queries (query token, head) as fit 16, so that the heads of a KV head stay together.
//   lane (i, kk) = (l % 16, l / 16): channels kk ROUNDS .. of mean i and of row i; result register r: mean 4 r + kk, row i
// The order in which channels are added does not matter (double precision), so each lane takes a contiguous quarter of its row.
typedef __attribute__((ext_vector_type(4))) double f64x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t bl_u32x4_t;

template <typename T, int ROUNDS> __device__ __forceinline__ void load_quarter(const T *row, int kk, bl_u32x4_t (&raw)[ROUNDS * sizeof(T) / 16])
{
#pragma unroll
    for (int i = 0; i < (int)(ROUNDS * sizeof(T) / 16); ++i) raw[i] = reinterpret_cast<const bl_u32x4_t *>(row + kk * ROUNDS)[i];
}
template <typename T> __device__ __forceinline__ double channel(const bl_u32x4_t *raw, int e);
template <> __device__ __forceinline__ double channel<float>(const bl_u32x4_t *raw, int e) { return (double)__uint_as_float(raw[e / 4][e % 4]); }
template <> __device__ __forceinline__ double channel<bf16_t>(const bl_u32x4_t *raw, int e)
{
    const uint32_t x = raw[e / 8][e % 8 / 2];
    return (double)__uint_as_float(e & 1 ? x & 0xFFFF0000u : x << 16);
}

template <typename T, int ROUNDS>
__global__ __launch_bounds__(256) void block_scores_mfma_kernel(CacheArgs a, const T *__restrict__ landmarks, float *__restrict__ scores, int n_c,
                                                                int per_tile)
{
    constexpr int PIECES = ROUNDS * sizeof(T) / 16, D = 4 * ROUNDS;
    __shared__ float sm[4][16][17];
    const int lane = lane_id(), w = wave_id(), i16 = lane & 15, kk = lane >> 4, n_rep = a.H_q / a.H_kv;
    const int g = blockIdx.y % a.H_kv, b = blockIdx.y / a.H_kv, t0 = blockIdx.z * per_tile;  // first query token of this tile
    const int tokens = a.N - t0 < per_tile ? a.N - t0 : per_tile;
    const int r = i16 < tokens * n_rep ? i16 : 0;  // (rows beyond repeat the first one)
    bl_u32x4_t raw[PIECES];
    load_quarter<T, ROUNDS>((const T *)a.q + (((size_t)b * a.N + t0 + r / n_rep) * a.H_q + g * n_rep + r % n_rep) * D, kk, raw);
    double Q[ROUNDS];
#pragma unroll
    for (int e = 0; e < ROUNDS; ++e) Q[e] = channel<T>(raw, e);
    int most = 0;  // rows that any of these queries sees
    for (int i = 0; i < tokens; ++i) {
        const int v = cache_rows(a, b * a.N + t0 + i);
        most = most > v ? most : v;
    }
    const T *means = landmarks + ((size_t)b * a.H_kv + g) * n_c * D;
    const int stride = gridDim.x * 64;
    for (int j0 = (blockIdx.x * 4 + w) * 16; j0 < n_c; j0 += stride) {
        f64x4_t S = {0.0, 0.0, 0.0, 0.0};
        if ((long long)j0 * a.c < most) {  // (else no query gets that far)
            load_quarter<T, ROUNDS>(means + (size_t)(j0 + i16 < n_c ? j0 + i16 : n_c - 1) * D, kk, raw);
#pragma unroll
            for (int e = 0; e < ROUNDS; ++e) S = __builtin_amdgcn_mfma_f64_16x16x4f64(channel<T>(raw, e), Q[e], S, 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int x = 0; x < 4; ++x) sm[w][4 * x + kk][i16] = (float)S[x];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        for (int i = kk; i < tokens; i += 4) {  // a lane per block and query token
            const int j = j0 + i16, z = b * a.N + t0 + i, v = cache_rows(a, z), last = v > 0 ? (v - 1) / a.c : -1;
            float best = -INFINITY;
            for (int h = 0; h < n_rep; ++h) best = fmaxf(best, sm[w][i16][i * n_rep + h]);
            best = j < last ? best : j == last ? INFINITY : -INFINITY;
            if (j < n_c) scores[((size_t)z * a.H_kv + g) * n_c + j] = best;
        }
    }
}

// Means of the blocks that hold the last N rows in use, over the rows in use.  A wavefront per block, lanes over the channels.
template <typename T>
__global__ __launch_bounds__(256) void landmarks_update_kernel(const T *__restrict__ K, const int32_t *__restrict__ lengths,
                                                               T *__restrict__ landmarks, int L, int d, int H_kv, int N, int c, int n_c)
{
    const int lane = lane_id(), row = blockIdx.y;
    int n = lengths ? lengths[row / H_kv] : L;
    n = n < 0 ? 0 : n < L ? n : L;
    const int j = (n > N ? n - N : 0) / c + blockIdx.x * 4 + wave_id(), t0 = j * c, t1 = t0 + c < n ? t0 + c : n;
    if (n == 0 || j > (n - 1) / c) return;
    const float inv = 1.0f / (float)(t1 - t0);
    for (int e = lane; e < d; e += kWave) {
        float sum = 0.0f;
        for (int t = t0; t < t1; ++t) sum += to_f32(K[((size_t)row * L + t) * d + e]);
        landmarks[((size_t)row * n_c + j) * d + e] = from_f32<T>(sum * inv);
    }
}

}  // namespace

hipError_t launch_block_scores(const xkv_shape &s, const CacheArgs &a, const void *landmarks, int n_c, float *scores, hipStream_t st)
{
    const int n_rep = a.H_q / a.H_kv, per_tile = 16 / n_rep < a.N ? 16 / n_rep : a.N, tiles = (a.N + per_tile - 1) / per_tile;
    if ((((uintptr_t)a.q | (uintptr_t)landmarks) & 15u) == 0 && (s.d_h == 128 || s.d_h == 64)) {
        // a wavefront takes 16 blocks a time; several times, to load its queries less often, once there are enough of them
        const long long waves = (long long)((n_c + 15) / 16) * a.H_kv * a.batch * tiles;
        int times = (int)(waves / 8192);
        times = times < 1 ? 1 : times > 16 ? 16 : times;
        const dim3 g((n_c + 64 * times - 1) / (64 * times), a.H_kv * a.batch, tiles);
        auto launch = [&](auto kernel, auto *marks) {
            hipLaunchKernelGGL(kernel, g, dim3(256), 0, st, a, marks, scores, n_c, per_tile);
            return hipGetLastError();
        };
        if (s.dtype == XKV_F32)
            return s.d_h == 128 ? launch(block_scores_mfma_kernel<float, 32>, (const float *)landmarks)
                                : launch(block_scores_mfma_kernel<float, 16>, (const float *)landmarks);
        return s.d_h == 128 ? launch(block_scores_mfma_kernel<bf16_t, 32>, (const bf16_t *)landmarks)
                            : launch(block_scores_mfma_kernel<bf16_t, 16>, (const bf16_t *)landmarks);
    }
    const dim3 grid((n_c + 15) / 16, a.H_kv, a.batch * a.N);
    if (s.dtype == XKV_F32)
        hipLaunchKernelGGL(block_scores_kernel<float>, grid, dim3(256), 0, st, a, (const float *)landmarks, scores, n_c);
    else
        hipLaunchKernelGGL(block_scores_kernel<bf16_t>, grid, dim3(256), 0, st, a, (const bf16_t *)landmarks, scores, n_c);
    return hipGetLastError();
}

hipError_t launch_landmarks_update(const xkv_shape &s, const void *K, const int32_t *lengths, int N, int c, void *landmarks, hipStream_t st)
{
    const int n_c = (s.L + c - 1) / c, most = (N + c - 1) / c + 1, blocks = most < n_c ? most : n_c;
    const dim3 grid((blocks + 3) / 4, s.batch * s.H_kv);
    if (s.dtype == XKV_F32)
        hipLaunchKernelGGL(landmarks_update_kernel<float>, grid, dim3(256), 0, st, (const float *)K, lengths, (float *)landmarks, s.L, s.d_h,
                           s.H_kv, N, c, n_c);
    else
        hipLaunchKernelGGL(landmarks_update_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t *)K, lengths, (bf16_t *)landmarks, s.L,
                           s.d_h, s.H_kv, N, c, n_c);
    return hipGetLastError();
}

}  // namespace xkv
