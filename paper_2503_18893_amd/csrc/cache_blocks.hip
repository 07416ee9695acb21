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
