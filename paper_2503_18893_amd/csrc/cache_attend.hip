// Attention over an uncompressed cache: trees of drafted tokens, one token whose weights are kept, selected blocks (cache.h).
//   z_t = scale <q, k_t>,  out = sum_t exp(z_t - max) v_t / sum_t exp(z_t - max)
// over the tokens that the query sees, split over the tokens: every workgroup leaves (maximum, sum, unnormalised output) of its
// part, and a second kernel merges them.
#include "cache.h"

namespace xkv {
namespace {

constexpr int kGenTokens = 64;  // tokens a round of the general kernel, a lane each
constexpr int kGenRows = 16;    // its rows (query token, head) per workgroup, four per wavefront

// ------------------------------------------------------------------------------------------
// General path, any type, width and alignment.  A round takes 64 tokens: their keys go to LDS in single precision and a lane
// multiplies one of them with the four queries of its wavefront, which are there, too; for the values lanes run over the
// columns, and the weights come from the lanes that hold them.
// ------------------------------------------------------------------------------------------
template <typename T, CacheMode MODE, int JP>
__global__ __launch_bounds__(256) void cache_attend_general_kernel(CacheArgs a)
{
    extern __shared__ float smem_f[];
    const int split = blockIdx.x % a.splits, tile = blockIdx.x / a.splits, g = blockIdx.y;
    const int lane = lane_id(), w = wave_id(), n_rep = a.H_q / a.H_kv, d = a.d_h, pitch = d | 1;
    // blocks: one query token per z; else all query tokens of a sequence
    const int seq = MODE == CacheMode::blocks ? blockIdx.z / a.N : blockIdx.z;
    const int first_token = MODE == CacheMode::blocks ? blockIdx.z % a.N : 0;
    const int M = MODE == CacheMode::blocks ? n_rep : a.N * n_rep;
    const int n = cache_rows(a, blockIdx.z), n_tok = cache_tokens(a, MODE, n);
    const int t_begin = split * a.chunk, t_end = t_begin + a.chunk < n_tok ? t_begin + a.chunk : n_tok;
    if (t_begin >= t_end) return;  // (the merge knows)
    float *kt = smem_f, *qs = kt + kGenTokens * pitch;

    const T *Kg = (const T *)a.K + ((size_t)seq * a.H_kv + g) * a.L * d, *Vg = (const T *)a.V + ((size_t)seq * a.H_kv + g) * a.L * d;
    const T *Kd = (const T *)a.K_draft + ((size_t)seq * a.H_kv + g) * a.N * d, *Vd = (const T *)a.V_draft + ((size_t)seq * a.H_kv + g) * a.N * d;
    const int32_t *sel = MODE == CacheMode::blocks ? a.sel + ((size_t)blockIdx.z * a.H_kv + g) * a.k_ch : nullptr;

    // row m of this workgroup: query token first_token + m / n_rep, head g n_rep + m % n_rep
    const int m0 = tile * kGenRows + 4 * w;
    size_t row_id[4];
    int token[4];
    float o[4][JP], mx[4], den[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int m = m0 + r < M ? m0 + r : M - 1;
        token[r] = first_token + m / n_rep;
        row_id[r] = ((size_t)seq * a.N + token[r]) * a.H_q + g * n_rep + m % n_rep;
        mx[r] = -INFINITY;
        den[r] = 0.0f;
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int j = lane + jj * kWave;
            o[r][jj] = 0.0f;
            if (j < d) qs[(4 * w + r) * d + j] = to_f32(((const T *)a.q)[row_id[r] * d + j]);
        }
    }
    for (int t0 = t_begin; t0 < t_end; t0 += kGenTokens) {
        // this lane's token (beyond the last one: that one again) and its row; drafted tokens are rows L, L + 1, ..
        const int t = t0 + lane < t_end ? t0 + lane : t_end - 1;
        const bool real = t0 + lane < t_end;
        int row = t;
        if (MODE == CacheMode::tree && t >= n) row = a.L + t - n;
        if (MODE == CacheMode::blocks) row = sel[t / a.c] * a.c + t % a.c;
        __syncthreads();
        for (int i = w; i < kGenTokens; i += 4) {
            const int rw = __builtin_amdgcn_readlane(row, i);
            const T *k = MODE == CacheMode::tree && rw >= a.L ? Kd + (size_t)(rw - a.L) * d : Kg + (size_t)rw * d;
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) {
                const int j = lane + jj * kWave;
                if (j < d) kt[i * pitch + j] = to_f32(k[j]);
            }
        }
        __syncthreads();
        float p[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < d; ++j) {
            const float x = kt[lane * pitch + j];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = fmaf(x, qs[(4 * w + r) * d + j], p[r]);
        }
        int used = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            bool sees = real;
            if (MODE == CacheMode::tree && t >= n)
                sees = real && (a.tree ? a.tree[((size_t)seq * a.N + token[r]) * a.words + ((t - n) >> 5)] >> ((t - n) & 31) & 1u
                                       : (uint32_t)(t - n <= token[r]));
            const float z = a.scale * p[r];
            if (MODE == CacheMode::weights && real && m0 + r < M) a.logits[row_id[r] * a.L + t] = z;
            const float m_new = fmaxf(mx[r], wave_max(sees ? z : -INFINITY));
            const float alpha = m_new == -INFINITY ? 1.0f : expf(mx[r] - m_new);
            p[r] = sees ? expf(z - m_new) : 0.0f;
            used |= sees;
            den[r] = den[r] * alpha + wave_sum(p[r]);
            mx[r] = m_new;
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) o[r][jj] *= alpha;
        }
        const int count = t_end - t0 < kGenTokens ? t_end - t0 : kGenTokens;
        for (int i0 = 0; i0 < count; i0 += 4) {
            float v[4][JP];
#pragma unroll
            for (int u = 0; u < 4; ++u) {  // (lanes from `count` on hold the last token again, with weight zero)
                const int rw = __builtin_amdgcn_readlane(row, i0 + u);
                const T *x = MODE == CacheMode::tree && rw >= a.L ? Vd + (size_t)(rw - a.L) * d : Vg + (size_t)rw * d;
                // a drafted token that none of these rows sees may be padding with anything in it
                const bool use = __builtin_amdgcn_readlane(used, i0 + u) != 0;
#pragma unroll
                for (int jj = 0; jj < JP; ++jj) {
                    const int j = lane + jj * kWave;
                    v[u][jj] = j < d && use ? to_f32(x[j]) : 0.0f;
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float pw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p[r]), i0 + u));
#pragma unroll
                    for (int jj = 0; jj < JP; ++jj) o[r][jj] = fmaf(pw, v[u][jj], o[r][jj]);
                }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (m0 + r >= M) break;
        const size_t slot = row_id[r] * a.splits + split;
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int j = lane + jj * kWave;
            if (j < d) a.part_o[slot * d + j] = o[r][jj];
        }
        if (lane == 0) {
            a.part_ml[2 * slot] = mx[r];
            a.part_ml[2 * slot + 1] = den[r];
        }
    }
}

// ------------------------------------------------------------------------------------------
// Merge: one workgroup per (query token, head).  Partials that no token went to were not written and are not read.
// ------------------------------------------------------------------------------------------
constexpr int kMaxCacheParts = 256;

template <typename T, CacheMode MODE>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheArgs a)
{
    __shared__ float sm_w[kMaxCacheParts], sm_o[4][256];
    const int lane = lane_id(), w = wave_id(), d = a.d_h;
    const size_t row = (size_t)blockIdx.y * a.H_q + blockIdx.x;  // y: (sequence, query token)
    const int n = cache_rows(a, MODE == CacheMode::tree ? blockIdx.y / a.N : blockIdx.y);
    const int n_tok = cache_tokens(a, MODE, n), parts = (n_tok + a.chunk - 1) / a.chunk;
    const float *ml = a.part_ml + row * a.splits * 2;
    float M = -INFINITY;
    for (int s = lane; s < parts; s += kWave) M = fmaxf(M, ml[2 * s]);
    M = wave_max(M);
    float den = 0.0f;
    for (int s = lane; s < parts; s += kWave) {
        const float wt = ml[2 * s] == -INFINITY ? 0.0f : expf(ml[2 * s] - M);
        if (w == 0) sm_w[s] = wt;
        den = fmaf(wt, ml[2 * s + 1], den);
    }
    den = wave_sum(den);
    __syncthreads();
    const float *po = a.part_o + row * a.splits * d;
    for (int j = lane; j < d; j += kWave) {
        float acc = 0.0f;
#pragma unroll 4
        for (int s = w; s < parts; s += 4) acc = fmaf(sm_w[s], po[(size_t)s * d + j], acc);
        sm_o[w][j] = acc;
    }
    __syncthreads();
    const int j = threadIdx.x;
    if (j < d) {
        const float num = (sm_o[0][j] + sm_o[1][j]) + (sm_o[2][j] + sm_o[3][j]);
        ((T *)a.out)[row * d + j] = from_f32<T>(den > 0.0f ? num / den : 0.0f);  // (a query that sees nothing: zeros)
    }
}

// ------------------------------------------------------------------------------------------
// weights[t] += sum over the query heads of a KV head of exp(z_t - max) / sum, from the kept logits.  The maximum and the sum
// of a head are merged from the partials by every workgroup.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void cache_weights_kernel(CacheArgs a, float *__restrict__ weights)
{
    __shared__ float sm_m[16], sm_r[16];
    const int lane = lane_id(), w = wave_id(), n_rep = a.H_q / a.H_kv, g = blockIdx.y, b = blockIdx.z;
    const int n = cache_rows(a, b), parts = (n + a.chunk - 1) / a.chunk;
    const int t0 = blockIdx.x * 1024;
    if (t0 >= n) return;
    const size_t head = (size_t)b * a.H_q + g * n_rep;
    for (int h = w; h < n_rep; h += 4) {
        const float *ml = a.part_ml + (head + h) * a.splits * 2;
        float M = -INFINITY, den = 0.0f;
        for (int s = lane; s < parts; s += kWave) M = fmaxf(M, ml[2 * s]);
        M = wave_max(M);
        for (int s = lane; s < parts; s += kWave) den = fmaf(expf(ml[2 * s] - M), ml[2 * s + 1], den);
        den = wave_sum(den);
        if (lane == 0) {
            sm_m[h] = M;
            sm_r[h] = 1.0f / den;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int t = t0 + 256 * u + threadIdx.x;
        if (t >= n) break;
        float sum = 0.0f;
        for (int h = 0; h < n_rep; ++h) sum = fmaf(expf(a.logits[(head + h) * a.L + t] - sm_m[h]), sm_r[h], sum);
        weights[((size_t)b * a.H_kv + g) * a.L + t] += sum;
    }
}

template <CacheMode MODE, typename T>
hipError_t launch_general(const CacheArgs &a, hipStream_t st)
{
    const int M = MODE == CacheMode::blocks ? a.H_q / a.H_kv : a.N * (a.H_q / a.H_kv);
    const dim3 grid(a.splits * ((M + kGenRows - 1) / kGenRows), a.H_kv, MODE == CacheMode::blocks ? a.batch * a.N : a.batch);
    const size_t lds = ((size_t)kGenTokens * (a.d_h | 1) + (size_t)kGenRows * a.d_h) * sizeof(float);
    auto launch = [&](auto kernel, DynamicLdsOnce &attr) {
        const hipError_t e = attr.ensure((const void *)kernel, lds > 65536 ? 160 * 1024 : lds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, a);
        return hipGetLastError();
    };
    static DynamicLdsOnce attr[3];
    return a.d_h <= 64 ? launch(cache_attend_general_kernel<T, MODE, 1>, attr[0])
         : a.d_h <= 128 ? launch(cache_attend_general_kernel<T, MODE, 2>, attr[1]) : launch(cache_attend_general_kernel<T, MODE, 4>, attr[2]);
}

template <CacheMode MODE>
hipError_t launch_mode(const xkv_shape &s, const CacheArgs &a, hipStream_t st)
{
    hipError_t e = s.dtype == XKV_F32 ? launch_general<MODE, float>(a, st) : launch_general<MODE, bf16_t>(a, st);
    if (e != hipSuccess) return e;
    const dim3 grid(a.H_q, a.batch * a.N);
    if (s.dtype == XKV_F32)
        hipLaunchKernelGGL((cache_merge_kernel<float, MODE>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((cache_merge_kernel<bf16_t, MODE>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attend(CacheMode mode, const xkv_shape &s, const CacheArgs &a, hipStream_t st)
{
    return mode == CacheMode::tree ? launch_mode<CacheMode::tree>(s, a, st)
         : mode == CacheMode::weights ? launch_mode<CacheMode::weights>(s, a, st) : launch_mode<CacheMode::blocks>(s, a, st);
}

hipError_t launch_cache_weights(const CacheArgs &a, float *weights, hipStream_t st)
{
    hipLaunchKernelGGL(cache_weights_kernel, dim3((a.L + 1023) / 1024, a.H_kv, a.batch), dim3(256), 0, st, a, weights);
    return hipGetLastError();
}

}  // namespace xkv
