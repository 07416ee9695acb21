// Attention over a cache held in 8 bits (cache8.h).
//   z_t = scale ks[t / c] <q, k8_t>,  out = sum_t exp(z_t - max) vs[t / c] v8_t / sum_t exp(z_t - max)
// over the rows that a query sees, split over the rows: every workgroup leaves (maximum, sum, unnormalised output) of its part, in
// powers of two, and a second kernel merges them.
#include "cache8.h"

namespace xkv {
namespace {

constexpr int kGenTokens = 64;  // rows of the cache a round of the general kernel, a lane each
constexpr int kGenRows = 16;    // its rows (query, head) per workgroup, four per wavefront
constexpr float kLog2e = 1.44269504088896340736f;

// What a workgroup takes: query rows tile * rows .. of KV head g of sequence seq, rows t_begin .. t_end - 1 of the cache.
struct Unit8 {
    int seq, g, tile, part, t_begin, t_end;
    bool some;
};

// The queries whose rows (query, head) a tile holds.
__device__ __forceinline__ void tile_queries(const Cache8Args &a, int tile, int &first, int &last)
{
    const int n_rep = a.H_q / a.H_kv;
    first = tile * a.rows / n_rep;
    const int upto = ((tile + 1) * a.rows - 1) / n_rep;
    last = upto < a.N ? upto : a.N - 1;
}
// Rows that any of a tile's queries sees.  All lanes of a wavefront call it together.
__device__ __forceinline__ int tile_sees(const Cache8Args &a, int seq, int tile)
{
    int first, last, n = 0;
    tile_queries(a, tile, first, last);
    for (int i = first + lane_id(); i <= last; i += kWave) n = MaxOp()(n, visible8(a, seq, i));
    return wave_all(n, MaxOp());
}
__device__ __forceinline__ int tile_chunk(const Cache8Args &a, int n)
{
    return ceil_div_dev(ceil_div_dev(n > 0 ? n : 1, a.parts), a.round) * a.round;
}

__device__ __forceinline__ Unit8 unit8(const Cache8Args &a)
{
    Unit8 u{};
    if (a.by_length) {
        const CacheUnit c = cache_unit(a, CacheMode::weights, 1);
        u.seq = c.seq, u.g = c.g, u.part = c.part, u.t_begin = c.t_begin, u.t_end = c.t_end, u.some = c.some;
        return u;
    }
    const int tiles = (int)(((long long)a.N * (a.H_q / a.H_kv) + a.rows - 1) / a.rows);
    int id = (int)blockIdx.x;
    u.tile = tiles - 1 - id % tiles;  // (of a prompt the last ones see most)
    id /= tiles;
    const int p = id % a.parts;
    id /= a.parts;
    u.g = id % a.H_kv;
    u.seq = id / a.H_kv;
    const int n = tile_sees(a, u.seq, u.tile), chunk = tile_chunk(a, n);
    u.part = u.seq * a.parts + p;
    u.t_begin = p * chunk;
    u.t_end = u.t_begin + chunk < n ? u.t_begin + chunk : n;
    u.some = u.t_begin < u.t_end;
    return u;
}

template <int CODE> __device__ __forceinline__ float value8(uint8_t x)
{
    return CODE == XKV_E4M3 ? __builtin_amdgcn_cvt_f32_fp8((int)x, 0) : (float)(int8_t)x;
}

// ------------------------------------------------------------------------------------------
// General path, any type, width and block.  A round takes 64 rows of the cache, whose keys and values, with their scales, go to LDS in single precision.
// For the logits a lane multiplies one of the keys with the four queries of its wavefront; for the sums lanes run over the channels, and
// the weights go through LDS.
// ------------------------------------------------------------------------------------------
__host__ __device__ inline int general_pitch(int d) { return ((d + 3) / 4 | 1) * 4; }  // floats; an odd number of 16-byte pieces

template <typename T, int CODE, int JP>
__global__ __launch_bounds__(256) void cache8_general_kernel(Cache8Args a)
{
    extern __shared__ __attribute__((aligned(16))) float smem_f[];
    const Unit8 u = unit8(a);
    if (!u.some) return;  // (the merge knows)
    const int lane = lane_id(), w = wave_id(), n_rep = a.H_q / a.H_kv, d = a.d_h, d4 = (d + 3) / 4 * 4, pitch = general_pitch(d);
    const int M = a.N * n_rep;
    float *kt = smem_f, *vt = kt + kGenTokens * pitch, *qs = vt + kGenTokens * pitch, *ps = qs + kGenRows * d4;
    const size_t head = (size_t)u.seq * a.H_kv + u.g;
    const uint8_t *K = a.K8 + head * a.L * d, *V = a.V8 + head * a.L * d;
    const float *ks = a.k_scales + head * a.n_c, *vs = a.v_scales + head * a.n_c, c = a.scale * kLog2e;

    const int m0 = u.tile * kGenRows + 4 * w;
    size_t row_id[4];
    int sees[4];
    float o[4][JP], mx[4], den[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int m = m0 + r < M ? m0 + r : M - 1, i = m / n_rep;
        row_id[r] = ((size_t)u.seq * a.N + i) * a.H_q + u.g * n_rep + m % n_rep;
        sees[r] = visible8(a, u.seq, i);
        mx[r] = -INFINITY;
        den[r] = 0.0f;
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int j = lane + jj * kWave;
            o[r][jj] = 0.0f;
            if (j < d4) qs[(4 * w + r) * d4 + j] = j < d ? to_f32(((const T *)a.q)[row_id[r] * d + j]) : 0.0f;
        }
    }
    for (int t0 = u.t_begin; t0 < u.t_end; t0 += kGenTokens) {
        __syncthreads();
        for (int i = w; i < kGenTokens; i += 4) {
            const int t = t0 + i < u.t_end ? t0 + i : u.t_end - 1;
            const float k_scale = ks[t >> a.shift], v_scale = vs[t >> a.shift];
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) {
                const int j = lane + jj * kWave;
                if (j >= d4) continue;
                kt[i * pitch + j] = j < d ? k_scale * value8<CODE>(K[(size_t)t * d + j]) : 0.0f;
                vt[i * pitch + j] = j < d ? v_scale * value8<CODE>(V[(size_t)t * d + j]) : 0.0f;
            }
        }
        __syncthreads();
        const int t = t0 + lane;
        float p[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < d4; j += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(kt + lane * pitch + j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float4 y = *reinterpret_cast<const float4 *>(qs + (4 * w + r) * d4 + j);
                p[r] = fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, p[r]))));
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool in = t < sees[r] && t < u.t_end;
            const float z = in ? c * p[r] : -INFINITY;
            const float m_new = fmaxf(mx[r], wave_all(z, MaxOp()));
            const float alpha = m_new == -INFINITY ? 1.0f : exp2f(mx[r] - m_new);
            p[r] = z == -INFINITY ? 0.0f : exp2f(z - m_new);
            den[r] = den[r] * alpha + wave_all(p[r], AddOp());
            mx[r] = m_new;
            p[r] = in ? p[r] : -0.0f;  // (weights are not negative: hidden from this row)
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) o[r][jj] *= alpha;
        }
        *reinterpret_cast<float4 *>(ps + 4 * (64 * w + lane)) = float4{p[0], p[1], p[2], p[3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        for (int i = 0; i < kGenTokens; ++i) {
            const float4 y = *reinterpret_cast<const float4 *>(ps + 4 * (64 * w + i));
            const float weight[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) {
                const int j = lane + jj * kWave;
                const float v = vt[i * pitch + (j < d ? j : 0)];
                // what a row does not see is not multiplied by zero: it may be anything
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r][jj] = fmaf(weight[r], __float_as_uint(weight[r]) == 0x80000000u ? 0.0f : v, o[r][jj]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (m0 + r >= M) break;
        const int m = m0 + r;
        const size_t slot = ((size_t)u.part * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep;
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
// Merge: a wavefront per row (query, head).  Partials of parts that have no rows were not written and are not read.
// ------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void cache8_merge_kernel(Cache8Args a, int rows)
{
    __shared__ float sm_w[4][kMaxCacheParts];
    const int lane = lane_id(), w = wave_id(), row = (int)blockIdx.x * 4 + w;
    if (row >= rows) return;  // (nothing below is waited for by other wavefronts)
    const int n_rep = a.H_q / a.H_kv, head = row % a.H_q, i = row / a.H_q % a.N, seq = row / a.H_q / a.N;
    int first, parts;
    if (a.by_length) {
        first = a.table[seq];
        parts = a.table[seq + 1] - first;
    } else {
        const int n = tile_sees(a, seq, (i * n_rep + head % n_rep) / a.rows);
        first = seq * a.parts;
        parts = ceil_div_dev(n, tile_chunk(a, n));
    }
    const size_t stride = (size_t)a.N * a.H_q, at = first * stride + (size_t)i * a.H_q + head;
    float m = -INFINITY, den = 0.0f;
    for (int s = lane; s < parts; s += kWave) m = fmaxf(m, a.part_ml[2 * (at + s * stride)]);
    m = wave_all(m, MaxOp());
    for (int s = lane; s < parts; s += kWave) {
        const float top = a.part_ml[2 * (at + s * stride)], wt = top == -INFINITY ? 0.0f : exp2f(top - m);
        sm_w[w][s] = wt;
        den = fmaf(wt, a.part_ml[2 * (at + s * stride) + 1], den);
    }
    den = wave_all(den, AddOp());
    // (the logits of all that a row sees may be -inf: 0 / 0; a NaN among them is in its sum)
    const bool none = visible8(a, seq, i) == 0;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int j = lane; j < a.d_h; j += kWave) {
        float o = 0.0f;
        for (int s = 0; s < parts; ++s) o = fmaf(sm_w[w][s], a.part_o[(at + s * stride) * a.d_h + j], o);
        ((T *)a.out)[(size_t)row * a.d_h + j] = result<T>(none ? 0.0f : o / den);
    }
}

template <typename T, int CODE>
hipError_t launch_general(const Cache8Args &a, hipStream_t st)
{
    const int M = a.N * (a.H_q / a.H_kv);
    const dim3 grid((unsigned)a.parts * a.H_kv * (a.by_length ? 1 : (unsigned)a.batch * ((M + a.rows - 1) / a.rows)));
    const size_t lds = (2 * (size_t)kGenTokens * general_pitch(a.d_h) + (size_t)kGenRows * ((a.d_h + 3) / 4 * 4) + 4 * 4 * kGenTokens) * sizeof(float);
    auto launch = [&](auto kernel, DynamicLdsOnce &attr) {
        const hipError_t e = attr.ensure((const void *)kernel, 160 * 1024);  // (at most 150 KiB, at 256 channels)
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, a);
        return hipGetLastError();
    };
    static DynamicLdsOnce attr[3];
    return a.d_h <= 64 ? launch(cache8_general_kernel<T, CODE, 1>, attr[0])
         : a.d_h <= 128 ? launch(cache8_general_kernel<T, CODE, 2>, attr[1]) : launch(cache8_general_kernel<T, CODE, 4>, attr[2]);
}

}  // namespace

hipError_t launch_cache8_attend(const xkv_shape &s, const Cache8Args &a, int code, bool mfma, hipStream_t st)
{
    (void)mfma;
    hipError_t e;
    if (s.dtype == XKV_F32)
        e = code == XKV_E4M3 ? launch_general<float, XKV_E4M3>(a, st) : launch_general<float, XKV_INT8>(a, st);
    else
        e = code == XKV_E4M3 ? launch_general<bf16_t, XKV_E4M3>(a, st) : launch_general<bf16_t, XKV_INT8>(a, st);
    if (e != hipSuccess) return e;
    const int rows = a.batch * a.N * a.H_q;
    if (s.dtype == XKV_F32)
        hipLaunchKernelGGL(cache8_merge_kernel<float>, dim3((rows + 3) / 4), dim3(256), 0, st, a, rows);
    else
        hipLaunchKernelGGL(cache8_merge_kernel<bf16_t>, dim3((rows + 3) / 4), dim3(256), 0, st, a, rows);
    return hipGetLastError();
}

}  // namespace xkv
