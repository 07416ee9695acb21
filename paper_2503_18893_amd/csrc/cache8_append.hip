// New rows into a cache held in 8 bits: the scale of a block of rows from their largest magnitude, codes, and older codes again where the
// scale grows.
#include "cache8.h"

namespace xkv {
namespace {

constexpr float kSmallest = 0x1p-126f;  // of a scale: quotients by it and products with it are ordinary numbers

template <int CODE> __device__ __forceinline__ float highest() { return CODE == XKV_E4M3 ? 448.0f : 127.0f; }

// Four numbers, at most the highest in magnitude, to the nearest codes (ties to even).
template <int CODE> __device__ __forceinline__ uint32_t code4(const float *x)
{
    if constexpr (CODE == XKV_E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    } else {
        uint32_t w = 0;
        for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(x[e]) & 0xFFu) << (8 * e);
        return w;
    }
}
template <int CODE> __device__ __forceinline__ uint8_t code1(float x)
{
    const float four[4] = {x, 0.0f, 0.0f, 0.0f};
    return (uint8_t)code4<CODE>(four);
}
template <int CODE> __device__ __forceinline__ float value1(uint8_t x)
{
    return CODE == XKV_E4M3 ? __builtin_amdgcn_cvt_f32_fp8((int)x, 0) : (float)(int8_t)x;
}

// ------------------------------------------------------------------------------------------
// A wavefront takes a block of a KV head of K or V: first the largest magnitude of its new rows, then their codes.  VEC: numbers of a row
// that a lane takes at once.
// ------------------------------------------------------------------------------------------
template <typename T, int CODE, int VEC>
__global__ __launch_bounds__(256) void cache8_append_kernel(Cache8Append a, unsigned units)
{
    const unsigned unit = blockIdx.x * 4 + (unsigned)wave_id();
    if (unit >= units) return;
    const int lane = lane_id(), g = (int)(unit % a.H_kv), of = (int)(unit / a.H_kv % 2), rest = (int)(unit / (2 * a.H_kv));
    const int place = rest % a.blocks, b = rest / a.blocks;
    int n = a.lengths ? a.lengths[b] : 0, count = a.counts ? a.counts[b] : a.N;
    n = n < 0 ? 0 : n < a.L ? n : a.L;
    count = count < 0 ? 0 : count < a.N ? count : a.N;
    count = count < a.L - n ? count : a.L - n;
    const int block = (n >> a.shift) + place;
    if (block >= a.n_c) return;
    const long long start = (long long)block << a.shift, end = start + (1LL << a.shift);
    const int r0 = start > n ? (int)start : n, r1 = end < (long long)n + count ? (int)end : n + count;  // new rows
    if (r0 >= r1) return;
    const xkv_rows &at = of ? a.V_at : a.K_at;
    const T *from = (const T *)(of ? a.V : a.K) + (b * at.sequence + g * at.head);
    uint8_t *to = (of ? a.V8 : a.K8) + ((size_t)b * a.H_kv + g) * a.L * a.d_h;
    float *scale = (of ? a.v_scales : a.k_scales) + ((size_t)b * a.H_kv + g) * a.n_c + block;
    const int pieces = a.d_h / VEC;
    const long long count_new = (long long)(r1 - r0) * pieces;

    float top = 0.0f;
    bool odd = false;
    for (long long i = lane; i < count_new; i += kWave) {
        const T *x = from + (r0 - n + i / pieces) * at.token + i % pieces * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float v = fabsf(to_f32(x[e]));
            odd |= !(v < INFINITY);
            top = fmaxf(top, v);
        }
    }
    top = wave_all(top, MaxOp());
    const float old = start < n ? *scale : 0.0f;
    float s = old;
    int up = 0;
    if (__ballot(odd) != 0) {
        s = __builtin_nanf("");
    } else if (old == 0.0f) {
        s = top > 0.0f ? fmaxf(top / highest<CODE>(), kSmallest) : 0.0f;
    } else {
        while (top > highest<CODE>() * s && up < 300) {  // (a scale from outside may be anything)
            s *= 2.0f;
            ++up;
        }
    }
    if (lane == 0) *scale = s;
    if (up > 0) {
        const float less = exp2f(-(float)up);
        const long long count_old = (n - start) * pieces;
        for (long long i = lane; i < count_old; i += kWave) {
            uint8_t *x = to + (size_t)(start + i / pieces) * a.d_h + i % pieces * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = code1<CODE>(value1<CODE>(x[e]) * less);
        }
    }
    const bool none = s == 0.0f || s != s;
    for (long long i = lane; i < count_new; i += kWave) {
        const T *x = from + (r0 - n + i / pieces) * at.token + i % pieces * VEC;
        uint8_t *y = to + (size_t)(r0 + i / pieces) * a.d_h + i % pieces * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = none ? 0 : code1<CODE>(to_f32(x[e]) / s);
    }
}

}  // namespace

hipError_t launch_cache8_append(const xkv_shape &s, const Cache8Append &a, int code, hipStream_t st)
{
    const unsigned units = (unsigned)a.blocks * 2 * a.H_kv * a.batch;  // (at most 2^31 - 1)
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((units + 3) / 4), dim3(256), 0, st, a, units);
        return hipGetLastError();
    };
    if (code == XKV_E4M3)
        return s.dtype == XKV_F32 ? launch(cache8_append_kernel<float, XKV_E4M3, 1>) : launch(cache8_append_kernel<bf16_t, XKV_E4M3, 1>);
    return s.dtype == XKV_F32 ? launch(cache8_append_kernel<float, XKV_INT8, 1>) : launch(cache8_append_kernel<bf16_t, XKV_INT8, 1>);
}

}  // namespace xkv
