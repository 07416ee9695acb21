// Rotary positions: pairs of channels of queries and keys turned by position times frequency.
#include "cache8.h"

namespace xkv {
namespace {

constexpr int kRopeThreads = 256;

__global__ void rope_frequencies_kernel(int d_rot, double theta, int scaling, double factor, double low, double high, double context, double *out)
{
    const int j = (int)threadIdx.x;
    if (2 * j >= d_rot) return;
    if (scaling == XKV_ROPE_BASE) theta *= pow(factor, d_rot / (d_rot - 2.0));
    double f = pow(theta, -2.0 * j / d_rot);
    if (scaling == XKV_ROPE_LINEAR) f /= factor;
    if (scaling == XKV_ROPE_TURNS) {
        const double t = fmin(fmax((context * f / 6.283185307179586476925 - low) / (high - low), 0.0), 1.0);
        f *= t + (1.0 - t) / factor;
    }
    out[j] = f;
}

// VEC numbers of a row at once (a piece of 16 bytes, or one).
template <typename T, int VEC> struct Piece {
    T x[VEC];
};
template <typename T, int VEC> __device__ __forceinline__ void load_piece(Piece<T, VEC> &p, const T *from)
{
    if constexpr (sizeof(p) == 16)
        __builtin_memcpy(&p, __builtin_assume_aligned(from, 16), 16);
    else
        for (int e = 0; e < VEC; ++e) p.x[e] = from[e];
}
template <typename T, int VEC> __device__ __forceinline__ void store_piece(T *to, const Piece<T, VEC> &p)
{
    if constexpr (sizeof(p) == 16)
        __builtin_memcpy(__builtin_assume_aligned(to, 16), &p, 16);
    else
        for (int e = 0; e < VEC; ++e) to[e] = p.x[e];
}

// ------------------------------------------------------------------------------------------
// A workgroup takes `tokens` tokens of a sequence: first the cosines and sines of their pairs (angles p f_j in double precision, whole turns
// taken off there, then fp32), which all heads share, into LDS; then, `width` threads a row (token, head), the pieces of the rows.
// ------------------------------------------------------------------------------------------
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rotate_kernel(RotateArgs a, int tokens, int lg_width)
{
    extern __shared__ float2 sm_unit[];  // [tokens][d_rot / 2]
    const int m = a.d_rot / 2, groups = (a.N + tokens - 1) / tokens;
    const int b = (int)(blockIdx.x / (unsigned)groups), first = (int)(blockIdx.x % (unsigned)groups) * tokens;
    const int here = a.N - first < tokens ? a.N - first : tokens;
    for (int i = (int)threadIdx.x; i < here * m; i += kRopeThreads) {
        const int t = first + i / m;
        const int p = a.positions ? a.positions[(size_t)b * a.N + t] : t;
        const double turns = (double)p * (a.frequencies[i % m] * 0.15915494309189533577);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        sm_unit[i] = float2{a.amplitude * c, a.amplitude * a.sign * s};
    }
    __syncthreads();
    const int heads = a.heads[0] + a.heads[1], width = 1 << lg_width;
    constexpr int PAIRS = INTERLEAVED ? (VEC > 1 ? VEC / 2 : 1) : VEC;  // pairs of a piece
    const int turned = m / PAIRS, items = turned + (a.d_h - a.d_rot) / VEC;
    for (int row = (int)threadIdx.x >> lg_width; row < here * heads; row += kRopeThreads >> lg_width) {
        const int t = row / heads, h = row % heads, of = h < a.heads[0] ? 0 : 1, head = h - (of ? a.heads[0] : 0);
        const T *x = (const T *)a.x[of] + (b * a.x_at[of].sequence + (first + t) * a.x_at[of].token + head * a.x_at[of].head);
        T *y = (T *)a.y[of] + (b * a.y_at[of].sequence + (first + t) * a.y_at[of].token + head * a.y_at[of].head);
        for (int i = (int)threadIdx.x & (width - 1); i < items; i += width) {
            if (i >= turned) {
                const int j = a.d_rot + (i - turned) * VEC;
                Piece<T, VEC> p;
                load_piece(p, x + j);
                store_piece(y + j, p);
                continue;
            }
            const float2 *unit = sm_unit + t * m + i * PAIRS;
            if constexpr (INTERLEAVED && VEC > 1) {
                Piece<T, VEC> p;
                load_piece(p, x + i * VEC);
#pragma unroll
                for (int e = 0; e < PAIRS; ++e) {
                    const float2 u = unit[e];
                    const float lo = to_f32(p.x[2 * e]), hi = to_f32(p.x[2 * e + 1]);
                    p.x[2 * e] = result<T>(fmaf(lo, u.x, -(hi * u.y)));
                    p.x[2 * e + 1] = result<T>(fmaf(hi, u.x, lo * u.y));
                }
                store_piece(y + i * VEC, p);
            } else {
                const int jl = INTERLEAVED ? 2 * i : i * VEC, jh = INTERLEAVED ? 2 * i + 1 : m + i * VEC;
                Piece<T, VEC> l, r;
                load_piece(l, x + jl);
                load_piece(r, x + jh);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 u = unit[e];
                    const float lo = to_f32(l.x[e]), hi = to_f32(r.x[e]);
                    l.x[e] = result<T>(fmaf(lo, u.x, -(hi * u.y)));
                    r.x[e] = result<T>(fmaf(hi, u.x, lo * u.y));
                }
                store_piece(y + jl, l);
                store_piece(y + jh, r);
            }
        }
    }
}

// Whether every piece of 16 bytes of these rows is aligned.
bool aligned16(const RotateArgs &a, size_t size)
{
    for (int i = 0; i < 2; ++i) {
        if (!a.x[i]) continue;
        for (const xkv_rows &r : {a.x_at[i], a.y_at[i]})
            if (((a.batch > 1 ? r.sequence : 0) | (a.N > 1 ? r.token : 0) | (a.heads[i] > 1 ? r.head : 0)) * (int64_t)size % 16) return false;
        if (((uintptr_t)a.x[i] | (uintptr_t)a.y[i]) % 16) return false;
    }
    return true;
}

template <typename T>
hipError_t launch_rotate_of(const RotateArgs &a, bool interleaved, hipStream_t st)
{
    constexpr int WIDE = 16 / sizeof(T);
    const int m = a.d_rot / 2;
    const bool wide = aligned16(a, sizeof(T)) && a.d_h % WIDE == 0 && (interleaved ? a.d_rot : m) % WIDE == 0;
    const int vec = wide ? WIDE : 1, pairs = interleaved ? (vec > 1 ? vec / 2 : 1) : vec, items = m / pairs + (a.d_h - a.d_rot) / vec;
    int lg = 0;
    while ((1 << lg) < items && lg < 8) ++lg;
    const long long rows = (long long)a.N * (a.heads[0] + a.heads[1]);
    int tokens = 1;
    while (tokens < 8 && tokens < a.N && a.batch * rows / tokens * (1 << lg) > 4096LL * kRopeThreads) tokens *= 2;
    const unsigned groups = (unsigned)((a.N + tokens - 1) / tokens);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(groups * (unsigned)a.batch), dim3(kRopeThreads), (size_t)tokens * m * sizeof(float2), st, a, tokens, lg);
        return hipGetLastError();
    };
    if (wide) return interleaved ? launch(rotate_kernel<T, WIDE, true>) : launch(rotate_kernel<T, WIDE, false>);
    return interleaved ? launch(rotate_kernel<T, 1, true>) : launch(rotate_kernel<T, 1, false>);
}

}  // namespace

hipError_t launch_rotate(const xkv_shape &s, const RotateArgs &a, bool interleaved, hipStream_t st)
{
    return s.dtype == XKV_F32 ? launch_rotate_of<float>(a, interleaved, st) : launch_rotate_of<bf16_t>(a, interleaved, st);
}

hipError_t launch_rope_frequencies(int d_rot, double theta, int scaling, double factor, double low, double high, double context, double *out,
                                   hipStream_t st)
{
    hipLaunchKernelGGL(rope_frequencies_kernel, dim3(1), dim3(128), 0, st, d_rot, theta, scaling, factor, low, high, context, out);
    return hipGetLastError();
}

}  // namespace xkv
