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
// A workgroup takes `tokens` tokens of a sequence, 2^lg_width threads a row (token, head), a piece each (two that belong together in the half
// layout).  The cosines and sines of the tokens' pairs, which all heads share, go to LDS first: angles p f_j in double precision, whole turns
// taken off there, then fp32.  The first rows are requested before that, and ROWS of them at a time.  It is bound by its bytes: 40 heads of 32768 tokens, bf16, 123 us,
// 5.5 TB/s read and written together; one token of 16 sequences 3.7 us.  Rows that are not aligned, or widths without whole pieces (VEC = 1), go one number
// at a time, a load and a store of 2 bytes a lane: twice the time in bf16 (32768 tokens 242 us), 1.08 times in fp32 (252 beside 233).
// ------------------------------------------------------------------------------------------
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rotate_kernel(RotateArgs a, int tokens, int lg_width)
{
    constexpr int PAIRS = INTERLEAVED ? (VEC > 1 ? VEC / 2 : 1) : VEC;  // pairs of a piece
    constexpr bool ONE = INTERLEAVED && VEC > 1;                        // a piece holds both channels of its pairs
    constexpr int ROWS = 4;
    extern __shared__ float2 sm_unit[];  // [tokens][d_rot / 2]
    const int m = a.d_rot / 2, groups = (a.N + tokens - 1) / tokens;
    const unsigned unit = long_grid_unit();
    const int b = (int)(unit / (unsigned)groups), first = (int)(unit % (unsigned)groups) * tokens;
    if (b >= a.batch) return;
    const int here = a.N - first < tokens ? a.N - first : tokens, heads = a.heads[0] + a.heads[1], rows = here * heads;
    const int turned = m / PAIRS, items = turned + (a.d_h - a.d_rot) / VEC;
    const int i = (int)threadIdx.x & ((1 << lg_width) - 1), row0 = (int)threadIdx.x >> lg_width, step = kRopeThreads >> lg_width;
    const bool turns = i < turned, works = i < items;
    // this thread's places in a row
    const int jl = !turns ? a.d_rot + (i - turned) * VEC : ONE ? i * VEC : INTERLEAVED ? 2 * i : i * VEC;
    const int jh = !turns || ONE ? jl : INTERLEAVED ? 2 * i + 1 : m + i * VEC;
    const float inv_heads = 1.0f / (float)heads;

    Piece<T, VEC> l[ROWS], r[ROWS];
    T *to[ROWS];
    int token[ROWS];
    auto request = [&](int row) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int at = row + k * step;
            if (!works || at >= rows) break;
            int t = (int)((float)at * inv_heads), h = at - t * heads;  // (at most 8, one off at most)
            if (h < 0) h += heads, --t;
            if (h >= heads) h -= heads, ++t;
            token[k] = t;
            const int of = h < a.heads[0] ? 0 : 1, head = h - (of ? a.heads[0] : 0);
            const xkv_rows &xs = a.x_at[of], &ys = a.y_at[of];
            const T *x = (const T *)a.x[of] + (b * xs.sequence + (first + t) * xs.token + head * xs.head);
            to[k] = (T *)a.y[of] + (b * ys.sequence + (first + t) * ys.token + head * ys.head);
            load_piece(l[k], x + jl);
            if (!ONE && turns) load_piece(r[k], x + jh);
        }
    };
    request(row0);
    for (int j = (int)threadIdx.x; j < here * m; j += kRopeThreads) {
        const int t = first + j / m;
        const int p = a.positions ? a.positions[(size_t)b * a.N + t] : t;
        const double revolutions = (double)p * (a.frequencies[j % m] * 0.15915494309189533577);
        float s, c;
        sincospif(2.0f * (float)(revolutions - rint(revolutions)), &s, &c);
        sm_unit[j] = float2{a.amplitude * c, a.amplitude * a.sign * s};
    }
    __syncthreads();
    for (int row = row0; row < rows; row += ROWS * step) {
        if (row > row0) request(row);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (!works || row + k * step >= rows) break;
            if (turns) {
                const float2 *unit = sm_unit + token[k] * m + i * PAIRS;
#pragma unroll
                for (int e = 0; e < PAIRS; ++e) {
                    const float2 u = unit[e];
                    T &x = ONE ? l[k].x[2 * e] : l[k].x[e], &y = ONE ? l[k].x[2 * e + 1] : r[k].x[e];
                    const float lo = to_f32(x), hi = to_f32(y);
                    x = result<T>(fmaf(lo, u.x, -(hi * u.y)));
                    y = result<T>(fmaf(hi, u.x, lo * u.y));
                }
                if (!ONE) store_piece(to[k] + jh, r[k]);
            }
            store_piece(to[k] + jl, l[k]);
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
    // Tokens of a workgroup: as few as give every thread a row's piece.  40 heads of 32768 tokens, 8 threads a row: 1 123 us, 2 126, 8 136; 8 heads of 4 x 16384
    // tokens, 1 63, 2 47, 4 43.5, 8 48.
    int tokens = 1;
    while (tokens < 8 && ((a.heads[0] + a.heads[1]) * tokens << lg) < kRopeThreads) tokens *= 2;
    const unsigned groups = (unsigned)((a.N + tokens - 1) / tokens);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, long_grid(groups * (unsigned)a.batch), dim3(kRopeThreads), (size_t)tokens * m * sizeof(float2), st, a, tokens, lg);
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
