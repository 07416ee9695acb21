// New rows into a cache held in 8 bits: the scale of a block of rows from their largest magnitude, codes, and older codes again where the
// scale grows.
#include "cache8.h"

namespace xkv {
namespace {

constexpr float kSmallest = 0x1p-126f;  // of a scale: quotients by it and products with it are ordinary numbers

template <int CODE> __device__ __forceinline__ float highest() { return CODE == XKV_E4M3 ? 448.0f : 127.0f; }

// Four numbers, at most the highest in magnitude, to the nearest codes (ties to even).
template <int CODE> __device__ __forceinline__ uint32_t code4(float a, float b, float c, float d)
{
    if constexpr (CODE == XKV_E4M3) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        // 2^23 + 2^22 + a whole number up to 127 in magnitude has its two's complement in the lower bits, and the addition rounds to nearest even
        constexpr float BIG = 12582912.0f;
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + BIG), __float_as_uint(a + BIG), 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + BIG), __float_as_uint(c + BIG), 0x04000C0Cu);
        return lo | hi;
    }
}
template <int CODE, int BYTE> __device__ __forceinline__ float value(uint32_t w)
{
    return CODE == XKV_E4M3 ? __builtin_amdgcn_cvt_f32_fp8((int)w, BYTE) : (float)(int8_t)(w >> (8 * BYTE));
}

// A quotient x / s of at most 2^9, rounded to nearest; inv is 1 / s rounded to nearest, s at least 2^-100.  The product with inv is off by at most 1.5 steps;
// what it leaves of x, taken exactly, makes it one of the two neighbours of the quotient, and once more the nearest (Markstein's theorem on
// division by a correctly rounded reciprocal).  Five operations where a division takes ten.  (Where a remainder is too small to be
// exact, the quotient is below 2^-20 and its code 0.)
__device__ __forceinline__ float quotient(float x, float s, float inv)
{
    float q = x * inv;
    q = fmaf(fmaf(-q, s, x), inv, q);
    return fmaf(fmaf(-q, s, x), inv, q);
}

// VEC numbers of a row, a piece of 16 bytes or one number, as they come.
template <typename T, int VEC> struct Piece {
    T x[VEC];
};

// Over the LANES lanes (16, 32, 64) that work together, in all of them.
template <int LANES, typename T, typename OP> __device__ __forceinline__ T lanes_all(T v, OP op)
{
    if constexpr (LANES == 64) return wave_all(v, op);
    auto with = [&](uint32_t o) { v = op(v, __builtin_bit_cast(T, o)); };
    with(lanes_by<0xB1>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x4E>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x141>(__builtin_bit_cast(uint32_t, v)));
    with(lanes_by<0x140>(__builtin_bit_cast(uint32_t, v)));
    if constexpr (LANES == 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        v = op(__builtin_bit_cast(T, (uint32_t)r[0]), __builtin_bit_cast(T, (uint32_t)r[1]));
    }
    return v;
}

// ------------------------------------------------------------------------------------------
// THREADS threads (part of a wavefront, one, or four) take a block of a KV head of K or V: first the largest magnitude of its new rows, then their codes.
// A thread's pieces, up to KEPT of them, stay in registers between the two; a larger block's are read again.  Codes of older rows are
// only touched where the scale grows.  Long appends are bound by their bytes: 32768 tokens of 8 KV heads, bf16 to e4m3, blocks of 32 rows, 41 us, 4.9 TB/s
// (48 with divisions in the place of `quotient`); one token of 16 sequences 4.4 us, a chain of two loads, the maximum and the quotients.  Blocks of one or two rows
// 74: a lane has one piece under way, and a scale is 4 bytes of a store of its own.  A block is one workgroup's, so that few large ones do not fill the card: of 256 rows 54, 1024 70,
// 4096 220, one for a head 1710.
// ------------------------------------------------------------------------------------------
template <typename T, int CODE, int VEC, int THREADS, int KEPT>
__global__ __launch_bounds__(256) void cache8_append_kernel(Cache8Append a, unsigned units)
{
    constexpr int WAVES = THREADS / kWave;  // (0: part of one)
    __shared__ float sm_top[WAVES > 1 ? WAVES : 1];
    __shared__ int sm_odd[WAVES > 1 ? WAVES : 1];
    const unsigned group = long_grid_unit();
    const unsigned unit = THREADS == 256 ? group : THREADS == 64 ? group * 4 + (unsigned)wave_id() : group * (256 / THREADS) + threadIdx.x / THREADS;
    if (unit >= units) return;
    const int lane = (int)threadIdx.x % THREADS, g = (int)(unit % a.H_kv), of = (int)(unit / a.H_kv % 2), rest = (int)(unit / (2 * a.H_kv));
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
    const T *from = (const T *)(of ? a.V : a.K) + (b * at.sequence + g * at.head + (r0 - n) * at.token);
    uint8_t *to = (of ? a.V8 : a.K8) + (((size_t)b * a.H_kv + g) * a.L + r0) * a.d_h;
    float *scale = (of ? a.v_scales : a.k_scales) + ((size_t)b * a.H_kv + g) * a.n_c + block;
    const int pieces = a.d_h / VEC;  // of a row
    const long long total = (long long)(r1 - r0) * pieces;
    const float old = start < n ? *scale : 0.0f;

    // piece `lane + THREADS i`: its row and place in the row; THREADS pieces further
    const int row_step = THREADS / pieces, place_step = THREADS % pieces;
    struct Cursor {
        int row, place;
    };
    const Cursor begin{lane / pieces, lane % pieces};
    auto advance = [&](Cursor &c) __attribute__((always_inline)) {
        c.row += row_step;
        c.place += place_step;
        if (c.place >= pieces) c.place -= pieces, ++c.row;
    };
    typedef Piece<T, VEC> piece_t;
    piece_t kept[KEPT];
    auto load = [&](piece_t &p, const Cursor &c) __attribute__((always_inline)) {
        const T *x = from + c.row * at.token + c.place * VEC;
        if constexpr (sizeof(piece_t) == 16) {
            __builtin_memcpy(&p, __builtin_assume_aligned(x, 16), 16);
        } else {
            for (int e = 0; e < VEC; ++e) p.x[e] = x[e];
        }
    };
    float top = 0.0f;
    bool odd = false;
    Cursor c = begin;
    for (long long i0 = lane; i0 < total; i0 += (long long)KEPT * THREADS) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            if (i0 + (long long)i * THREADS < total) {
                load(kept[i], c);
            } else {
                for (int e = 0; e < VEC; ++e) kept[i].x[e] = T(0);
            }
            advance(c);
        }
#pragma unroll
        for (int i = 0; i < KEPT; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float v = fabsf(to_f32(kept[i].x[e]));
                odd |= !(v < INFINITY);
                top = fmaxf(top, v);
            }
    }
    top = lanes_all<THREADS < kWave ? THREADS : kWave>(top, MaxOp());
    odd = lanes_all<THREADS < kWave ? THREADS : kWave>((int)odd, MaxOp()) != 0;
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) sm_top[wave_id()] = top, sm_odd[wave_id()] = odd;
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) {
            top = fmaxf(top, sm_top[i]);
            odd |= sm_odd[i] != 0;
        }
    }
    float s = old;
    int up = 0;
    if (odd) {
        s = __builtin_nanf("");
    } else if (old == 0.0f) {
        s = top > 0.0f ? fmaxf(top / highest<CODE>(), kSmallest) : 0.0f;
    } else {
        while (top > highest<CODE>() * s && up < 300) {  // (a scale from outside may be anything)
            s *= 2.0f;
            ++up;
        }
    }
    // (all of them have read the old scale: where they are several, there was a barrier since)
    if (lane == 0) *scale = s;
    if (up > 0) {
        const float less = exp2f(-(float)up);
        const long long older = (long long)(r0 - start) * a.d_h;
        uint8_t *x = to - older;
        if (VEC > 1) {  // (rows are whole words then)
            for (long long i = lane; i < older / 4; i += THREADS) {
                uint32_t *word = reinterpret_cast<uint32_t *>(x) + i;
                const uint32_t w = *word;
                *word = code4<CODE>(value<CODE, 0>(w) * less, value<CODE, 1>(w) * less, value<CODE, 2>(w) * less, value<CODE, 3>(w) * less);
            }
        } else {
            for (long long i = lane; i < older; i += THREADS) x[i] = (uint8_t)code4<CODE>(value<CODE, 0>(x[i]) * less, 0.0f, 0.0f, 0.0f);
        }
    }
    const bool none = s == 0.0f || s != s;
    const float by = none ? 1.0f : s, inv = 1.0f / by;
    const bool small = by < 0x1p-100f;
    c = begin;
    for (long long i0 = lane; i0 < total; i0 += (long long)KEPT * THREADS) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            if (i0 + (long long)i * THREADS >= total) break;
            if (total > (long long)KEPT * THREADS) load(kept[i], c);
            uint8_t *y = to + (size_t)c.row * a.d_h + c.place * VEC;
            advance(c);
            if constexpr (VEC > 1) {
                uint32_t w[VEC / 4];
#pragma unroll
                for (int e = 0; e < VEC; e += 4) {
                    float q[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[j] = small ? to_f32(kept[i].x[e + j]) / by : quotient(to_f32(kept[i].x[e + j]), by, inv);
                    w[e / 4] = none ? 0u : code4<CODE>(q[0], q[1], q[2], q[3]);
                }
                __builtin_memcpy(__builtin_assume_aligned(y, VEC), w, VEC);
            } else {
                *y = none ? (uint8_t)0 : (uint8_t)code4<CODE>(small ? to_f32(kept[i].x[0]) / by : quotient(to_f32(kept[i].x[0]), by, inv), 0.0f, 0.0f, 0.0f);
            }
        }
    }
}

// Whether a row's pieces of 16 bytes are aligned wherever it lies, and so are the codes of those.
bool wide_ok(const Cache8Append &a, int size)
{
    const int vec = 16 / size;
    if (a.d_h % vec != 0 || ((uintptr_t)a.K8 | (uintptr_t)a.V8) % vec != 0 || ((uintptr_t)a.K | (uintptr_t)a.V) % 16 != 0) return false;
    for (const xkv_rows &r : {a.K_at, a.V_at})
        if (((a.batch > 1 ? r.sequence : 0) | (a.N > 1 ? r.token : 0) | (a.H_kv > 1 ? r.head : 0)) * (int64_t)size % 16 != 0) return false;
    return true;
}

template <typename T, int CODE>
hipError_t launch_append(const Cache8Append &a, hipStream_t st)
{
    constexpr int WIDE = 16 / sizeof(T);
    const unsigned units = (unsigned)a.blocks * 2 * a.H_kv * a.batch;  // (at most 2^31 - 1)
    const bool wide = wide_ok(a, (int)sizeof(T));
    // As few threads as hold a block's new rows in registers, and as few registers as that takes.  32768 tokens of 8 KV heads, bf16: blocks of 64 rows by four
    // wavefronts 49 us, by one 59, of 32 78 and 40; blocks of 8 rows in 2 pieces a thread 47, with room for 8 76;
    // blocks of one row by 16 lanes 74, by 64 268.
    const long long rows = a.N < (1LL << a.shift) ? a.N : 1LL << a.shift, pieces = rows * (a.d_h / (wide ? WIDE : 1));
    auto launch = [&](auto kernel, int threads) {
        const unsigned of = 256 / threads;
        hipLaunchKernelGGL(kernel, long_grid((units + of - 1) / of), dim3(256), 0, st, a, units);
        return hipGetLastError();
    };
    if (!wide) return pieces <= 16 * kWave ? launch(cache8_append_kernel<T, CODE, 1, 64, 16>, 64) : launch(cache8_append_kernel<T, CODE, 1, 256, 16>, 256);
    return pieces <= 16 ? launch(cache8_append_kernel<T, CODE, WIDE, 16, 1>, 16) : pieces <= 32 ? launch(cache8_append_kernel<T, CODE, WIDE, 32, 1>, 32)
         : pieces <= kWave ? launch(cache8_append_kernel<T, CODE, WIDE, 64, 1>, 64) : pieces <= 2 * kWave ? launch(cache8_append_kernel<T, CODE, WIDE, 64, 2>, 64)
         : pieces <= 4 * kWave ? launch(cache8_append_kernel<T, CODE, WIDE, 64, 4>, 64) : pieces <= 8 * kWave ? launch(cache8_append_kernel<T, CODE, WIDE, 64, 8>, 64)
                                                                                        : launch(cache8_append_kernel<T, CODE, WIDE, 256, 8>, 256);
}

}  // namespace

hipError_t launch_cache8_append(const xkv_shape &s, const Cache8Append &a, int code, hipStream_t st)
{
    if (code == XKV_E4M3) return s.dtype == XKV_F32 ? launch_append<float, XKV_E4M3>(a, st) : launch_append<bf16_t, XKV_E4M3>(a, st);
    return s.dtype == XKV_F32 ? launch_append<float, XKV_INT8>(a, st) : launch_append<bf16_t, XKV_INT8>(a, st);
}

}  // namespace xkv
