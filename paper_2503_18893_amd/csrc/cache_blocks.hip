// Blocks of an uncompressed cache: how well their means agree with a query, and the means themselves (cache.h).
#include "cache.h"

namespace xkv {
namespace {

// The score of the block that ends with the query's last visible row: the number with the largest order key, above +inf.
#define XKV_OWN_BLOCK __uint_as_float(0x7FFFFFFFu)

// S[j] = max over the query heads of a KV head of <q_h, mean_j>; XKV_OWN_BLOCK for the query's own, -inf for those behind it.  The sums
// decide which block is read, so they are taken in double precision and rounded once to single: then the order of addition does not
// show in the selection.  A wavefront per block, lanes over the channels.
template <typename T>
__global__ __launch_bounds__(256) void block_scores_kernel(CacheArgs a, const T *__restrict__ landmarks, float *__restrict__ scores,
                                                           int n_c)
{
    const int lane = lane_id(), w = wave_id(), g = blockIdx.y, z = blockIdx.z, b = z / a.N, d = a.d_h, n_rep = a.H_q / a.H_kv;
    const int v = cache_rows(a, z), last = v > 0 ? (v - 1) / a.c : -1;
    const T *q = (const T *)a.q + ((size_t)z * a.H_q + g * n_rep) * d;
    for (int j = blockIdx.x * 4 + w; j < n_c; j += gridDim.x * 4) {
        float best = j == last ? XKV_OWN_BLOCK : -INFINITY;
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
            best = j < last ? best : j == last ? XKV_OWN_BLOCK : -INFINITY;
            if (j < n_c) scores[((size_t)z * a.H_kv + g) * n_c + j] = best;
        }
    }
}

// ------------------------------------------------------------------------------------------
// bf16 means of 128 channels: scores in single precision on the bf16 matrix cores, and how far they may be off; block_select_kernel
// takes the few that this leaves undecided again in double precision.  A product of two bf16 numbers is exact in fp32, so a sum over
// the channels is off by at most 128 roundings of A = sum |q_e m_e|, 2^-17 A to the nearest; 2^-16 A is
// allowed for, which holds for rounding towards zero as well.  reach [..][n_c / 16]: the largest A
// of 16 blocks and the heads.  As above otherwise, a wavefront per 16 blocks and the queries that fit 16 rows:
//   lane (i, kk) = (l % 16, l / 16): channels 32 f + 8 kk .. of mean i and of row i; result register r: mean 4 kk + r, row i
// ------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) __bf16 bl_bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float bl_f32x4_t;

template <int QT>
__global__ __launch_bounds__(256) void block_scores_bf16_kernel(CacheArgs a, const bf16_t *__restrict__ landmarks, float *__restrict__ scores,
                                                                float *__restrict__ reach, int n_c, int per_tile)
{
    __shared__ float sm[4][2][16][17];
    const int lane = lane_id(), w = wave_id(), i16 = lane & 15, kk = lane >> 4, n_rep = a.H_q / a.H_kv;
    const int g = blockIdx.y % a.H_kv, b = blockIdx.y / a.H_kv, t0 = blockIdx.z * per_tile * QT;  // first query token of these tiles
    const int n_t = (n_c + 15) / 16;
    bl_u32x4_t Q[QT][4];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int t = t0 + x * per_tile, left = a.N - t, tokens = left < per_tile ? left : per_tile;
        const int r = i16 < tokens * n_rep ? i16 : 0, tc = tokens > 0 ? t + r / n_rep : a.N - 1;  // (rows beyond repeat another)
        const bl_u32x4_t *q = reinterpret_cast<const bl_u32x4_t *>((const bf16_t *)a.q + (((size_t)b * a.N + tc) * a.H_q + g * n_rep + r % n_rep) * 128);
#pragma unroll
        for (int f = 0; f < 4; ++f) Q[x][f] = q[4 * f + kk];
    }
    // the queries' own blocks; those before them are scored
    __shared__ int sm_own[QT * 16];
    const int all = a.N - t0 < per_tile * QT ? a.N - t0 : per_tile * QT;
    int most = 0;
    if (lane < all) {
        const int v = cache_rows(a, b * a.N + t0 + lane);
        most = v > 0 ? (v - 1) / a.c : 0;
        if (w == 0) sm_own[lane] = most;
    }
    most = wave_all(most, MaxOp());
    __syncthreads();
    const bl_u32x4_t *means = reinterpret_cast<const bl_u32x4_t *>(landmarks + ((size_t)b * a.H_kv + g) * n_c * 128);
    const int stride = gridDim.x * 64;
    bl_u32x4_t raw[4];
    auto request = [&](int j0) __attribute__((always_inline)) {
        const bl_u32x4_t *m = means + (size_t)(j0 + i16 < n_c ? j0 + i16 : n_c - 1) * 16;
#pragma unroll
        for (int f = 0; f < 4; ++f) raw[f] = m[4 * f + kk];
    };
    int j0 = (blockIdx.x * 4 + w) * 16;
    if (j0 < most) request(j0);
    for (; j0 < most; j0 += stride) {
        bl_f32x4_t S[QT], A[QT];
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            S[x] = A[x] = bl_f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                S[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bl_bf16x8_t, raw[f]), __builtin_bit_cast(bl_bf16x8_t, Q[x][f]), S[x], 0, 0, 0);
                A[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bl_bf16x8_t, raw[f] & 0x7FFF7FFFu),
                                                               __builtin_bit_cast(bl_bf16x8_t, Q[x][f] & 0x7FFF7FFFu), A[x], 0, 0, 0);
            }
        }
        if (j0 + stride < most) request(j0 + stride);
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            const int t = t0 + x * per_tile, left = a.N - t, tokens = left < per_tile ? left : per_tile;
            if (tokens <= 0) break;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sm[w][0][4 * kk + i][i16] = S[x][i];
                sm[w][1][4 * kk + i][i16] = A[x][i];
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            for (int i = kk; i < ((tokens + 3) & ~3); i += 4) {  // a lane per block and query token
                const int ic = i < tokens ? i : tokens - 1, j = j0 + i16, z = b * a.N + t + ic, last = sm_own[x * per_tile + ic];
                float best = -INFINITY, far = 0.0f;
                for (int h = 0; h < n_rep; ++h) {
                    best = fmaxf(best, sm[w][0][i16][ic * n_rep + h]);
                    far = fmaxf(far, sm[w][1][i16][ic * n_rep + h]);
                }
                if (j >= last) far = 0.0f;  // (its mean is not used and may be anything)
                far = fmaxf(far, __uint_as_float(lanes_by<0xB1>(__float_as_uint(far))));
                far = fmaxf(far, __uint_as_float(lanes_by<0x4E>(__float_as_uint(far))));
                far = fmaxf(far, __uint_as_float(lanes_by<0x141>(__float_as_uint(far))));
                far = fmaxf(far, __uint_as_float(lanes_by<0x140>(__float_as_uint(far))));
                const size_t zg = (size_t)z * a.H_kv + g;
                if (i < tokens && j < last) scores[zg * n_c + j] = best;
                if (i < tokens && i16 == 0) reach[zg * n_t + j0 / 16] = far;
            }
        }
    }
}

// Sum over the 16 lanes of a row, in all of them.
template <int CTRL> __device__ __forceinline__ double lanes_by64(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)lanes_by<CTRL>((uint32_t)(u >> 32)) << 32 | lanes_by<CTRL>((uint32_t)u));
}
__device__ __forceinline__ double row_sum64(double x)
{
    x += lanes_by64<0xB1>(x);
    x += lanes_by64<0x4E>(x);
    x += lanes_by64<0x141>(x);
    return x + lanes_by64<0x140>(x);
}

// ------------------------------------------------------------------------------------------
// The blocks of a query and KV head, ascending: one workgroup, the scores in registers, KPT a thread (element i of a lane is block
// (w KPT + i) 64 + lane).  The scores' range is cut into 2048 bins; the bin that the k-th largest falls into, and with estimates (reach)
// what is within 2 E of it, is open: the k-th largest of the exact scores is within E of the k-th largest estimate, so everything above is
// taken and nothing below.  The open ones, a few, are scored again in double precision (16 lanes each) and ranked one against another.
// Where more than kOpen are open (many equal scores, infinite ones) all are scored again and a radix selection over all digits follows
// instead: 16 queries and KV heads, 1000 / 4000 / 16000 equal means of 4 heads, the whole call 46 / 127 / 286 us, else 21 / 26 / 42.
// ------------------------------------------------------------------------------------------
constexpr int kOpen = 128;

template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void block_select_kernel(CacheArgs a, const bf16_t *__restrict__ landmarks, const float *__restrict__ scores,
                                                               const float *__restrict__ reach, int32_t *__restrict__ blocks, int n_c)
{
    constexpr int WAVES = THREADS / 64, COPIES = 16, BINS = 2048, PER = BINS / THREADS;
    __shared__ uint32_t hist[256 * COPIES];
    __shared__ uint32_t sh_pick[3], sh_wave[2][WAVES];
    __shared__ float sh_min[WAVES], sh_max[WAVES], sh_far[WAVES];
    __shared__ int open_id[kOpen];
    __shared__ uint32_t open_key[kOpen], open_taken[kOpen];
    const int zg = blockIdx.x, z = zg / a.H_kv, g = zg % a.H_kv, lane = lane_id(), w = wave_id(), tid = threadIdx.x, n_rep = a.H_q / a.H_kv;
    const int v = cache_rows(a, z), own = v > 0 ? (v - 1) / a.c : -1, k_ch = a.k_ch;  // candidates: 0 .. own - 1
    int32_t *out = blocks + (size_t)zg * k_ch;
    if (own < k_ch) {  // all that there are, and the next ones
        for (int i = tid; i < k_ch; i += THREADS) out[i] = i;
        return;
    }
    const uint32_t k = (uint32_t)k_ch - 1u;
    if (k == 0u) {
        if (tid == 0) out[0] = own;
        return;
    }
    const bf16_t *means = landmarks + ((size_t)(z / a.N) * a.H_kv + g) * n_c * 128, *q = (const bf16_t *)a.q + ((size_t)z * a.H_q + g * n_rep) * 128;
    auto block_of = [&](int i) { return (w * KPT + i) * 64 + lane; };
    auto below = [&](uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)); };
    float S[KPT], s_min = INFINITY, s_max = -INFINITY, far = 0.0f;
#pragma unroll
    for (int i = 0; i < KPT; ++i) S[i] = scores[(size_t)zg * n_c + (block_of(i) < own ? block_of(i) : 0)];
    if (reach)
        for (int i = tid; i < (own + 15) / 16; i += THREADS) far = fmaxf(far, reach[(size_t)zg * ((n_c + 15) / 16) + i]);
    for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        s_min = fminf(s_min, block_of(i) < own ? S[i] : INFINITY);
        s_max = fmaxf(s_max, block_of(i) < own ? S[i] : -INFINITY);
    }
    s_min = -wave_all(-s_min, MaxOp());
    s_max = wave_all(s_max, MaxOp());
    far = wave_all(far, MaxOp());
    if (lane == 0) {
        sh_min[w] = s_min;
        sh_max[w] = s_max;
        sh_far[w] = far;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        s_min = fminf(s_min, sh_min[i]);
        s_max = fmaxf(s_max, sh_max[i]);
        far = fmaxf(far, sh_far[i]);
    }
    const float range = s_max - s_min, scale = (BINS - 1) / range;
    bool few = scale > 0.0f && scale < INFINITY;  // (the same in every thread; not where all are equal or sums overflow)
    float lo = 0.0f, hi = 0.0f;
    uint32_t in = 0, open = 0, open_before = 0;
    if (few) {
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (block_of(i) < own) {
                const int bin = (int)((S[i] - s_min) * scale);
                atomicAdd(&hist[bin < BINS ? bin : BINS - 1], 1u);
            }
        __syncthreads();
        uint32_t c[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            c[i] = hist[PER * tid + i];
            sum += c[i];
        }
        uint32_t upto = sum;  // in this thread's bins and those of higher threads
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const uint32_t o = __shfl_down(upto, off, kWave);
            upto += lane + off < kWave ? o : 0u;
        }
        if (lane == 0) sh_wave[0][w] = upto;
        __syncthreads();
        for (int i = w + 1; i < WAVES; ++i) upto += sh_wave[0][i];
        uint32_t above = upto - sum;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
            if (above < k && k <= above + c[i]) sh_pick[0] = PER * tid + i;
            above += c[i];
        }
        __syncthreads();
        const float width = range / (BINS - 1), at = s_min + width * (float)sh_pick[0];
        const float slack = fmaxf(fabsf(s_min), fabsf(s_max)) * 0x1p-20f + far * 0x1p-15f;  // rounding of the bins' ends; 2 E, E = 2^-16 A
        lo = at - slack;
        hi = at + width + slack;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            in += (uint32_t)__popcll(__ballot(block_of(i) < own && S[i] > hi));
            open += (uint32_t)__popcll(__ballot(block_of(i) < own && S[i] >= lo && S[i] <= hi));
        }
        if (lane == 0) {
            sh_wave[0][w] = in;
            sh_wave[1][w] = open;
        }
        __syncthreads();
        in = open = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            in += sh_wave[0][i];
            open_before += i < w ? sh_wave[1][i] : 0u;
            open += sh_wave[1][i];
        }
        few = open <= kOpen;
    }
    uint32_t key[KPT];  // 0: no candidate; what is above T and the first `ties` of what is T are taken
    uint32_t T, ties;
    if (few) {
        uint32_t at = open_before;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool mine = block_of(i) < own && S[i] >= lo && S[i] <= hi;
            const uint64_t m = __ballot(mine);
            if (mine) {
                open_id[at + below(m)] = block_of(i);
                open_key[at + below(m)] = order_key(S[i]);
            }
            at += (uint32_t)__popcll(m);
        }
        __syncthreads();
        if (reach && in + open > k) {  // (else all of them are taken)
            const int grp = tid >> 4, l = tid & 15;
            for (uint32_t e = grp; e < open; e += THREADS / 16) {
                const bl_u32x4_t x = reinterpret_cast<const bl_u32x4_t *>(means + (size_t)open_id[e] * 128)[l];
                float best = -INFINITY;
#pragma unroll 4
                for (int h = 0; h < n_rep; ++h) {
                    const bl_u32x4_t y = reinterpret_cast<const bl_u32x4_t *>(q + 128 * h)[l];
                    double sum = 0.0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fma(channel<bf16_t>(&x, i), channel<bf16_t>(&y, i), sum);
                    best = fmaxf(best, (float)row_sum64(sum));
                }
                if (l == 0) open_key[e] = order_key(best);
            }
            __syncthreads();
        }
        for (uint32_t e = tid; e < open; e += THREADS) {
            const uint32_t mine = open_key[e];
            uint32_t rank = in;
            for (uint32_t f = 0; f < open; ++f) rank += open_key[f] > mine || (open_key[f] == mine && f < e);
            open_taken[e] = rank < k;
        }
        __syncthreads();
        at = open_before;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool is_open = block_of(i) < own && S[i] >= lo && S[i] <= hi;
            const uint64_t m = __ballot(is_open);
            key[i] = block_of(i) < own && (is_open ? open_taken[at + below(m)] != 0u : S[i] > hi);
            at += (uint32_t)__popcll(m);
        }
        T = 0;
        ties = 0;
    } else {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            if (reach && (w * KPT + i) * 64 < own) {  // every one of them exactly, 16 lanes each
                const int b0 = (w * KPT + i) * 64, grp = lane >> 4, l16 = lane & 15;
                bl_u32x4_t x[4];  // blocks b0 + 4 step + grp, four steps at once
#pragma unroll 1
                for (int s4 = 0; s4 < 16; s4 += 4) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int j = b0 + 4 * (s4 + t) + grp;
                        x[t] = reinterpret_cast<const bl_u32x4_t *>(means + (size_t)(j < own ? j : own - 1) * 128)[l16];
                    }
                    float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    for (int h = 0; h < n_rep; ++h) {
                        const bl_u32x4_t y = reinterpret_cast<const bl_u32x4_t *>(q + 128 * h)[l16];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            double sum = 0.0;
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum = fma(channel<bf16_t>(&x[t], e), channel<bf16_t>(&y, e), sum);
                            best[t] = fmaxf(best[t], (float)row_sum64(sum));
                        }
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {  // to lane 4 step + grp
                        const float mine = __shfl(best[t], 16 * (lane & 3), kWave);
                        S[i] = lane >> 2 == s4 + t ? mine : S[i];
                    }
                }
            }
            const uint32_t x = order_key(S[i]);
            key[i] = block_of(i) < own ? (x ? x : 1u) : 0u;
        }
        uint32_t prefix = 0, k_rem = k;
#pragma unroll
        for (int level = 0; level < 4; ++level) {  // counters in 16 copies: many are equal
            __syncthreads();
            for (int i = tid; i < 256 * COPIES; i += THREADS) hist[i] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < KPT; ++i)
                if (level == 0 || key[i] >> (32 - 8 * level) == prefix) atomicAdd(&hist[(key[i] >> (24 - 8 * level) & 255u) * COPIES + (lane & (COPIES - 1))], 1u);
            __syncthreads();
            if (tid < 256) {
                uint32_t c = 0;
#pragma unroll
                for (int i = 0; i < COPIES; ++i) c += hist[tid * COPIES + ((i + tid) & (COPIES - 1))];
                hist[tid * COPIES] = c;  // (only this thread reads the others)
            }
            __syncthreads();
            if (w == 0) {  // the bin b with (keys in bins above b) < k_rem <= (keys in bins >= b)
                uint32_t c[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[i] = hist[(4 * lane + i) * COPIES];
                    sum += c[i];
                }
                uint32_t upto = sum;
#pragma unroll
                for (int off = 1; off < kWave; off <<= 1) {
                    const uint32_t o = __shfl_down(upto, off, kWave);
                    upto += lane + off < kWave ? o : 0u;
                }
                uint32_t above = upto - sum;
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    if (above < k_rem && k_rem <= above + c[i]) {
                        sh_pick[1] = 4 * lane + i;
                        sh_pick[2] = k_rem - above;
                    }
                    above += c[i];
                }
            }
            __syncthreads();
            prefix = prefix << 8 | sh_pick[1];
            k_rem = sh_pick[2];
        }
        T = prefix;
        ties = k_rem;
    }
    // in order: what is above T, and the first of those equal to it
    uint32_t gt = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        gt += (uint32_t)__popcll(__ballot(key[i] > T));
        if (ties) eq += (uint32_t)__popcll(__ballot(key[i] == T));
    }
    __syncthreads();
    if (lane == 0) {
        sh_wave[0][w] = gt;
        sh_wave[1][w] = eq;
    }
    __syncthreads();
    gt = eq = 0;
    for (int i = 0; i < w; ++i) {
        gt += sh_wave[0][i];
        eq += sh_wave[1][i];
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const uint64_t mg = __ballot(key[i] > T), me = ties ? __ballot(key[i] == T) : 0;
        const uint32_t g_at = gt + below(mg), e_at = eq + below(me);
        if (key[i] > T || (ties && key[i] == T && e_at < ties)) out[g_at + (e_at < ties ? e_at : ties)] = block_of(i);
        gt += (uint32_t)__popcll(mg);
        eq += (uint32_t)__popcll(me);
    }
    if (tid == 0) out[k] = own;
}

// Means of the blocks that hold the last N rows in use, over the rows in use.  A wavefront per block, lanes over the channels.
template <typename T>
__global__ __launch_bounds__(256) void landmarks_update_kernel(const T *__restrict__ K, const int32_t *__restrict__ lengths,
                                                               T *__restrict__ landmarks, int L, int d, int H_kv, int N, int c, int n_c)
{
    const int lane = lane_id(), row = blockIdx.y;
    int n = lengths ? lengths[row / H_kv] : L;
    n = n < 0 ? 0 : n < L ? n : L;
    const int j = (n > N ? n - N : 0) / c + blockIdx.x * 4 + wave_id();
    if (n == 0 || j > (n - 1) / c) return;
    const int t0 = j * c, t1 = n - t0 > c ? t0 + c : n;
    const float inv = 1.0f / (float)(t1 - t0);
    for (int e = lane; e < d; e += kWave) {
        float sum = 0.0f;
#pragma unroll 8
        for (int t = t0; t < t1; ++t) sum += to_f32(K[((size_t)row * L + t) * d + e]);
        landmarks[((size_t)row * n_c + j) * d + e] = from_f32<T>(sum * inv);
    }
}

}  // namespace

bool block_select_ok(int n_c) { return n_c <= 16384; }

hipError_t launch_block_select(const xkv_shape &s, const CacheArgs &a, const void *landmarks, int n_c, float *scores, float *reach, int32_t *blocks,
                               hipStream_t st)
{
    const int n_rep = a.H_q / a.H_kv;
    const bool estimate = s.dtype == XKV_BF16 && s.d_h == 128 && (((uintptr_t)a.q | (uintptr_t)landmarks) & 15u) == 0;
    if (a.k_ch < n_c) {  // (else there is nothing to choose)
        if (estimate) {
            // four row tiles a wavefront share the means that it reads, where there are that many; 16 blocks a time, several times once
            // there are wavefronts enough
            const int per_tile = 16 / n_rep < a.N ? 16 / n_rep : a.N, qt = a.N > 2 * per_tile ? 4 : 1, tiles = (a.N + per_tile * qt - 1) / (per_tile * qt);
            const long long waves = (long long)((n_c + 15) / 16) * a.H_kv * a.batch * tiles;
            const int times = waves < 8192 ? 1 : waves < 65536 ? (int)(waves / 4096) : 16;
            const dim3 grid((n_c + 64 * times - 1) / (64 * times), a.H_kv * a.batch, tiles);
            auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, (const bf16_t *)landmarks, scores, reach, n_c, per_tile); };
            qt == 4 ? launch(block_scores_bf16_kernel<4>) : launch(block_scores_bf16_kernel<1>);
        } else {
            const hipError_t e = launch_block_scores(s, a, landmarks, n_c, scores, st);
            if (e != hipSuccess) return e;
        }
    }
    auto select = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3(a.batch * a.N * a.H_kv), dim3(threads), 0, st, a, (const bf16_t *)landmarks, scores, estimate ? reach : nullptr, blocks, n_c);
        return hipGetLastError();
    };
    // Eight wavefronts where a workgroup has a compute unit to itself and more than 1024 blocks.  A whole call with four / eight, us: 8 queries
    // and KV heads, 2048 blocks 22.4 / 21.5, 128 of them 77.6 / 76.3, 1024 of them 263 / 268; 16 with 4000 blocks 25.9 / 24.2; 8 with 1000 the same.
    const bool few = a.batch * a.N * a.H_kv <= 256;
    return n_c <= 1024 ? select(block_select_kernel<256, 4>, 256)
         : n_c <= 2048 ? (few ? select(block_select_kernel<512, 4>, 512) : select(block_select_kernel<256, 8>, 256))
         : n_c <= 4096 ? (few ? select(block_select_kernel<512, 8>, 512) : select(block_select_kernel<256, 16>, 256))
                       : select(block_select_kernel<1024, 16>, 1024);
}

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
    const int n_c = (s.L - 1) / c + 1, most = (N - 1) / c + 2, blocks = most < n_c ? most : n_c;  // (N rows: one block more if they begin inside one)
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
