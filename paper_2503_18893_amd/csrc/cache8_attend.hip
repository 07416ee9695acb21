// Attention over a cache held in 8 bits (cache8.h).
//   z_t = scale ks[t / c] <q, k8_t>,  out = sum_t exp(z_t - max) vs[t / c] v8_t / sum_t exp(z_t - max)
// over the rows that a query sees, split over the rows: every workgroup leaves (maximum, sum, unnormalised output) of its part, in
// powers of two, and a second kernel merges them.
#include <type_traits>

#include "cache8.h"
#include "cache_tile.h"

namespace xkv {
namespace {

using namespace cache_tile;

constexpr int kGenTokens = 64;  // rows of the cache a round of the general kernel, a lane each
constexpr int kGenRows = 16;    // its rows (query, head) per workgroup, four per wavefront
constexpr float kLog2e = 1.44269504088896340736f;

// What a workgroup takes: query rows tile * rows .. of KV head g of sequence seq, rows t_begin .. t_end - 1 of the cache.
struct Unit8 {
    int seq, g, tile, part, t_begin, t_end;
    bool some;  // whether the merge reads this part (it may have no rows all the same)
};
__device__ __forceinline__ Unit8 same_in_all_lanes(const Unit8 &u)
{
    auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    return Unit8{same(u.seq), same(u.g), same(u.tile), same(u.part), same(u.t_begin), same(u.t_end), same(u.some) != 0};
}

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
    const int tiles = ceil_div_dev(a.N * (a.H_q / a.H_kv), a.rows);
    if (a.by_length) {
        __shared__ int sm_rows[kCutBatch];
        const bool many = a.N > 1 && a.visible;
        if (many) {  // every workgroup looks at all of them
            for (int i = (int)threadIdx.x; i < a.batch; i += (int)blockDim.x) sm_rows[i] = 0;
            __syncthreads();
            for (int i = (int)threadIdx.x; i < a.batch * a.N; i += (int)blockDim.x) atomicMax(&sm_rows[i / a.N], a.visible[i]);
            __syncthreads();
        }
        const CacheUnit c = cache_unit(Cache8Cut{many ? sm_rows : nullptr, a.visible, a.table, a.L, a.H_kv, a.batch, a.round, a.parts}, CacheMode::weights, tiles);
        u.seq = c.seq, u.g = c.g, u.tile = tiles - 1 - c.tile, u.part = c.part, u.t_begin = c.t_begin, u.t_end = c.t_end, u.some = c.some;
        if (many && u.some) {  // (of a prompt the tiles see different numbers of rows)
            const int n = tile_sees(a, u.seq, u.tile);
            u.t_end = n < u.t_end ? n : u.t_end;
        }
        return u;
    }
    // workgroups go to the eight XCDs in turn: the row tiles of a part, which share its rows of the cache, to one XCD, one after the other
    const int x = (int)blockIdx.x;
    int id = x / tiles, tile = x % tiles;
    if ((int)gridDim.x % (8 * tiles) == 0) {
        tile = x / 8 % tiles;
        id = x / (8 * tiles) * 8 + x % 8;
    }
    u.tile = tiles - 1 - tile;  // (of a prompt the last ones see most)
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

// A part that has no rows for this tile: a sum that none has, by which the merge knows that there is no output.
__device__ __forceinline__ void leave_nothing(const Cache8Args &a, const Unit8 &u)
{
    const int n_rep = a.H_q / a.H_kv, M = a.N * n_rep;
    for (int i = (int)threadIdx.x; i < a.rows; i += (int)blockDim.x) {
        const int m = u.tile * a.rows + i;
        if (m >= M) break;
        const size_t slot = ((size_t)u.part * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep;
        a.part_ml[2 * slot] = -INFINITY;
        a.part_ml[2 * slot + 1] = -1.0f;
    }
}

template <int CODE> __device__ __forceinline__ float value8(uint8_t x)
{
    return CODE == XKV_E4M3 ? __builtin_amdgcn_cvt_f32_fp8((int)x, 0) : (float)(int8_t)x;
}

// ------------------------------------------------------------------------------------------
// General path, any type, width and block.  A round takes 64 rows of the cache, whose keys and values, with their scales, go to LDS in single precision.
// For the logits a lane multiplies one of the keys with the four queries of its wavefront; for the sums lanes run over the channels, and
// the weights go through LDS.  Far from its bytes: one query of 4 heads on each of 8 KV heads after 32768 rows of 96 channels, 107 us (10 at the rate of a copy).
// ------------------------------------------------------------------------------------------
__host__ __device__ inline int general_pitch(int d) { return ((d + 3) / 4 | 1) * 4; }  // floats; an odd number of 16-byte pieces

template <typename T, int CODE, int JP>
__global__ __launch_bounds__(256) void cache8_general_kernel(Cache8Args a, bool direct)
{
    extern __shared__ __attribute__((aligned(16))) float smem_f[];
    constexpr int TOGETHER = 16 / JP;  // rows of a wavefront that are requested together
    const Unit8 u = unit8(a);
    if (!u.some && !direct) return;  // (the merge knows)
    if (u.t_begin >= u.t_end && !direct) return leave_nothing(a, u);
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
        for (int i0 = w; i0 < kGenTokens; i0 += 4 * TOGETHER) {
            uint8_t kx[TOGETHER][JP], vx[TOGETHER][JP];
            float k_scale[TOGETHER], v_scale[TOGETHER];
#pragma unroll
            for (int x = 0; x < TOGETHER; ++x) {
                const int t = t0 + i0 + 4 * x < u.t_end ? t0 + i0 + 4 * x : u.t_end - 1;
                k_scale[x] = ks[t >> a.shift];
                v_scale[x] = vs[t >> a.shift];
#pragma unroll
                for (int jj = 0; jj < JP; ++jj) {
                    const int j = lane + jj * kWave, jc = j < d ? j : 0;
                    kx[x][jj] = K[(size_t)t * d + jc];
                    vx[x][jj] = V[(size_t)t * d + jc];
                }
            }
#pragma unroll
            for (int x = 0; x < TOGETHER; ++x)
#pragma unroll
                for (int jj = 0; jj < JP; ++jj) {
                    const int j = lane + jj * kWave, i = i0 + 4 * x;
                    if (j >= d4) continue;
                    kt[i * pitch + j] = j < d ? k_scale[x] * value8<CODE>(kx[x][jj]) : 0.0f;
                    vt[i * pitch + j] = j < d ? v_scale[x] * value8<CODE>(vx[x][jj]) : 0.0f;
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
        const size_t slot = ((size_t)(direct ? u.seq : u.part) * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep;
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int j = lane + jj * kWave;
            if (j >= d) continue;
            if (direct)
                ((T *)a.out)[slot * d + j] = result<T>(sees[r] == 0 ? 0.0f : o[r][jj] / den[r]);
            else
                a.part_o[slot * d + j] = o[r][jj];
        }
        if (!direct && lane == 0) {
            a.part_ml[2 * slot] = mx[r];
            a.part_ml[2 * slot + 1] = den[r];
        }
    }
}

// ------------------------------------------------------------------------------------------
// Matrix-core path: D channels.  A wavefront takes tiles of 32 rows of the cache on its own and 16 RT rows (query,
// head):
//   S^T [32 tokens x rows] = codes of K x Q^T (bf16),  P^T = exp2(c ks S^T - m),  O^T [channels x rows] += codes of V^T x (vs P^T) (fp16)
// Codes are bf16 and fp16 numbers as they are (3 or 7 bits of mantissa), so both products take them exactly, and the scales, one for four tokens of
// a lane (FINE: blocks of one or two rows, one for each), multiply logits and weights.  A lane holds one row of S^T, P^T and O^T (rows n16), so that the statistics are its own, and P^T is the
// second product's operand as it comes.  Keys and values go from memory to registers: a lane's pieces of K are its operands but for the
// conversion; of V it reads the tokens that it has weights of, D / 16 channels of each (a row of the cache is read by 16 lanes), and pairs
// up neighbouring tokens by permuting bytes.
// The maximum is only raised when a logit outgrows it by 2^8.  Weights times scales enter as fp16, 2^-12: `inv`, a power of two, brings the largest scale met
// so far to between 2^6 and 2^7, so that they are at most 2^15, and down to 2^-20 of that scale keep their 11 bits (what is smaller is held to 2^-31 of it;
// scales below 2^-119 stay as `inv` begins, 2^126, and their weights are held to 2^-151).
// Beside the output's own rounding that is not seen: the error against 64 bits is 0.0017 of the results' root mean square, with bf16 pairs in its place as well.
// fp32: a query is three terms of bf16, a weight two of fp16, and scales are multiplied in after the exponential.
// It is a stream: one query after 32768 rows of 8 KV heads, 67 MB, 15 us with its start and end (6.4 TB/s with 16 sequences of 65536); 16 heads 15, 20 rows 20,
// 32 rows 23; from there on row tiles of their own, which read the same rows of the cache (64 rows 24, 128 38).  A wavefront takes 0.8 to 1.3 us a tile, a
// chain of products, a maximum and exponentials; two of them to a vector unit keep 64 KB a compute unit under way.
// ------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;

template <int CODE> __device__ __forceinline__ bf16x8_t codes8(uint32_t lo, uint32_t hi)
{
    u32x4_t x;
    if constexpr (CODE == XKV_E4M3) {
        x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
        x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
        x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
        x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = (i < 2 ? lo : hi) >> (16 * (i & 1));
            x[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(w >> 8)), __float_as_uint((float)(int8_t)w), 0x07060302u);  // (exact)
        }
    }
    return __builtin_bit_cast(bf16x8_t, x);
}

// Eight codes as fp16 numbers.
template <int CODE> __device__ __forceinline__ f16x8_t values8(uint32_t lo, uint32_t hi)
{
    u32x4_t x;
    if constexpr (CODE == XKV_E4M3) {
        x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
        x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
        x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
        x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = (i < 2 ? lo : hi) ^ 0x80808080u;
            const uint32_t two = __builtin_amdgcn_perm(w, w, i % 2 ? 0x0C030C02u : 0x0C010C00u) | 0x64006400u;
            x[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, two) - (_Float16)1152.0f);
        }
    }
    return __builtin_bit_cast(f16x8_t, x);
}

// Four channels of eight tokens, w[e] those of token e, as operands: x[j] channel j of the tokens.
template <int CODE> __device__ __forceinline__ void codes_by_channel(const uint32_t (&w)[8], f16x8_t (&x)[4])
{
    u32x4_t y[4];
    if constexpr (CODE == XKV_E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t a = __builtin_bit_cast(uint32_t, h ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i], 1.0f, true)
                                                                  : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i], 1.0f, false));
                const uint32_t b = __builtin_bit_cast(uint32_t, h ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + 1], 1.0f, true)
                                                                  : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + 1], 1.0f, false));
                y[2 * h][i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                y[2 * h + 1][i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            }
    } else {
        // 1024 + 128 + a code is an fp16 number with the code, its sign bit turned, in its lower bits
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = w[2 * i] ^ 0x80808080u, b = w[2 * i + 1] ^ 0x80808080u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t two = __builtin_amdgcn_perm(b, a, 0x0C040C00u + 0x00010001u * j) | 0x64006400u;
                y[j][i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, two) - (_Float16)1152.0f);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __builtin_bit_cast(f16x8_t, y[j]);
}

// 4 B per lane from global memory into LDS at lds_base + lane * 4 (lds_base is wave-uniform); see copy16_global_to_lds.
__device__ __forceinline__ void copy4_to_lds(const void *gptr, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_base), "v"(gptr) : "memory", "m0");
}

// Words of a row of the cache; ONCE: past the caches, where nobody else reads them.
template <int N> struct Words {
    uint32_t x[N];
};
template <int N, bool ONCE> __device__ __forceinline__ Words<N> load_words(const uint8_t *from)
{
    typedef __attribute__((ext_vector_type(N))) uint32_t vec_t;
    Words<N> r;
    if constexpr (N == 1) {
        r.x[0] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(from)) : *reinterpret_cast<const uint32_t *>(from);
    } else {
        const vec_t v = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const vec_t *>(from)) : *reinterpret_cast<const vec_t *>(from);
#pragma unroll
        for (int i = 0; i < N; ++i) r.x[i] = v[i];
    }
    return r;
}

__device__ __forceinline__ float largest4(const f32x4_t &x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }

constexpr float kFarUp = 0x1p126f;  // `inv` before any scale was met
constexpr float kLeast = 0x1p-60f;  // scales by `inv` that are less count as this: their weights are zeros in fp16

template <typename T, int CODE, int D, int RT, bool ONCE, bool FINE>
__global__ __launch_bounds__(256, D < 256 ? 2 : 1) void cache8_mfma_kernel(Cache8Args a, bool direct)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int TERMS = F32 ? 3 : 1;  // of a query
    constexpr int SCALES = FINE ? 8 : 2;  // of a lane's eight tokens: each has its own, or four have one
    constexpr bool AFTER = F32 || FINE;   // weights are multiplied with scales after the exponential
    static_assert(!F32 || RT == 1, "queries in registers");
    constexpr int KP = D / 64, VW = D / 64, JC = D / 16, STEPS = D / 32, PITCH = D / 4;  // pieces of K, words of V, channels of a lane; products; 16-byte pieces of a row
    constexpr bool Q_LDS = RT > 1;
    __shared__ f32x4_t sm_o[4][16 * PITCH];
    __shared__ float sm_m[4][16], sm_l[4][16];
    __shared__ u32x4_t sm_q[Q_LDS ? RT * STEPS * 64 : 1];
    const Unit8 u = unit8(a);
    const int lane = lane_id(), w = wave_id(), n16 = lane & 15, kk = lane >> 4, n_rep = a.H_q / a.H_kv, M = a.N * n_rep;
    if (!u.some && !direct) return;  // (the merge knows)
    if (u.t_begin >= u.t_end && !direct) return leave_nothing(a, u);
    const size_t head = (size_t)u.seq * a.H_kv + u.g;
    const uint8_t *K = a.K8 + head * a.L * D, *V = a.V8 + head * a.L * D;
    const float *ks = a.k_scales + head * a.n_c, *vs = a.v_scales + head * a.n_c, c = a.scale * kLog2e;

    Words<4> kr[2][KP];
    Words<VW> vr[8];
    float ksr[SCALES], vsr[SCALES];
    const uint32_t k_off = n16 * D + 16 * kk, v_off = 4 * kk * D + 4 * VW * n16;
    auto request_scales = [&](float (&r)[SCALES], const float *from, int t, int last) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            const int row = FINE ? 16 * (i / 4) + 4 * kk + i % 4 : 16 * i + 4 * kk;
            r[i] = from[(t + (row < last ? row : last)) >> a.shift];
        }
    };
    auto request_k = [&](int t) __attribute__((always_inline)) {
        const uint8_t *base = K + (size_t)t * D;
        const int last = u.t_end - 1 - t;  // (rows behind the last one: that one again)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = 16 * h + n16;
            const uint32_t off = last >= 31 ? k_off + 16 * h * D : (row < last ? row : last) * D + 16 * kk;
#pragma unroll
            for (int f = 0; f < KP; ++f) kr[h][f] = load_words<4, ONCE>(base + off + 64 * f);
        }
        request_scales(ksr, ks, t, last);
    };
    auto request_v = [&](int t) __attribute__((always_inline)) {
        const uint8_t *base = V + (size_t)t * D;
        const int last = u.t_end - 1 - t;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = 16 * (e / 4) + e % 4 + 4 * kk;
            const uint32_t off = last >= 31 ? v_off + (16 * (e / 4) + e % 4) * D : (row < last ? row : last) * D + 4 * VW * n16;
            vr[e] = load_words<VW, ONCE>(base + off);
        }
        request_scales(vsr, vs, t, last);
    };
    constexpr int STEP = 128;  // of a workgroup
    int t = u.t_begin + 32 * w;
    if (t < u.t_end) {
        request_k(t);
        request_v(t);
    }

    // Q^T operands: lane (row n16, kk), product s, position e: channel 64 (s / 2) + 16 kk + 8 (s % 2) + e, as the pieces of K have them
    u32x4_t Q[TERMS][STEPS];
    int sees[RT], least = 0x7FFFFFFF;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int m = (u.tile * RT + rt) * 16 + n16, m_in = m < M ? m : M - 1, i = m_in / n_rep;
        const T *q = (const T *)a.q + (((size_t)u.seq * a.N + i) * a.H_q + u.g * n_rep + m_in % n_rep) * D;
        sees[rt] = visible8(a, u.seq, i);
        least = sees[rt] < least ? sees[rt] : least;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (Q_LDS && (rt * STEPS + s) % 4 != w) continue;
            const T *from = q + 64 * (s / 2) + 16 * kk + 8 * (s % 2);
            if constexpr (F32) {  // three terms of bf16 hold a query's 24 bits
                f32x8_t x = *reinterpret_cast<const f32x8_t *>(from);
#pragma unroll
                for (int i = 0; i < TERMS; ++i) {
                    const bf16x8_t y = __builtin_convertvector(x, bf16x8_t);
                    Q[i][s] = __builtin_bit_cast(u32x4_t, y);
                    x -= __builtin_convertvector(y, f32x8_t);
                }
            } else {
                const u32x4_t x = *reinterpret_cast<const u32x4_t *>(from);
                if (Q_LDS)
                    sm_q[(rt * STEPS + s) * 64 + lane] = x;
                else
                    Q[0][s] = x;
            }
        }
    }
    least = -wave_all(-least, MaxOp());  // rows that all of them see
    least = __builtin_amdgcn_readfirstlane(least < u.t_end ? least : u.t_end);
    if (Q_LDS) __syncthreads();

    f32x4_t O[RT][JC];
    float m_run[RT], l_run[RT], inv = kFarUp;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.0f;
#pragma unroll
        for (int j = 0; j < JC; ++j) O[rt][j] = f32x4_t(0.0f);
    }

    // A tile; MIXED: rows see different tokens of it.
    auto tile = [&](int t, auto mixed) __attribute__((always_inline)) {
        constexpr bool MIXED = decltype(mixed)::value;
        const bool next = t + STEP < u.t_end;
        f32x4_t S[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) S[rt][0] = S[rt][1] = f32x4_t(0.0f);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            bf16x8_t kb[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) kb[h] = codes8<CODE>(kr[h][s / 2].x[2 * (s % 2)], kr[h][s / 2].x[2 * (s % 2) + 1]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                for (int i = TERMS - 1; i >= 0; --i) {
                    const bf16x8_t qf = __builtin_bit_cast(bf16x8_t, Q_LDS ? sm_q[(rt * STEPS + s) * 64 + lane] : Q[i][s]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) S[rt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[h], qf, S[rt][h], 0, 0, 0);
                }
            }
        }
        // of element e of the lane's eight: scale e, or e / 4
        auto of = [](int e) { return FINE ? e : e / 4; };
        float kc[SCALES], largest = vsr[0];
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            kc[i] = ksr[i] * c;
            largest = fmaxf(largest, vsr[i]);
        }
        if (next) request_k(t + STEP);
        // element v of half h: token t + 16 h + 4 kk + v
        uint32_t seen[RT];
        float top[RT];
        bool raise = !(largest * inv <= 128.0f);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (MIXED) {
                const int left = sees[rt] < u.t_end ? sees[rt] - t : u.t_end - t;
                seen[rt] = left >= 32 ? 0xFFFFFFFFu : left > 0 ? (1u << left) - 1u : 0u;
                seen[rt] >>= 4 * kk;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    S[rt][e / 4][e % 4] = seen[rt] >> (16 * (e / 4) + e % 4) & 1u ? S[rt][e / 4][e % 4] * kc[of(e)] : -INFINITY;
            } else if (FINE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) S[rt][e / 4][e % 4] *= kc[of(e)];
            }
            float lo, hi, most[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                most[h] = largest4(S[rt][h]);
                if (!MIXED && !FINE) most[h] *= kc[h];  // (scales are not negative)
            }
            quarters(fmaxf(most[0], most[1]), lo, hi);
            halves(fmaxf(lo, hi), lo, hi);
            top[rt] = fmaxf(lo, hi);
            raise |= !(top[rt] - m_run[rt] <= 8.0f);
        }
        if (__ballot(raise)) {
            largest = wave_all(largest, MaxOp());  // (NaN is passed over)
            float less = 1.0f;
            if (largest * inv > 128.0f && largest < INFINITY) {
                const float now = __uint_as_float((254u + 6u - (__float_as_uint(largest) >> 23 & 0xFFu)) << 23);  // 2^6 by its power of two
                less = now * __uint_as_float((254u << 23) - __float_as_uint(inv));                                 // (inv is a power of two)
                inv = now;
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float m_new = fmaxf(m_run[rt], top[rt]), alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
                l_run[rt] *= alpha;
#pragma unroll
                for (int j = 0; j < JC; ++j) O[rt][j] *= alpha * less;
                m_run[rt] = m_new;
            }
        }
        // vs P = exp2(z - m + log2 vs), whose sum by 1 / vs is that of the weights (AFTER: one after the other)
        float lv[2], rv[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float v = AFTER ? 1.0f : vsr[h] * inv < kLeast ? kLeast : vsr[h] * inv;  // (NaN stays)
            lv[h] = AFTER ? 0.0f : __builtin_amdgcn_logf(v);
            rv[h] = AFTER ? 1.0f : __builtin_amdgcn_rcpf(v);
        }
        f16x8_t P[RT], R[RT];  // .. (fp32) and what P leaves
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float less = m_run[rt] == -INFINITY ? 0.0f : m_run[rt], add[2] = {lv[0] - less, lv[1] - less};
            f32x8_t z;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                z[e] = __builtin_amdgcn_exp2f(MIXED || FINE ? S[rt][e / 4][e % 4] + add[e / 4] : fmaf(S[rt][e / 4][e % 4], kc[of(e)], add[e / 4]));
            if (MIXED) {  // (a scale that is not seen may be NaN)
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = seen[rt] >> (16 * (e / 4) + e % 4) & 1u ? z[e] : 0.0f;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float by = MIXED && !(seen[rt] >> (16 * h) & 0xFu) ? 0.0f : rv[h];
                l_run[rt] = fmaf((z[4 * h] + z[4 * h + 1]) + (z[4 * h + 2] + z[4 * h + 3]), by, l_run[rt]);
            }
            if constexpr (AFTER) {
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] *= MIXED && !(seen[rt] >> (16 * (e / 4) + e % 4) & 1u) ? 0.0f : vsr[of(e)] * inv;
            }
            P[rt] = __builtin_convertvector(z, f16x8_t);
            if constexpr (F32) R[rt] = __builtin_convertvector(z - __builtin_convertvector(P[rt], f32x8_t), f16x8_t);
        }
        if (CODE == XKV_E4M3 && MIXED) {
            // Codes of V that are NaN reach the rows that see them, not the others: where there are any, the NaN of a channel that a row sees are
            // counted, a product of ones, and the codes become zeros.
            uint32_t odd = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int i = 0; i < VW; ++i) odd |= ((vr[e].x[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
            if (__ballot(odd != 0)) {
#pragma unroll
                for (int i = 0; i < VW; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u32x4_t ones;
#pragma unroll
                        for (int p = 0; p < 4; ++p)
                            ones[p] = ((vr[2 * p].x[i] >> (8 * j) & 0x7Fu) == 0x7Fu ? 0x3C00u : 0u) |
                                      ((vr[2 * p + 1].x[i] >> (8 * j) & 0x7Fu) == 0x7Fu ? 0x3C000000u : 0u);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            u32x4_t sees_it;
#pragma unroll
                            for (int p = 0; p < 4; ++p) {
                                const uint32_t two = seen[rt] >> (16 * (p / 2) + 2 * (p % 2));
                                sees_it[p] = (two & 1u ? 0x3C00u : 0u) | (two & 2u ? 0x3C000000u : 0u);
                            }
                            const f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, ones), __builtin_bit_cast(f16x8_t, sees_it),
                                                                                         f32x4_t(0.0f), 0, 0, 0);
#pragma unroll
                            for (int v = 0; v < 4; ++v) O[rt][4 * i + j][v] = count[v] > 0.0f ? __builtin_nanf("") : O[rt][4 * i + j][v];
                        }
                    }
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int i = 0; i < VW; ++i)
                        vr[e].x[i] &= ~(((((vr[e].x[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u);
            }
        }
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            f16x8_t vb[4];
            const uint32_t word[8] = {vr[0].x[i], vr[1].x[i], vr[2].x[i], vr[3].x[i], vr[4].x[i], vr[5].x[i], vr[6].x[i], vr[7].x[i]};
            codes_by_channel<CODE>(word, vb);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    f32x4_t &o = O[rt][4 * i + j];
                    if (F32) o = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb[j], R[rt], o, 0, 0, 0);
                    o = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb[j], P[rt], o, 0, 0, 0);
                }
        }
        if (next) request_v(t + STEP);
    };
    for (; t < u.t_end; t += STEP) {
        if (t + 32 <= least)
            tile(t, std::false_type{});
        else
            tile(t, std::true_type{});
    }

    // merge the wavefronts through LDS, 16 rows at a time: 16-byte piece p of row n16 sits at (p + n16) % PITCH; channel JC (4 kk + v) + j is
    // register v of O[j]
    const float undo = __uint_as_float((254u << 23) - __float_as_uint(inv));
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float lo, hi;
        quarters(l_run[rt], lo, hi);
        halves(lo + hi, lo, hi);
        if (rt > 0) __syncthreads();
        if (kk == 0) {
            sm_m[w][n16] = m_run[rt];
            sm_l[w][n16] = lo + hi;
        }
        __syncthreads();
        const float top = fmaxf(fmaxf(sm_m[0][n16], sm_m[1][n16]), fmaxf(sm_m[2][n16], sm_m[3][n16]));
        const float f = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - top) * undo;
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int j = 0; j < JC; j += 4)
                sm_o[w][PITCH * n16 + (((4 * kk + v) * JC + j) / 4 + n16) % PITCH] =
                    f32x4_t{f * O[rt][j][v], f * O[rt][j + 1][v], f * O[rt][j + 2][v], f * O[rt][j + 3][v]};
        __syncthreads();
        for (int item = (int)threadIdx.x; item < 16 * PITCH; item += 256) {
            const int row = item / PITCH, p = item % PITCH, m = (u.tile * RT + rt) * 16 + row;
            if (m >= M) continue;
            f32x4_t x = f32x4_t(0.0f);
            float den = 0.0f, most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x += sm_o[i][PITCH * row + (p + row) % PITCH];
                most = fmaxf(most, sm_m[i][row]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)  // (a wavefront without a maximum: 0, or NaN)
                den += sm_l[i][row] * (sm_m[i][row] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sm_m[i][row] - most));
            if (direct) {
                const bool none = visible8(a, u.seq, m / n_rep) == 0;
                T *out = (T *)a.out + (((size_t)u.seq * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep) * D + 4 * p;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = result<T>(none ? 0.0f : x[e] / den);
                continue;
            }
            const size_t slot = ((size_t)u.part * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep;
            *reinterpret_cast<f32x4_t *>(a.part_o + slot * D + 4 * p) = x;
            if (p == 0) {
                a.part_ml[2 * slot] = most;
                a.part_ml[2 * slot + 1] = den;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// The same for many rows, 128 channels: 32 rows a wavefront, eight of them to a workgroup, which share tiles of 64 rows of the cache.  Codes go from
// memory to LDS as they are, four tiles ahead, and are converted there once for all wavefronts, K to bf16 and V to fp16; V^T is read by
// the transposing LDS read.  The logits of a tile are multiplied beside the exponentials of the one before, so that the matrix cores and the
// vector units work at once; the tile after it is converted beside that one's second product.  Nothing in the loop waits for a load of
// its own: scales take the way of the codes (a load into a register would first have to wait for all tiles that are under way).
// 256 queries of 7 heads after 131072 rows (1792 rows a KV head): 508 us with the merge, 492 without, 0.95 PFLOP/s of 4 d flops a logit (a 8192^3 library product 1.2); logits and
// exponentials one after the other 631; codes and scales through registers 525; by 32 rows that share nothing 783.  With few rows a
// tile still takes 2.4 us, the latency of its steps: the streams are faster up to 128 rows.
// LDS: 16-byte piece p of row t of K sits at p ^ (t % 16), 32-byte piece u of V at u ^ (t % 8), so that neither the fragment reads (16
// rows at a time, one piece each) nor the transposing reads (4 rows at a time, two pieces each) meet in a bank.
// ------------------------------------------------------------------------------------------
template <int CODE>
__global__ __launch_bounds__(512, 2) void cache8_rows_kernel(Cache8Args a, bool direct)
{
    constexpr int D = 128, RT = 2, WAVES = 8, TILE = 64, KV = TILE * 2 * D, AHEAD = 4;  // bytes of a tile of K or V; tiles of codes under way
    __shared__ __attribute__((aligned(1024))) unsigned char smem[(5 + AHEAD) * KV];  // K, K, V, V, V, and codes of tiles that are under way (K and V)
    __shared__ float sm_scale[8][64];  // of tile i in i % 8: of K, four tokens each, of V, and both again
    __shared__ uint32_t sm_odd[4][2];  // of this tile, the next one, the one after it and one that is cleared
    const Unit8 u = same_in_all_lanes(unit8(a));
    const int lane = lane_id(), w = wave_id(), n16 = lane & 15, kk = lane >> 4, n_rep = a.H_q / a.H_kv, M = a.N * n_rep;
    if (!u.some && !direct) return;  // (the merge knows)
    if (u.t_begin >= u.t_end && !direct) return leave_nothing(a, u);
    const size_t head = (size_t)u.seq * a.H_kv + u.g;
    const uint8_t *K = a.K8 + head * a.L * D, *V = a.V8 + head * a.L * D;
    const float *ks = a.k_scales + head * a.n_c, *vs = a.v_scales + head * a.n_c, c = a.scale * kLog2e;

    // This thread's 16 codes of a tile, of row p_row, from channel 16 p on; they go straight to LDS, where only this wavefront reads them.
    // WHOLE: no row is behind the last one (those are the last one again).
    const int p_row = (int)threadIdx.x / 8, p = (int)threadIdx.x % 8;
    const uint32_t scale0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)&sm_scale[0][0];
    const uint32_t raw0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + 5 * KV + 1024 * w;
    const float *const scales = lane & 16 ? vs : ks;
    const int quad = 4 * (lane & 15);
    auto request = [&](int t, int i, auto whole) __attribute__((always_inline)) {  // tile i
        const int slot = i % AHEAD;
        if (w == i % 8) {  // (a load more than the others have makes its waits longer)
            const int last = u.t_end - 1 - t;
            copy4_to_lds(scales + ((t + (decltype(whole)::value || quad < last ? quad : last)) >> a.shift), scale0 + 256 * (i % 8));
        }
        uint32_t off = 16 * threadIdx.x;
        if constexpr (!decltype(whole)::value) {
            const int last = u.t_end - 1 - t;
            off = (p_row < last ? p_row : last) * D + 16 * p;
        }
        copy16_to_lds(K + (size_t)t * D, off, raw0 + KV * slot);
        copy16_to_lds(V + (size_t)t * D, off, raw0 + KV * slot + KV / 2);
    };
    constexpr std::true_type whole{};
    constexpr std::false_type any{};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (u.t_begin + i * TILE < u.t_end) request(u.t_begin + i * TILE, i, any);

    // Q^T operands: lane (row n16, kk), product s, position e: channel 32 s + 8 kk + e
    bf16x8_t Q[RT][4];
    int sees[RT], most = 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int m = ((u.tile * WAVES + w) * RT + rt) * 16 + n16, m_in = m < M ? m : M - 1, i = m_in / n_rep;
        const bf16_t *q = (const bf16_t *)a.q + (((size_t)u.seq * a.N + i) * a.H_q + u.g * n_rep + m_in % n_rep) * D;
        sees[rt] = visible8(a, u.seq, i);
        most = sees[rt] > most ? sees[rt] : most;
#pragma unroll
        for (int s = 0; s < 4; ++s) Q[rt][s] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(q + 32 * s + 8 * kk));
    }
    if (((u.tile * WAVES + w) * RT) * 16 >= M) most = 0;             // (no rows)
    most = __builtin_amdgcn_readfirstlane(wave_all(most, MaxOp()));  // rows of the cache that any of this wavefront's rows sees, ..
    int all = 0x7FFFFFFF;                                            // .. and all rows of the workgroup
    {
        int first, last;
        tile_queries(a, u.tile, first, last);
        for (int i = first + lane; i <= last; i += kWave) {
            const int n = visible8(a, u.seq, i);
            all = n < all ? n : all;
        }
        all = -wave_all(-all, MaxOp());
        all = __builtin_amdgcn_readfirstlane(all < u.t_end ? all : u.t_end);
    }
    if (threadIdx.x < 8) sm_odd[threadIdx.x / 2][threadIdx.x % 2] = 0u;
    __syncthreads();

    // Converted codes of a tile into LDS.  NaN among the values of a tile that rows see different tokens of become zeros, and their tokens are noted
    // (WHOLE: all see all).
    unsigned char *const to_k = smem + 256 * p_row + 16 * ((2 * p) ^ (p_row & 15)), *const to_v = smem + 2 * KV + 256 * p_row + 32 * (p ^ (p_row & 7));
    auto store = [&](int t, int i, int kbuf, int vbuf, auto whole) __attribute__((always_inline)) {
        // (requests are answered in order: those of the tiles behind this one may be under way, others in between make the wait longer)
        if (decltype(whole)::value || t + (AHEAD - 1) * TILE < u.t_end)
            XKV_WAIT_VMCNT(2 * (AHEAD - 1));
        else
            XKV_WAIT_VMCNT(0);
        asm volatile("" : : : "memory");
        const unsigned char *raw = smem + 5 * KV + KV * (i % AHEAD) + 16 * threadIdx.x;
        const u32x4_t kr = *reinterpret_cast<const u32x4_t *>(raw);
        u32x4_t vr = *reinterpret_cast<const u32x4_t *>(raw + KV / 2);
        *reinterpret_cast<bf16x8_t *>(to_k + KV * kbuf) = codes8<CODE>(kr[0], kr[1]);
        *reinterpret_cast<bf16x8_t *>(smem + ((uint32_t)(to_k - smem) ^ 16u) + KV * kbuf) = codes8<CODE>(kr[2], kr[3]);
        if (CODE == XKV_E4M3 && !decltype(whole)::value && t + TILE > all) {
            uint32_t odd = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t nan = (((vr[e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
                odd |= nan;
                vr[e] &= ~(nan * 255u);
            }
            if (odd) atomicOr(&sm_odd[i % 4][p_row >> 5], 1u << (p_row & 31));
        }
        *reinterpret_cast<f16x8_t *>(to_v + KV * vbuf) = values8<CODE>(vr[0], vr[1]);
        *reinterpret_cast<f16x8_t *>(to_v + KV * vbuf + 16) = values8<CODE>(vr[2], vr[3]);
    };

    // fragment f of K is at kat ^ (64 f), block of 16 channels db of V at vat ^ (32 db)
    const int rl = 4 * kk + (n16 >> 2);
    const uint32_t kat = 256 * n16 + 16 * (kk ^ n16), vat = 256 * rl + 32 * (rl & 7) + 8 * (lane & 3);
    f32x4_t O[RT][8];
    float m_run[RT], l_run[RT], inv = kFarUp;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) O[rt][j] = f32x4_t(0.0f);
    }
    float ksr[4], vsr[4];  // of tokens 16 h + 4 kk .. + 3 of a tile
    auto scales_of = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            ksr[h] = sm_scale[i % 8][4 * h + kk];
            vsr[h] = sm_scale[i % 8][16 + 4 * h + kk];
        }
    };

    f32x4_t S[RT][4];
    // Logits of tokens 16 h .. + 15.  What is read from LDS is requested a step before it is used, and stays before that step's arithmetic.
    bf16x8_t kf[2][4];
    auto keys = [&](int kbuf, int h) __attribute__((always_inline)) {
        const unsigned char *lds = smem + KV * kbuf + 4096 * h;
#pragma unroll
        for (int f = 0; f < 4; ++f) kf[h % 2][f] = *reinterpret_cast<const bf16x8_t *>(lds + (kat ^ (64u * f)));
    };
    auto logits = [&](int h) __attribute__((always_inline)) {
        f32x4_t x[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt] = f32x4_t(0.0f);
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) x[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[h % 2][f], Q[rt][f], x[rt], 0, 0, 0);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) S[rt][h] = x[rt];
    };

    // A tile, whose logits are there; those of the next one, if there is any, take their place.
    auto tile = [&](int t, int i, int kbuf, int vbuf, bool next, auto mixed, auto beside) __attribute__((always_inline)) {
        constexpr bool MIXED = decltype(mixed)::value;
        const unsigned char *lds = smem + KV * (2 + vbuf);
        if (next) keys(kbuf ^ 1, 0);
        float kc[4], largest = vsr[0];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            kc[h] = ksr[h] * c;
            largest = fmaxf(largest, vsr[h]);
        }
        uint64_t seen[RT];
        float top[RT];
        bool raise = !(largest * inv <= 128.0f);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (MIXED) {
                const int left = (sees[rt] < u.t_end ? sees[rt] : u.t_end) - t;
                seen[rt] = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1ull : 0ull;
                seen[rt] >>= 4 * kk;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    S[rt][e / 4][e % 4] = seen[rt] >> (16 * (e / 4) + e % 4) & 1u ? S[rt][e / 4][e % 4] * kc[e / 4] : -INFINITY;
            }
            float lo, hi, x = -INFINITY;
#pragma unroll
            for (int h = 0; h < 4; ++h) x = fmaxf(x, MIXED ? largest4(S[rt][h]) : largest4(S[rt][h]) * kc[h]);  // (scales are not negative)
            quarters(x, lo, hi);
            halves(fmaxf(lo, hi), lo, hi);
            top[rt] = fmaxf(lo, hi);
            raise |= !(top[rt] - m_run[rt] <= 8.0f);
        }
        if (__ballot(raise)) {
            largest = wave_all(largest, MaxOp());  // (NaN is passed over)
            float less = 1.0f;
            if (largest * inv > 128.0f && largest < INFINITY) {
                const float now = __uint_as_float((254u + 6u - (__float_as_uint(largest) >> 23 & 0xFFu)) << 23);  // 2^6 by its power of two
                less = now * __uint_as_float((254u << 23) - __float_as_uint(inv));                                 // (inv is a power of two)
                inv = now;
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float m_new = fmaxf(m_run[rt], top[rt]), alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
                l_run[rt] *= alpha;
#pragma unroll
                for (int j = 0; j < 8; ++j) O[rt][j] *= alpha * less;
                m_run[rt] = m_new;
            }
        }
        f16x8_t P[RT][2];
        auto weights = [&](int h) __attribute__((always_inline)) {  // of tokens 16 h .. + 15
            const float v = vsr[h] * inv < kLeast ? kLeast : vsr[h] * inv;  // (NaN stays)
            const float lv = __builtin_amdgcn_logf(v), rv = __builtin_amdgcn_rcpf(v);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float add = lv - (m_run[rt] == -INFINITY ? 0.0f : m_run[rt]);
                f32x4_t z;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = __builtin_amdgcn_exp2f(MIXED ? S[rt][h][e] + add : fmaf(S[rt][h][e], kc[h], add));
                    if (MIXED) z[e] = seen[rt] >> (16 * h + e) & 1u ? z[e] : 0.0f;  // (a scale that is not seen may be NaN)
                }
                const float by = MIXED && !(seen[rt] >> (16 * h) & 0xFu) ? 0.0f : rv;
                l_run[rt] = fmaf((z[0] + z[1]) + (z[2] + z[3]), by, l_run[rt]);
#pragma unroll
                for (int e = 0; e < 4; ++e) P[rt][h / 2][4 * (h % 2) + e] = (_Float16)z[e];
            }
        };
        if (next) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (h < 3) keys(kbuf ^ 1, h + 1);
                __builtin_amdgcn_sched_barrier(0);
                weights(h);
                logits(h);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h) weights(h);
        }
        f16x8_t v[3][2];
        auto values = [&](int db) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                // position e of lane (channel, kk): token 32 k + 16 (e / 4) + 4 kk + e % 4, as in P
                const unsigned char *from = lds + (vat ^ (32u * db)) + 8192 * k;
                const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)from);
                const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(from + 4096));
                v[db % 3][k] = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        values(0);
        values(1);
        beside();
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            if (db < 6) values(db + 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[rt][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[db % 3][k], P[rt][k], O[rt][db], 0, 0, 0);
        }
        if (CODE == XKV_E4M3 && MIXED) {  // NaN of noted tokens to the rows that see them
            for (int x = 0; x < 2; ++x)
                for (uint32_t bits = __builtin_amdgcn_readfirstlane(sm_odd[i % 4][x]); bits; bits &= bits - 1) {
                    const int j = t + 32 * x + __builtin_ctz(bits);
                    const uint8_t *v = V + (size_t)(j < u.t_end ? j : u.t_end - 1) * D + 4 * kk;
#pragma unroll
                    for (int db = 0; db < 8; ++db)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool nan = (v[16 * db + e] & 0x7F) == 0x7F;
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) O[rt][db][e] = nan && j < sees[rt] && j < u.t_end ? __builtin_nanf("") : O[rt][db][e];
                        }
                }
        }
    };

    // Tile i of this part: its codes in i % AHEAD, converted ones in i % 2 (K) and i % 3 (V), scales in i % 8, notes in i % 4.
    auto convert = [&](int t, int i, int kbuf, int vbuf) __attribute__((always_inline)) {
        if (t >= u.t_end) return;
        store(t, i, kbuf, vbuf, any);
        wait_lds();
        if (t + AHEAD * TILE < u.t_end) request(t + AHEAD * TILE, i + AHEAD, any);
    };
    convert(u.t_begin, 0, 0, 0);
    lds_barrier();
    convert(u.t_begin + TILE, 1, 1, 1);
    if (u.t_begin < u.t_end) {
        scales_of(0);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            keys(0, h);
            logits(h);
        }
    }
    lds_barrier();
    int kbuf = 0, vbuf = 0, i = 0, t = u.t_begin;
    auto then = [&]() __attribute__((always_inline)) {
        lds_barrier();
        kbuf ^= 1;
        vbuf = vbuf < 2 ? vbuf + 1 : 0;
        ++i;
    };
    for (; t + (AHEAD + 3) * TILE <= all; t += TILE) {  // all rows see all of the tiles that are dealt with here
        tile(t, i, kbuf, vbuf, true, std::false_type{}, [&]() __attribute__((always_inline)) {
            scales_of(i + 1);
            store(t + 2 * TILE, i + 2, kbuf, vbuf > 0 ? vbuf - 1 : 2, whole);
            wait_lds();
            request(t + (2 + AHEAD) * TILE, i + 2 + AHEAD, whole);
        });
        then();
    }
    for (; t < u.t_end; t += TILE) {
        if (CODE == XKV_E4M3 && threadIdx.x < 2) sm_odd[(i + 3) % 4][threadIdx.x] = 0u;  // (read before the last barrier, written after the next)
        auto beside = [&]() __attribute__((always_inline)) {
            scales_of(i + 1);
            convert(t + 2 * TILE, i + 2, kbuf, vbuf > 0 ? vbuf - 1 : 2);
        };
        if (t < most)
            tile(t, i, kbuf, vbuf, t + TILE < u.t_end, std::true_type{}, beside);
        else  // (nor do its rows see anything further)
            beside();
        then();
    }

    const float undo = __uint_as_float((254u << 23) - __float_as_uint(inv));
    float den[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float lo, hi;
        quarters(l_run[rt], lo, hi);
        halves(lo + hi, lo, hi);
        den[rt] = lo + hi;
#pragma unroll
        for (int db = 0; db < 8; ++db) O[rt][db] *= undo;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int m = ((u.tile * WAVES + w) * RT + rt) * 16 + n16;
        if (m >= M) continue;
        const size_t row = ((size_t)(direct ? u.seq : u.part) * a.N + m / n_rep) * a.H_q + u.g * n_rep + m % n_rep;
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            if (direct) {
                typedef __attribute__((ext_vector_type(4))) uint16_t u16x4_t;
                u16x4_t x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = result<bf16_t>(sees[rt] == 0 ? 0.0f : O[rt][db][e] / den[rt]);
                __builtin_memcpy((bf16_t *)a.out + row * D + 16 * db + 4 * kk, &x, sizeof x);  // (wherever `out` lies)
            } else {
                *reinterpret_cast<f32x4_t *>(a.part_o + row * D + 16 * db + 4 * kk) = O[rt][db];
            }
        }
        if (!direct && kk == 0) {
            a.part_ml[2 * row] = m_run[rt];
            a.part_ml[2 * row + 1] = den[rt];
        }
    }
}

// ------------------------------------------------------------------------------------------
// Merge.  A group of 2^lg lanes covers the columns of a row (query, head), VEC a lane.  Where there are many rows, a group per row; where there are few,
// the groups of a workgroup share a row's partials and are added up in LDS: latency is all there is to it then, and the first partials are
// requested before their weights are known.  Partials of parts that have no rows were not written and do not count; all others do, also with a
// weight of zero: a NaN among a row's values is in its output alone, however little the part weighs.  64 parts of 32 rows 4.4 us, most of
// it a launch's own time; a group per row there 9.
// ------------------------------------------------------------------------------------------
template <typename T, int VEC>
__global__ __launch_bounds__(256) void cache8_merge_kernel(Cache8Args a, int lg, int share, int rows)
{
    typedef __attribute__((ext_vector_type(VEC))) float vec_t;
    constexpr int BATCH = 8;
    __shared__ vec_t sm[256];
    __shared__ float sm_w[32][kMaxCacheParts];
    const int width = 1 << lg, l = (int)threadIdx.x & (width - 1), grp = (int)threadIdx.x >> lg, groups = 256 >> lg;
    const int col = ((int)blockIdx.y * width + l) * VEC;
    const int item = share ? (int)blockIdx.x : (int)blockIdx.x * groups + grp, row = item < rows ? item : rows - 1;
    const int n_rep = a.H_q / a.H_kv, head = row % a.H_q, i = row / a.H_q % a.N, seq = row / a.H_q / a.N;
    int first, parts;
    if (a.by_length) {
        first = a.table[seq];
        parts = a.table[seq + 1] - first;
    } else {
        int lo, hi, n = 0;
        tile_queries(a, (i * n_rep + head % n_rep) / a.rows, lo, hi);
        for (int j = lo + l; j <= hi; j += width) n = MaxOp()(n, visible8(a, seq, j));
        for (int off = 1; off < width; off <<= 1) n = MaxOp()(n, __shfl_xor(n, off, kWave));
        first = seq * a.parts;
        parts = ceil_div_dev(n, tile_chunk(a, n));
    }
    const bool none = visible8(a, seq, i) == 0;  // (the logits of all that a row sees may be -inf: 0 / 0; a NaN among them is in its sum)
    const size_t stride = (size_t)a.N * a.H_q, at = first * stride + (size_t)i * a.H_q + head;
    const float *ml = a.part_ml + 2 * at, *po = a.part_o + at * a.d_h + (col < a.d_h ? col : 0);
    const int step = share ? groups : 1, begin = share ? grp : 0;
    vec_t v[BATCH];
    auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = s0 + u * step < parts ? s0 + u * step : 0;
            v[u] = parts > 0 ? *reinterpret_cast<const vec_t *>(po + (size_t)s * stride * a.d_h) : vec_t(0.0f);
        }
    };
    request(begin);
    float m = -INFINITY, den = 0.0f;
    for (int s = l; s < parts; s += width) m = fmaxf(m, ml[2 * s * stride]);
    for (int off = 1; off < width; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    for (int s = l; s < parts; s += width) {
        const float top = ml[2 * s * stride], sum = ml[2 * s * stride + 1], wt = top == -INFINITY ? 0.0f : exp2f(top - m);
        const bool left = sum < 0.0f;  // (nothing)
        sm_w[grp][s] = left ? -1.0f : wt;
        den = left ? den : fmaf(top == -INFINITY ? 1.0f : wt, sum, den);  // (a part without a maximum: 0, or NaN)
    }
    for (int off = 1; off < width; off <<= 1) den += __shfl_xor(den, off, kWave);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // (a group is part of a wavefront)
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    vec_t acc = vec_t(0.0f);
    for (int s0 = begin; s0 < parts; s0 += BATCH * step) {
        if (s0 > begin) request(s0);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = s0 + u * step;
            const float wt = s < parts ? sm_w[grp][s] : -1.0f;
            acc += wt < 0.0f ? vec_t(0.0f) : wt * v[u];
        }
    }
    if (share) {
        sm[threadIdx.x] = acc;
        __syncthreads();
        if (grp > 0) return;
        for (int k = 1; k < groups; ++k) acc += sm[(k << lg) + l];
    }
    if (item >= rows || col >= a.d_h) return;
    T *out = (T *)a.out + (size_t)row * a.d_h + col;
#pragma unroll
    for (int e = 0; e < VEC; ++e) out[e] = result<T>(none ? 0.0f : acc[e] / den);
}

template <typename T>
hipError_t launch_merge(const Cache8Args &a, hipStream_t st)
{
    const int vec = a.d_h % 4 == 0 ? 4 : 1, rows = a.batch * a.N * a.H_q;
    int lg = 3;
    while (lg < 6 && (vec << lg) < a.d_h) ++lg;
    const int share = rows < 2048, groups = 256 >> lg;
    const dim3 grid(share ? rows : (rows + groups - 1) / groups, (a.d_h + (vec << lg) - 1) / (vec << lg));
    if (vec == 4)
        hipLaunchKernelGGL((cache8_merge_kernel<T, 4>), grid, dim3(256), 0, st, a, lg, share, rows);
    else
        hipLaunchKernelGGL((cache8_merge_kernel<T, 1>), grid, dim3(256), 0, st, a, lg, share, rows);
    return hipGetLastError();
}

dim3 unit_grid(const Cache8Args &a)
{
    const int M = a.N * (a.H_q / a.H_kv);
    return dim3((unsigned)a.parts * a.H_kv * ((M + a.rows - 1) / a.rows) * (a.by_length ? 1u : (unsigned)a.batch));
}

template <typename T, int CODE>
hipError_t launch_general(const Cache8Args &a, bool direct, hipStream_t st)
{
    const size_t lds = (2 * (size_t)kGenTokens * general_pitch(a.d_h) + (size_t)kGenRows * ((a.d_h + 3) / 4 * 4) + 4 * 4 * kGenTokens) * sizeof(float);
    auto launch = [&](auto kernel, DynamicLdsOnce &attr) {
        const hipError_t e = attr.ensure((const void *)kernel, 150 * 1024);  // (what 256 channels take)
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, unit_grid(a), dim3(256), lds, st, a, direct);
        return hipGetLastError();
    };
    static DynamicLdsOnce attr[3];
    return a.d_h <= 64 ? launch(cache8_general_kernel<T, CODE, 1>, attr[0])
         : a.d_h <= 128 ? launch(cache8_general_kernel<T, CODE, 2>, attr[1]) : launch(cache8_general_kernel<T, CODE, 4>, attr[2]);
}

template <typename T, int CODE, int D>
hipError_t launch_mfma(const Cache8Args &a, bool direct, hipStream_t st)
{
    auto launch = [&](auto kernel, int threads = 256) {
        hipLaunchKernelGGL(kernel, unit_grid(a), dim3(threads), 0, st, a, direct);
        return hipGetLastError();
    };
    const bool once = a.rows >= a.N * (a.H_q / a.H_kv);
    if (a.shift < 2) return launch(cache8_mfma_kernel<T, CODE, D, 1, false, true>);
    if (a.rows == 16) return once ? launch(cache8_mfma_kernel<T, CODE, D, 1, true, false>) : launch(cache8_mfma_kernel<T, CODE, D, 1, false, false>);
    if constexpr (sizeof(T) == 2 && D < 256) {
        if (a.rows == 32) return once ? launch(cache8_mfma_kernel<T, CODE, D, 2, true, false>) : launch(cache8_mfma_kernel<T, CODE, D, 2, false, false>);
        if constexpr (D == 128) return launch(cache8_rows_kernel<CODE>, 512);
    }
    return hipErrorInvalidValue;
}

template <typename T, int CODE>
hipError_t launch_of(Cache8Args a, bool matrix, bool direct, hipStream_t st)
{
    if (matrix)
        return a.d_h == 64 ? launch_mfma<T, CODE, 64>(a, direct, st) : a.d_h == 128 ? launch_mfma<T, CODE, 128>(a, direct, st)
                                                                                     : launch_mfma<T, CODE, 256>(a, direct, st);
    return launch_general<T, CODE>(a, direct, st);
}

}  // namespace

hipError_t launch_cache8_attend(const xkv_shape &s, const Cache8Args &given, int code, bool mfma, hipStream_t st)
{
    Cache8Args a = given;
    const bool matrix = mfma && ((uintptr_t)a.K8 | (uintptr_t)a.V8 | (uintptr_t)a.q) % 16 == 0;
    const bool direct = !a.part_o;
    if (!matrix || a.shift < 2) a.rows = kGenRows;  // (.. of the plan's 16, 32 or 256; its rounds divide the plan's)
    const hipError_t e = s.dtype == XKV_F32 ? code == XKV_E4M3 ? launch_of<float, XKV_E4M3>(a, matrix, direct, st) : launch_of<float, XKV_INT8>(a, matrix, direct, st)
                       : code == XKV_E4M3   ? launch_of<bf16_t, XKV_E4M3>(a, matrix, direct, st)
                                            : launch_of<bf16_t, XKV_INT8>(a, matrix, direct, st);
    if (e != hipSuccess || direct) return e;
    return s.dtype == XKV_F32 ? launch_merge<float>(a, st) : launch_merge<bf16_t>(a, st);
}

}  // namespace xkv
