// Attention over an uncompressed cache: trees of drafted tokens, one token whose weights are kept, selected blocks (cache.h).
//   z_t = scale <q, k_t>,  out = sum_t exp(z_t - max) v_t / sum_t exp(z_t - max)
// over the tokens that the query sees, split over the tokens: every workgroup leaves (maximum, sum, unnormalised output) of its
// part, and a second kernel merges them.
#include <type_traits>

#include "cache_tile.h"

namespace xkv {
namespace {

using namespace cache_tile;

constexpr int kGenTokens = 64;  // tokens a round of the general kernel, a lane each
constexpr int kGenRows = 16;    // its rows (query token, head) per workgroup, four per wavefront

// Bits of the drafted tokens 32 k .. 32 k + 31 that `token` of a sequence sees; k < 0: rows of the cache, all of them.
__device__ __forceinline__ uint32_t draft_word(const CacheArgs &a, int seq, int token, int k)
{
    uint32_t x;
    if (a.tree) {  // (the same in every lane)
        const int kc = k < 0 ? 0 : k < a.words ? k : a.words - 1;
        x = a.tree[((size_t)seq * a.N + token) * a.words + kc];
    } else {
        const int up = token - 32 * k;
        x = up >= 31 ? 0xFFFFFFFFu : up >= 0 ? (2u << up) - 1u : 0u;
    }
    return k < 0 ? 0xFFFFFFFFu : k < a.words ? x : 0u;
}

// The same for the 32 places from drafted token j on (j < 0: they begin in the cache).
__device__ __forceinline__ uint32_t draft_bits(const CacheArgs &a, int seq, int token, int j)
{
    const uint32_t lo = draft_word(a, seq, token, j >> 5), hi = draft_word(a, seq, token, (j >> 5) + 1);
    return (uint32_t)(((uint64_t)hi << 32 | lo) >> (j & 31));
}

// ------------------------------------------------------------------------------------------
// General path, any type, width and alignment.  A round takes 64 tokens, whose keys and values go to LDS in single precision (the
// next round's are requested before this one is computed).  For the logits a lane multiplies one of the keys with the four queries
// of its wavefront, four channels a time; for the sums lanes run over the channels, and the weights go through LDS.  With few rows its time
// is that of one round, latencies: 8 drafted tokens of 4 heads after 512 tokens, fp32, 9.1 us.  Long caches are far from their bytes: 32768 tokens
// of 8 KV heads with 4 query heads, one token, fp32 x 64 72 us (26 at the rate of a copy), x 128 107 (53), bf16 x 64 67 (13), x 256 296 (53).
// ------------------------------------------------------------------------------------------
__host__ __device__ inline int general_pitch(int d) { return ((d + 3) / 4 | 1) * 4; }  // floats; an odd number of 16-byte pieces

template <typename T, CacheMode MODE, int JP>
__global__ __launch_bounds__(256) void cache_attend_general_kernel(CacheArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float smem_f[];
    constexpr int PER_WAVE = kGenTokens / 4;
    const int lane = lane_id(), w = wave_id(), n_rep = a.H_q / a.H_kv, d = a.d_h, d4 = (d + 3) / 4 * 4, pitch = general_pitch(d);
    const int M = MODE == CacheMode::blocks ? n_rep : a.N * n_rep;
    const CacheUnit u = cache_unit(a, MODE, (M + kGenRows - 1) / kGenRows);
    if (!u.some) return;  // (the merge knows)
    const int tile = u.tile, g = u.g, n = u.n, t_begin = u.t_begin, t_end = u.t_end;
    // blocks: one query token; else all query tokens of a sequence
    const int seq = MODE == CacheMode::blocks ? u.seq / a.N : u.seq, first_token = MODE == CacheMode::blocks ? u.seq % a.N : 0;
    float *kt = smem_f, *vt = kt + kGenTokens * pitch, *qs = vt + kGenTokens * pitch, *ps = qs + kGenRows * d4;

    const T *Kg = (const T *)a.K + ((size_t)seq * a.H_kv + g) * a.L * d, *Vg = (const T *)a.V + ((size_t)seq * a.H_kv + g) * a.L * d;
    const T *Kd = (const T *)a.K_draft + ((size_t)seq * a.H_kv + g) * a.N * d, *Vd = (const T *)a.V_draft + ((size_t)seq * a.H_kv + g) * a.N * d;
    const int32_t *sel = MODE == CacheMode::blocks ? a.sel + ((size_t)u.seq * a.H_kv + g) * a.k_ch : nullptr;

    // The row of this lane's token of a round (beyond the last one: that one again); drafted tokens are rows L, L + 1, ..
    auto row_of = [&](int t0) __attribute__((always_inline)) {
        const int t = t0 + lane < t_end ? t0 + lane : t_end - 1;
        if (MODE == CacheMode::blocks) return sel[t / a.c] * a.c + t % a.c;
        return MODE == CacheMode::tree && t >= n ? a.L + t - n : t;
    };
    T kr[PER_WAVE][JP], vr[PER_WAVE][JP];
    auto request = [&](int row) __attribute__((always_inline)) {  // tokens w, w + 4, .. of a round
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int rw = __builtin_amdgcn_readlane(row, 4 * i + w);
            const bool draft = MODE == CacheMode::tree && rw >= a.L;
            const T *k = draft ? Kd + (size_t)(rw - a.L) * d : Kg + (size_t)rw * d, *v = draft ? Vd + (size_t)(rw - a.L) * d : Vg + (size_t)rw * d;
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) {
                const int j = lane + jj * kWave, jc = j < d ? j : 0;
                kr[i][jj] = k[jc];
                vr[i][jj] = v[jc];
            }
        }
    };
    request(row_of(t_begin));

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
            if (j < d4) qs[(4 * w + r) * d4 + j] = j < d ? to_f32(((const T *)a.q)[row_id[r] * d + j]) : 0.0f;
        }
    }
    for (int t0 = t_begin; t0 < t_end; t0 += kGenTokens) {
        const int t = t0 + lane < t_end ? t0 + lane : t_end - 1;
        const bool real = t0 + lane < t_end;
        const bool mixed = MODE == CacheMode::tree && t0 + kGenTokens > n;  // rows see different tokens of this round
        uint32_t bits[4] = {1u, 1u, 1u, 1u};                                  // whether the rows see this lane's token (requested here, used after the logits)
        if (mixed) {
#pragma unroll
            for (int r = 0; r < 4; ++r) bits[r] = draft_bits(a, seq, token[r], t - n);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i)
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) {
                const int j = lane + jj * kWave;
                if (j < d4) {
                    kt[(4 * i + w) * pitch + j] = j < d ? to_f32(kr[i][jj]) : 0.0f;
                    vt[(4 * i + w) * pitch + j] = t0 + 4 * i + w < t_end ? to_f32(vr[i][jj]) : 0.0f;
                }
            }
        __syncthreads();
        if (t0 + kGenTokens < t_end) request(row_of(t0 + kGenTokens));
        float p[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int j = 0; j < d4; j += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(kt + lane * pitch + j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float4 y = *reinterpret_cast<const float4 *>(qs + (4 * w + r) * d4 + j);
                p[r] = fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, p[r]))));
            }
        }
        float z[4], top[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            z[r] = a.scale * p[r];
            if (MODE == CacheMode::weights && real && m0 + r < M) a.logits[row_id[r] * a.L + t] = z[r];
            if (!real) z[r] = -INFINITY;
        }
        if (MODE == CacheMode::tree) {
#pragma unroll
            for (int r = 0; r < 4; ++r) z[r] = bits[r] & 1u ? z[r] : -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) top[r] = wave_all(z[r], MaxOp());
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float m_new = fmaxf(mx[r], top[r]);
            const float alpha = m_new == -INFINITY ? 1.0f : expf(mx[r] - m_new);
            p[r] = z[r] == -INFINITY ? 0.0f : expf(z[r] - m_new);
            den[r] = den[r] * alpha + wave_all(p[r], AddOp());
            mx[r] = m_new;
#pragma unroll
            for (int jj = 0; jj < JP; ++jj) o[r][jj] *= alpha;
        }
        if (mixed) {
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = bits[r] & 1u ? p[r] : -0.0f;  // (weights are not negative: hidden from this row)
        }
        // the four weights of a token to every lane
        *reinterpret_cast<float4 *>(ps + 4 * (64 * w + lane)) = float4{p[0], p[1], p[2], p[3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int count = t_end - t0 < kGenTokens ? t_end - t0 : kGenTokens;
        auto add_values = [&](auto take) __attribute__((always_inline)) {
            for (int i0 = 0; i0 < count; i0 += 8) {  // (places from `count` on hold zeros)
                float v[8][JP];
                float4 y[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    y[x] = *reinterpret_cast<const float4 *>(ps + 4 * (64 * w + i0 + x));
#pragma unroll
                    for (int jj = 0; jj < JP; ++jj) {
                        const int j = lane + jj * kWave;
                        v[x][jj] = vt[(i0 + x) * pitch + (j < d ? j : 0)];
                    }
                }
#pragma unroll
                for (int x = 0; x < 8; ++x)
#pragma unroll
                    for (int jj = 0; jj < JP; ++jj) {
                        o[0][jj] = fmaf(y[x].x, take(y[x].x, v[x][jj]), o[0][jj]);
                        o[1][jj] = fmaf(y[x].y, take(y[x].y, v[x][jj]), o[1][jj]);
                        o[2][jj] = fmaf(y[x].z, take(y[x].z, v[x][jj]), o[2][jj]);
                        o[3][jj] = fmaf(y[x].w, take(y[x].w, v[x][jj]), o[3][jj]);
                    }
            }
        };
        // what a row does not see is not multiplied by zero: it may be padding with anything in it, or other rows' infinities
        if (mixed)
            add_values([](float weight, float value) { return __float_as_uint(weight) == 0x80000000u ? 0.0f : value; });
        else
            add_values([](float, float value) { return value; });
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (m0 + r >= M) break;
        const size_t slot = part_row(a, MODE, u.part, token[r], g * n_rep + (m0 + r) % n_rep);
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
// Matrix-core path: bf16, 128 channels.  A workgroup has WR x WT wavefronts: WR groups of 32 rows (query token, head), WT groups of
// tokens.  Tiles of 32 SUB WT tokens of K and V go from memory straight to LDS, two of them in turn; all row groups read them, or, where
// there is one, every wavefront its own part alone, without barriers:
//   S^T [tokens x rows] = K tile x Q^T (registers),  P^T = exp2(c S^T - c m),  O^T [channels x rows] += V^T x P^T
// A lane holds one row of S^T, P^T and O^T: the softmax statistics are its own (with the lane 32 further), rescaling needs no exchange, and
// P^T is the second product's operand as it comes.  V^T is read from its tile by the transposing LDS read.
// The maximum m is only raised when a row's logits outgrow it by a factor of 2^8: until then weights reach 2^8, sums stay exact to
// single precision, and the accumulators need not be rescaled.
// Weights are operands of two products, their upper 16 bits and what is left of them rounded to bf16, so that they keep 2^-15: the error
// against 64 bits is the output's rounding alone, 0.0017 of the results' root mean square (0.0023 with weights rounded to bf16).  What the
// second product costs: up to 16 rows nothing, the stream covers it; 64 rows after 32768 tokens 34.6 -> 36.0 us; 256 rows of four sequences
// of 16K to 64K 193 -> 258, 231 rows 62 -> 76, where the matrix cores bound it.  Logits, statistics and sums are fp32.
// LDS: row t of a tile is 256 B; its 16-byte piece p of K sits at (p + t) % 16, its 32-byte piece u of V at (u + 2 t) % 8, so
// that neither the fragment reads (16 rows at a time, one piece each) nor the transposing reads (4 rows at a time, two pieces each)
// meet in a bank.
// ------------------------------------------------------------------------------------------
__device__ const u32x4_t kZeroRow[16] = {};  // stands for drafted tokens that nothing sees, and for places behind the last token

// Rows see different drafted tokens, but a product with the values takes all of them, with weight zero where they are hidden: infinities and
// NaN must not be among them.  A wavefront that has received rows of values of drafted tokens sets such values to zero where they lie in LDS
// and notes the tokens; when rows leave, they are added to those that see them.  (Without any it is a look at the last tiles.)
//   clear_odd: 4 LOADS rows at `at` (this lane's 16 bytes of the first four), those from `skip` on -> a bit for each row that had some
template <int LOADS> __device__ __forceinline__ uint32_t clear_odd(unsigned char *at, int skip)
{
    uint32_t rows = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        u32x4_t x = *reinterpret_cast<const u32x4_t *>(at + 1024 * i);
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool lo = (x[e] & 0x7F80u) == 0x7F80u, hi = (x[e] & 0x7F800000u) == 0x7F800000u;
            x[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
            odd |= lo || hi;
        }
        odd &= 4 * i + (lane_id() >> 4) >= skip;
        const uint64_t m = __ballot(odd);
        if (m == 0) continue;
        if (odd) *reinterpret_cast<u32x4_t *>(at + 1024 * i) = x;
#pragma unroll
        for (int r = 0; r < 4; ++r) rows |= (m >> (16 * r) & 0xFFFFu) ? 1u << (4 * i + r) : 0u;
    }
    return rows;
}
// bit i of rows: drafted token j + i (j may be negative, such bits are not set), in all wavefronts' notes
__device__ __forceinline__ void note_odd(uint32_t *notes, uint32_t rows, int j)
{
    if (rows == 0 || lane_id() != 0) return;
    const uint64_t bits = j < 0 ? rows >> -j : (uint64_t)rows << (j & 31);
    const int k = j < 0 ? 0 : j >> 5;
    if ((uint32_t)bits) atomicOr(&notes[k], (uint32_t)bits);
    if (bits >> 32) atomicOr(&notes[k + 1], (uint32_t)(bits >> 32));
}
__device__ __forceinline__ f32x4_t add_odd(const CacheArgs &a, const uint32_t *notes, const bf16_t *values, int seq, int token, int channel, f32x4_t x)
{
    for (int k = 0; k < a.words; ++k)
        for (uint32_t bits = notes[k] & draft_word(a, seq, token, k); bits; bits &= bits - 1) {
            const bf16_t *v = values + (size_t)(32 * k + __builtin_ctz(bits)) * 128 + channel;
            for (int e = 0; e < 4; ++e)
                if ((v[e] & 0x7F80) == 0x7F80) x[e] += bf16_to_f32(v[e]);
        }
    return x;
}

template <int WR, int WT, int SUB, int RT>
__global__ __launch_bounds__(64 * WR * WT, WR == 1 ? 1 : 2) void cache_tree_kernel(CacheArgs a)
{
    constexpr CacheMode MODE = CacheMode::tree;
    constexpr bool OWN = WR == 1;  // tiles that only one wavefront reads
    constexpr int WAVES = WR * WT, TILE = 32 * SUB * WT, STAGE = 512 * TILE, RPW = TILE / WAVES, LOADS = RPW / 4, KTILE = OWN ? 8192 : 256 * TILE, VBASE = OWN ? KTILE : 2 * KTILE;
    static_assert(!OWN || SUB == 1, "a wavefront's tile is 32 tokens");
    static_assert(RPW % 8 == 0, "rotations by i");
    constexpr int MERGE = WAVES * RT * 16384;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE >= MERGE ? 2 * STAGE : MERGE];
    __shared__ float sm_m[WT][32 * WR * RT], sm_l[WT][32 * WR * RT];
    __shared__ uint32_t sm_seen[32], sm_odd[32], sm_slot[32 * WR * RT];
    const int lane = lane_id(), w = wave_id(), rg = w % WR, tg = w / WR, n32 = lane & 31, hf = lane >> 5, n_rep = a.H_q / a.H_kv;
    const int M = a.N * n_rep;
    const CacheUnit u = cache_unit(a, MODE, (M + 32 * WR * RT - 1) / (32 * WR * RT));
    if (!u.some) return;  // (the merge knows)
    const int tile = u.tile, g = u.g, n = u.n, t_begin = u.t_begin, t_end = u.t_end;
    const int seq = u.seq;
    const float c = a.scale * 1.44269504088896340736f;

    const bf16_t *Kg = (const bf16_t *)a.K + ((size_t)seq * a.H_kv + g) * a.L * 128, *Vg = (const bf16_t *)a.V + ((size_t)seq * a.H_kv + g) * a.L * 128;
    const bf16_t *Kd = (const bf16_t *)a.K_draft + ((size_t)seq * a.H_kv + g) * a.N * 128;
    const bf16_t *Vd = (const bf16_t *)a.V_draft + ((size_t)seq * a.H_kv + g) * a.N * 128;

    // Q^T fragments: lane (row n32, hf), fragment f, position e: channel 16 f + 8 hf + e
    int m_row[RT], token[RT];
    bf16x8_t Qf[RT][8];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_row[rt] = ((tile * WR + rg) * RT + rt) * 32 + n32;
        const int m_in = m_row[rt] < M ? m_row[rt] : M - 1;
        token[rt] = m_in / n_rep;
        const size_t q_row = ((size_t)seq * a.N + token[rt]) * a.H_q + g * n_rep + m_in % n_rep;
#pragma unroll
        for (int f = 0; f < 8; ++f)
            Qf[rt][f] = __builtin_bit_cast(bf16x8_t, reinterpret_cast<const u32x4_t *>((const bf16_t *)a.q + q_row * 128)[2 * f + hf]);
    }

    if (t_end > n) {  // which drafted tokens any token sees
        if (threadIdx.x < 32) sm_seen[threadIdx.x] = a.tree ? 0u : 0xFFFFFFFFu, sm_odd[threadIdx.x] = 0u;
        __syncthreads();
        if (a.tree)
            for (int i = threadIdx.x; i < a.N * a.words; i += 64 * WAVES) {
                const uint32_t x = a.tree[(size_t)seq * a.N * a.words + i];
                if (x) atomicOr(&sm_seen[i % a.words], x);
            }
        __syncthreads();
    }

    // Where this wavefront puts rows: its share of a tile that all read (WR > 1), or tiles of 32 rows of its own.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + (OWN ? 32768 * w : 256 * RPW * w);
    const int r4 = lane >> 4, x16 = lane & 15;
    uint32_t koff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) koff[i] = 256 * r4 + 16 * ((x16 - (OWN ? 0 : RPW * w) - 4 * i - r4) & 15);
    const uint32_t voff = 256 * r4 + 32 * (((x16 >> 1) - 2 * r4) & 7) + 16 * (x16 & 1);
    const int plain_end = n < t_end ? n : t_end;  // rows of the cache end here
    auto stage_plain = [&](int first, int buf, auto values) __attribute__((always_inline)) {  // RPW rows of the cache
        constexpr bool is_v = decltype(values)::value;
        const uint32_t at = lds0 + buf * (OWN ? 2 * KTILE : KTILE) + (is_v ? VBASE : 0);
        const unsigned char *base = (const unsigned char *)((is_v ? Vg : Kg) + (size_t)first * 128);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (OWN)
                copy16_to_lds_once(base + 1024 * i, is_v ? voff : koff[i & 3], at + 1024 * i);
            else
                copy16_to_lds(base + 1024 * i, is_v ? voff : koff[i & 3], at + 1024 * i);
        }
    };
    auto stage = [&](int first, int buf, auto values) __attribute__((always_inline)) {  // RPW tokens from `first` on
        constexpr bool is_v = decltype(values)::value;
        const uint32_t at = lds0 + buf * (OWN ? 2 * KTILE : KTILE) + (is_v ? VBASE : 0);
        const bf16_t *rows = is_v ? Vg : Kg;
        if (first + RPW <= plain_end) {  // (wave-uniform)
            stage_plain(first, buf, values);
            return;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int t = first + 4 * i + r4, j = t - n;
            const bool draft = t < t_end && j >= 0 && (sm_seen[(j >> 5) & 31] >> (j & 31) & 1u);
            const bf16_t *from = t < n ? rows + (size_t)t * 128 : draft ? (is_v ? Vd : Kd) + (size_t)j * 128 : (const bf16_t *)kZeroRow;
            copy16_global_to_lds((const unsigned char *)from + ((is_v ? voff : koff[i & 3]) - 256 * r4), at + 1024 * i);
        }
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};

    // this lane's places in a tile: fragment f of K, block of 32 channels db of V
    constexpr int TG = OWN ? 0 : 1;
    const unsigned char *lds_w = smem + (OWN ? 32768 * w : 0);
    uint32_t kat[8], vat[4];
#pragma unroll
    for (int f = 0; f < 8; ++f) kat[f] = 256 * (32 * SUB * TG * tg + n32) + 16 * ((2 * f + hf + n32) & 15);
    {
        const int rl = 4 * hf + ((lane & 15) >> 2);
#pragma unroll
        for (int db = 0; db < 4; ++db)
            vat[db] = VBASE + 256 * (32 * SUB * TG * tg + rl) + 32 * ((2 * db + ((lane >> 4) & 1) + 2 * rl) & 7) + 8 * (lane & 3);
    }

    // Row tile rt, part s of a tile of tokens: S[rt SUB + s]; its weights as operands: P[2 (rt SUB + s)] and the next one.
    constexpr int PARTS = RT * SUB;
    f32x16_t O[RT][4];
    float m_run[RT], l_run[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.0f;
#pragma unroll
        for (int db = 0; db < 4; ++db) O[rt][db] = f32x16_t(0.0f);
    }
    // logits of a tile of keys
    auto logits = [&](const unsigned char *lds, f32x16_t (&S)[PARTS]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < PARTS; ++s) S[s] = f32x16_t(0.0f);
#pragma unroll
        for (int f = 0; f < 8; ++f)
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const u32x4_t kf = *reinterpret_cast<const u32x4_t *>(lds + kat[f] + 8192 * s);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    S[rt * SUB + s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf), Qf[rt][f], S[rt * SUB + s], 0, 0, 0);
            }
    };
    // register v of part s is token tw + 32 s + 8 (v / 4) + 4 hf + v % 4: what this row does not see
    auto hide = [&](int tw, f32x16_t (&S)[PARTS]) __attribute__((always_inline)) {
        if (tw + 32 * SUB > plain_end) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const int t = tw + 32 * (p % SUB), left = t_end - t;
                uint32_t sees = left >= 32 ? 0xFFFFFFFFu : left > 0 ? (1u << left) - 1u : 0u;
                sees &= draft_bits(a, seq, token[p / SUB], t - n);
                sees >>= 4 * hf;
#pragma unroll
                for (int v = 0; v < 16; ++v) S[p][v] = sees >> (8 * (v / 4) + v % 4) & 1u ? S[p][v] : -INFINITY;
            }
        }
    };
    auto top_of = [&](const f32x16_t (&S)[PARTS], float (&m_loc)[RT]) __attribute__((always_inline)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float m = S[rt * SUB][0], lo, hi;
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int v = 0; v < 16; ++v) m = fmaxf(m, S[rt * SUB + s][v]);
            halves(m, lo, hi);
            m_loc[rt] = fmaxf(lo, hi);
        }
    };
    auto raise = [&](const float (&m_loc)[RT]) __attribute__((always_inline)) {
        bool any = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) any |= !((m_loc[rt] - m_run[rt]) * c <= 8.0f);
        if (__ballot(any)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float m_new = fmaxf(m_run[rt], m_loc[rt]), alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run[rt] - m_new) * c);
                l_run[rt] *= alpha;
#pragma unroll
                for (int db = 0; db < 4; ++db)
#pragma unroll
                    for (int v = 0; v < 16; ++v) O[rt][db][v] *= alpha;
                m_run[rt] = m_new;
            }
        }
    };
    // logits to weights, as operands of two products
    auto weigh = [&](f32x16_t (&S)[PARTS], bf16x8_t (&P)[2 * PARTS], bf16x8_t (&R)[2 * PARTS]) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int rt = p / SUB;
            const float less = m_run[rt] == -INFINITY ? 0.0f : -m_run[rt] * c;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int v = 8 * j; v < 8 * j + 8; ++v) S[p][v] = __builtin_amdgcn_exp2f(fmaf(S[p][v], c, less));
                const f32x8_t x = eight(S[p], j);
                l_run[rt] = sum8(x, l_run[rt]);
                P[2 * p + j] = upper8(x);
                R[2 * p + j] = lower8(x);
            }
        }
    };
    auto add_values = [&](const unsigned char *lds, const bf16x8_t (&P)[2 * PARTS], const bf16x8_t (&R)[2 * PARTS]) __attribute__((always_inline)) {
#pragma unroll
        for (int sj = 0; sj < 2 * SUB; ++sj)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                // position e of lane (channel, hf): token 16 sj + 8 (e / 4) + 4 hf + e % 4, as in P
                const unsigned char *from = lds + vat[db] + 4096 * sj;
                const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)from);
                const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(from + 2048));
                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[rt][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, R[2 * SUB * rt + sj], O[rt][db], 0, 0, 0);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[rt][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, P[2 * SUB * rt + sj], O[rt][db], 0, 0, 0);
            }
    };
    if constexpr (OWN) {
        // A wavefront keeps two tiles of its own and waits for nobody: the keys of the tile after the next are requested as soon as the
        // logits are there, its values as soon as the products are.  (Counted waits: requests are answered in order.)
        const int t_first = t_begin + 32 * w;
        if (t_first < t_end) {
            stage(t_first, 0, keys);
            stage(t_first, 0, values);
        }
        if (t_first + TILE < t_end) {
            stage(t_first + TILE, 1, keys);
            stage(t_first + TILE, 1, values);
        }
        int buf = 0;
        for (int t = t_first; t < t_end; t += TILE, buf ^= 1) {
            const unsigned char *lds = lds_w + 16384 * buf;
            const bool next = t + TILE < t_end, then = t + 2 * TILE < t_end;
            if (next)
                XKV_WAIT_VMCNT(3 * LOADS);
            else
                XKV_WAIT_VMCNT(LOADS);
            asm volatile("" : : : "memory");
            f32x16_t S[PARTS];
            bf16x8_t P[2 * PARTS], R[2 * PARTS];
            logits(lds, S);
            if (then) {
                wait_lds();
                stage(t + 2 * TILE, buf, keys);
            }
            hide(t, S);
            float m_loc[RT];
            top_of(S, m_loc);
            raise(m_loc);
            weigh(S, P, R);
            if (then)
                XKV_WAIT_VMCNT(3 * LOADS);
            else if (next)
                XKV_WAIT_VMCNT(2 * LOADS);
            else
                XKV_WAIT_VMCNT(0);
            asm volatile("" : : : "memory");
            if (t_end > n && t + 32 > n) note_odd(sm_odd, clear_odd<LOADS>(smem + 32768 * w + 16384 * buf + VBASE + 16 * lane, n - t), t - n);
            add_values(lds, P, R);
            if (then) {
                wait_lds();
                stage(t + 2 * TILE, buf, values);
            }
        }
    } else {
        // One tile ahead with the logits: the products of tile i + 1 with the keys run beside the exponentials of tile i, those of tile i
        // with the values beside the maximum of tile i + 1.  Keys i + 1 and values i are there at the barrier, and nobody reads keys i
        // and values i - 1 any more, whose places keys i + 2 and values i + 1 take.
        stage(t_begin + RPW * w, 0, keys);
        stage(t_begin + RPW * w, 0, values);
        if (t_begin + TILE < t_end) stage(t_begin + TILE + RPW * w, 1, keys);
        if (t_begin + TILE < t_end)
            XKV_WAIT_VMCNT(2 * LOADS);
        else
            XKV_WAIT_VMCNT(LOADS);
        __syncthreads();
        f32x16_t S[PARTS];
        float m_loc[RT];
        logits(lds_w, S);
        hide(t_begin + 32 * SUB * tg, S);
        top_of(S, m_loc);
        auto step = [&](int t0, auto which, f32x16_t (&S)[PARTS], f32x16_t (&S1)[PARTS]) __attribute__((always_inline)) {
            constexpr int BUF = decltype(which)::value, READS = 8 * SUB, STEPS = READS * RT, AHEAD = 3;
            XKV_WAIT_VMCNT(0);
            __syncthreads();
            stage_plain(t0 + 2 * TILE + RPW * w, BUF, keys);
            stage_plain(t0 + TILE + RPW * w, BUF ^ 1, values);
            raise(m_loc);
            const unsigned char *kt = lds_w + (BUF ^ 1) * KTILE, *vt = lds_w + BUF * KTILE;
            bf16x8_t P[2 * PARTS], R[RT];
            // each product with the keys beside two exponentials
            u32x4_t kf[READS];
            auto read_key = [&](int k) __attribute__((always_inline)) {
                kf[k] = *reinterpret_cast<const u32x4_t *>(kt + kat[k / SUB] + 8192 * (k % SUB));
            };
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) read_key(k);
            float less[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) less[rt] = m_run[rt] == -INFINITY ? 0.0f : -m_run[rt] * c;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int k = i / RT, rt = i % RT, p = rt * SUB + k % SUB;
                if (rt == 0 && k + AHEAD < READS) read_key(k + AHEAD);
                if (k < SUB) S1[p] = f32x16_t(0.0f);
                S1[p] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[k]), Qf[rt][k / SUB], S1[p], 0, 0, 0);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int v = 2 * i + x;
                    S[v / 16][v % 16] = __builtin_amdgcn_exp2f(fmaf(S[v / 16][v % 16], c, less[v / 16 / SUB]));
                }
                if (i % 4 == 3) {
                    const f32x8_t x = eight(S[i / 8], i / 4 % 2);
                    l_run[i / 8 / SUB] = sum8(x, l_run[i / 8 / SUB]);
                    P[i / 4] = upper8(x);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // each product with the values beside its share of the next maximum
            s16x4_t vf[READS][2];
            auto read_values = [&](int k) __attribute__((always_inline)) {
                const unsigned char *from = vt + vat[k % 4] + 4096 * (k / 4);
                vf[k][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)from);
                vf[k][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(from + 2048));
            };
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) read_values(k);
            float m_next[2 * RT];
#pragma unroll
            for (int i = 0; i < 2 * RT; ++i) m_next[i] = -INFINITY;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int k = i / RT, rt = i % RT;
                if (rt == 0 && k + AHEAD < READS) read_values(k + AHEAD);
                if (k % 4 == 0) R[rt] = lower8(eight(S[(2 * SUB * rt + k / 4) / 2], k / 4 % 2));  // (not before: the exponentials keep the other half busy)
                const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(vf[k][0], vf[k][1], 0, 1, 2, 3, 4, 5, 6, 7));
                O[rt][k % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v8, R[rt], O[rt][k % 4], 0, 0, 0);
                O[rt][k % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v8, P[2 * SUB * rt + k / 4], O[rt][k % 4], 0, 0, 0);
                if (i >= STEPS / 2) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int v = 4 * (i - STEPS / 2) + x, m = 2 * (v / 16 / SUB) + (x >> 1);
                        m_next[m] = fmaxf(m_next[m], S1[v / 16][v % 16]);
                        if (x & 1) asm volatile("" : "+v"(m_next[m]));  // (here, not at the end)
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float lo, hi;
                halves(fmaxf(m_next[2 * rt], m_next[2 * rt + 1]), lo, hi);
                m_loc[rt] = fmaxf(lo, hi);
            }
        };
        int buf = 0, t0 = t_begin;
        for (; t0 + 4 * TILE <= plain_end; t0 += 2 * TILE) {  // the next three tiles are whole
            f32x16_t S1[PARTS];
            step(t0, std::integral_constant<int, 0>{}, S, S1);
            step(t0 + TILE, std::integral_constant<int, 1>{}, S1, S);
        }
        for (; t0 < t_end; t0 += TILE, buf ^= 1) {
            XKV_WAIT_VMCNT(0);
            if (t_end > n && t0 + TILE > n) {
                asm volatile("" : : : "memory");
                const int first = t0 + RPW * w;
                note_odd(sm_odd, clear_odd<LOADS>(smem + 256 * RPW * w + buf * KTILE + VBASE + 16 * lane, n - first), first - n);
            }
            __syncthreads();
            if (t0 + 2 * TILE < t_end) stage(t0 + 2 * TILE + RPW * w, buf, keys);
            if (t0 + TILE < t_end) stage(t0 + TILE + RPW * w, buf ^ 1, values);
            raise(m_loc);
            f32x16_t S1[PARTS];
            bf16x8_t P[2 * PARTS], R[2 * PARTS];
            logits(lds_w + (buf ^ 1) * KTILE, S1);  // (behind the last tile: of whatever is there, not used)
            weigh(S, P, R);
            if (t0 + TILE < t_end) hide(t0 + TILE + 32 * SUB * tg, S1);
            add_values(lds_w + buf * KTILE, P, R);
            top_of(S1, m_loc);
#pragma unroll
            for (int s = 0; s < PARTS; ++s) S[s] = S1[s];
        }
    }

    // merge the token groups through LDS, where rows come together as well: 16-byte piece p of row n32 of a row tile sits at (p + n32) % 32
    // (all row tiles at once, places found by a thread per row, four rows of a thread on their way: 2.4 us; one after the other 5)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float lo, hi;
        halves(l_run[rt], lo, hi);
        if (hf == 0) {
            sm_m[tg][32 * (rg * RT + rt) + n32] = m_run[rt];
            sm_l[tg][32 * (rg * RT + rt) + n32] = lo + hi;
        }
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < WT; ++i) top = fmaxf(top, sm_m[i][32 * (rg * RT + rt) + n32]);
        const float f = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run[rt] - top) * c);
        f32x4_t *ot = reinterpret_cast<f32x4_t *>(smem) + 1024 * (w * RT + rt) + 32 * n32;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                ot[(8 * db + v / 2 + hf + n32) & 31] = f32x4_t{f * O[rt][db][v], f * O[rt][db][v + 1], f * O[rt][db][v + 2], f * O[rt][db][v + 3]};
    }
    constexpr int ROWS = 32 * WR * RT, AT_ONCE = 2 * WAVES, BATCH = 4;
    static_assert(ROWS <= 64 * WAVES && ROWS % (AT_ONCE * BATCH) == 0, "a thread per row, then whole rounds of 32 threads per row");
    if (threadIdx.x < ROWS) {  // a row's place and statistics, once
        const int m = tile * ROWS + (int)threadIdx.x;
        float top = -INFINITY, den = 0.0f;
#pragma unroll
        for (int i = 0; i < WT; ++i) top = fmaxf(top, sm_m[i][threadIdx.x]);
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            const float mi = sm_m[i][threadIdx.x];
            den += sm_l[i][threadIdx.x] * (mi == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((mi - top) * c));  // (without a maximum: 0, or NaN)
        }
        const size_t slot = part_row(a, MODE, u.part, m / n_rep, g * n_rep + m % n_rep);
        sm_slot[threadIdx.x] = m < M ? (uint32_t)slot : 0xFFFFFFFFu;
        if (m < M) {
            a.part_ml[2 * slot] = top * a.scale;
            a.part_ml[2 * slot + 1] = den;
        }
    }
    __syncthreads();
    const int p = threadIdx.x & 31, r0 = threadIdx.x >> 5;
    const bool odd = t_end > n && __ballot(sm_odd[n32] != 0u);
#pragma unroll
    for (int s0 = 0; s0 < ROWS / AT_ONCE; s0 += BATCH) {
        f32x4_t x[BATCH];
        uint32_t slot[BATCH];
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const int row = r0 + (s0 + s) * AT_ONCE;
            slot[s] = sm_slot[row];
            x[s] = f32x4_t(0.0f);
#pragma unroll
            for (int i = 0; i < WT; ++i) x[s] += reinterpret_cast<const f32x4_t *>(smem)[1024 * i * WR * RT + 32 * row + ((p + row) & 31)];
        }
        if (odd) {
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
                if (slot[s] != 0xFFFFFFFFu) x[s] = add_odd(a, sm_odd, Vd, seq, (tile * ROWS + r0 + (s0 + s) * AT_ONCE) / n_rep, 4 * p, x[s]);
        }
#pragma unroll
        for (int s = 0; s < BATCH; ++s)
            if (slot[s] != 0xFFFFFFFFu) *reinterpret_cast<f32x4_t *>(a.part_o + (size_t)slot[s] * 128 + 4 * p) = x[s];
    }
}

// ------------------------------------------------------------------------------------------
// Up to 16 rows (a token's query heads, selected blocks, short drafts): the same products in 16 x 16 tiles, so that half as many logits are
// formed per lane and no chain of products is longer than four.  A wavefront streams tiles of 32 tokens of its own, four in a workgroup.
//   S^T: lane (row l % 16, kk = l / 16), part h, register r: token 16 h + 4 kk + r;  O^T: block db, register r: channel 16 db + 4 kk + r
// LDS: the 16-byte piece p of row t of K at p ^ t % 16 (a fragment read takes two neighbouring pieces of 8 rows each at a time), the 32-byte
// piece u of row t of V at (u + t) % 8 (a transposing read takes one piece of 8 rows at a time).
// In 32 x 32 tiles, half of them empty, against 16 x 16 (with one product for a weight): 256 queries of a 128K prompt 240 / 223 us, weights over
// 8 x 32768 tokens 26.3 / 25.6.  The second product: the whole calls 263 -> 269 and 31.0 -> 31.4.
// ------------------------------------------------------------------------------------------
constexpr int kHeldLogits = 32;  // rows of 32 logits that a wavefront holds back

template <CacheMode MODE>
__global__ __launch_bounds__(256, 1) void cache_stream_kernel(CacheArgs a)
{
    constexpr int TILE = 128, LOADS = 8, KTILE = 8192;
    constexpr bool BLK = MODE == CacheMode::blocks, KEEP = MODE == CacheMode::weights;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * 4 * KTILE];
    __shared__ float sm_m[4][16], sm_l[4][16];
    __shared__ uint32_t sm_seen[32], sm_odd[32];
    __shared__ __attribute__((aligned(16))) float sm_z[KEEP ? 4 : 1][KEEP ? kHeldLogits : 1][36];  // logits of a few tiles
    __shared__ int sm_rows[BLK ? kPartBlocks + 2 : 1];                                              // first rows of this part's blocks
    const int lane = lane_id(), w = wave_id(), n16 = lane & 15, kk = lane >> 4, n_rep = a.H_q / a.H_kv;
    const int M = BLK ? n_rep : a.N * n_rep;
    const CacheUnit u = cache_unit(a, MODE, 1);
    const bool direct = BLK && a.parts == 1;  // a query's only part: the result instead of a partial
    if (!u.some) {  // (the merge knows)
        if (direct)
            for (int i = threadIdx.x; i < n_rep * 128; i += 256) ((bf16_t *)a.out)[((size_t)u.seq * a.H_q + u.g * n_rep) * 128 + i] = 0;
        return;
    }
    const int g = u.g, n = u.n, t_begin = u.t_begin, t_end = u.t_end;
    const int seq = BLK ? u.seq / a.N : u.seq, first_token = BLK ? u.seq % a.N : 0;
    const float c = a.scale * 1.44269504088896340736f;

    const bf16_t *Kg = (const bf16_t *)a.K + ((size_t)seq * a.H_kv + g) * a.L * 128, *Vg = (const bf16_t *)a.V + ((size_t)seq * a.H_kv + g) * a.L * 128;
    const bf16_t *Kd = (const bf16_t *)a.K_draft + ((size_t)seq * a.H_kv + g) * a.N * 128;
    const bf16_t *Vd = (const bf16_t *)a.V_draft + ((size_t)seq * a.H_kv + g) * a.N * 128;

    // Q^T fragments: lane (row n16, kk), fragment f, position e: channel 32 f + 8 kk + e
    const int m_in = n16 < M ? n16 : M - 1, token = first_token + m_in / n_rep;
    bf16x8_t Qf[4];
    {
        const u32x4_t *q = reinterpret_cast<const u32x4_t *>((const bf16_t *)a.q + (((size_t)seq * a.N + token) * a.H_q + g * n_rep + m_in % n_rep) * 128);
#pragma unroll
        for (int f = 0; f < 4; ++f) Qf[f] = __builtin_bit_cast(bf16x8_t, q[4 * f + kk]);
    }
    if (MODE == CacheMode::tree && t_end > n) {  // which drafted tokens any token sees
        if (threadIdx.x < 32) sm_seen[threadIdx.x] = a.tree ? 0u : 0xFFFFFFFFu, sm_odd[threadIdx.x] = 0u;
        __syncthreads();
        if (a.tree)
            for (int i = threadIdx.x; i < a.N * a.words; i += 256) {
                const uint32_t x = a.tree[(size_t)seq * a.N * a.words + i];
                if (x) atomicOr(&sm_seen[i % a.words], x);
            }
        __syncthreads();
    }
    // Blocks: a load of a block's number between the requests of rows would be waited for together with them, so the numbers go to LDS first.
    // A lane's next tokens are TILE further on: `ahead` whole blocks and `rest` rows.
    int in_list[8], in_block[8], rows_of[8], ahead = 0, rest = 0;
    if constexpr (BLK) {
        const int32_t *sel = a.sel + ((size_t)u.seq * a.H_kv + g) * a.k_ch;
        const int b0 = t_begin / a.c, b1 = (t_end - 1) / a.c;  // b1 - b0 <= kPartBlocks
        for (int i = threadIdx.x; i <= b1 - b0; i += 256) sm_rows[i] = sel[b0 + i] * a.c;
        __syncthreads();
        ahead = TILE / a.c;
        rest = TILE % a.c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = t_begin + 32 * w + 4 * i + (lane >> 4), j = t / a.c;
            in_list[i] = j - b0;
            in_block[i] = t - j * a.c;
        }
    }


    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + 4 * KTILE * w;
    const int r4 = lane >> 4, x16 = lane & 15;
    uint32_t koff[4], voff[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) koff[i] = 256 * r4 + 16 * (x16 ^ (4 * i + r4));
#pragma unroll
    for (int i = 0; i < 2; ++i) voff[i] = 256 * r4 + 32 * (((x16 >> 1) - 4 * i - r4) & 7) + 16 * (x16 & 1);
    const int plain_end = MODE == CacheMode::tree && n < t_end ? n : t_end;  // rows of the cache end here
    auto stage = [&](int first, int buf, auto values) __attribute__((always_inline)) {  // 32 tokens from `first` on
        constexpr bool is_v = decltype(values)::value;
        const uint32_t at = lds0 + buf * 2 * KTILE + (is_v ? KTILE : 0);
        const bf16_t *rows = is_v ? Vg : Kg;
        if constexpr (BLK) {  // called for the tiles in turn, keys before values
            if constexpr (!is_v) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool real = first + 4 * i + r4 < t_end;
                    rows_of[i] = real ? sm_rows[real ? in_list[i] : 0] + in_block[i] : -1;
                    in_list[i] += ahead;
                    in_block[i] += rest;
                    if (in_block[i] >= a.c) {
                        in_block[i] -= a.c;
                        ++in_list[i];
                    }
                }
            }
            auto copy = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const bf16_t *from = decltype(whole)::value || rows_of[i] >= 0 ? rows + (size_t)rows_of[i] * 128 : (const bf16_t *)kZeroRow;
                    copy16_global_to_lds((const unsigned char *)from + ((is_v ? voff[i & 1] : koff[i & 3]) - 256 * r4), at + 1024 * i);
                }
            };
            if (first + 32 <= t_end)  // (wave-uniform)
                copy(std::true_type{});
            else
                copy(std::false_type{});
            return;
        }
        if (first + 32 <= plain_end) {  // (wave-uniform)
            const unsigned char *base = (const unsigned char *)(rows + (size_t)first * 128);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) copy16_to_lds_once(base + 1024 * i, is_v ? voff[i & 1] : koff[i & 3], at + 1024 * i);
            return;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int t = first + 4 * i + r4, j = t - n;
            const bf16_t *from = t < plain_end ? rows + (size_t)t * 128 : (const bf16_t *)kZeroRow;
            if (MODE == CacheMode::tree && t < t_end && j >= 0 && (sm_seen[(j >> 5) & 31] >> (j & 31) & 1u)) from = (is_v ? Vd : Kd) + (size_t)j * 128;
            copy16_global_to_lds((const unsigned char *)from + ((is_v ? voff[i & 1] : koff[i & 3]) - 256 * r4), at + 1024 * i);
        }
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};

    uint32_t kat[4], vat[8];
#pragma unroll
    for (int f = 0; f < 4; ++f) kat[f] = 256 * n16 + 16 * ((4 * f + kk) ^ n16);
    {
        const int rl = 4 * kk + (n16 >> 2);
#pragma unroll
        for (int db = 0; db < 8; ++db) vat[db] = KTILE + 256 * rl + 32 * ((db + rl) & 7) + 8 * (lane & 3);
    }
    f32x4_t O[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) O[db] = f32x4_t(0.0f);
    float m_run = -INFINITY, l_run = 0.0f;
    int held = 0;  // tiles whose logits wait, of `hold`
    const int hold = n_rep <= kHeldLogits / 8 ? 8 : kHeldLogits / n_rep;

    // A wavefront keeps two tiles and waits for nobody: the keys of the tile after the next are requested as soon as the logits are there,
    // its values as soon as the products are.  (Counted waits: requests are answered in order; others in between, of logits that are
    // stored, make a wait longer, not shorter.)
    const int t_first = t_begin + 32 * w;
    if (t_first < t_end) {
        stage(t_first, 0, keys);
        stage(t_first, 0, values);
    }
    if (t_first + TILE < t_end) {
        stage(t_first + TILE, 1, keys);
        stage(t_first + TILE, 1, values);
    }
    int buf = 0;
    for (int t = t_first; t < t_end; t += TILE, buf ^= 1) {
        const unsigned char *lds = smem + 4 * KTILE * w + 2 * KTILE * buf;
        const bool next = t + TILE < t_end, then = t + 2 * TILE < t_end;
        if (next)
            XKV_WAIT_VMCNT(3 * LOADS);
        else
            XKV_WAIT_VMCNT(LOADS);
        asm volatile("" : : : "memory");
        f32x4_t S[2];
        S[0] = S[1] = f32x4_t(0.0f);
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4_t kf = *reinterpret_cast<const u32x4_t *>(lds + kat[f] + 4096 * h);
                S[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), Qf[f], S[h], 0, 0, 0);
            }
        if (then) {
            wait_lds();
            stage(t + 2 * TILE, buf, keys);
        }
        if (t + 32 > plain_end) {
            const int left = t_end - t;
            uint32_t sees = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
            if (MODE == CacheMode::tree) sees &= draft_bits(a, seq, token, t - n);
            sees >>= 4 * kk;
#pragma unroll
            for (int v = 0; v < 8; ++v) S[v / 4][v % 4] = sees >> (16 * (v / 4) + v % 4) & 1u ? S[v / 4][v % 4] : -INFINITY;
        }
        // The logits of a few tiles wait in LDS and leave together, a line of 32 per head and tile: small stores between the requests of a
        // stream slow it down by more than their share of its bytes.
        if constexpr (KEEP) {
            if (n16 < n_rep) {
#pragma unroll
                for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4_t *>(&sm_z[w][held * n_rep + n16][16 * h + 4 * kk]) = a.scale * S[h];
            }
            if (++held == hold || !next) {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                const int n32 = lane & 31;
                float *to = a.logits + ((size_t)seq * a.H_q + g * n_rep) * a.L + n32;
                for (int i = 0; i < held; ++i) {
                    const int ti = t - TILE * (held - 1 - i);
                    for (int h = lane >> 5; h < n_rep; h += 2)
                        if (ti + n32 < t_end) to[(size_t)h * a.L + ti] = sm_z[w][i * n_rep + h][n32];
                }
                __builtin_amdgcn_wave_barrier();
                held = 0;
            }
        }
        float m_loc = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
        float lo, hi;
        quarters(m_loc, lo, hi);
        halves(fmaxf(lo, hi), lo, hi);
        m_loc = fmaxf(lo, hi);
        if (__ballot(!((m_loc - m_run) * c <= 8.0f))) {
            const float m_new = fmaxf(m_run, m_loc), alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - m_new) * c);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < 8; ++db) O[db] *= alpha;
            m_run = m_new;
        }
        const float less = m_run == -INFINITY ? 0.0f : -m_run * c;
        f32x8_t p;
#pragma unroll
        for (int v = 0; v < 8; ++v) p[v] = __builtin_amdgcn_exp2f(fmaf(S[v / 4][v % 4], c, less));
        l_run = sum8(p, l_run);
        const bf16x8_t P = upper8(p), R = lower8(p);
        if (then)
            XKV_WAIT_VMCNT(3 * LOADS);
        else if (next)
            XKV_WAIT_VMCNT(2 * LOADS);
        else
            XKV_WAIT_VMCNT(0);
        asm volatile("" : : : "memory");
        if (MODE == CacheMode::tree && t_end > n && t + 32 > n)
            note_odd(sm_odd, clear_odd<LOADS>(smem + 4 * KTILE * w + 2 * KTILE * buf + KTILE + 16 * lane, n - t), t - n);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            // position e of lane (channel, kk): token 16 (e / 4) + 4 kk + e % 4, as in P
            const unsigned char *from = lds + vat[db];
            const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)from);
            const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(from + 4096));
            const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
            O[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, R, O[db], 0, 0, 0);
            O[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P, O[db], 0, 0, 0);
        }
        if (then) {
            wait_lds();
            stage(t + 2 * TILE, buf, values);
        }
    }

    // merge the wavefronts through LDS: 16-byte piece p of row n16 sits at (p + n16) % 32
    {
        float lo, hi;
        quarters(l_run, lo, hi);
        halves(lo + hi, lo, hi);
        if (kk == 0) {
            sm_m[w][n16] = m_run;
            sm_l[w][n16] = lo + hi;
        }
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(sm_m[0][n16], sm_m[1][n16]), fmaxf(sm_m[2][n16], sm_m[3][n16]));
    const float f = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - top) * c);
    f32x4_t *ot = reinterpret_cast<f32x4_t *>(smem) + 512 * w;
#pragma unroll
    for (int db = 0; db < 8; ++db) ot[32 * n16 + ((4 * db + kk + n16) & 31)] = f * O[db];
    __syncthreads();
    const bool odd = MODE == CacheMode::tree && t_end > n && __ballot(sm_odd[lane & 31] != 0u);
    for (int item = threadIdx.x; item < 512; item += 256) {
        const int row = item >> 5, p = item & 31;
        if (row >= M) continue;
        f32x4_t x = f32x4_t(0.0f);
        float den = 0.0f, most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x += reinterpret_cast<const f32x4_t *>(smem)[512 * i + 32 * row + ((p + row) & 31)];
            most = fmaxf(most, sm_m[i][row]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) den += sm_l[i][row] * (sm_m[i][row] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((sm_m[i][row] - most) * c));
        if (direct) {
            bf16_t *out = (bf16_t *)a.out + ((size_t)u.seq * a.H_q + g * n_rep + row) * 128 + 4 * p;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = f32_to_bf16(x[e] / den);
            continue;
        }
        if (odd) x = add_odd(a, sm_odd, Vd, seq, row / n_rep, 4 * p, x);
        const size_t slot = part_row(a, MODE, u.part, row / n_rep, g * n_rep + row % n_rep);
        *reinterpret_cast<f32x4_t *>(a.part_o + slot * 128 + 4 * p) = x;
        if (p == 0) {
            a.part_ml[2 * slot] = most * a.scale;
            a.part_ml[2 * slot + 1] = den;
        }
    }
}

// Whether query z (sequence, query token) sees no token at all: its result is zeros.
__device__ __forceinline__ bool sees_nothing(const CacheArgs &a, CacheMode mode, int z)
{
    if (cache_rows(a, mode == CacheMode::tree ? z / a.N : z) > 0) return false;
    if (mode != CacheMode::tree) return true;
    if (!a.tree) return false;  // (it sees itself)
    uint32_t any = 0;
    for (int k = 0; k < a.words; ++k) any |= a.tree[(size_t)z * a.words + k] & (32 * k + 32 <= a.N ? 0xFFFFFFFFu : (1u << (a.N & 31)) - 1u);
    return any == 0;
}

// ------------------------------------------------------------------------------------------
// Merge.  A group of 2^lg lanes covers the columns of a row (query token, head), VEC a lane.  Where there are many rows, a group per row;
// where there are few, all groups of a workgroup share a row's partials between them and are added up in LDS: latency is all there is to
// it then.  Partials that no token went to were
// not written and are not read.
// ------------------------------------------------------------------------------------------
template <typename T, CacheMode MODE, int VEC>
__device__ __forceinline__ void merge_block(const CacheArgs &a, int lg, int share, int rows)
{
    typedef __attribute__((ext_vector_type(VEC))) float vec_t;
    constexpr int BATCH = 4;
    __shared__ vec_t sm[256];
    __shared__ float sm_w[32][kMaxCacheParts];
    const int width = 1 << lg, l = (int)threadIdx.x & (width - 1), grp = (int)threadIdx.x >> lg, groups = 256 >> lg;
    const int col = ((int)blockIdx.y * width + l) * VEC;
    const int item = share ? (int)blockIdx.x : (int)blockIdx.x * groups + grp, row = item < rows ? item : rows - 1;
    const int z = row / a.H_q, head = row % a.H_q;  // z: (sequence, query token)
    int first, parts;
    cache_parts(a, MODE, MODE == CacheMode::tree ? z / a.N : z, first, parts);
    const size_t at = part_row(a, MODE, first, z % a.N, head), stride = part_row(a, MODE, 1, 0, 0);  // its first partial; to the next one
    const float *ml = a.part_ml + at * 2;
    float M = -INFINITY, den = 0.0f;
    for (int s = l; s < parts; s += width) M = fmaxf(M, ml[2 * s * stride]);
    for (int off = 1; off < width; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, kWave));
    for (int s = l; s < parts; s += width) {
        const float m = ml[2 * s * stride], wt = m == -INFINITY ? 0.0f : expf(m - M);
        sm_w[grp][s] = wt;
        den = fmaf(wt, ml[2 * s * stride + 1], den);
    }
    for (int off = 1; off < width; off <<= 1) den += __shfl_xor(den, off, kWave);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // (a group is part of a wavefront)
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const float *po = a.part_o + at * a.d_h + (col < a.d_h ? col : 0);
    const int step = share ? groups : 1;
    vec_t acc = vec_t(0.0f);
    for (int s1 = share ? grp : 0; s1 < parts; s1 += BATCH * step) {
        vec_t v[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = s1 + u * step < parts ? s1 + u * step : parts - 1;
            v[u] = *reinterpret_cast<const vec_t *>(po + (size_t)s * stride * a.d_h);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = s1 + u * step;
            acc += (s < parts ? sm_w[grp][s] : 0.0f) * (s < parts ? v[u] : vec_t(0.0f));
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
    const bool none = den == 0.0f && sees_nothing(a, MODE, z);  // (a sum of zero otherwise: logits of -inf alone, 0 / 0)
#pragma unroll
    for (int e = 0; e < VEC; ++e) out[e] = from_f32<T>(none ? 0.0f : acc[e] / den);
}

// ------------------------------------------------------------------------------------------
// weights[t] += sum over the query heads of a KV head of exp(z_t - max) / sum, from the kept logits.  The maximum and the sum
// of a head are merged from the partials by every workgroup.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void weights_block(const CacheArgs &a, int block)
{
    __shared__ float sm_m[16], sm_r[16];
    const int per_head = (a.L + 1023) / 1024, g = block / per_head % a.H_kv, b = block / per_head / a.H_kv;
    const int lane = lane_id(), w = wave_id(), n_rep = a.H_q / a.H_kv;
    const int n = cache_rows(a, b), t0 = block % per_head * 1024;
    if (t0 >= n) return;
    const size_t head = (size_t)b * a.H_q + g * n_rep, stride = a.H_q;
    int first, parts;
    cache_parts(a, CacheMode::weights, b, first, parts);
    for (int h = w; h < n_rep; h += 4) {
        const float *ml = a.part_ml + part_row(a, CacheMode::weights, first, 0, g * n_rep + h) * 2;
        float M = -INFINITY, den = 0.0f;
        for (int s = lane; s < parts; s += kWave) M = fmaxf(M, ml[2 * s * stride]);
        M = wave_all(M, MaxOp());
        for (int s = lane; s < parts; s += kWave) den = fmaf(expf(ml[2 * s * stride] - M), ml[2 * s * stride + 1], den);
        den = wave_all(den, AddOp());
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
        a.weights[((size_t)b * a.H_kv + g) * a.L + t] += sum;
    }
}

// x: workgroups of the merge, then (weights) those of the weights.
template <typename T, CacheMode MODE, int VEC>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheArgs a, int lg, int share, int rows, int merges)
{
    if (MODE != CacheMode::weights || (int)blockIdx.x < merges)
        merge_block<T, MODE, VEC>(a, lg, share, rows);
    else if (blockIdx.y == 0)
        weights_block(a, (int)blockIdx.x - merges);
}

dim3 unit_grid(const CacheArgs &a, CacheMode mode, int M)
{
    return dim3((unsigned)a.parts * a.H_kv * ((M + a.rows - 1) / a.rows) * (mode == CacheMode::blocks ? a.batch * a.N : 1));
}

template <CacheMode MODE, typename T>
hipError_t launch_general(const CacheArgs &a, hipStream_t st)
{
    const int M = MODE == CacheMode::blocks ? a.H_q / a.H_kv : a.N * (a.H_q / a.H_kv);
    const dim3 grid = unit_grid(a, MODE, M);
    const size_t lds = (2 * (size_t)kGenTokens * general_pitch(a.d_h) + (size_t)kGenRows * ((a.d_h + 3) / 4 * 4) + 4 * 4 * kGenTokens) * sizeof(float);
    auto launch = [&](auto kernel, DynamicLdsOnce &attr) {
        const hipError_t e = attr.ensure((const void *)kernel, 160 * 1024);  // (at most 150 KiB, at 256 channels)
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, a);
        return hipGetLastError();
    };
    static DynamicLdsOnce attr[3];
    return a.d_h <= 64 ? launch(cache_attend_general_kernel<T, MODE, 1>, attr[0])
         : a.d_h <= 128 ? launch(cache_attend_general_kernel<T, MODE, 2>, attr[1]) : launch(cache_attend_general_kernel<T, MODE, 4>, attr[2]);
}

template <CacheMode MODE>
hipError_t launch_mfma(const CacheArgs &a, hipStream_t st)
{
    const int M = MODE == CacheMode::blocks ? a.H_q / a.H_kv : a.N * (a.H_q / a.H_kv);
    const dim3 grid = unit_grid(a, MODE, M);
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a); };
    if (a.rows == 16) {
        launch(cache_stream_kernel<MODE>, 256);
    } else if constexpr (MODE == CacheMode::tree) {
        a.rows == 256 ? launch(cache_tree_kernel<8, 1, 2, 1>, 512) : a.rows == 128 ? launch(cache_tree_kernel<4, 1, 2, 1>, 256)
            : a.rows == 64 ? launch(cache_tree_kernel<1, 4, 1, 2>, 256) : launch(cache_tree_kernel<1, 4, 1, 1>, 256);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <CacheMode MODE>
hipError_t launch_mode(const xkv_shape &s, const CacheArgs &a, hipStream_t st)
{
    const uintptr_t bits = (uintptr_t)a.K | (uintptr_t)a.V | (uintptr_t)a.q | (uintptr_t)a.K_draft | (uintptr_t)a.V_draft;
    CacheArgs gen = a;
    gen.rows = kGenRows;  // (its rounds divide those of the plan)
    const bool matrix = a.mfma && bits % 16 == 0;
    hipError_t e = matrix ? launch_mfma<MODE>(a, st)
                 : s.dtype == XKV_F32 ? launch_general<MODE, float>(gen, st) : launch_general<MODE, bf16_t>(gen, st);
    if (e != hipSuccess || (MODE == CacheMode::blocks && a.parts == 1 && matrix)) return e;
    const int vec = a.d_h % 4 == 0 ? 4 : 1, rows = a.batch * a.N * a.H_q;
    int lg = 3;
    while (lg < 6 && (vec << lg) < a.d_h) ++lg;
    const int share = rows < 2048, groups = 256 >> lg;
    const int merges = share ? rows : (rows + groups - 1) / groups;
    const unsigned more = MODE == CacheMode::weights ? (unsigned)(a.batch * a.H_kv) * ((a.L + 1023) / 1024) : 0u;
    const dim3 grid(merges + more, (a.d_h + (vec << lg) - 1) / (vec << lg));
    auto merge = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, lg, share, rows, merges);
        return hipGetLastError();
    };
    if (s.dtype == XKV_F32) return vec == 4 ? merge(cache_merge_kernel<float, MODE, 4>) : merge(cache_merge_kernel<float, MODE, 1>);
    return vec == 4 ? merge(cache_merge_kernel<bf16_t, MODE, 4>) : merge(cache_merge_kernel<bf16_t, MODE, 1>);
}

}  // namespace

hipError_t launch_cache_attend(CacheMode mode, const xkv_shape &s, const CacheArgs &a, hipStream_t st)
{
    return mode == CacheMode::tree ? launch_mode<CacheMode::tree>(s, a, st)
         : mode == CacheMode::weights ? launch_mode<CacheMode::weights>(s, a, st) : launch_mode<CacheMode::blocks>(s, a, st);
}

}  // namespace xkv
