// Eviction from an uncompressed cache: of every KV head's rows the first `sink`, the last `recent` and those of the largest
// accumulated weight are kept, k altogether, in their order (cache.h).
#include "cache.h"

namespace xkv {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

// What the selection of longer rows (launch_topk) goes by, numbers whose order keys are: the largest key for rows that are kept anyway, the
// smallest one for rows that are not in use (behind those in use, whose places are smaller), and the weight's own between the two.
__global__ __launch_bounds__(256) void evict_keys_kernel(EvictArgs a)
{
    const int t = blockIdx.x * 256 + threadIdx.x, row = blockIdx.y, b = row / a.H_kv;
    int n = a.lengths ? a.lengths[b] : a.L;
    n = n < 0 ? 0 : n < a.L ? n : a.L;
    if (t == 0 && row == b * a.H_kv) a.n[b] = n;
    if (t >= a.L) return;
    const size_t at = (size_t)row * a.L + t;
    const float x = a.weights[at];
    const uint32_t key = order_key(x);
    const bool kept = t < a.sink || t >= n - a.recent;
    const float first = __uint_as_float(0x7FFFFFFFu), before = __uint_as_float(0x7FFFFFFEu), last = __uint_as_float(0xFFFFFFFEu);  // keys 2^32 - 1, 2^32 - 2, 1
    a.keys[at] = t >= n ? last : kept ? first : key == 0xFFFFFFFFu ? before : key < 1u ? last : x;
}

// The rows that stay, for caches of up to 1024 KPT rows: one workgroup per (sequence, KV head), the order keys of the weights in
// registers (element i of a lane is row (w KPT + i) 64 + lane; rows that are kept anyway have the largest key, rows that are not in use
// 0).  The range of the other keys is cut into up to 2048 bins, the bin of the k-th largest again, and so on until all or none of a bin
// is taken: keys are logarithms of the weights, nearly, so two rounds do.  Its time is instructions per row of one compute unit.  A whole
// eviction of rows of 32 bytes, with the keys written out and launch_topk on them / with this kernel, us: 32 x 4352 down to 4096 16.0 /
// 14.2, 128 x 16384 to 1024 28.5 / 21.8, 32 x 32768 to 1024 27.0 / 25.2, to 16384 40.8 / 41.3; with 64 keys per lane 32 x 65536 to 1024
// 36.0 / 41.2, to 8192 29 / 40 (the selection alone), so longer rows go the other way.
constexpr int kEvictThreads = 1024;
template <int KPT>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a)
{
    constexpr int WAVES = kEvictThreads / 64, BINS = 2048, PER = BINS / kEvictThreads;
    __shared__ uint32_t hist[BINS];
    __shared__ uint32_t sh_pick[2], sh_lo[WAVES], sh_hi[WAVES], sh_wave[2][WAVES];
    const int row = blockIdx.x, b = row / a.H_kv, lane = lane_id(), w = wave_id(), tid = threadIdx.x;
    int n = a.lengths ? a.lengths[b] : a.L;
    n = n < 0 ? 0 : n < a.L ? n : a.L;
    if (tid == 0 && row == b * a.H_kv) a.n[b] = n;
    int32_t *out = a.sel + (size_t)row * a.k;
    if (n <= a.k) {
        for (int i = tid; i < a.k; i += kEvictThreads) out[i] = i;
        return;
    }
    const float *weights = a.weights + (size_t)row * a.L;
    uint32_t key[KPT], lo = 0xFFFFFFFFu, hi = 0u;
    const int base = w * KPT * 64 + lane;
    if ((w + 1) * KPT * 64 <= n) {  // (one lane offset for all loads)
        const float *mine = weights + w * KPT * 64;
#pragma unroll
        for (int i = 0; i < KPT; ++i) key[i] = __float_as_uint(mine[64 * i + lane]);
    } else {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int t = base + 64 * i;
            key[i] = __float_as_uint(weights[t < n ? t : n - 1]);
            if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);  // bounds the address registers alive at once
        }
    }
    int base_v = base;  // (the rows' numbers are made again in each phase; all KPT of them would not fit the registers)
    asm volatile("" : "+v"(base_v));
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int t = base_v + 64 * i;
        const uint32_t x = order_key(__uint_as_float(key[i])), y = x < 1u ? 1u : x > 0xFFFFFFFEu ? 0xFFFFFFFEu : x;
        const bool kept = t < a.sink || t >= n - a.recent, used = t < n;
        key[i] = !used ? 0u : kept ? 0xFFFFFFFFu : y;
        lo = used && !kept && y < lo ? y : lo;
        hi = used && !kept && y > hi ? y : hi;
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
    lo = ~wave_all(~lo, UMaxOp());
    hi = wave_all(hi, UMaxOp());
    if (lane == 0) {
        sh_lo[w] = lo;
        sh_hi[w] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        lo = sh_lo[i] < lo ? sh_lo[i] : lo;
        hi = sh_hi[i] > hi ? sh_hi[i] : hi;
    }
    uint32_t rem = (uint32_t)(a.k - a.sink - a.recent);  // of the others (n > k: those that are kept anyway are distinct)
    uint32_t T = 0xFFFFFFFEu, ties = 0;                  // what is above T is taken, and the first `ties` of what is T
    while (rem > 0) {
        const uint32_t span = hi - lo;
        const int bits = 32 - __builtin_clz(span | 1u), shift = bits > 11 ? bits - 11 : 0;
        for (int i = tid; i < BINS; i += kEvictThreads) hist[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (key[i] - lo <= span) atomicAdd(&hist[(key[i] - lo) >> shift], 1u);
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
            if (above < rem && rem <= above + c[i]) {
                sh_pick[0] = PER * tid + i;
                sh_pick[1] = above;
                sh_lo[0] = c[i];
            }
            above += c[i];
        }
        __syncthreads();
        const uint32_t first = lo + (sh_pick[0] << shift), in_bin = sh_lo[0];
        rem -= sh_pick[1];
        if (in_bin == rem || shift == 0) {
            T = in_bin == rem ? first - 1u : first;
            ties = in_bin == rem ? 0u : rem;
            break;
        }
        const uint32_t end = first + ((1u << shift) - 1u);
        hi = end < hi ? end : hi;
        lo = first;
        __syncthreads();  // (the counters and sh_pick are read)
    }
    uint32_t gt = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        gt += (uint32_t)__popcll(__ballot(key[i] > T));
        if (ties) eq += (uint32_t)__popcll(__ballot(key[i] == T));
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
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
    // (the comparisons are made again rather than kept, for the same reason: the compiler must not know that T is the same)
    int base_w = base;
    asm volatile("" : "+v"(T), "+v"(base_w));
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const uint64_t mg = __ballot(key[i] > T), me = ties ? __ballot(key[i] == T) : 0;
        const uint32_t g_at = __builtin_amdgcn_mbcnt_hi((uint32_t)(mg >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mg, gt));
        const uint32_t e_at = __builtin_amdgcn_mbcnt_hi((uint32_t)(me >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)me, eq));
        if (key[i] > T || (ties && key[i] == T && e_at < ties)) out[g_at + (e_at < ties ? e_at : ties)] = base_w + 64 * i;
        gt += (uint32_t)__popcll(mg);
        eq += (uint32_t)__popcll(me);
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
}

// Rows to new places elsewhere: a workgroup per step of rows, z: keys or values.  All of a thread's rows are requested at once; what
// bounds it is the copy.
constexpr int kMoveRows = 8;  // rows per thread and step
template <typename P>
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a, int pieces, int log_threads)
{
    const int row = blockIdx.y, b = row / a.H_kv;
    const int piece = (int)threadIdx.x & ((1 << log_threads) - 1), at_once = 256 >> log_threads, step = at_once * kMoveRows;
    const int32_t *sel = a.sel + (size_t)row * a.k;
    const bool of_v = blockIdx.z;
    const int i0 = (int)blockIdx.x * step, r0 = (int)threadIdx.x >> log_threads;
    int src[kMoveRows];
#pragma unroll
    for (int u = 0; u < kMoveRows; ++u) src[u] = sel[i0 + u * at_once + r0 < a.k ? i0 + u * at_once + r0 : a.k - 1];
    const int n = a.n[b], m = n < a.k ? n : a.k;
    if (i0 < m) {
        const P *from = (const P *)(of_v ? a.V : a.K) + (size_t)row * a.L * pieces + (piece < pieces ? piece : 0);
        P *to = (P *)(of_v ? a.V_out : a.K_out) + (size_t)row * a.L_out * pieces + piece;
        P x[kMoveRows];
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) x[u] = __builtin_nontemporal_load(from + (size_t)src[u] * pieces);  // (any entry of sel is a row)
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            const int i = i0 + u * at_once + r0;
            if (piece < pieces && i < m) __builtin_nontemporal_store(x[u], to + (size_t)i * pieces);
        }
    }
    if (of_v) return;
    for (int i = i0 + (int)threadIdx.x; i < i0 + step && i < a.k; i += 256) {
        const int t = sel[i];
        if (i < m) a.weights_out[(size_t)row * a.L_out + i] = a.weights[(size_t)row * a.L + t];
        if (a.rows_out) a.rows_out[(size_t)row * a.k + i] = i < m ? t : -1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && row == b * a.H_kv && a.lengths_out) a.lengths_out[b] = m;
}

// Rows to new places in the same cache.  A row's new place is never behind its old one, so that a workgroup which takes the rows in
// order and reads a step's rows (and those of the next one, which lie behind everything it writes) before it writes any of them may
// work in place.  z: keys or values, and slices of `width` pieces of the rows, which move independently of each other and make four
// workgroups of a KV head whose rows have 256 bytes.
// A use of a loaded value: it is waited for here.
__device__ __forceinline__ void arrived(u32x4_t &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void arrived(uint32_t &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void arrived(uint16_t &x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void arrived(float &x) { asm volatile("" : "+v"(x)); }

template <typename P>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int pieces, int width, int log_threads)
{
    const int row = blockIdx.y, b = row / a.H_kv, n = a.n[b], m = n < a.k ? n : a.k;
    const bool of_v = blockIdx.z & 1;
    const int in_slice = (int)threadIdx.x & ((1 << log_threads) - 1), piece = (int)(blockIdx.z >> 1) * width + in_slice;
    const bool mine = in_slice < width && piece < pieces;
    const int at_once = 256 >> log_threads, step = at_once * kMoveRows, r0 = (int)threadIdx.x >> log_threads;
    const int32_t *sel = a.sel + (size_t)row * a.k;
    P *rows = (P *)(of_v ? a.V_out : a.K_out) + (size_t)row * a.L * pieces + piece;
    const bool head = blockIdx.z == 0;  // weights and row numbers are moved here
    P x[2][kMoveRows];
    int src[2][kMoveRows];  // -1: nothing to move
    float w[2][kMoveRows];  // of rows i0 + 256 u + threadIdx.x of a step
    int wsrc[2][kMoveRows];
    int later[kMoveRows];  // entries of sel for the step that is read next
    auto look_up = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) later[u] = sel[i0 + u * at_once + r0 < a.k ? i0 + u * at_once + r0 : a.k - 1];
    };
    auto read = [&](int i0, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            const int i = i0 + u * at_once + r0;
            src[s][u] = mine && i < m && later[u] != i ? later[u] : -1;
        }
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            x[s][u] = P{};
            if (src[s][u] >= 0) x[s][u] = rows[(size_t)src[s][u] * pieces];
        }
        look_up(i0 + step);
        if (head) {
#pragma unroll
            for (int u = 0; u < kMoveRows; ++u) {
                const int r = 256 * u + (int)threadIdx.x, i = i0 + r;
                wsrc[s][u] = r < step && i < m ? sel[i] : -1;
                w[s][u] = wsrc[s][u] >= 0 ? a.weights_out[(size_t)row * a.L + wsrc[s][u]] : 0.0f;
            }
        }
    };
    auto write = [&](int i0, int s) __attribute__((always_inline)) {
        // every thread has what it reads in this step before any of them writes (the requests of the next step may be on their way)
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) arrived(x[s][u]);
        if (head) {
#pragma unroll
            for (int u = 0; u < kMoveRows; ++u) arrived(w[s][u]);
        }
        lds_barrier();
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u)
            if (src[s][u] >= 0) rows[(size_t)(i0 + u * at_once + r0) * pieces] = x[s][u];
        if (head) {
#pragma unroll
            for (int u = 0; u < kMoveRows; ++u) {
                const int r = 256 * u + (int)threadIdx.x, i = i0 + r;
                if (r >= step || i >= a.k) continue;
                if (wsrc[s][u] >= 0) a.weights_out[(size_t)row * a.L + i] = w[s][u];
                if (a.rows_out) a.rows_out[(size_t)row * a.k + i] = wsrc[s][u];
            }
        }
    };
    look_up(0);
    read(0, 0);
    for (int i0 = 0; i0 < a.k; i0 += 2 * step) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = i0 + s * step;
            if (at >= a.k) break;
            if (a.k - at > step) read(at + step, s ^ 1);
            write(at, s);
        }
    }
    if (head && threadIdx.x == 0 && row == b * a.H_kv && a.lengths_out) a.lengths_out[b] = m;
}

}  // namespace

bool evict_select_ok(int L) { return L <= 32768; }

hipError_t launch_evict(const xkv_shape &s, const CachePlan &p, const EvictArgs &a, uint32_t *hist, uint32_t *state, hipStream_t st)
{
    const int rows = a.batch * a.H_kv;
    hipError_t e;
    auto select = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(rows), dim3(kEvictThreads), 0, st, a);
        return hipGetLastError();
    };
    if (evict_select_ok(a.L)) {
        e = a.L <= 8192 ? select(evict_select_kernel<8>) : a.L <= 16384 ? select(evict_select_kernel<16>) : select(evict_select_kernel<32>);
    } else {
        hipLaunchKernelGGL(evict_keys_kernel, dim3((a.L + 255) / 256, rows), dim3(256), 0, st, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && !evict_select_ok(a.L)) e = launch_topk(p.sel_shape, p.sel_plan, a.keys, a.sel, hist, state, false, st);
    if (e != hipSuccess) return e;
    const size_t row_bytes = (size_t)a.d_h * (s.dtype == XKV_F32 ? 4 : 2);
    const uintptr_t bits = (uintptr_t)a.K | (uintptr_t)a.V | (uintptr_t)a.K_out | (uintptr_t)a.V_out | row_bytes;
    const bool in_place = a.K_out == a.K;
    auto launch = [&](auto copy, auto move, int piece) {
        const int pieces = (int)(row_bytes / piece);
        // in place: slices of whole 128-byte lines, so that more than two workgroups work on a KV head
        const int width = in_place && row_bytes % 128 == 0 ? 128 / piece : pieces, slices = (pieces + width - 1) / width;
        int log_threads = 0;
        while ((1 << log_threads) < width) ++log_threads;
        const int step = (256 >> log_threads) * kMoveRows;
        if (in_place)
            hipLaunchKernelGGL(move, dim3(1, rows, 2 * slices), dim3(256), 0, st, a, pieces, width, log_threads);
        else
            hipLaunchKernelGGL(copy, dim3((a.k + step - 1) / step, rows, 2), dim3(256), 0, st, a, pieces, log_threads);
        return hipGetLastError();
    };
    return bits % 16 == 0 ? launch(evict_copy_kernel<u32x4_t>, evict_move_kernel<u32x4_t>, 16)
         : s.dtype == XKV_F32 ? launch(evict_copy_kernel<uint32_t>, evict_move_kernel<uint32_t>, 4)
                              : launch(evict_copy_kernel<uint16_t>, evict_move_kernel<uint16_t>, 2);
}

}  // namespace xkv
