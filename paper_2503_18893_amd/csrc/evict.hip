// Eviction from an uncompressed cache: of every KV head's rows the first `sink`, the last `recent` and those of the largest
// accumulated weight are kept, k altogether, in their order (cache.h).
#include "cache.h"

namespace xkv {
namespace {

// What the selection goes by: the weight, +inf for rows that are kept anyway, and below every number for rows that are not in use.
__global__ __launch_bounds__(256) void evict_keys_kernel(EvictArgs a)
{
    const int t = blockIdx.x * 256 + threadIdx.x, row = blockIdx.y, b = row / a.H_kv;
    int n = a.lengths ? a.lengths[b] : a.L;
    n = n < 0 ? 0 : n < a.L ? n : a.L;
    if (t == 0 && row == b * a.H_kv) a.n[b] = n;
    if (t >= a.L) return;
    const size_t at = (size_t)row * a.L + t;
    a.keys[at] = t >= n ? -INFINITY : (t < a.sink || t >= n - a.recent) ? INFINITY : a.weights[at];
}

// Rows to their new places.  A row's new place is never behind its old one, so that a workgroup which takes the rows in order and
// reads a step's rows before it writes any of them may work in place; elsewhere steps are workgroups of their own.
template <typename P>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int pieces)
{
    constexpr int STEP = 8;  // pieces per thread and step
    const int row = blockIdx.y, b = row / a.H_kv, n = a.n[b], m = n < a.k ? n : a.k;
    const int32_t *sel = a.sel + (size_t)row * a.k;
    const P *Ks = (const P *)a.K + (size_t)row * a.L * pieces, *Vs = (const P *)a.V + (size_t)row * a.L * pieces;
    P *Kd = (P *)a.K_out + (size_t)row * a.L_out * pieces, *Vd = (P *)a.V_out + (size_t)row * a.L_out * pieces;
    const long long all = (long long)m * pieces;
    for (long long p0 = (long long)blockIdx.x * 256 * STEP; p0 < all; p0 += (long long)gridDim.x * 256 * STEP) {
        P k[STEP], v[STEP];
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            const long long p = p0 + u * 256 + threadIdx.x;
            if (p < all) {
                const size_t from = (size_t)sel[p / pieces] * pieces + p % pieces;
                k[u] = Ks[from];
                v[u] = Vs[from];
            }
        }
        XKV_WAIT_VMCNT(0);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            const long long p = p0 + u * 256 + threadIdx.x;
            if (p < all) {
                Kd[p] = k[u];
                Vd[p] = v[u];
            }
        }
    }
    if (blockIdx.x > 0) return;
    for (int i0 = 0; i0 < a.k; i0 += 256) {
        const int i = i0 + threadIdx.x;
        const bool real = i < m;
        const float x = real ? a.weights[(size_t)row * a.L + sel[i]] : 0.0f;
        XKV_WAIT_VMCNT(0);
        __syncthreads();
        if (real) a.weights_out[(size_t)row * a.L_out + i] = x;
        if (i < a.k && a.rows_out) a.rows_out[(size_t)row * a.k + i] = real ? sel[i] : -1;
    }
    if (threadIdx.x == 0 && row == b * a.H_kv && a.lengths_out) a.lengths_out[b] = m;
}

}  // namespace

hipError_t launch_evict(const xkv_shape &s, const CachePlan &p, const EvictArgs &a, uint32_t *hist, uint32_t *state, hipStream_t st)
{
    const int rows = a.batch * a.H_kv;
    hipLaunchKernelGGL(evict_keys_kernel, dim3((a.L + 255) / 256, rows), dim3(256), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = launch_topk(p.sel_shape, p.sel_plan, a.keys, a.sel, hist, state, false, st);
    if (e != hipSuccess) return e;
    const size_t row_bytes = (size_t)a.d_h * (s.dtype == XKV_F32 ? 4 : 2);
    const uintptr_t bits = (uintptr_t)a.K | (uintptr_t)a.V | (uintptr_t)a.K_out | (uintptr_t)a.V_out | row_bytes;
    const bool in_place = a.K_out == a.K || a.V_out == a.V || a.weights_out == a.weights;
    auto launch = [&](auto kernel, int piece) {
        const int pieces = (int)(row_bytes / piece);
        const long long steps = ((long long)a.k * pieces + 2047) / 2048;
        hipLaunchKernelGGL(kernel, dim3(in_place ? 1 : (unsigned)steps, rows), dim3(256), 0, st, a, pieces);
        return hipGetLastError();
    };
    return bits % 16 == 0 ? launch(evict_move_kernel<uint4>, 16) : s.dtype == XKV_F32 ? launch(evict_move_kernel<uint32_t>, 4)
                                                                                        : launch(evict_move_kernel<uint16_t>, 2);
}

}  // namespace xkv
