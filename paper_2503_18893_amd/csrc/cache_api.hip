// C ABI of the calls on an uncompressed cache that grows and shrinks: argument checks, plans, workspace, launch order.
#include <cmath>
#include <cstring>

#include "cache.h"

namespace xkv {

static inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
static inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
static inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
template <typename T> static inline T *at(void *ws, size_t off) { return reinterpret_cast<T *>((char *)ws + off); }
static inline xkv_status hip_status(hipError_t e) { return e == hipSuccess ? XKV_OK : XKV_ERR_HIP; }

constexpr int kMaxDraft = 1024;        // drafted tokens of a sequence
constexpr int kMaxBlocks = kMaxCacheParts * (kPartBlocks - 128);  // blocks of a query, as many as all parts of the longest round hold, for any type
constexpr int kMaxPlaces = 1 << 30;    // rows and drafted tokens of a sequence: sums of two places are ints

// Scratch of launch_topk for p.sel_shape, and room for what it selects from and for the ids.
static size_t plan_selection(CachePlan &p, size_t off)
{
    make_plan(p.sel_shape, p.sel_plan);
    const Plan &q = p.sel_plan;
    const size_t rows = (size_t)(q.rows > 0 ? q.rows : 1);
    p.off_hist = off;
    off = align_up(off + rows * q.topk_chunks * kTopkLevels * kTopkBins * sizeof(uint32_t), 256);
    p.off_state = off;
    off = align_up(off + rows * (kStateWords + kTopkLevels * kTopkBins + q.topk_chunks) * sizeof(uint32_t), 256);
    p.off_keys = off;
    off = align_up(off + rows * p.sel_shape.L * sizeof(float), 256);
    p.off_sel = off;
    return align_up(off + rows * p.sel_shape.k * sizeof(int32_t), 256);
}

xkv_status plan_cache_attend(const xkv_shape &s, CacheMode mode, int N, int c, CachePlan &p)
{
    std::memset(&p, 0, sizeof p);
    if (N < 1) return XKV_ERR_INVALID_ARG;
    if (mode == CacheMode::tree && N > kMaxDraft) return XKV_ERR_UNSUPPORTED;
    p.n_rep = s.H_q / s.H_kv;
    p.words = ceil_div(N, 32);
    p.scale = s.scale > 0.0f ? s.scale : 1.0f / std::sqrt((float)s.d_h);
    const long long batch = s.batch > 0 ? s.batch : 1;
    // One limit for all calls.  It is needed where blocks are selected by launch_topk or scored by block_scores_kernel: rows are y, queries z of a grid.
    if (batch * N * s.H_kv > 65535LL) return XKV_ERR_UNSUPPORTED;
    if ((long long)s.L + N > kMaxPlaces) return XKV_ERR_UNSUPPORTED;
    size_t off = 0;
    long long most = s.L + (mode == CacheMode::tree ? N : 0);  // tokens of a query
    if (mode == CacheMode::blocks) {
        if (c < 1) return XKV_ERR_INVALID_ARG;
        p.n_c = ceil_div(s.L, c);
        p.k_ch = ceil_div(s.k, c) < p.n_c ? ceil_div(s.k, c) : p.n_c;
        if ((long long)p.k_ch * c < most) most = (long long)p.k_ch * c;
        if ((long long)p.k_ch * c > kMaxPlaces || p.k_ch > kMaxBlocks) return XKV_ERR_UNSUPPORTED;
        p.sel_shape = xkv_shape{1, s.H_kv, s.H_kv, 1, 1, 1, p.n_c, p.k_ch, (int32_t)(batch * N), XKV_F32, 1.0f};
        if (block_select_ok(p.n_c)) {
            const size_t rows = (size_t)batch * N * s.H_kv;
            p.off_keys = off;
            off = align_up(off + rows * p.n_c * sizeof(float), 256);
            p.off_reach = off;
            off = align_up(off + rows * ceil_div(p.n_c, 16) * sizeof(float), 256);
            p.off_sel = off;
            off = align_up(off + rows * p.k_ch * sizeof(int32_t), 256);
        } else {
            off = plan_selection(p, off);
        }
    }
    // The matrix-core kernel: as many rows per workgroup as there are, up to 256 (128 where that leaves fewer of them empty), one workgroup
    // to a compute unit (two of 128 rows).  The general one: 16 rows, rounds of 64 tokens, four workgroups.  384 rows by 128 / by 256, us:
    // one sequence of 32768 tokens 99 / 103, four of 65536 571 / 680, two of 9457 73 / 65, two of 1000 28 / 29; 640 rows, 32768 tokens 161 /
    // 226; 260 rows, 32768 tokens 91 / 93, 280 rows of four sequences 302 / 350; 512 rows of four sequences 728 / 716.
    const int M = mode == CacheMode::blocks ? p.n_rep : N * p.n_rep;
    p.mfma = s.dtype == XKV_BF16 && s.d_h == 128;
    p.rows = !p.mfma || M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : (ceil_div(M, 128) & 1) ? 128 : 256;
    p.round = p.mfma && p.rows <= 64 ? 128 : 64;
    int want = !p.mfma ? 1024 : p.rows == 128 ? 512 : 256;
    // Streams (up to 64 rows) of several sequences, whose lengths differ: up to three workgroups one after the other on a compute unit, so
    // that those of short sequences fill in, where each has 8192 tokens; a workgroup costs about 5 us beside its tokens.  Up to 65536
    // tokens of 16 sequences with 8 KV heads: 488 us with one, 460 with two, 454 with three, 464 with six; one sequence of 32768 tokens 36, 42, 47.
    if (p.mfma && p.rows <= 64 && mode != CacheMode::blocks && batch > 1) want *= clampi((int)(batch * s.H_kv * most / (256 * 8192)), 1, 3);
    const long long tiles = (long long)s.H_kv * ceil_div(M, p.rows);
    const int longest = ceil_div(most, p.round);  // parts that the longest sequence can have
    if (mode == CacheMode::blocks) {
        p.parts = clampi(ceil_div(want, tiles * batch * N), 1, clampi(longest, 1, kMaxCacheParts));
        // (a part is a multiple of the round: blocks of few rows, up to a round more of them)
        const int least = ceil_div(p.k_ch, kPartBlocks - p.round);  // (at most kMaxCacheParts)
        if (p.parts < least) p.parts = least;
    } else {
        const long long all = batch * longest;
        p.parts = clampi(ceil_div(want, tiles), (int)batch, (int)(all < (1 << 30) ? all : 1 << 30));
        if (p.parts > batch + kMaxCacheParts - 1) p.parts = (int)batch + kMaxCacheParts - 1;
    }
    const long long part_rows = mode == CacheMode::blocks ? batch * N * p.parts * s.H_q : (long long)p.parts * N * s.H_q;
    p.off_table = off;
    off = align_up(off + ((size_t)batch + 1) * sizeof(int32_t), 256);
    if (mode == CacheMode::weights) {
        p.off_logits = off;
        off = align_up(off + (size_t)batch * s.H_q * s.L * sizeof(float), 256);
    }
    p.off_part_o = off;
    off = align_up(off + (size_t)part_rows * s.d_h * sizeof(float), 256);
    p.off_part_ml = off;
    p.total = align_up(off + (size_t)part_rows * 2 * sizeof(float), 256);
    return XKV_OK;
}

xkv_status plan_evict(const xkv_shape &s, CachePlan &p)
{
    std::memset(&p, 0, sizeof p);
    if (s.L > kMaxPlaces) return XKV_ERR_UNSUPPORTED;
    p.sel_shape = xkv_shape{1, s.H_kv, s.H_kv, 1, 1, 1, s.L, s.k, s.batch > 0 ? s.batch : 1, XKV_F32, 1.0f};
    if (evict_select_ok(s.L))
        p.off_n = align_up((size_t)p.sel_shape.batch * s.H_kv * s.k * sizeof(int32_t), 256);  // the rows, at 0
    else
        p.off_n = plan_selection(p, 0);
    p.total = align_up(p.off_n + (size_t)p.sel_shape.batch * sizeof(int32_t), 256);
    return XKV_OK;
}

namespace {

xkv_status check_workspace(void *ws, size_t bytes, size_t need)
{
    if (!ws || ((uintptr_t)ws & 255u)) return XKV_ERR_INVALID_ARG;
    return bytes < need ? XKV_ERR_WORKSPACE : XKV_OK;
}

CacheArgs attend_args(const xkv_shape &s, const CachePlan &p, const void *K, const void *V, const int32_t *lengths, const void *q, int N,
                      void *out, void *ws)
{
    CacheArgs a{};
    a.K = K;
    a.V = V;
    a.q = q;
    a.lengths = lengths;
    a.out = out;
    a.part_o = at<float>(ws, p.off_part_o);
    a.part_ml = at<float>(ws, p.off_part_ml);
    a.L = s.L;
    a.H_kv = s.H_kv;
    a.H_q = s.H_q;
    a.d_h = s.d_h;
    a.batch = s.batch;
    a.N = N;
    a.words = p.words;
    a.k_ch = p.k_ch;
    a.table = at<int32_t>(ws, p.off_table);
    a.rows = p.rows;
    a.round = p.round;
    a.parts = p.parts;
    a.mfma = p.mfma;
    a.scale = p.scale;
    return a;
}

}  // namespace
}  // namespace xkv

using namespace xkv;

extern "C" {

xkv_status xkv_cache_workspace_bytes(const xkv_shape *shape, int32_t N, int32_t c, size_t *bytes)
{
    if (!bytes) return XKV_ERR_INVALID_ARG;
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    if (N < 1 || c < 0) return XKV_ERR_INVALID_ARG;
    CachePlan p;
    size_t most = 0;
    auto take = [&](xkv_status got) {
        if (got == XKV_OK && p.total > most) most = p.total;
        return got;
    };
    take(plan_evict(*shape, p));
    if ((st = take(plan_cache_attend(*shape, CacheMode::weights, 1, 0, p))) != XKV_OK) return st;
    if (c > 0) {
        if ((st = take(plan_cache_attend(*shape, CacheMode::blocks, N, c, p))) != XKV_OK) return st;
        if (N <= kMaxDraft) take(plan_cache_attend(*shape, CacheMode::tree, N, 0, p));
    } else if ((st = take(plan_cache_attend(*shape, CacheMode::tree, N, 0, p))) != XKV_OK) {
        return st;
    }
    *bytes = most;
    return XKV_OK;
}

xkv_status xkv_tree_decode(const xkv_shape *shape, const void *K, const void *V, const int32_t *lengths, const void *q,
                           const void *K_draft, const void *V_draft, const int32_t *tree, int32_t N, void *out, void *workspace,
                           size_t workspace_bytes, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    CachePlan p;
    if ((st = plan_cache_attend(*shape, CacheMode::tree, N, 0, p)) != XKV_OK) return st;
    if (!K || !V || !q || !K_draft || !V_draft || !out) return XKV_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes, p.total)) != XKV_OK) return st;
    if (shape->batch == 0) return XKV_OK;
    CacheArgs a = attend_args(*shape, p, K, V, lengths, q, N, out, workspace);
    a.K_draft = K_draft;
    a.V_draft = V_draft;
    a.tree = reinterpret_cast<const uint32_t *>(tree);
    return hip_status(launch_cache_attend(CacheMode::tree, *shape, a, (hipStream_t)hip_stream));
}

xkv_status xkv_block_decode(const xkv_shape *shape, const void *K, const void *V, const int32_t *visible, const void *q, int32_t N,
                            const void *landmarks, int32_t c, void *out, int32_t *blocks_out, void *workspace, size_t workspace_bytes,
                            void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    CachePlan p;
    if ((st = plan_cache_attend(*shape, CacheMode::blocks, N, c, p)) != XKV_OK) return st;
    if (!K || !V || !q || !landmarks || !out) return XKV_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes, p.total)) != XKV_OK) return st;
    if (shape->batch == 0) return XKV_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    CacheArgs a = attend_args(*shape, p, K, V, visible, q, N, out, workspace);
    a.c = c;
    float *scores = at<float>(workspace, p.off_keys);
    int32_t *sel = blocks_out ? blocks_out : at<int32_t>(workspace, p.off_sel);
    a.sel = sel;
    hipError_t e;
    if (block_select_ok(p.n_c)) {
        e = launch_block_select(*shape, a, landmarks, p.n_c, scores, at<float>(workspace, p.off_reach), sel, stream);
    } else {
        e = launch_block_scores(*shape, a, landmarks, p.n_c, scores, stream);
        if (e == hipSuccess)
            e = launch_topk(p.sel_shape, p.sel_plan, scores, sel, at<uint32_t>(workspace, p.off_hist), at<uint32_t>(workspace, p.off_state), false,
                            stream);
    }
    if (e == hipSuccess) e = launch_cache_attend(CacheMode::blocks, *shape, a, stream);
    return hip_status(e);
}

xkv_status xkv_landmarks_update(const xkv_shape *shape, const void *K, const int32_t *lengths, int32_t N, int32_t c, void *landmarks,
                                void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    if (N < 1 || c < 1 || !K || !landmarks) return XKV_ERR_INVALID_ARG;
    if (shape->L > kMaxPlaces) return XKV_ERR_UNSUPPORTED;
    if (shape->batch == 0) return XKV_OK;
    return hip_status(launch_landmarks_update(*shape, K, lengths, N, c, landmarks, (hipStream_t)hip_stream));
}

xkv_status xkv_dense_decode_weights(const xkv_shape *shape, const void *K, const void *V, const int32_t *lengths, const void *q, void *out,
                                    float *weights, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    CachePlan p;
    if ((st = plan_cache_attend(*shape, CacheMode::weights, 1, 0, p)) != XKV_OK) return st;
    if (!K || !V || !q || !out || !weights) return XKV_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes, p.total)) != XKV_OK) return st;
    if (shape->batch == 0) return XKV_OK;
    CacheArgs a = attend_args(*shape, p, K, V, lengths, q, 1, out, workspace);
    a.logits = at<float>(workspace, p.off_logits);
    a.weights = weights;
    return hip_status(launch_cache_attend(CacheMode::weights, *shape, a, (hipStream_t)hip_stream));
}

xkv_status xkv_evict(const xkv_shape *shape, const void *K, const void *V, const float *weights, const int32_t *lengths, int32_t sink,
                     int32_t recent, int32_t L_out, void *K_out, void *V_out, float *weights_out, int32_t *rows_out, int32_t *lengths_out,
                     void *workspace, size_t workspace_bytes, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    if (!K || !V || !weights || !K_out || !V_out || !weights_out) return XKV_ERR_INVALID_ARG;
    if (sink < 0 || recent < 0 || (long long)sink + recent > shape->k || L_out < shape->k) return XKV_ERR_INVALID_ARG;
    // in place: all of it, with the same room for rows
    const bool in_place = K_out == K || V_out == V || weights_out == weights;
    if (in_place && (K_out != K || V_out != V || weights_out != weights || L_out != shape->L)) return XKV_ERR_INVALID_ARG;
    CachePlan p;
    if ((st = plan_evict(*shape, p)) != XKV_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes, p.total)) != XKV_OK) return st;
    if (shape->batch == 0) return XKV_OK;
    const EvictArgs a{K, V, weights, lengths, K_out, V_out, weights_out, rows_out, lengths_out, at<float>(workspace, p.off_keys),
                      at<int32_t>(workspace, p.off_sel), at<int32_t>(workspace, p.off_n), shape->L, L_out, shape->H_kv, shape->d_h, shape->k,
                      sink, recent, shape->batch};
    return hip_status(launch_evict(*shape, p, a, at<uint32_t>(workspace, p.off_hist), at<uint32_t>(workspace, p.off_state),
                                   (hipStream_t)hip_stream));
}

}  // extern "C"
