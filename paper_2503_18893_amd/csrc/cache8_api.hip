// C ABI of rotary positions and of the cache held in 8 bits: argument checks, plans, workspace.
#include <cmath>
#include <cstring>

#include "cache8.h"

namespace xkv {

static inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
static inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
static inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
static inline xkv_status hip_status(hipError_t e) { return e == hipSuccess ? XKV_OK : XKV_ERR_HIP; }

namespace {

// Where rows [sequences][tokens][heads] of d numbers lie; false for negative strides.
bool rows_at(const xkv_rows *at, int N, int heads, int d, xkv_rows &r)
{
    r = at ? *at : xkv_rows{(int64_t)N * heads * d, (int64_t)heads * d, d};
    return r.sequence >= 0 && r.token >= 0 && r.head >= 0;
}

// Whether no two rows share a number: in the order of their strides, each reaches beyond all that is inside it.
bool rows_apart(const xkv_rows &r, int batch, int N, int heads, int d)
{
    struct { int64_t stride; int64_t count; } axis[3] = {{r.sequence, batch}, {r.token, N}, {r.head, heads}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (axis[j].stride > axis[j + 1].stride) std::swap(axis[j], axis[j + 1]);
    unsigned __int128 reach = d;
    for (const auto &x : axis) {
        if (x.count <= 1) continue;
        if ((unsigned __int128)x.stride < reach) return false;
        reach += (unsigned __int128)x.stride * (uint64_t)(x.count - 1);
    }
    return reach < ((unsigned __int128)1 << 62);
}

bool same_rows(const xkv_rows &x, const xkv_rows &y, int batch, int N, int heads)
{
    return (batch <= 1 || x.sequence == y.sequence) && (N <= 1 || x.token == y.token) && (heads <= 1 || x.head == y.head);
}

xkv_status check_blocks(const xkv_shape &s, int32_t code, int32_t c, int &shift, int &n_c)
{
    if (code != XKV_E4M3 && code != XKV_INT8) return XKV_ERR_INVALID_ARG;
    if (c < 1) return XKV_ERR_INVALID_ARG;
    if ((c & (c - 1)) != 0 || s.L > (1 << 30)) return XKV_ERR_UNSUPPORTED;
    shift = __builtin_ctz((unsigned)c);
    n_c = ceil_div(s.L, c);
    return XKV_OK;
}

xkv_status plan_cache8(const xkv_shape &s, int N, Cache8Plan &p)
{
    std::memset(&p, 0, sizeof p);
    if (N < 1) return XKV_ERR_INVALID_ARG;
    const long long batch = s.batch > 0 ? s.batch : 1;
    if (s.L > (1 << 30) || batch * N > (1LL << 26) || batch * N * s.H_q > (1LL << 26)) return XKV_ERR_UNSUPPORTED;
    p.n_rep = s.H_q / s.H_kv;
    p.scale = s.scale > 0.0f ? s.scale : 1.0f / std::sqrt((float)s.d_h);
    const long long M = (long long)N * p.n_rep;
    p.mfma = s.d_h == 64 || s.d_h == 128 || s.d_h == 256;
    // Rows of a workgroup.  Two workgroups of the matrix-core kernels to a compute unit, one of 256 rows or channels; four of the general one.
    // (More than 128 rows of 128 channels: 256 that share tiles.  Microseconds by 32 / by 256, 8 KV heads: 64 rows after 32768 rows of the cache 29 / 47, 96
    // 41 / 50, 128 42 / 52, 192 73 / 61; four sequences of up to 65536 rows, 72 rows 132 / 197, 128 171 / 201, 192 243 / 208.  By 16 / by 32, one sequence of 32768 rows, int8:
    // 128 channels, 4 rows 20 / 23, 20 rows 25 / 26, 64 rows 39 / 32, 128 65 / 49; 64 channels 17 / 19, 21 / 21, 30 / 25, 48 / 37; 256 channels, where 32 rows leave
    // no registers for the stream, 32 / 84, 44 / 88, 72 / 146, 129 / 228.  fp32: a query's three terms take the registers of 32 rows; 4, 20, 64 and 256 rows
    // of 128 channels 22, 29, 45 and 135.)
    p.rows = !p.mfma || M <= 16 || s.d_h == 256 || s.dtype == XKV_F32 ? 16 : M <= 128 || s.d_h != 128 ? 32 : 256;
    p.round = p.mfma ? 128 : 64;
    const int slots = !p.mfma ? 1024 : p.rows == 256 || s.d_h == 256 ? 256 : 512;
    const int row_tiles = ceil_div(M, p.rows), longest = ceil_div(s.L, p.round);
    const long long units = (long long)s.H_kv * row_tiles;  // workgroups of a part
    // A cache of up to 512 rows and few queries, or many sequences: one part, whose result needs no merge.  4 heads after 512 rows of 128 channels in bf16 8.0 us, cut 9.2 (16
    // sequences with 32 heads 9.9, cut 13.7); after 1024 rows 11.4 and 9.4 (15.5 and 17.2).
    const bool one = s.L <= 512 && (M <= 64 || units * batch >= 64);
    // Otherwise, where sequences alone do not fill the compute units, parts are cut by the lengths, for which every workgroup looks at those of all
    // queries (unless they are very many).  Four sequences of up to 65536 rows, 1024 rows of queries, 128 tiles of them 777 us, tiles cut in
    // equal parts 1094; 16 of up to 4096, 512 tiles 243, not cut 175.  (Where sequences take most of the slots, or all of them, parts are coarse beside their differences:
    // lengths from 16384 / b to 16384, 8 KV heads, b = 32 4.8 TB/s, 48 4.1, 64 4.8, 80 and more 6.2 to 6.4; 16 4.7, most of which is the start and end of 60 us.)
    p.by_length = !one && units * batch < slots && batch <= kCutBatch && (N == 1 || batch * N <= kCutQueries);
    if (one) {
        p.parts = 1;
    } else if (batch > 1 && p.by_length) {
        // (More of them, so that those of short sequences fill in, do not pay: 16 sequences of 4096 to 65536 rows, 8 KV heads, 197 us, with 1.5 times as
        // many 195, twice 211, three times 198; three of up to 40001, 4 KV heads, 23.9, 26.5, 28.8, 29.2.)
        const long long all = batch * longest, most = all < batch + kMaxCacheParts - 1 ? all : batch + kMaxCacheParts - 1;
        p.parts = clampi((int)(slots / units), (int)batch, (int)most);
    } else {
        // As few as fill the compute units well (one where units alone do that 64 times over).  A part costs about what 4 rounds take beside its own.
        long long best = 0;
        p.parts = 1;
        for (int parts = 1; parts <= kMaxCacheParts && parts <= longest && units * batch * (parts - 1) < 64 * slots; ++parts) {
            const long long time = ((units * batch * parts + slots - 1) / slots) * (ceil_div(longest, parts) + 4);
            if (parts == 1 || time < best) best = time, p.parts = parts;
        }
    }
    // Where there is one part of every row tile, and a workgroup for it also if it has no rows, results leave at once.
    p.direct = p.parts == 1 && (!p.by_length || batch == 1);
    const size_t part_rows = p.direct ? 0 : (size_t)p.parts * (p.by_length ? 1 : batch) * N * s.H_q;
    size_t off = align_up(((size_t)batch + 1) * sizeof(int32_t), 256);
    p.off_part_o = off;
    off = align_up(off + part_rows * s.d_h * sizeof(float), 256);
    p.off_part_ml = off;
    p.total = align_up(off + part_rows * 2 * sizeof(float), 256);
    return XKV_OK;
}

}  // namespace
}  // namespace xkv

using namespace xkv;

extern "C" {

xkv_status xkv_rope_frequencies(int32_t d_rot, float theta, int32_t scaling, float factor, float low, float high, float context,
                                double *frequencies, void *hip_stream)
{
    if (!frequencies || d_rot < 2 || d_rot % 2 || d_rot > 256 || scaling < XKV_ROPE_PLAIN || scaling > XKV_ROPE_TURNS) return XKV_ERR_INVALID_ARG;
    if (!(theta > 0.0f) || !std::isfinite(theta)) return XKV_ERR_INVALID_ARG;
    if (scaling != XKV_ROPE_PLAIN && (!(factor > 0.0f) || !std::isfinite(factor))) return XKV_ERR_INVALID_ARG;
    if (scaling == XKV_ROPE_BASE && d_rot == 2) return XKV_ERR_INVALID_ARG;
    if (scaling == XKV_ROPE_TURNS && (!(low >= 0.0f) || !(high > low) || !std::isfinite(high) || !(context > 0.0f) || !std::isfinite(context)))
        return XKV_ERR_INVALID_ARG;
    return hip_status(launch_rope_frequencies(d_rot, theta, scaling, factor, low, high, context, frequencies, (hipStream_t)hip_stream));
}

xkv_status xkv_rotate(const xkv_shape *shape, int32_t d_rot, int32_t layout, int32_t direction, float amplitude, const double *frequencies,
                      const int32_t *positions, int32_t N, const void *q, const xkv_rows *q_at, void *q_out, const xkv_rows *q_out_at,
                      const void *K, const xkv_rows *K_at, void *K_out, const xkv_rows *K_out_at, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    const xkv_shape &s = *shape;
    if (N < 1 || d_rot < 2 || d_rot % 2 || d_rot > s.d_h || !frequencies) return XKV_ERR_INVALID_ARG;
    if ((layout != XKV_ROPE_HALF && layout != XKV_ROPE_INTERLEAVED) || direction < XKV_ROPE_FORWARD || direction > XKV_ROPE_GRADIENT)
        return XKV_ERR_INVALID_ARG;
    if (!(amplitude >= 0.0f) || !std::isfinite(amplitude) || (amplitude > 0.0f && !std::isfinite(1.0f / amplitude))) return XKV_ERR_INVALID_ARG;
    if (!q != !q_out || !K != !K_out || (!q && !K)) return XKV_ERR_INVALID_ARG;
    if ((long long)s.batch * N > (1LL << 30) || (long long)s.batch * N * ((long long)s.H_q + s.H_kv) > (1LL << 40)) return XKV_ERR_UNSUPPORTED;
    const float m = amplitude > 0.0f ? amplitude : 1.0f;
    RotateArgs a{};
    a.x[0] = q, a.x[1] = K;
    a.y[0] = q_out, a.y[1] = K_out;
    const xkv_rows *in[2] = {q_at, K_at}, *to[2] = {q_out_at, K_out_at};
    for (int i = 0; i < 2; ++i) {
        if (!a.x[i]) continue;
        a.heads[i] = i == 0 ? s.H_q : s.H_kv;
        if (!rows_at(in[i], N, a.heads[i], s.d_h, a.x_at[i]) || !rows_at(to[i], N, a.heads[i], s.d_h, a.y_at[i])) return XKV_ERR_INVALID_ARG;
        if (!rows_apart(a.y_at[i], s.batch, N, a.heads[i], s.d_h)) return XKV_ERR_INVALID_ARG;
        if (a.x[i] == a.y[i] && !same_rows(a.x_at[i], a.y_at[i], s.batch, N, a.heads[i])) return XKV_ERR_INVALID_ARG;
    }
    if (s.batch == 0) return XKV_OK;
    a.positions = positions;
    a.frequencies = frequencies;
    a.batch = s.batch;
    a.N = N;
    a.d_h = s.d_h;
    a.d_rot = d_rot;
    a.amplitude = direction == XKV_ROPE_INVERSE ? 1.0f / m : m;
    a.sign = direction == XKV_ROPE_FORWARD ? 1.0f : -1.0f;
    return hip_status(launch_rotate(s, a, layout == XKV_ROPE_INTERLEAVED, (hipStream_t)hip_stream));
}

xkv_status xkv_cache8_append(const xkv_shape *shape, const void *K, const xkv_rows *K_at, const void *V, const xkv_rows *V_at,
                             const int32_t *lengths, const int32_t *counts, int32_t N, int32_t code, int32_t c, void *K8, void *V8,
                             float *k_scales, float *v_scales, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    const xkv_shape &s = *shape;
    Cache8Append a{};
    if (N < 1 || !K || !V || !K8 || !V8 || !k_scales || !v_scales) return XKV_ERR_INVALID_ARG;
    if ((st = check_blocks(s, code, c, a.shift, a.n_c)) != XKV_OK) return st;
    if (!rows_at(K_at, N, s.H_kv, s.d_h, a.K_at) || !rows_at(V_at, N, s.H_kv, s.d_h, a.V_at)) return XKV_ERR_INVALID_ARG;
    const int most = N < s.L ? N : s.L;  // rows that there is room for
    a.blocks = (int)(((long long)most - 1) / c) + 2 < a.n_c ? (int)(((long long)most - 1) / c) + 2 : a.n_c;
    if ((long long)a.blocks * 2 * s.H_kv * s.batch > 0x7FFFFFFFLL) return XKV_ERR_UNSUPPORTED;
    if (s.batch == 0) return XKV_OK;
    a.K = K, a.V = V;
    a.lengths = lengths;
    a.counts = counts;
    a.K8 = (uint8_t *)K8, a.V8 = (uint8_t *)V8;
    a.k_scales = k_scales, a.v_scales = v_scales;
    a.N = N;
    a.L = s.L;
    a.H_kv = s.H_kv;
    a.d_h = s.d_h;
    a.batch = s.batch;
    return hip_status(launch_cache8_append(s, a, code, (hipStream_t)hip_stream));
}

xkv_status xkv_cache8_workspace_bytes(const xkv_shape *shape, int32_t N, size_t *bytes)
{
    if (!bytes) return XKV_ERR_INVALID_ARG;
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    Cache8Plan p;
    if ((st = plan_cache8(*shape, N, p)) != XKV_OK) return st;
    *bytes = p.total;
    return XKV_OK;
}

xkv_status xkv_cache8_decode(const xkv_shape *shape, const void *K8, const void *V8, const float *k_scales, const float *v_scales,
                             int32_t code, int32_t c, const int32_t *visible, const void *q, int32_t N, void *out, void *workspace,
                             size_t workspace_bytes, void *hip_stream)
{
    xkv_status st = validate(shape);
    if (st != XKV_OK) return st;
    const xkv_shape &s = *shape;
    Cache8Args a{};
    Cache8Plan p;
    if (!K8 || !V8 || !k_scales || !v_scales || !q || !out) return XKV_ERR_INVALID_ARG;
    if ((st = check_blocks(s, code, c, a.shift, a.n_c)) != XKV_OK) return st;
    if ((st = plan_cache8(s, N, p)) != XKV_OK) return st;
    if (!workspace || ((uintptr_t)workspace & 255u)) return XKV_ERR_INVALID_ARG;
    if (workspace_bytes < p.total) return XKV_ERR_WORKSPACE;
    if (s.batch == 0) return XKV_OK;
    a.K8 = (const uint8_t *)K8, a.V8 = (const uint8_t *)V8;
    a.k_scales = k_scales, a.v_scales = v_scales;
    a.q = q;
    a.visible = visible;
    a.out = out;
    a.table = (int32_t *)((char *)workspace + p.off_table);
    if (!p.direct) {
        a.part_o = (float *)((char *)workspace + p.off_part_o);
        a.part_ml = (float *)((char *)workspace + p.off_part_ml);
    }
    a.L = s.L;
    a.H_kv = s.H_kv;
    a.H_q = s.H_q;
    a.d_h = s.d_h;
    a.batch = s.batch;
    a.N = N;
    a.rows = p.rows;
    a.round = p.round;
    a.parts = p.parts;
    a.by_length = p.by_length;
    a.scale = p.scale;
    return hip_status(launch_cache8_attend(s, a, code, p.mfma, (hipStream_t)hip_stream));
}

}  // extern "C"
