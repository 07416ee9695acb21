// Prints what plan_cache_attend decides for lines "mode H_kv H_q d_h L k batch dtype N c" on stdin (mode 0 tree, 1 weights, 2 blocks), as
// name=value pairs.  Linked with the library's objects by tests/test_cache_plan.py; host only.
#include <cstdio>

#include "cache.h"

int main()
{
    int mode, N, c;
    xkv_shape s{1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 0.0f};
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &mode, &s.H_kv, &s.H_q, &s.d_h, &s.L, &s.k, &s.batch, &s.dtype, &N, &c) == 10) {
        xkv::CachePlan p;
        const int status = xkv::plan_cache_attend(s, (xkv::CacheMode)mode, N, c, p);
        std::printf("status=%d mfma=%d rows=%d round=%d parts=%d k_ch=%d n_c=%d total=%zu max_parts=%d part_blocks=%d\n", status, (int)p.mfma, p.rows,
                    p.round, p.parts, p.k_ch, p.n_c, p.total, xkv::kMaxCacheParts, xkv::kPartBlocks);
    }
    return 0;
}
