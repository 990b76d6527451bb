// Launchers of attention over the paged 8-bit cache for one query type (compiled once with
// -DAASD_DT=0 for fp32 and once with -DAASD_DT=1 for bf16).
#include "aasd_kvb_attend.cuh"
#include "aasd_kv_host.h"

#ifndef AASD_DT
#error "compile with -DAASD_DT=0 (fp32) or -DAASD_DT=1 (bf16)"
#endif

namespace aasd {

#if AASD_DT == 0
int launch_kvb_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
#else
int launch_kvb_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
#endif
    constexpr int DT = AASD_DT;
    KvAttendArgs a = args;
    *launches = 1;
    const unsigned int grid = (unsigned int)(a.p.n_tokens * a.p.n_q_heads);
    if (a.p.head_dim == 64) launch(kvb_attend_plain_kernel<DT, 64>, grid, 128u, 0, env.stream, a);
    else if (a.p.head_dim == 128) launch(kvb_attend_plain_kernel<DT, 128>, grid, 128u, 0, env.stream, a);
    else launch(kvb_attend_plain_kernel<DT, 256>, grid, 128u, 0, env.stream, a);
    return AASD_OK;
}

}  // namespace aasd
