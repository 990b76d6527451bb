// Launchers of attention over the paged 4-bit cache for one query type (compiled once with
// -DAASD_DT=0 for fp32 and once with -DAASD_DT=1 for bf16).
#include "aasd_kv_host.h"

#ifndef AASD_DT
#error "compile with -DAASD_DT=0 (fp32) or -DAASD_DT=1 (bf16)"
#endif

namespace aasd {

#if AASD_DT == 0
int launch_kv_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches) {
#else
int launch_kv_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches) {
#endif
    constexpr int DT = AASD_DT;
    (void)sm_count;
    (void)scratch;
    const unsigned int grid = (unsigned int)((a.p.n_tokens * a.p.n_q_heads + 7) / 8);
    if (a.p.head_dim == 64) launch(kv_attend_kernel<DT, 64>, grid, 256u, 0, env.stream, a);
    else if (a.p.head_dim == 128) launch(kv_attend_kernel<DT, 128>, grid, 256u, 0, env.stream, a);
    else launch(kv_attend_kernel<DT, 256>, grid, 256u, 0, env.stream, a);
    *launches = 1;
    return AASD_OK;
}

}  // namespace aasd
