// Launchers of attention over the paged 8-bit cache for one query type (compiled once with
// -DAASD_DT=0 for fp32 and once with -DAASD_DT=1 for bf16).
#include "aasd_kvb_attend.cuh"
#include "aasd_kv_host.h"
#include "aasd_kvb_tile.cuh"

#ifndef AASD_DT
#error "compile with -DAASD_DT=0 (fp32) or -DAASD_DT=1 (bf16)"
#endif

namespace aasd {

namespace {

// Rows per key/value head up to which the split kernel takes bf16 queries: it goes over the pages once for every 16 rows, but
// shares them among all warps of the device.  Measured with trees over 32 query and 8 key heads of 128 channels, split kernel
// against tiles, graph replays: 64 sequences of 4000 tokens: 16 rows 130 and 178 us, 24 rows 217 and 197 us, 48 rows 313 and 199
// us; 8 of 4000: 16 rows 39 and 43 us, 24 rows 47 and 45 us; one of 16000: 16 rows 35 and 33 us, 24 rows 37 and 35 us.  With 64
// channels, where a page is half as long to fetch: 64 of 4000: 24 rows 119 and 154 us, 32 rows 123 and 156 us; 8 of 4000: 33 and 37, 35
// and 37 us; one of 16000: 27 and 29, 29 and 29 us.  With 256 channels (16 and 4 heads), where the split kernel has eight rows at a time: 64 of
// 4000: 8 rows 127 and 143 us, 16 rows 209 and 149 us; 8 of 4000: 35 and 45, 43 and 48 us; one of 16000: 41 and 37, 38 and 43 us (48 rows: 517 and
// 156, 86 and 51, 55 and 45 us).
constexpr int64_t split_rows(int head_dim) { return head_dim == 64 ? 32 : head_dim == 128 ? 16 : 8; }

template <int DT, int D, int NT>
int launch_split(const LaunchEnv& env, int sm_count, const KvAttendArgs& a) {
    constexpr auto kernel = kvb_attend_split_kernel<DT, D, NT>;
    constexpr size_t smem = sizeof(KvbSplitShared<DT, D, NT>);
    static_assert(smem <= 227 * 1024, "fits an SM");
    if (enable_smem<kernel, smem>(env.device) != AASD_OK) return AASD_ERR_CUDA;
    launch(kernel, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)KvbSplitShape<DT, D, NT>::kThreads, smem, env.stream, a);
    return AASD_OK;
}

#if AASD_DT == 1
template <int D, bool PAIR>
int launch_tile(const LaunchEnv& env, int sm_count, const KvAttendArgs& a) {
    constexpr auto kernel = kvb_attend_tile_kernel<D, PAIR>;
    constexpr size_t smem = sizeof(KvbTileShared<D, PAIR>) + 1024;   // (its first member wants a 1024-byte boundary)
    static_assert(smem <= 227 * 1024, "fits an SM");
    constexpr KvScratch L = kv_attend_scratch(D);
    static_assert((size_t)kKvMaxCtas * 2 * KvbTileShared<D, PAIR>::R * (D + 2) * 4 <= L.off_warp - L.off_cta, "the parts fit the scratch");
    if (enable_smem<kernel, smem>(env.device) != AASD_OK) return AASD_ERR_CUDA;
    // the softmax warps wait for registers that the launch must have brought along
    static const bool enough = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, kernel) == cudaSuccess && f.numRegs >= KvbTileShape<D>::kLaunchRegs;
    }();
    if (!enough) return AASD_ERR_UNSUPPORTED;
    launch(kernel, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)KvbTileShape<D>::kThreads, smem, env.stream, a);
    launch_grid2(kv_tile_join_kernel<D, PAIR>, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)kTileJoinCtas,
                 (unsigned int)kTileJoinThreads, env.stream, a);
    return AASD_OK;
}
#endif

}  // namespace

#if AASD_DT == 0
int launch_kvb_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
#else
int launch_kvb_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
#endif
    constexpr int DT = AASD_DT;
    KvAttendArgs a = args;
    const KvScratch L = kv_attend_scratch(a.p.head_dim);
    char* ws = static_cast<char*>(scratch);
    a.tickets = reinterpret_cast<unsigned int*>(ws);
    a.cta_parts = reinterpret_cast<float*>(ws + L.off_cta);
    a.tile_open = reinterpret_cast<KvTileOpen*>(ws + L.off_open);
    a.warp_parts = reinterpret_cast<float*>(ws + L.off_warp);
    // rows per key/value head that a sequence brings (packed rows: on average)
    const int64_t per_seq = a.p.rows_per_seq > 0 ? a.p.rows_per_seq : (a.p.n_tokens + a.p.n_seqs - 1) / (a.p.n_seqs > 0 ? a.p.n_seqs : 1);
    const int64_t rows = per_seq * (a.p.n_q_heads / a.p.n_kv_heads);
    *launches = 1;
#if AASD_DT == 1
    if (rows > split_rows(a.p.head_dim)) {
        // (Two row tiles of the same pages, or two groups on alternate pages of one.)
        *launches = 2;
        if (a.p.head_dim == 256) return launch_tile<256, false>(env, sm_count, a);
        if (a.p.head_dim == 64) return rows > kTileRows ? launch_tile<64, true>(env, sm_count, a) : launch_tile<64, false>(env, sm_count, a);
        return rows > kTileRows ? launch_tile<128, true>(env, sm_count, a) : launch_tile<128, false>(env, sm_count, a);
    }
#endif
    if (a.p.head_dim == 64)
        return rows > 8 ? launch_split<DT, 64, 2>(env, sm_count, a) : launch_split<DT, 64, 1>(env, sm_count, a);
    if (a.p.head_dim == 128)
        return rows > 8 ? launch_split<DT, 128, 2>(env, sm_count, a) : launch_split<DT, 128, 1>(env, sm_count, a);
    return launch_split<DT, 256, 1>(env, sm_count, a);
}

}  // namespace aasd
