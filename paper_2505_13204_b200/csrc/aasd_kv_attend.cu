// Launchers of attention over the paged 4-bit cache for one query type (compiled once with
// -DAASD_DT=0 for fp32 and once with -DAASD_DT=1 for bf16).
#include "aasd_kv_host.h"

#ifndef AASD_DT
#error "compile with -DAASD_DT=0 (fp32) or -DAASD_DT=1 (bf16)"
#endif

namespace aasd {

namespace {

// Rows per key/value head up to which the split kernel takes bf16 queries: it goes over the pages once
// for every 16 rows, but shares them among all warps of the device and fetches nothing a page does not
// hold.  Measured with trees over 32 query and 8 key heads of 128 channels, split kernel against tiles:
//   64 sequences of 4000 tokens: 32 rows 164 and 276 us, 48 rows 235 and 283 us, 64 rows 304 and 276 us; of 2000 tokens:
//   96 rows 245 and 184 us;  8 of 4000: 32 rows 38 and 47 us, 48 rows 49 and 48 us, 96 rows 74 and 50 us;  one of 16000: 16
//   rows 26.6 and 28.3 us, 32 rows 30.0 and 29.0 us.
constexpr int64_t kSplitRows = 48;

template <int DT, int D, int NT>
int launch_split(const LaunchEnv& env, int sm_count, const KvAttendArgs& a) {
    constexpr auto kernel = kv_attend_split_kernel<DT, D, NT>;
    constexpr size_t smem = sizeof(KvSplitShared<DT, D, NT>);
    static_assert(smem <= 227 * 1024, "fits an SM");
    if (enable_smem<kernel, smem>(env.device) != AASD_OK) return AASD_ERR_CUDA;
    launch(kernel, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)KvSplitShape<DT, D, NT>::kThreads, smem, env.stream, a);
    return AASD_OK;
}

#if AASD_DT == 1
template <int D, bool PAIR>
int launch_tile(const LaunchEnv& env, int sm_count, const KvAttendArgs& a) {
    constexpr auto kernel = kv_attend_tile_kernel<D, PAIR>;
    constexpr size_t smem = sizeof(KvTileShared<D, PAIR>) + 1024;   // (its first member wants a 1024-byte boundary)
    static_assert(smem <= 227 * 1024, "fits an SM");
    if (enable_smem<kernel, smem>(env.device) != AASD_OK) return AASD_ERR_CUDA;
    // the softmax warps wait for registers that the launch must have brought along
    static const bool enough = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, kernel) == cudaSuccess && f.numRegs >= kTileLaunchRegs;
    }();
    if (!enough) return AASD_ERR_UNSUPPORTED;
    launch(kernel, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)kTileThreads, smem, env.stream, a);
    launch_grid2(kv_tile_join_kernel<D, PAIR>, (unsigned int)(sm_count < kKvMaxCtas ? sm_count : kKvMaxCtas), (unsigned int)kTileJoinCtas,
                 (unsigned int)kTileJoinThreads, env.stream, a);
    return AASD_OK;
}
#endif

}  // namespace

#if AASD_DT == 0
int launch_kv_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
#else
int launch_kv_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& args, void* scratch, int* launches) {
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
    if (rows > kSplitRows && a.p.head_dim <= 128) {
        // Two row tiles of the same pages, or two groups on alternate pages of one: with 8 sequences of 4000 tokens the pair
        // takes 55.0 us for 128 rows and 58.8 us for 132, the single tile 51.8 and 82.0 us (64 of 2000: 196 and 195 us, and 184 and 328).
        *launches = 2;
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
