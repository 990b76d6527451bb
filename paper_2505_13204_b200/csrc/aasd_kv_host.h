// Host-side internals of the paged 4-bit cache, shared by aasd_kv.cu and aasd_kv_attend.cu.
#pragma once

#include <initializer_list>
#include <type_traits>

#include "aasd_host.h"
#include "aasd_kv.cuh"
#include "aasd_kv_attend.cuh"
#include "aasd_kv_tile.cuh"

namespace aasd {

// Scratch of the attention kernels: tickets (zero between calls), then per CTA two partial
// results, then per warp one.
struct KvScratch {
    size_t zero_bytes, off_open, off_cta, off_warp, bytes;
};
constexpr KvScratch kv_attend_scratch(int head_dim) {
    KvScratch L{};
    // a scratch for one head dimension serves the smaller ones too
    const size_t D = (size_t)head_dim, W = 12;
    const size_t part = 2 * kTileRows * ((D < 128 ? D : 128) + 2);   // the largest: two tiles of 128 rows (head_dim 256 has parts of 8 rows)
    L.zero_bytes = align_up(4 * kKvMaxCtas, 256);
    L.off_open = L.zero_bytes;
    L.off_cta = align_up(L.off_open + kKvMaxCtas * sizeof(KvTileOpen), 256);
    L.off_warp = align_up(L.off_cta + kKvMaxCtas * 2 * part * 4, 256);
    L.bytes = align_up(L.off_warp + kKvMaxCtas * W * 16 * (D + 4) * 4, 256);
    return L;
}

// A launch with a second grid dimension (see launch()).
template <class... Params, class... Args>
void launch_grid2(void (*kernel)(Params...), unsigned int gx, unsigned int gy, unsigned int block, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(gx, gy, 1);
    cfg.blockDim = dim3(block, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    cfg.attrs = attr;
    cudaLaunchKernelEx(&cfg, kernel, Params(args)...);   // errors surface in cudaGetLastError
}

int launch_kv_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);
int launch_kv_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);

}  // namespace aasd
