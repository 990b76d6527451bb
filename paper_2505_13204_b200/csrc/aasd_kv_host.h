// Host-side internals of the paged caches (4 and 8 bits), shared by the files that launch their kernels.
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
    const size_t part = 2 * kTileRows * ((D < 128 ? D : 128) + 2);   // the largest: two tiles of 128 rows (one with head_dim 256)
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

inline bool kv_head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }
inline bool kv_dtype_ok(int d) { return d == AASD_F32 || d == AASD_BF16; }
inline size_t kv_elt_size(int dtype) { return dtype == AASD_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether two arrays have a byte in common.
inline bool overlap(const void* x, int64_t x_bytes, const void* y, int64_t y_bytes) {
    const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
    return x != nullptr && y != nullptr && x_bytes > 0 && y_bytes > 0 && a < b + (uintptr_t)y_bytes && b < a + (uintptr_t)x_bytes;
}

// Calls f with the head dimension, or the type, as a constant.
template <class F>
void with_dim(int head_dim, F&& f) {
    if (head_dim == 64) f(std::integral_constant<int, 64>());
    else if (head_dim == 128) f(std::integral_constant<int, 128>());
    else f(std::integral_constant<int, 256>());
}
template <class F>
void with_type(int dtype, F&& f) {
    if (dtype == AASD_F32) f(std::integral_constant<int, AASD_F32>());
    else f(std::integral_constant<int, AASD_BF16>());
}

// What calls on either cache check alike (aasd_kv.cu).
struct KvCommitArgs;
int kv_check_write(const aasd_kv_write_params& p, int64_t n_tokens);
int kv_prepare_attend(aasd_ctx* ctx, const void* q, const void* pages, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len,
                      const int32_t* tok_offsets, const int32_t* node_parent, const aasd_kv_attend_params* p, void* workspace, size_t workspace_bytes,
                      const aasd_kv_attend_out* o, KvAttendArgs& a);
int kv_prepare_commit(aasd_ctx* ctx, void* pages, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len, const int32_t* tok_offsets,
                      const int32_t* best_node, const int32_t* node_parent, const aasd_kv_commit_params* p, int32_t* new_len, int64_t head_bytes,
                      KvCommitArgs& a);
int kv_check_read(aasd_ctx* ctx, const void* pages, const int32_t* slots, int64_t n, int32_t n_pages, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                  const void* k_out, const void* v_out);

int launch_kv_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);
int launch_kv_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);
int launch_kvb_attend_f32(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);
int launch_kvb_attend_bf16(const LaunchEnv& env, int sm_count, const KvAttendArgs& a, void* scratch, int* launches);

}  // namespace aasd
