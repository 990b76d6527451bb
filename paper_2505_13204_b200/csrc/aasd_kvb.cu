// Host side of the paged 8-bit cache (aasd_kvb_* in include/aasd.h) and the kernels of aasd_kvb.cuh; the
// attention kernels are launched from aasd_kvb_attend.cu.
#define AASD_KVB_TU 1
#include "aasd_host.h"
#include "aasd_kv_host.h"
#include "aasd_kvb.cuh"

using namespace aasd;

extern "C" {

int aasd_kvb_head_bytes(int32_t head_dim, size_t* bytes) {
    if (bytes == nullptr) return AASD_ERR_INVALID_ARG;
    if (!kv_head_dim_ok(head_dim)) return AASD_ERR_UNSUPPORTED;
    *bytes = (size_t)kvb_head_bytes(head_dim);
    return AASD_OK;
}

int aasd_kvb_write(aasd_ctx* ctx, const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight, const float* cos_sin,
                   const int32_t* positions, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len,
                   const int32_t* tok_offsets, int64_t n_tokens, const aasd_kvb_write_params* params, void* pages, void* q_out, void* k_out) {
    TraceRange trace("aasd_kvb_write");
    if (ctx == nullptr || params == nullptr) return AASD_ERR_INVALID_ARG;
    const aasd_kv_write_params* p = &params->rows;
    if (const int rc = kv_check_write(*p, n_tokens)) return rc;
    const int hq = p->n_q_heads, hkv = p->n_kv_heads, D = p->head_dim, B = params->n_seqs;
    if (B < 0 || params->max_pages < 1 || params->max_pages > 0x7FFFFFFF / kPage || params->rows_per_seq < 0 || n_tokens > 0x7FFFFFFFLL)
        return AASD_ERR_BAD_SHAPE;
    if (params->rows_per_seq > 0 && (int64_t)B * params->rows_per_seq != n_tokens) return AASD_ERR_BAD_SHAPE;
    if (n_tokens == 0 || hq + hkv == 0) return AASD_OK;
    if (!positions || (p->rotary_dim > 0 && !cos_sin)) return AASD_ERR_INVALID_ARG;
    if (hq > 0 && (!q || !q_out)) return AASD_ERR_INVALID_ARG;
    if (hkv > 0 && (!k || !v || !pages || !aligned16(pages))) return AASD_ERR_INVALID_ARG;
    if (hkv > 0 && B > 0 && (!block_table || !cached_len || !kv_len || (params->rows_per_seq == 0 && !tok_offsets))) return AASD_ERR_INVALID_ARG;
    const size_t es = kv_elt_size(p->dtype);
    for (const void* x : {q, k, v, q_weight, k_weight, (const void*)q_out, (const void*)k_out})
        if (((uintptr_t)x % es) != 0) return AASD_ERR_INVALID_ARG;
    // Rows are read by the lanes that write them, other rows in no order with them: an output lies where its own rows lie, or apart.
    struct Rows {
        const void* at;
        int64_t stride, bytes;   // elements between rows; bytes from the first element to behind the last
    };
    const auto rows = [&](const void* x, int64_t stride, int heads) {
        const int64_t n = (int64_t)heads * D;
        return Rows{x, stride, n == 0 ? 0 : ((n_tokens - 1) * stride + n) * (int64_t)es};
    };
    const auto apart = [](const Rows& x, const Rows& y) { return !overlap(x.at, x.bytes, y.at, y.bytes); };
    const auto in_place = [&](const Rows& out, const Rows& in) { return out.at == in.at && (n_tokens == 1 || in.stride == out.stride); };
    const Rows qi = rows(q, p->q_stride, hq), ki = rows(k, p->k_stride, hkv), vi = rows(v, p->v_stride, hkv);
    const Rows qo = rows(q_out, (int64_t)hq * D, hq), ko = rows(k_out, (int64_t)hkv * D, hkv);
    if (!(apart(qo, qi) || in_place(qo, qi)) || !(apart(ko, ki) || in_place(ko, ki)) || !apart(qo, ki) || !apart(qo, vi) || !apart(ko, qi) || !apart(ko, vi) ||
        !apart(qo, ko))
        return AASD_ERR_INVALID_ARG;
    KvbWriteArgs a{};
    a.w = KvWriteArgs{q, k, v, q_weight, k_weight, cos_sin, positions, nullptr, n_tokens, *p, static_cast<uint8_t*>(pages), q_out, k_out,
                      ctx->state, 0u, make_float2(-0.f, -0.f)};
    a.block_table = block_table;
    a.cached_len = cached_len;
    a.kv_len = kv_len;
    a.tok_offsets = tok_offsets;
    a.n_seqs = B;
    a.max_pages = params->max_pages;
    a.rows_per_seq = params->rows_per_seq;
    // 16-byte accesses where every row of every operand starts on a 16-byte boundary
    bool vec = p->rotary_dim == 0 || aligned16(cos_sin);
    for (const void* x : {q, k, v, q_weight, k_weight, (const void*)q_out, (const void*)k_out}) vec = vec && aligned16(x);
    if (hq > 0) vec = vec && (p->q_stride * es) % 16 == 0;
    if (hkv > 0) vec = vec && (p->k_stride * es) % 16 == 0 && (p->v_stride * es) % 16 == 0;
    const bool full = p->rotary_dim == D && !(p->flags & AASD_KV_ROPE_INTERLEAVED);
    const int lanes = D / 16;
    const int64_t units = hkv > 0 && B > 0 ? (n_tokens / kPage + 2 * (int64_t)B) * hkv * 2 : 0;
    const int64_t query_blocks = (n_tokens * hq * lanes + kByteThreads - 1) / kByteThreads;
    if (units > 0x7FFFFFFFLL || query_blocks > 0x3FFFFFFFLL) return AASD_ERR_BAD_SHAPE;
    if (units + query_blocks == 0) return AASD_OK;
    a.units = (unsigned int)units;
    // A warp for each page, head and half, or a CTA.  A CTA holds a page's rows in registers, but most of its warps idle with few rows;
    // a warp goes through its rows twice, four of 128 channels at a time.  A CTA where all of them run at once, or with more
    // than 32 rows per sequence.  Measured with 32 query and 8 key heads of 128 channels, warps against CTAs, in us (read-back included,
    // 5 to 12): 64 sequences of 1 row 16 and 25, 8 rows 18 and 27, 16 rows 25 and 31, 33 rows 39 and 39, 64 rows 57 and 55;
    // 4 sequences of 1 row 12 and 12, 8 rows 14 and 12, 33 rows 27 and 14, 128 rows 41 and 16.
    AASD_CUDA(cudaSetDevice(ctx->device));
    with_type(p->dtype, [&](auto dt) {
        with_dim(D, [&](auto d) {
            auto go = [&](auto kernel, int warps) {
                const int per = kByteThreads / 32 / warps;
                a.store_blocks = (unsigned int)((units + per - 1) / per);
                launch(kernel, a.store_blocks + (unsigned int)query_blocks, (unsigned int)kByteThreads, 0, ctx->stream, a);
            };
            const bool few = units > (int64_t)kWriteCtas * ctx->sm_count && n_tokens <= 32 * (int64_t)B;
            if (vec && full) few ? go(kvb_write_kernel<dt(), d(), true, true, 1>, 1) : go(kvb_write_kernel<dt(), d(), true, true, 8>, 8);
            else if (vec) few ? go(kvb_write_kernel<dt(), d(), true, false, 1>, 1) : go(kvb_write_kernel<dt(), d(), true, false, 8>, 8);
            else few ? go(kvb_write_kernel<dt(), d(), false, false, 1>, 1) : go(kvb_write_kernel<dt(), d(), false, false, 8>, 8);
        });
    });
    return after_launch(ctx, 1);
}

int aasd_kvb_read(aasd_ctx* ctx, const void* pages, const int32_t* slots, int64_t n, int32_t n_pages, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                  void* k_out, void* v_out) {
    TraceRange trace("aasd_kvb_read");
    const int rc = kv_check_read(ctx, pages, slots, n, n_pages, n_kv_heads, head_dim, dtype, k_out, v_out);
    if (rc != AASD_OK || n == 0 || (!k_out && !v_out)) return rc;
    KvReadArgs a{static_cast<const uint8_t*>(pages), slots, n, n_pages, n_kv_heads, k_out, v_out, ctx->state};
    const int64_t per_cta = kByteThreads / (head_dim / 16);
    if (n > 0x7FFFFFFFLL / n_kv_heads) return AASD_ERR_BAD_SHAPE;
    const unsigned int grid = (unsigned int)((n * n_kv_heads + per_cta - 1) / per_cta);
    const bool vec = aligned16(k_out) && aligned16(v_out);
    AASD_CUDA(cudaSetDevice(ctx->device));
    with_type(dtype, [&](auto dt) {
        with_dim(head_dim, [&](auto d) {
            if (vec) launch(kvb_read_kernel<dt(), d(), true>, grid, (unsigned int)kByteThreads, 0, ctx->stream, a);
            else launch(kvb_read_kernel<dt(), d(), false>, grid, (unsigned int)kByteThreads, 0, ctx->stream, a);
        });
    });
    return after_launch(ctx, 1);
}

int aasd_kvb_commit(aasd_ctx* ctx, void* pages, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len, const int32_t* tok_offsets,
                    const int32_t* best_node, const int32_t* node_parent, const aasd_kv_commit_params* p, int32_t* new_len) {
    TraceRange trace("aasd_kvb_commit");
    if (p == nullptr || !kv_head_dim_ok(p->head_dim)) return p == nullptr ? AASD_ERR_INVALID_ARG : AASD_ERR_UNSUPPORTED;
    KvCommitArgs a{};
    const int rc = kv_prepare_commit(ctx, pages, block_table, cached_len, kv_len, tok_offsets, best_node, node_parent, p, new_len,
                                     kvb_head_bytes(p->head_dim), a);
    if (rc != AASD_OK || p->n_seqs == 0) return rc;
    const int64_t items = (int64_t)p->n_layers * p->n_kv_heads * 2;
    int64_t groups = (items + kCommitThreads / 32 - 1) / (kCommitThreads / 32);
    groups = groups < 1 ? 1 : groups > 64 ? 64 : groups;
    AASD_CUDA(cudaSetDevice(ctx->device));
    with_dim(p->head_dim, [&](auto d) {
        launch_grid2(kvb_commit_kernel<d()>, (unsigned int)p->n_seqs, (unsigned int)groups, (unsigned int)kCommitThreads, ctx->stream, a);
    });
    return after_launch(ctx, 1);
}

int aasd_kvb_attend(aasd_ctx* ctx, const void* q, const void* pages, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len,
                    const int32_t* tok_offsets, const int32_t* node_parent, const aasd_kv_attend_params* p, void* workspace, size_t workspace_bytes,
                    const aasd_kv_attend_out* o) {
    TraceRange trace("aasd_kvb_attend");
    KvAttendArgs a{};
    int rc = kv_prepare_attend(ctx, q, pages, block_table, cached_len, kv_len, tok_offsets, node_parent, p, workspace, workspace_bytes, o, a);
    if (rc != AASD_OK || p->n_tokens == 0) return rc;
    AASD_CUDA(cudaSetDevice(ctx->device));
    const LaunchEnv env{ctx->stream, ctx->device};
    int launches = 0;
    rc = p->dtype == AASD_F32 ? launch_kvb_attend_f32(env, ctx->sm_count, a, workspace, &launches)
                              : launch_kvb_attend_bf16(env, ctx->sm_count, a, workspace, &launches);
    if (rc != AASD_OK) return rc;
    return after_launch(ctx, launches);
}

}  // extern "C"
