// Host side of the paged 4-bit cache (aasd_kv_* in include/aasd.h) and the kernels of
// aasd_kv.cuh; the attention kernels are launched from aasd_kv_attend.cu.
#define AASD_KV_TU 1
#include "aasd_host.h"
#include "aasd_kv_host.h"

using namespace aasd;

namespace {

bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }
bool dtype_ok(int d) { return d == AASD_F32 || d == AASD_BF16; }
size_t elt_size(int dtype) { return dtype == AASD_F32 ? 4 : 2; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether two arrays have a byte in common.
bool overlap(const void* x, int64_t x_bytes, const void* y, int64_t y_bytes) {
    const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
    return x != nullptr && y != nullptr && a < b + (uintptr_t)y_bytes && b < a + (uintptr_t)x_bytes;
}

// Calls f with the head dimension as a constant.
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

// Token rows up to which the planning CTA writes the token arrays itself, and from which a second launch
// does: 256 tokens 3.3 us inline and 7.3 us in two launches, 1024 tokens 5.0 and 7.1, 2048 tokens 7.4 and 6.2, 4096 tokens
// 11.8 and 6.1.
constexpr int64_t kInlineTokens = 1024;
// Sequences up to which the planning CTA has 256 threads, one for each: its scans cost a barrier per warp (4 to
// 256 sequences take 3.5 us with them and 8.2 us with 1024 threads; 300 sequences, a second round for the 256, 22.6 and 8.6).
constexpr int kPlanManySeqs = 256;

}  // namespace

extern "C" {

int aasd_kv_head_bytes(int32_t head_dim, size_t* bytes) {
    if (bytes == nullptr) return AASD_ERR_INVALID_ARG;
    if (!head_dim_ok(head_dim)) return AASD_ERR_UNSUPPORTED;
    *bytes = (size_t)kv_head_bytes(head_dim);
    return AASD_OK;
}

int aasd_kv_plan(aasd_ctx* ctx, const int32_t* cached_len, const int32_t* n_new, const int32_t* node_depth,
                 const aasd_kv_plan_params* p, const aasd_kv_plan_state* s, const aasd_kv_plan_out* o) {
    TraceRange trace("aasd_kv_plan");
    if (ctx == nullptr || p == nullptr || s == nullptr || o == nullptr) return AASD_ERR_INVALID_ARG;
    if (p->n_seqs < 0 || p->n_pages < 0 || p->max_pages < 1 || p->rows_per_seq < 0 || p->n_tokens < 0) return AASD_ERR_BAD_SHAPE;
    if (p->rows_per_seq > 0 && (int64_t)p->n_seqs * p->rows_per_seq != p->n_tokens) return AASD_ERR_BAD_SHAPE;
    if (p->n_tokens > 0x7FFFFFFFLL || p->n_pages > 0x7FFFFFFF / kPage || p->max_pages > 0x7FFFFFFF / kPage) return AASD_ERR_BAD_SHAPE;
    if (p->n_seqs == 0 && p->n_tokens == 0) return AASD_OK;
    if (!s->n_free || !s->free_pages || (p->n_seqs > 0 && (!cached_len || !n_new || !s->block_table || !s->seq_pages || !o->kv_len)))
        return AASD_ERR_INVALID_ARG;
    if (p->n_tokens > 0 && (!o->slot_map || !o->positions)) return AASD_ERR_INVALID_ARG;
    if (p->rows_per_seq == 0 && !o->tok_offsets) return AASD_ERR_INVALID_ARG;
    // a token's slot and position are found from the old length and the new one
    const int64_t n4 = 4 * (int64_t)p->n_seqs;
    if (overlap(cached_len, n4, o->kv_len, n4) || overlap(cached_len, n4, o->tok_offsets, n4 + 4) ||
        overlap(cached_len, n4, o->slot_map, 4 * p->n_tokens) || overlap(cached_len, n4, o->positions, 4 * p->n_tokens))
        return AASD_ERR_INVALID_ARG;
    KvPlanArgs a{cached_len, n_new, node_depth, *p, *s, *o, ctx->state, 0};
    const bool many = p->n_seqs > kPlanManySeqs;
    a.tokens_inline = p->n_tokens <= kInlineTokens && p->n_seqs <= (many ? kPlanThreadsMany : kPlanThreads);
    AASD_CUDA(cudaSetDevice(ctx->device));
    if (many) launch(kv_plan_kernel<kPlanThreadsMany>, 1u, (unsigned int)kPlanThreadsMany, 0, ctx->stream, a);
    else launch(kv_plan_kernel<kPlanThreads>, 1u, (unsigned int)kPlanThreads, 0, ctx->stream, a);
    if (a.tokens_inline || p->n_tokens == 0) return after_launch(ctx, 1);
    launch(kv_tokens_kernel, (unsigned int)((p->n_tokens + 1023) / 1024), 256u, 0, ctx->stream, a);
    return after_launch(ctx, 2);
}

int aasd_kv_write(aasd_ctx* ctx, const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                  const float* cos_sin, const int32_t* positions, const int32_t* slot_map, int64_t n_tokens,
                  const aasd_kv_write_params* p, void* pages, void* q_out, void* k_out) {
    TraceRange trace("aasd_kv_write");
    if (ctx == nullptr || p == nullptr) return AASD_ERR_INVALID_ARG;
    if (!dtype_ok(p->dtype)) return AASD_ERR_BAD_DTYPE;
    if (!head_dim_ok(p->head_dim)) return AASD_ERR_UNSUPPORTED;
    const int hq = p->n_q_heads, hkv = p->n_kv_heads, D = p->head_dim;
    if (n_tokens < 0 || hq < 0 || hkv < 0 || p->n_pages < 0 || p->n_pages > 0x7FFFFFFF / kPage) return AASD_ERR_BAD_SHAPE;
    if (p->rotary_dim < 0 || p->rotary_dim > D || (p->rotary_dim & 1) || p->max_positions < 0) return AASD_ERR_BAD_SHAPE;
    if ((hq > 0 && p->q_stride < (int64_t)hq * D) || (hkv > 0 && (p->k_stride < (int64_t)hkv * D || p->v_stride < (int64_t)hkv * D)))
        return AASD_ERR_BAD_SHAPE;
    if (!(p->eps >= 0.f) || (p->flags & ~AASD_KV_ROPE_INTERLEAVED)) return AASD_ERR_INVALID_ARG;
    if (n_tokens == 0 || hq + hkv == 0) return AASD_OK;
    if (!positions || (p->rotary_dim > 0 && !cos_sin)) return AASD_ERR_INVALID_ARG;
    if (hq > 0 && (!q || !q_out)) return AASD_ERR_INVALID_ARG;
    if (hkv > 0 && (!k || !v || !slot_map || !pages || !aligned16(pages))) return AASD_ERR_INVALID_ARG;
    const size_t es = elt_size(p->dtype);
    for (const void* x : {q, k, v, q_weight, k_weight, (const void*)q_out, (const void*)k_out})
        if (((uintptr_t)x % es) != 0) return AASD_ERR_INVALID_ARG;
    KvWriteArgs a{q, k, v, q_weight, k_weight, cos_sin, positions, slot_map, n_tokens, *p, static_cast<uint8_t*>(pages), q_out, k_out,
                  ctx->state, 0u, make_float2(-0.f, -0.f)};
    // 16-byte accesses where every row of every operand starts on a 16-byte boundary
    bool vec = p->rotary_dim == 0 || aligned16(cos_sin);
    for (const void* x : {q, k, v, q_weight, k_weight, (const void*)q_out, (const void*)k_out}) vec = vec && aligned16(x);
    if (hq > 0) vec = vec && (p->q_stride * es) % 16 == 0;
    if (hkv > 0) vec = vec && (p->k_stride * es) % 16 == 0 && (p->v_stride * es) % 16 == 0;
    const int lanes = D / 16;
    const int64_t rows = n_tokens * (hq + hkv);
    const bool full = p->rotary_dim == D && !(p->flags & AASD_KV_ROPE_INTERLEAVED);
    const int64_t value_blocks = (n_tokens + kValueTokens - 1) / kValueTokens * hkv;
    const int64_t blocks = value_blocks + (rows * lanes + kWriteThreads - 1) / kWriteThreads;
    if (blocks > 0x7FFFFFFFLL) return AASD_ERR_BAD_SHAPE;
    a.value_blocks = (unsigned int)value_blocks;
    AASD_CUDA(cudaSetDevice(ctx->device));
    with_type(p->dtype, [&](auto dt) {
        with_dim(D, [&](auto d) {
            auto go = [&](auto kernel) { launch(kernel, (unsigned int)blocks, (unsigned int)kWriteThreads, 0, ctx->stream, a); };
            if (vec && full) go(kv_write_kernel<dt(), d(), true, true>);
            else if (vec) go(kv_write_kernel<dt(), d(), true, false>);
            else go(kv_write_kernel<dt(), d(), false, false>);
        });
    });
    return after_launch(ctx, 1);
}

int aasd_kv_read(aasd_ctx* ctx, const void* pages, const int32_t* slots, int64_t n, int32_t n_pages, int32_t n_kv_heads,
                 int32_t head_dim, int32_t dtype, void* k_out, void* v_out) {
    TraceRange trace("aasd_kv_read");
    if (ctx == nullptr) return AASD_ERR_INVALID_ARG;
    if (!dtype_ok(dtype)) return AASD_ERR_BAD_DTYPE;
    if (!head_dim_ok(head_dim)) return AASD_ERR_UNSUPPORTED;
    if (n < 0 || n_kv_heads < 1 || n_pages < 0 || n_pages > 0x7FFFFFFF / kPage) return AASD_ERR_BAD_SHAPE;
    if (n == 0 || (!k_out && !v_out)) return AASD_OK;
    if (!pages || !aligned16(pages) || !slots) return AASD_ERR_INVALID_ARG;
    const size_t es = elt_size(dtype);
    if (((uintptr_t)k_out % es) != 0 || ((uintptr_t)v_out % es) != 0) return AASD_ERR_INVALID_ARG;
    KvReadArgs a{static_cast<const uint8_t*>(pages), slots, n, n_pages, n_kv_heads, k_out, v_out, ctx->state};
    const int64_t blocks = (n + kValueTokens - 1) / kValueTokens * n_kv_heads;
    if (blocks > 0x7FFFFFFFLL) return AASD_ERR_BAD_SHAPE;
    const bool vec = aligned16(k_out) && aligned16(v_out);
    AASD_CUDA(cudaSetDevice(ctx->device));
    const unsigned int grid = (unsigned int)blocks;
    with_type(dtype, [&](auto dt) {
        with_dim(head_dim, [&](auto d) {
            if (vec) launch(kv_read_kernel<dt(), d(), true>, grid, (unsigned int)kWriteThreads, 0, ctx->stream, a);
            else launch(kv_read_kernel<dt(), d(), false>, grid, (unsigned int)kWriteThreads, 0, ctx->stream, a);
        });
    });
    return after_launch(ctx, 1);
}

int aasd_kv_commit(aasd_ctx* ctx, void* pages, const int32_t* block_table, const int32_t* cached_len, const int32_t* kv_len,
                   const int32_t* tok_offsets, const int32_t* best_node, const int32_t* node_parent,
                   const aasd_kv_commit_params* p, int32_t* new_len) {
    TraceRange trace("aasd_kv_commit");
    if (ctx == nullptr || p == nullptr) return AASD_ERR_INVALID_ARG;
    if (!head_dim_ok(p->head_dim)) return AASD_ERR_UNSUPPORTED;
    if (p->n_seqs < 0 || p->n_kv_heads < 1 || p->n_pages < 0 || p->n_pages > 0x7FFFFFFF / kPage || p->max_pages < 1 ||
        p->max_pages > 0x7FFFFFFF / kPage || p->rows_per_seq < 0 || p->n_layers < 0 || p->layer_stride < 0 || (p->layer_stride % 16) != 0)
        return AASD_ERR_BAD_SHAPE;
    if (p->n_seqs == 0) return AASD_OK;
    if (!block_table || !cached_len || !kv_len || !best_node || !node_parent || !new_len) return AASD_ERR_INVALID_ARG;
    if (p->rows_per_seq == 0 && !tok_offsets) return AASD_ERR_INVALID_ARG;
    if (p->n_layers > 0 && (!pages || !aligned16(pages))) return AASD_ERR_INVALID_ARG;
    // Every CTA of a sequence reads its inputs for itself, in no order with the one that writes the new length.
    const int64_t n4 = 4 * (int64_t)p->n_seqs;
    const int64_t pool = (int64_t)p->n_pages * p->n_kv_heads * kv_head_bytes(p->head_dim);
    if (overlap(new_len, n4, cached_len, n4) || overlap(new_len, n4, kv_len, n4) || overlap(new_len, n4, best_node, n4) ||
        overlap(new_len, n4, tok_offsets, n4 + 4) || overlap(new_len, n4, block_table, n4 * p->max_pages) ||
        overlap(new_len, n4, node_parent, p->rows_per_seq > 0 ? n4 * p->rows_per_seq : 4) ||
        (p->n_layers > 0 && overlap(new_len, n4, pages, (p->n_layers - 1) * p->layer_stride + pool)))
        return AASD_ERR_INVALID_ARG;
    KvCommitArgs a{static_cast<uint8_t*>(pages), block_table, cached_len, kv_len, tok_offsets, best_node, node_parent, *p, new_len,
                   ctx->state};
    const int64_t items = (int64_t)p->n_layers * p->n_kv_heads;
    int64_t groups = (items + kCommitThreads / 32 - 1) / (kCommitThreads / 32);
    groups = groups < 1 ? 1 : groups > 64 ? 64 : groups;
    AASD_CUDA(cudaSetDevice(ctx->device));
    with_dim(p->head_dim, [&](auto d) {
        launch_grid2(kv_commit_kernel<d()>, (unsigned int)p->n_seqs, (unsigned int)groups, (unsigned int)kCommitThreads, ctx->stream, a);
    });
    return after_launch(ctx, 1);
}

int aasd_kv_workspace_bytes(int32_t head_dim, size_t* bytes) {
    if (bytes == nullptr) return AASD_ERR_INVALID_ARG;
    if (!head_dim_ok(head_dim)) return AASD_ERR_UNSUPPORTED;
    *bytes = kv_attend_scratch(head_dim).bytes;
    return AASD_OK;
}

int aasd_kv_workspace_init(aasd_ctx* ctx, void* workspace, size_t bytes, int32_t head_dim) {
    if (ctx == nullptr || workspace == nullptr || (uintptr_t)workspace % 256 != 0) return AASD_ERR_INVALID_ARG;
    if (!head_dim_ok(head_dim)) return AASD_ERR_UNSUPPORTED;
    const KvScratch L = kv_attend_scratch(head_dim);
    if (bytes < L.bytes) return AASD_ERR_WORKSPACE_TOO_SMALL;
    AASD_CUDA(cudaMemsetAsync(workspace, 0, L.zero_bytes, ctx->stream));
    try {
        ctx->kv_workspaces[workspace] = head_dim;
    } catch (...) {
        return AASD_ERR_CUDA;
    }
    return AASD_OK;
}

int aasd_kv_attend(aasd_ctx* ctx, const void* q, const void* pages, const int32_t* block_table, const int32_t* cached_len,
                   const int32_t* kv_len, const int32_t* tok_offsets, const int32_t* node_parent, const aasd_kv_attend_params* p,
                   void* workspace, size_t workspace_bytes, const aasd_kv_attend_out* o) {
    TraceRange trace("aasd_kv_attend");
    if (ctx == nullptr || p == nullptr || o == nullptr) return AASD_ERR_INVALID_ARG;
    if (!dtype_ok(p->dtype)) return AASD_ERR_BAD_DTYPE;
    if (!head_dim_ok(p->head_dim)) return AASD_ERR_UNSUPPORTED;
    if (p->n_seqs < 0 || p->n_tokens < 0 || p->n_kv_heads < 1 || p->n_q_heads < 1 || p->n_q_heads > 65536 || p->n_q_heads % p->n_kv_heads != 0 ||
        p->n_pages < 0 || p->n_pages > 0x7FFFFFFF / kPage || p->max_pages < 1 || p->max_pages > 0x7FFFFFFF / kPage || p->rows_per_seq < 0 ||
        p->q_stride < (int64_t)p->n_q_heads * p->head_dim)
        return AASD_ERR_BAD_SHAPE;
    if (p->rows_per_seq > 0 && (int64_t)p->n_seqs * p->rows_per_seq != p->n_tokens) return AASD_ERR_BAD_SHAPE;
    if (!(p->scale >= 0.f) || !(p->scale <= 3.0e38f)) return AASD_ERR_INVALID_ARG;
    if (p->n_tokens == 0) return AASD_OK;
    if (p->n_tokens > 0x7FFFFFFFLL / p->n_q_heads) return AASD_ERR_BAD_SHAPE;
    if (!q || !o->out) return AASD_ERR_INVALID_ARG;
    if (p->n_seqs > 0 && (!block_table || !cached_len || !kv_len || !pages || !aligned16(pages))) return AASD_ERR_INVALID_ARG;
    if (p->rows_per_seq == 0 && p->n_seqs > 0 && !tok_offsets) return AASD_ERR_INVALID_ARG;
    const size_t es = elt_size(p->dtype);
    if (((uintptr_t)q % es) != 0 || ((uintptr_t)o->out % es) != 0) return AASD_ERR_INVALID_ARG;
    const auto it = ctx->kv_workspaces.find(workspace);
    if (workspace == nullptr || it == ctx->kv_workspaces.end()) return AASD_ERR_INVALID_ARG;
    if (it->second < p->head_dim || workspace_bytes < kv_attend_scratch(p->head_dim).bytes) return AASD_ERR_WORKSPACE_TOO_SMALL;
    KvAttendArgs a{};
    a.q = q;
    a.pages = static_cast<const uint8_t*>(pages);
    a.block_table = block_table;
    a.cached_len = cached_len;
    a.kv_len = kv_len;
    a.tok_offsets = tok_offsets;
    a.node_parent = node_parent;
    a.p = *p;
    a.o = *o;
    a.q_vec = aligned16(q) && (p->q_stride * es) % 16 == 0;
    a.out_vec = aligned16(o->out);
    a.scale_log2 = (p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->head_dim)) * kLog2e;
    a.state = ctx->state;
    a.wait_limit = kWaitLimit;
    a.withhold_page = -1;
    if (ctx->withhold_item >= 0) {
        a.wait_limit = ctx->test_wait_limit;
        a.withhold_page = ctx->withhold_item < 0x7FFFFFFF ? (int)ctx->withhold_item : 0x7FFFFFFF;
        ctx->withhold_item = -1;
    }
    AASD_CUDA(cudaSetDevice(ctx->device));
    const LaunchEnv env{ctx->stream, ctx->device};
    int launches = 0;
    const int rc = p->dtype == AASD_F32 ? launch_kv_attend_f32(env, ctx->sm_count, a, workspace, &launches)
                                        : launch_kv_attend_bf16(env, ctx->sm_count, a, workspace, &launches);
    if (rc != AASD_OK) return rc;
    return after_launch(ctx, launches);
}

}  // extern "C"
