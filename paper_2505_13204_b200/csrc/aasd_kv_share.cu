// Host side of the page operators (aasd_kv_free, _fork, _copy, _compact in include/aasd.h).
#include "aasd_host.h"
#include "aasd_kv_host.h"
#include "aasd_kv_share.cuh"

using namespace aasd;

namespace {

// Sequences up to which the collecting CTA goes through the tables itself, a warp for two of them: a launch less for the host.
// Freeing and compacting, on the device: 16 sequences 14 us either way, 48 20 us against 16 with a launch for the tables.
constexpr int kDropInline = 16;
// Pages up to which the kernels with one CTA have few threads, one round of a scan: a round costs a barrier of all warps.  Freeing
// and compacting with few threads and with many: 100 pages 14 and 18 us, 1300 20 and 22, 2300 27 and 24, 8000 51 and 37.
constexpr int kFewPages = kShareThreads * kShareEach;

// Calls f with the number of threads as a constant.
template <class F>
void one_cta(bool few, F&& f) {
    if (few) f(std::integral_constant<int, kShareThreads>());
    else f(std::integral_constant<int, kShareThreadsMany>());
}

int check_books(const aasd_kv_books_params* p, const aasd_kv_books* k) {
    if (p == nullptr || k == nullptr) return AASD_ERR_INVALID_ARG;
    if (p->n_seqs < 0 || p->n_pages < 0 || p->n_pages > 0x7FFFFFFF / kPage || p->max_pages < 1 || p->max_pages > 0x7FFFFFFF / kPage) return AASD_ERR_BAD_SHAPE;
    if (!k->n_free || (p->n_pages > 0 && (!k->free_pages || !k->page_shares)) || (p->n_seqs > 0 && (!k->block_table || !k->seq_pages)))
        return AASD_ERR_INVALID_ARG;
    return AASD_OK;
}

int check_pool(const aasd_kv_pool* p) {
    if (p == nullptr) return AASD_ERR_INVALID_ARG;
    if (p->n_layers < 0 || p->page_bytes < 0 || p->page_bytes % 16 != 0 || p->layer_stride < 0 || p->layer_stride % 16 != 0) return AASD_ERR_BAD_SHAPE;
    if (p->n_layers > 0 && p->page_bytes > 0 && (!p->pages || !aligned16(p->pages))) return AASD_ERR_INVALID_ARG;
    return AASD_OK;
}

// Whether an array lies over one of the books, or over the layers' pools.
bool over_books(const void* x, int64_t bytes, const aasd_kv_books_params& p, const aasd_kv_books& k) {
    const int64_t b4 = 4 * (int64_t)p.n_seqs, n4 = 4 * (int64_t)p.n_pages;
    return overlap(x, bytes, k.block_table, b4 * p.max_pages) || overlap(x, bytes, k.seq_pages, b4) || overlap(x, bytes, k.free_pages, n4) ||
           overlap(x, bytes, k.n_free, 4) || overlap(x, bytes, k.page_shares, n4);
}
bool over_pool(const void* x, int64_t bytes, const aasd_kv_pool& p, int32_t n_pages) {
    return p.n_layers > 0 && overlap(x, bytes, p.pages, (p.n_layers - 1) * p.layer_stride + n_pages * p.page_bytes);
}

KvCopyArgs copy_args(const aasd_ctx* ctx, const aasd_kv_pool& p, int32_t n_pages, const int32_t* src, const int32_t* dst, int step, int32_t n, const int32_t* count) {
    return KvCopyArgs{static_cast<uint8_t*>(p.pages), p.layer_stride, p.page_bytes, p.page_bytes > 0 ? p.n_layers : 0, n_pages, src, dst, step, n, count, ctx->state};
}

// CTAs for the chunks of n pages: no more than there are, and no more than fit the device at a time.
unsigned int copy_grid(const aasd_ctx* ctx, const aasd_kv_pool& p, int64_t n) {
    const int64_t chunks = n * p.n_layers * ((p.page_bytes + kCopyChunk - 1) / kCopyChunk), most = (int64_t)ctx->sm_count * kCopyCtas;
    return (unsigned int)(chunks < 1 ? 1 : chunks < most ? chunks : most);
}

}  // namespace

extern "C" {

int aasd_kv_free(aasd_ctx* ctx, const int32_t* keep_len, const int32_t* n_new, const aasd_kv_books_params* p, const aasd_kv_books* k) {
    TraceRange trace("aasd_kv_free");
    if (ctx == nullptr) return AASD_ERR_INVALID_ARG;
    if (const int rc = check_books(p, k)) return rc;
    if (p->n_seqs == 0 || p->n_pages == 0) return AASD_OK;
    if (!keep_len) return AASD_ERR_INVALID_ARG;
    KvFreeArgs a{keep_len, n_new, *k, *p, ctx->state};
    AASD_CUDA(cudaSetDevice(ctx->device));
    const bool drop = p->n_seqs <= kDropInline;
    if (!drop) launch(kv_drop_kernel, (unsigned int)((p->n_seqs + 7) / 8), 256u, 0, ctx->stream, a);
    one_cta(p->n_pages <= kFewPages, [&](auto nt) {
        if (drop) launch(kv_collect_kernel<nt(), true>, 1u, (unsigned int)nt(), 0, ctx->stream, a);
        else launch(kv_collect_kernel<nt(), false>, 1u, (unsigned int)nt(), 0, ctx->stream, a);
    });
    return after_launch(ctx, drop ? 1 : 2);
}

int aasd_kv_copy(aasd_ctx* ctx, const aasd_kv_pool* pool, int32_t n_pages, const int32_t* src, const int32_t* dst, int32_t n) {
    TraceRange trace("aasd_kv_copy");
    if (ctx == nullptr) return AASD_ERR_INVALID_ARG;
    if (const int rc = check_pool(pool)) return rc;
    if (n_pages < 0 || n_pages > 0x7FFFFFFF / kPage || n < 0) return AASD_ERR_BAD_SHAPE;
    if (n == 0 || pool->n_layers == 0 || pool->page_bytes == 0) return AASD_OK;
    if (!src || !dst) return AASD_ERR_INVALID_ARG;
    AASD_CUDA(cudaSetDevice(ctx->device));
    launch(kv_copy_kernel, copy_grid(ctx, *pool, n), (unsigned int)kCopyThreads, 0, ctx->stream, copy_args(ctx, *pool, n_pages, src, dst, 1, n, nullptr));
    return after_launch(ctx, 1);
}

int aasd_kv_fork(aasd_ctx* ctx, const int32_t* src_seq, const int32_t* dst_seq, const int32_t* fork_len, int32_t n_forks, const aasd_kv_books_params* p,
                 const aasd_kv_books* k, int32_t* cached_len, const aasd_kv_pool* pool, const aasd_kv_fork_out* o) {
    TraceRange trace("aasd_kv_fork");
    if (ctx == nullptr || o == nullptr) return AASD_ERR_INVALID_ARG;
    if (const int rc = check_books(p, k)) return rc;
    if (const int rc = check_pool(pool)) return rc;
    if (n_forks < 0) return AASD_ERR_BAD_SHAPE;
    if (n_forks == 0) return AASD_OK;
    if (!src_seq || !dst_seq || !o->new_len || !o->copy_src || !o->copy_dst || (p->n_seqs > 0 && !cached_len)) return AASD_ERR_INVALID_ARG;
    // what the forks are made from is read again when their outputs have been written
    const int64_t n4 = 4 * (int64_t)n_forks, b4 = 4 * (int64_t)p->n_seqs;
    for (const int32_t* x : {o->new_len, o->copy_src, o->copy_dst})
        if (overlap(x, n4, src_seq, n4) || overlap(x, n4, dst_seq, n4) || overlap(x, n4, fork_len, n4) || overlap(x, n4, cached_len, b4) ||
            over_books(x, n4, *p, *k) || over_pool(x, n4, *pool, p->n_pages))
            return AASD_ERR_INVALID_ARG;
    if (overlap(o->new_len, n4, o->copy_src, n4) || overlap(o->new_len, n4, o->copy_dst, n4) || overlap(o->copy_src, n4, o->copy_dst, n4)) return AASD_ERR_INVALID_ARG;
    KvForkArgs a{src_seq, dst_seq, fork_len, n_forks, *k, *p, cached_len, o->new_len, o->copy_src, o->copy_dst,
                 copy_args(ctx, *pool, p->n_pages, o->copy_src, o->copy_dst, 1, n_forks, nullptr), ctx->state};
    AASD_CUDA(cudaSetDevice(ctx->device));
    one_cta(n_forks <= kShareThreads, [&](auto nt) { launch(kv_fork_kernel<nt()>, 1u, (unsigned int)nt(), 0, ctx->stream, a); });
    unsigned int grid = copy_grid(ctx, *pool, n_forks);
    const unsigned int tables = (unsigned int)((n_forks + 7) / 8);
    if (grid < tables) grid = tables < 1024 ? tables : 1024;
    launch(kv_fork_copy_kernel, grid, (unsigned int)kCopyThreads, 0, ctx->stream, a);
    return after_launch(ctx, 2);
}

int aasd_kv_compact(aasd_ctx* ctx, const aasd_kv_books_params* p, const aasd_kv_books* k, const aasd_kv_pool* pool, int32_t* page_map, int32_t* moves,
                    int32_t* n_moved) {
    TraceRange trace("aasd_kv_compact");
    if (ctx == nullptr) return AASD_ERR_INVALID_ARG;
    if (const int rc = check_books(p, k)) return rc;
    if (const int rc = check_pool(pool)) return rc;
    if (!n_moved || (p->n_pages > 0 && (!page_map || !moves))) return AASD_ERR_INVALID_ARG;
    const int64_t n4 = 4 * (int64_t)p->n_pages;
    if (overlap(page_map, n4, moves, n4) || overlap(n_moved, 4, page_map, n4) || overlap(n_moved, 4, moves, n4)) return AASD_ERR_INVALID_ARG;
    for (const int32_t* x : {page_map, moves, n_moved}) {
        const int64_t bytes = x == n_moved ? 4 : n4;
        if (over_books(x, bytes, *p, *k) || over_pool(x, bytes, *pool, p->n_pages)) return AASD_ERR_INVALID_ARG;
    }
    KvCompactArgs a{*k, *p, page_map, moves, n_moved, copy_args(ctx, *pool, p->n_pages, moves, moves + 1, 2, p->n_pages / 2, n_moved), ctx->state};
    AASD_CUDA(cudaSetDevice(ctx->device));
    one_cta(p->n_pages <= kFewPages, [&](auto nt) { launch(kv_compact_kernel<nt()>, 1u, (unsigned int)nt(), 0, ctx->stream, a); });
    launch(kv_compact_copy_kernel, copy_grid(ctx, *pool, p->n_pages), (unsigned int)kCopyThreads, 0, ctx->stream, a);
    return after_launch(ctx, 2);
}

}  // extern "C"
