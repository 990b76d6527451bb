// Pages with several holders: forking sequences, freeing pages, moving those in use to the front of the pool.
// The kernels move whole pages as bytes, so they serve the 4-bit and the 8-bit cache alike.
#pragma once

#include "aasd_kv.cuh"

namespace aasd {

constexpr int kShareThreads = 256, kShareThreadsMany = 1024;   // of the kernels with one CTA: a scan costs a barrier for every warp
constexpr int kShareEach = 8;              // pages that a thread looks at per round of a scan over the pool

// The count on the stack, held to what the pool has.
__device__ __forceinline__ int kv_free_count(const int32_t* n_free, int n_pages, unsigned int& bits) {
    const int n = *n_free;
    if (n < 0 || n > n_pages) bits |= AASD_STATUS_BAD_OFFSETS;
    return n < 0 ? 0 : n > n_pages ? n_pages : n;
}

// ---- freeing ----------------------------------------------------------------------------------------

struct KvFreeArgs {
    const int32_t* keep_len;
    const int32_t* n_new;                  // may be NULL
    aasd_kv_books k;
    aasd_kv_books_params p;
    DeviceState* state;
};

// A warp takes a sequence: the table's entries past what is kept go, and each takes a holder off its page.
__device__ __forceinline__ void kv_drop(const KvFreeArgs& a, int b) {
    const int lane = threadIdx.x & 31;
    const int keep = a.keep_len[b], held = a.k.seq_pages[b], fresh = a.n_new ? a.n_new[b] : 0;
    if (keep == AASD_NONE) return;
    if (keep < 0 || fresh < 0 || held < 0 || held > a.p.max_pages) {
        if (lane == 0) raise(a.state, AASD_STATUS_BAD_OFFSETS);
        return;
    }
    const long long need = ((long long)keep + fresh + kPage - 1) / kPage;
    if (need >= held) return;
    int32_t* row = a.k.block_table + (int64_t)b * a.p.max_pages;
    for (int j = (int)need + lane; j < held; j += 32) {
        const int page = row[j];
        row[j] = AASD_NONE;
        if (page >= 0 && page < a.p.n_pages) atomicSub(a.k.page_shares + page, 1);
        else raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    if (lane == 0) a.k.seq_pages[b] = (int)need;
}
__global__ void __launch_bounds__(256) kv_drop_kernel(const KvFreeArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int b = (int)((blockIdx.x * 256u + threadIdx.x) >> 5);
    if (b < a.p.n_seqs) kv_drop(a, b);
}

// Whether the new tokens of a warp's 32 sequences (from b0 on) are going to be stored to a page that others hold too: a sequence was cut
// inside what it shares.  Holders are those left when every sequence has dropped its pages.  A lane looks at its sequence's
// first page, as a rule the only one that is there; the warp at what follows.
__device__ __forceinline__ bool kv_writes_shared(const KvFreeArgs& a, int b0) {
    const int lane = threadIdx.x & 31, b = b0 + lane;
    int j = 0, end = 0;
    if (b < a.p.n_seqs) {
        const int keep = a.keep_len[b], fresh = a.n_new[b], held = a.k.seq_pages[b];
        if (keep >= 0 && fresh > 0 && held >= 0 && held <= a.p.max_pages) {
            j = keep / kPage;
            end = (int)min((long long)held, ((long long)keep + fresh + kPage - 1) / kPage);
        }
    }
    const auto shared = [&](int seq, int at) {
        const int page = a.k.block_table[(int64_t)seq * a.p.max_pages + at];
        return page >= 0 && page < a.p.n_pages && __ldcg(a.k.page_shares + page) > 0;   // (the atomics' own level)
    };
    bool found = j < end && shared(b, j);
    unsigned int more = __ballot_sync(0xFFFFFFFFu, j + 1 < end);
    while (more) {
        const int k = __ffs(more) - 1, from = __shfl_sync(0xFFFFFFFFu, j, k) + 1, to = __shfl_sync(0xFFFFFFFFu, end, k);
        more &= more - 1;
        for (int i = from + lane; i < to; i += 32) found = found || shared(b0 + k, i);
    }
    return found;
}

// One CTA: pages without a holder go on the stack, in order of their numbers (whatever order the atomics came in).
// DROP: a small batch's tables are gone through first, without a launch of their own.
template <int NT, bool DROP>
__global__ void __launch_bounds__(NT) kv_collect_kernel(const KvFreeArgs a) {
    __shared__ long long s_warp[NT / 32];
    pdl_launch_dependents();
    pdl_wait();
    if (DROP) {
        for (int b = (int)threadIdx.x >> 5; b < a.p.n_seqs; b += NT / 32) kv_drop(a, b);
        __syncthreads();
    }
    unsigned int bits = 0;
    if (a.n_new != nullptr)
        for (int b0 = (int)threadIdx.x & ~31; b0 < a.p.n_seqs; b0 += NT)
            if (kv_writes_shared(a, b0)) bits |= AASD_STATUS_BAD_OFFSETS;
    const int N = a.p.n_pages;
    long long n = kv_free_count(a.k.n_free, N, bits);
    for (int base = 0; base < N; base += NT * kShareEach) {
        const int first = base + (int)threadIdx.x * kShareEach;
        int v[kShareEach], mine = 0;
#pragma unroll
        for (int e = 0; e < kShareEach; ++e) {
            v[e] = first + e < N ? __ldcg(a.k.page_shares + first + e) : 0;   // (the atomics' own level)
            mine += v[e] < 0;
            if (v[e] < -1) bits |= AASD_STATUS_BAD_OFFSETS;      // listed more often than it had holders
        }
        long long total;
        long long at = n + block_scan<NT>(mine, s_warp, total);
#pragma unroll
        for (int e = 0; e < kShareEach; ++e) {
            if (v[e] >= 0) continue;
            a.k.page_shares[first + e] = 0;
            if (at < N) a.k.free_pages[at] = first + e;
            else bits |= AASD_STATUS_BAD_OFFSETS;
            ++at;
        }
        n += total;
        if (n > N) n = N;
    }
    __syncthreads();
    if (threadIdx.x == 0) *a.k.n_free = (int)n;
    if (bits) raise(a.state, bits);
}

// ---- copying ----------------------------------------------------------------------------------------

struct KvCopyArgs {
    uint8_t* pages;
    int64_t layer_stride, page_bytes;
    int n_layers, n_pages;
    const int32_t* src;            // pages, `step` entries apart, n of them (or *count)
    const int32_t* dst;
    int step, n;
    const int32_t* count;          // may be NULL
    DeviceState* state;
};

constexpr int kCopyThreads = 256, kCopyCtas = 6;                  // CTAs per SM at most
constexpr int kCopyVectors = 8;                                   // 16-byte loads under way per thread
constexpr int kCopyChunk = kCopyThreads * kCopyVectors * 16;      // bytes that a CTA moves at a time

// The chunks of all pages and layers, shared by the CTAs in turn: 16 bytes and eight loads under way per thread, 32 KB per CTA.
// Bound by memory: 317 pages of 8 layers of 8 heads of 128 channels, 665 MB read and written, 107 us, 6.2 TB/s, 95 % of the copy rate.
__device__ __forceinline__ void kv_copy_pages(const KvCopyArgs& a, unsigned int cta, unsigned int ctas) {
    const int64_t parts = (a.page_bytes + kCopyChunk - 1) / kCopyChunk;
    const int64_t n = a.count ? min(max(*a.count, 0), a.n) : a.n;
    const int64_t total = n * a.n_layers * parts;
    for (int64_t c = cta; c < total; c += ctas) {
        const int64_t part = c % parts, rest = c / parts;
        const int layer = (int)(rest % a.n_layers);
        const int64_t i = rest / a.n_layers;
        const int from = a.src[i * a.step], to = a.dst[i * a.step];
        if (from == AASD_NONE || to == AASD_NONE) continue;
        if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) {
            raise(a.state, AASD_STATUS_ID_RANGE);
            continue;
        }
        const uint4* x = reinterpret_cast<const uint4*>(a.pages + layer * a.layer_stride + from * a.page_bytes + part * kCopyChunk);
        uint4* y = reinterpret_cast<uint4*>(a.pages + layer * a.layer_stride + to * a.page_bytes + part * kCopyChunk);
        const int vectors = (int)(min((int64_t)kCopyChunk, a.page_bytes - part * kCopyChunk) / 16);
        uint4 v[kCopyVectors];
#pragma unroll
        for (int k = 0; k < kCopyVectors; ++k)
            if ((int)threadIdx.x + k * kCopyThreads < vectors) v[k] = x[threadIdx.x + k * kCopyThreads];
#pragma unroll
        for (int k = 0; k < kCopyVectors; ++k)
            if ((int)threadIdx.x + k * kCopyThreads < vectors) y[threadIdx.x + k * kCopyThreads] = v[k];
    }
}
__global__ void __launch_bounds__(kCopyThreads) kv_copy_kernel(const KvCopyArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    kv_copy_pages(a, blockIdx.x, gridDim.x);
}

// ---- forking ----------------------------------------------------------------------------------------

struct KvForkArgs {
    const int32_t *src_seq, *dst_seq, *fork_len;   // fork_len may be NULL
    int n_forks;
    aasd_kv_books k;
    aasd_kv_books_params p;
    int32_t* cached_len;
    int32_t *new_len, *copy_src, *copy_dst;        // [n_forks]
    KvCopyArgs c;
    DeviceState* state;
};

// One CTA: who forks, what each gets, and the pages for the parts that are begun.
// A sequence that is to be made is claimed by the first fork that names it: its held count (0) becomes that fork's number less
// n_forks.  Counts are set when every fork has been looked at, so that no fork sees what another one of the call made.
template <int NT>
__global__ void __launch_bounds__(NT) kv_fork_kernel(const KvForkArgs a) {
    __shared__ long long s_warp[NT / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int B = a.p.n_seqs, N = a.p.n_pages, F = a.n_forks;
    unsigned int bits = 0;
    const long long n_free = kv_free_count(a.k.n_free, N, bits);
    for (int i = threadIdx.x; i < F; i += NT) {
        const int d = a.dst_seq[i];
        if (d >= 0 && d < B && a.k.seq_pages[d] <= 0) atomicMin(a.k.seq_pages + d, i - F);
    }
    __syncthreads();
    long long asked = 0, taken = 0;
    for (int base = 0; base < F; base += NT) {
        const int i = base + (int)threadIdx.x;
        int len = AASD_NONE, page = AASD_NONE;
        bool claimed = false;
        if (i < F) {
            const int s = a.src_seq[i], d = a.dst_seq[i];
            claimed = d >= 0 && d < B && a.k.seq_pages[d] == i - F;
            if (claimed && s >= 0 && s < B) {
                const int held = a.k.seq_pages[s], cached = a.cached_len[s];
                len = a.fork_len ? a.fork_len[i] : cached;
                if (len < 0 || len > cached || held < 0 || held > a.p.max_pages || (long long)held * kPage < len) len = AASD_NONE;
            }
            if (len == AASD_NONE) bits |= AASD_STATUS_BAD_OFFSETS;
            else if (len % kPage) page = a.k.block_table[(int64_t)s * a.p.max_pages + len / kPage];
        }
        const int want = len != AASD_NONE && len % kPage ? 1 : 0;
        long long total, got;
        const long long rank = asked + block_scan<NT>(want, s_warp, total);
        const bool served = len != AASD_NONE && (!want || rank < n_free);
        block_scan<NT>(want && served, s_warp, got);
        int to = AASD_NONE;
        if (want && served) {
            to = a.k.free_pages[n_free - 1 - rank];
            a.k.free_pages[n_free - 1 - rank] = AASD_NONE;
            if (to < 0 || to >= N || page < 0 || page >= N) bits |= AASD_STATUS_BAD_OFFSETS;
        }
        if (len != AASD_NONE && !served) bits |= AASD_STATUS_KV_FULL;
        if (i < F) {
            // (a fork that is not served but has claimed its sequence says so, for the counts below)
            a.new_len[i] = served ? len : claimed ? AASD_NONE - 1 : AASD_NONE;
            a.copy_src[i] = want && served ? page : AASD_NONE;
            a.copy_dst[i] = to;
        }
        asked += total;
        taken += got;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < F; i += NT) {
        const int len = a.new_len[i];
        if (len == AASD_NONE) continue;
        const int d = a.dst_seq[i];
        a.k.seq_pages[d] = len < 0 ? 0 : (len + kPage - 1) / kPage;
        if (len >= 0) a.cached_len[d] = len;
        else a.new_len[i] = AASD_NONE;
    }
    if (threadIdx.x == 0) *a.k.n_free = (int)(n_free - taken);
    if (bits) raise(a.state, bits);
}

// The tables of the new sequences and the holders of their pages (a warp per fork), and the pages that are begun.
__global__ void __launch_bounds__(kCopyThreads) kv_fork_copy_kernel(const KvForkArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    for (int i = (int)((blockIdx.x * kCopyThreads + threadIdx.x) >> 5); i < a.n_forks; i += (int)(gridDim.x * kCopyThreads / 32)) {
        const int len = a.new_len[i];
        if (len < 0) continue;
        const int32_t* from = a.k.block_table + (int64_t)a.src_seq[i] * a.p.max_pages;
        int32_t* to = a.k.block_table + (int64_t)a.dst_seq[i] * a.p.max_pages;
        const int whole = len / kPage;
        for (int j = lane; j < whole; j += 32) {
            const int page = from[j];
            to[j] = page;
            if (page >= 0 && page < a.p.n_pages) atomicAdd(a.k.page_shares + page, 1);
            else raise(a.state, AASD_STATUS_BAD_OFFSETS);
        }
        if (lane == 0 && len % kPage) to[whole] = a.copy_dst[i];
    }
    kv_copy_pages(a.c, blockIdx.x, gridDim.x);
}

// ---- compacting -------------------------------------------------------------------------------------

struct KvCompactArgs {
    aasd_kv_books k;
    aasd_kv_books_params p;
    int32_t *page_map, *moves, *n_moved;           // [n_pages], [n_pages] pairs, [1]
    KvCopyArgs c;
    DeviceState* state;
};

// One CTA: the k-th page in use behind the last place moves to the k-th free one before it.
template <int NT>
__global__ void __launch_bounds__(NT) kv_compact_kernel(const KvCompactArgs a) {
    __shared__ long long s_warp[NT / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int N = a.p.n_pages, tid = threadIdx.x;
    unsigned int bits = 0;
    const int n_free = kv_free_count(a.k.n_free, N, bits), used = N - n_free;
    for (int i = tid; i < N; i += NT) a.page_map[i] = i;
    __syncthreads();
    for (int i = tid; i < n_free; i += NT) {
        const int page = a.k.free_pages[i];
        if (page < 0 || page >= N) bits |= AASD_STATUS_BAD_OFFSETS;
        else if (atomicExch(a.page_map + page, AASD_NONE) == AASD_NONE) bits |= AASD_STATUS_BAD_OFFSETS;   // twice on the stack
    }
    const bool bad = __syncthreads_or(bits != 0) != 0;
    long long far = 0, holes = 0;
    for (int base = 0; !bad && base < N; base += NT * kShareEach) {
        const int first = base + tid * kShareEach;
        int v[kShareEach], out = 0, in = 0;
#pragma unroll
        for (int e = 0; e < kShareEach; ++e) {
            v[e] = first + e < N ? a.page_map[first + e] : first + e;
            if (first + e >= N) continue;
            out += v[e] != AASD_NONE && first + e >= used;
            in += v[e] == AASD_NONE && first + e < used;
        }
        long long total;
        const long long both = block_scan<NT>((long long)out << 32 | in, s_warp, total);
        long long o = far + (both >> 32), h = holes + (both & 0xFFFFFFFFLL);
#pragma unroll
        for (int e = 0; e < kShareEach; ++e) {
            if (first + e >= N) continue;
            if (v[e] != AASD_NONE && first + e >= used) a.moves[2 * o++] = first + e;
            if (v[e] == AASD_NONE && first + e < used) a.moves[2 * h++ + 1] = first + e;
        }
        far += total >> 32;
        holes += total & 0xFFFFFFFFLL;
    }
    __syncthreads();
    // (a stack without repetitions has as many pages in front of the last place as pages in use lie behind it)
    for (int i = tid; i < (int)far; i += NT) {
        const int from = a.moves[2 * i], to = a.moves[2 * i + 1];
        a.page_map[from] = to;
        a.k.page_shares[to] = a.k.page_shares[from];
        a.k.page_shares[from] = 0;
    }
    for (int i = tid; i < n_free; i += NT)
        if (!bad) a.k.free_pages[i] = N - 1 - i;
    if (bad)
        for (int i = tid; i < N; i += NT) a.page_map[i] = i;
    if (tid == 0) *a.n_moved = (int)far;
    if (bits) raise(a.state, bits);
}

__global__ void __launch_bounds__(kCopyThreads) kv_compact_copy_kernel(const KvCompactArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    // (whether anything moves or not: a table that names a free page is found here)
    const int64_t entries = (int64_t)a.p.n_seqs * a.p.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kCopyThreads) {
        const int page = a.k.block_table[i];
        if (page == AASD_NONE) continue;
        const int to = page >= 0 && page < a.p.n_pages ? a.page_map[page] : AASD_NONE;
        if (to == AASD_NONE) raise(a.state, AASD_STATUS_BAD_OFFSETS);     // not in use, or not in the pool
        else if (to != page) a.k.block_table[i] = to;
    }
    kv_copy_pages(a.c, blockIdx.x, gridDim.x);
}

}  // namespace aasd
