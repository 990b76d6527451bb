// The paged 8-bit cache: layout, codes, and the kernels that keep it (norm + rotation + store, moving an accepted
// path, reading entries back).  Attention over it is in aasd_kvb_attend.cuh and aasd_kvb_tile.cuh.
//
// A value is an e4m3 code times the scale of its page, head and half (keys, values): a power of two, so that codes
// whose page's scale grows change by an exponent and lose nothing above the subnormal numbers.
#pragma once

#include <cuda_fp8.h>

#include "aasd_kv.cuh"

namespace aasd {

constexpr int kByteLeast = -64;            // least exponent of a scale
constexpr int kByteMost = 120;             // largest: fp32 numbers end at 2^128 < 448 * 2^120

// Offsets inside one head's block of a page (see include/aasd.h).
__host__ __device__ constexpr int kvb_head_bytes(int D) { return 2 * kPage * D + 16; }
__host__ __device__ constexpr int kvb_value_offset(int D) { return kPage * D; }
__host__ __device__ constexpr int kvb_scale_offset(int D) { return 2 * kPage * D; }
// Byte of token t's 16-byte chunk `chunk` (channels 16 chunk ..) inside the keys or the values: rows of 128 bytes (64 with D = 64)
// whose chunks lie in the swizzle that the tensor cores read operands in, so that a page is one as it comes.
__host__ __device__ constexpr int kvb_chunk_offset(int D, int t, int chunk) {
    return D == 64 ? t * 64 + ((chunk ^ ((t >> 1) & 3)) << 4) : (chunk >> 3) * (kPage * 128) + t * 128 + (((chunk & 7) ^ (t & 7)) << 4);
}

__device__ __forceinline__ float kvb_pow2(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }   // -126 <= e <= 127
// A stored scale, and its exponent.  (What a page holds that was never written is held to the range.)
__device__ __forceinline__ unsigned int kvb_scale_bits(unsigned int scale) {
    return min(max(scale & 0x7F800000u, (unsigned int)(kByteLeast + 127) << 23), (unsigned int)(kByteMost + 127) << 23);
}
__device__ __forceinline__ int kvb_exponent(unsigned int scale) { return (int)(kvb_scale_bits(scale) >> 23) - 127; }
// Least exponent e >= -64 with top <= 448 * 2^e = 1.75 * 2^(e + 8); top: bits of a finite magnitude.
__device__ __forceinline__ int kvb_fit(unsigned int top) { return max(kByteLeast, (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0)); }

// Codes of two values that are at most 448, rounded to nearest (ties to even).
__device__ __forceinline__ unsigned int kvb_codes(float2 x) { return __nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 kvb_values(unsigned int codes) {   // of the low 16 bits; exact
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// Eight codes times a power of two at most 1, as codes again.
__device__ __forceinline__ u64 kvb_rescale(u64 codes, float f) {
    u64 r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 x = kvb_values((unsigned int)(codes >> (16 * e)) & 0xFFFFu);
        r |= (u64)kvb_codes(make_float2(x.x * f, x.y * f)) << (16 * e);
    }
    return r;
}
__device__ __forceinline__ u64 kvb_row_codes(const float2 (&x)[4], float f) {
    u64 r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) r |= (u64)kvb_codes(make_float2(x[e].x * f, x[e].y * f)) << (16 * e);
    return r;
}

struct KvbWriteArgs {
    KvWriteArgs w;                 // (slot_map: none)
    const int32_t* block_table;
    const int32_t* cached_len;
    const int32_t* kv_len;
    const int32_t* tok_offsets;    // packed rows
    int n_seqs, max_pages, rows_per_seq;
    unsigned int units;            // pages that rows may be stored to (an upper bound), times heads, times two
    unsigned int store_blocks;     // CTAs that store; the others take queries
};

#ifdef AASD_KVB_TU

constexpr int kByteThreads = 256;

// A page's unit number: sequences have pages enough between tok_offsets / 64 + 2 b and the next one's, wherever in a page they
// go on (n rows touch at most n / 64 + 2 pages, one less where n % 64 is 0 or 1).
__device__ __forceinline__ int64_t kvb_first_unit(const KvbWriteArgs& a, int b) {
    const int64_t row = a.rows_per_seq > 0 ? (int64_t)b * a.rows_per_seq : a.tok_offsets[b];
    return (row < 0 ? 0 : row) / kPage + 2 * (int64_t)b;
}

// What a unit stores: rows [i0, i1) of sequence b (counted from its first new one) to one page.
struct KvbUnit {
    int64_t row0;      // token row of the sequence's first new token
    int i0, i1;
    int page;          // -1: none
    int place;         // of row i0
    int older;         // live older places of the page
};

// W warps store the rows of one page, head and half (a unit): they are normed and rotated (keys), the largest magnitude
// gives the page's scale, and the codes follow.  Rows of a page that fit the unit's registers are held between the two,
// others are made again.  Queries are rows of their own (D / 16 lanes each), as in the 4-bit store.
//
// The scale makes a page, head and half the unit: what it shares has to be known before its first code is stored.  Bound by
// latency: with prompts a unit's trips to memory stand in a row (lengths, table, rows, positions, cosines; each row read once and
// held), and the registers of the held rows leave 21 of an SM's 64 warps to fill the time.  They wait for memory a third of it, for
// the operation before a fifth, and issue in 55 % of the slots; DRAM is at 21 %.  With a step's tokens it is one pass of the chain.
// Measured (32 query and 8 key heads of 128 channels, bf16): four prompts of 4150 tokens in all 30 us, 93 MB at 3.1 TB/s
// (two CTAs per SM, whose registers are not held to 80, 39 us); 4 trees of 5 tokens 6 us.
constexpr int kWriteCtas = 3;              // CTAs per SM that registers are kept free for
template <int DT, int D, bool VEC, bool FULL, int W>
__global__ void __launch_bounds__(kByteThreads, D == 256 ? 1 : kWriteCtas) kvb_write_kernel(const KvbWriteArgs a) {
    constexpr int L = D / 16, H = D / 2;
    constexpr int T = 32 * W, U = kByteThreads / T;      // threads of a unit, units of a CTA
    constexpr int kRows = T / L;                         // rows of a pass
    constexpr int kHold = W == 8 ? kPage / kRows : 1;    // passes whose rows are held
    __shared__ float s_rows[FULL ? 1 : kByteThreads / L * D];
    __shared__ unsigned int s_top[kByteThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int hq = a.w.p.n_q_heads, hkv = a.w.p.n_kv_heads;
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    float* mine = s_rows + (FULL ? 0 : group * D);
    unsigned int bits = 0;
    if (blockIdx.x >= a.store_blocks) {
        // ---- queries
        const int64_t g = ((int64_t)(blockIdx.x - a.store_blocks) * kByteThreads + threadIdx.x) / L;
        const bool live = g < a.w.n_tokens * hq;
        const int64_t t = live ? g / hq : 0;
        const int h = live ? (int)(g - t * hq) : 0;
        Raw8<DT, VEC> rx, ry;
        rx.clear();
        ry.clear();
        if (live) {
            const int64_t at = t * a.w.p.q_stride + (int64_t)h * D + 8 * l;
            rx.load(a.w.q, at);
            ry.load(a.w.q, at + H);
        }
        int pos = AASD_NONE, slot;
        if (live) bits |= kv_write_token(a.w, t, false, pos, slot);
        const bool used = live && pos != AASD_NONE;
        if (!used) {
            rx.clear();
            ry.clear();
        }
        float2 u[4], v[4];
        kv_norm_rotate<DT, D, VEC, FULL>(a.w, rx, ry, l, used, pos, a.w.q_weight, mine, u, v);
        if (live) {
            const int64_t at = (t * hq + h) * D + 8 * l;
            store8<DT, VEC>(a.w.q_out, at, u);
            store8<DT, VEC>(a.w.q_out, at + H, v);
        }
        if (bits) raise(a.w.state, bits);
        return;
    }
    // ---- keys and values
    const unsigned int unit = blockIdx.x * U + threadIdx.x / T;
    const int ut = threadIdx.x % T, lane = threadIdx.x & 31;
    const bool value = (unit & 1u) != 0;
    const int head = (int)((unit >> 1) % (unsigned int)hkv);
    const int64_t pu = (unit >> 1) / (unsigned int)hkv;
    // the unit's sequence: the last one whose first unit is not behind it (a 32nd of the range at a time)
    int b = 0;
    if (a.rows_per_seq > 0 && a.n_seqs > 0) {
        const int64_t each = a.rows_per_seq;
        b = (int)min((int64_t)a.n_seqs - 1, pu * kPage / (each + 2 * kPage) );
        while (b + 1 < a.n_seqs && kvb_first_unit(a, b + 1) <= pu) ++b;
    } else {
        int n = a.n_seqs;
        while (n > 1) {
            const int step = (n + 31) / 32, at = b + lane * step;
            const unsigned int below = __ballot_sync(0xFFFFFFFFu, at < b + n && kvb_first_unit(a, at) <= pu);
            const int k = below ? 31 - __clz(below) : 0;
            n = min(step, b + n - (b + k * step));
            b += k * step;
        }
    }
    KvbUnit q{0, 0, 0, -1, 0, 0};
    if (unit < a.units && a.n_seqs > 0) {
        const int cached = a.cached_len[b];
        int64_t fresh = (int64_t)a.kv_len[b] - cached, rows = a.rows_per_seq;
        q.row0 = (int64_t)b * a.rows_per_seq;
        if (a.rows_per_seq == 0) {
            q.row0 = a.tok_offsets[b];
            rows = (int64_t)a.tok_offsets[b + 1] - q.row0;
        }
        const bool inside = q.row0 >= 0 && rows >= 0 && q.row0 + rows <= a.w.n_tokens && cached >= 0;
        fresh = inside ? (fresh < rows ? fresh : rows) : 0;
        const int64_t k = cached / kPage + (pu - kvb_first_unit(a, b)), lo = k * kPage > cached ? k * kPage : cached;
        const int64_t end = (int64_t)cached + fresh, hi = (k + 1) * kPage < end ? (k + 1) * kPage : end;
        if (cached >= 0 && lo < hi && pu >= kvb_first_unit(a, b)) {
            q.i0 = (int)(lo - cached);
            q.i1 = (int)(hi - cached);
            q.place = (int)(lo - k * kPage);
            q.older = k * kPage < cached ? q.place : 0;
            q.page = k < a.max_pages ? a.block_table[(int64_t)b * a.max_pages + k] : -1;
            if (q.page < 0 || q.page >= a.w.p.n_pages) {
                bits |= AASD_STATUS_BAD_OFFSETS;
                q.page = -1;
            }
        }
    }
    const int n = q.i1 - q.i0;
    uint8_t* block = a.w.pages + ((int64_t)(q.page < 0 ? 0 : q.page) * hkv + head) * kvb_head_bytes(D);
    uint8_t* base = block + (value ? kvb_value_offset(D) : 0);
    unsigned int* scale = reinterpret_cast<unsigned int*>(block + kvb_scale_offset(D)) + (value ? 1 : 0);
    const unsigned int was = q.page >= 0 && q.older > 0 ? *scale : 0u;
    // Row r of the unit, as it is to be stored.  Every lane of the warp comes here; rows with a NaN or infinity, and rows without a
    // position, become zeros.  first: what there is to say of the row is said; last: it is not read again, and k_out, which may be
    // the row's own place, gets it.
    auto row = [&](int r, bool first, bool last, float2(&u)[4], float2(&v)[4]) {
        const bool on = r < n;
        const int64_t t = q.row0 + q.i0 + (on ? r : 0);
        Raw8<DT, VEC> rx, ry;
        rx.clear();
        ry.clear();
        if (on) {
            const int64_t at = t * (value ? a.w.p.v_stride : a.w.p.k_stride) + (int64_t)head * D + 8 * l;
            rx.load(value ? a.w.v : a.w.k, at);
            ry.load(value ? a.w.v : a.w.k, at + H);
        }
        int pos = AASD_NONE, slot;
        unsigned int said = on ? kv_write_token(a.w, t, false, pos, slot) : 0u;
        const bool used = on && pos != AASD_NONE;
        if (!used) {
            rx.clear();
            ry.clear();
        }
        if (value) {
            rx.unpack(u);
            ry.unpack(v);
        } else {
            kv_norm_rotate<DT, D, VEC, FULL>(a.w, rx, ry, l, used, pos, a.w.k_weight, mine, u, v);
            if (last && on && a.w.k_out != nullptr) {
                const int64_t at = (t * hkv + head) * D + 8 * l;
                store8<DT, VEC>(a.w.k_out, at, u);
                store8<DT, VEC>(a.w.k_out, at + H, v);
            }
        }
        unsigned int top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            top = max(top, max(__float_as_uint(fabsf(u[e].x)), __float_as_uint(fabsf(u[e].y))));
            top = max(top, max(__float_as_uint(fabsf(v[e].x)), __float_as_uint(fabsf(v[e].y))));
        }
#pragma unroll
        for (int o = 1; o < L; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (top >= 0x7F800000u) {
            said |= AASD_STATUS_BAD_ROW;
            top = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = v[e] = make_float2(0.f, 0.f);
        }
        if (first) bits |= said;
        return top;
    };
    float2 u[kHold][4], v[kHold][4];
    unsigned int top = 0;
    const int r0 = ut / L;
    const int rounds = q.page < 0 ? 0 : (n + kRows - 1) / kRows;
    // (the warps of a unit take the same number of rounds; rows are held from the last ones on)
    if constexpr (kHold > 1) {
#pragma unroll
        for (int p = 0; p < kHold; ++p)
            if (p < rounds) top = max(top, row(p * kRows + r0, true, true, u[p], v[p]));
    } else {
#pragma unroll 1
        for (int p = 0; p < rounds; ++p) top = max(top, row(p * kRows + r0, true, p == rounds - 1, u[0], v[0]));
    }
#pragma unroll
    for (int o = L; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (W > 1) {
        if (lane == 0) s_top[threadIdx.x >> 5] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = max(top, s_top[(threadIdx.x / T) * W + w]);
    }
    if (q.page >= 0 && AASD_IN_RANGE(q.page < a.w.p.n_pages && head < hkv && q.place + n <= kPage, a.w.state)) {
        const int old = kvb_exponent(was);
        int e = kvb_fit(top);
        if (q.older > 0) e = max(e, old);
        const float f = kvb_pow2(-e);
        auto put = [&](int r, const float2(&x)[4], const float2(&y)[4]) {
            if (r >= n) return;
            const int t = q.place + r;
            *reinterpret_cast<u64*>(base + kvb_chunk_offset(D, t, l >> 1) + 8 * (l & 1)) = kvb_row_codes(x, f);
            *reinterpret_cast<u64*>(base + kvb_chunk_offset(D, t, (H / 16) + (l >> 1)) + 8 * (l & 1)) = kvb_row_codes(y, f);
        };
        if constexpr (kHold > 1) {
#pragma unroll
            for (int p = 0; p < kHold; ++p)
                if (p < rounds) put(p * kRows + r0, u[p], v[p]);
        } else {
            if (rounds > 0) put((rounds - 1) * kRows + r0, u[0], v[0]);
#pragma unroll 1
            for (int p = 0; p < rounds - 1; ++p) {
                row(p * kRows + r0, false, true, u[0], v[0]);
                put(p * kRows + r0, u[0], v[0]);
            }
        }
        // older entries follow a scale that grows
        if (q.older > 0 && e > old) {
            const float g = e - old > 126 ? 0.f : kvb_pow2(old - e);
            for (int i = ut; i < q.older * (D / 8); i += T) {
                const int t = i / (D / 8), c = i % (D / 8);
                u64* at = reinterpret_cast<u64*>(base + kvb_chunk_offset(D, t, c >> 1) + 8 * (c & 1));
                *at = kvb_rescale(*at, g);
            }
        }
        if (ut == 0) *scale = (unsigned int)(e + 127) << 23;
    }
    if (bits) raise(a.w.state, bits);
}

// ---- entries as values -----------------------------------------------------------------------------

// A lane per 16 bytes of a row (16 channels): keys and values of (slot, head), in the order of the outputs.  4150 slots of 8 heads
// of 128 channels 8 us, 26 MB at half the copy rate; a few slots 4 us.  Both are one trip to memory behind another (slot, codes and
// scale, stores): with many slots the warps wait for memory half of their time and for their stores to leave a seventh, in CTAs
// that go through the chain once; DRAM is at 12 %, L1 at 68.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(kByteThreads) kvb_read_kernel(const KvReadArgs a) {
    constexpr int C = D / 16;              // 16-byte chunks of a row
    pdl_launch_dependents();
    pdl_wait();
    const int hkv = a.n_kv_heads;
    const int64_t g = (int64_t)blockIdx.x * kByteThreads + threadIdx.x;
    const int64_t row = g / C;
    const int c = (int)(g % C);
    if (row >= a.n * hkv) return;
    const int64_t i = row / hkv;
    const int head = (int)(row - i * hkv);
    int slot = a.slots[i];
    if (slot < AASD_NONE || slot / kPage >= a.n_pages) {
        if (head == 0 && c == 0) raise(a.state, AASD_STATUS_ID_RANGE);
        slot = AASD_NONE;
    }
    const bool on = slot != AASD_NONE && AASD_IN_RANGE(slot >= 0 && slot / kPage < a.n_pages, a.state);
    const uint8_t* block = a.pages + ((int64_t)(on ? slot / kPage : 0) * hkv + head) * kvb_head_bytes(D);
    const int at = kvb_chunk_offset(D, on ? slot % kPage : 0, c);
    uint4 w[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    uint2 scale = make_uint2(0u, 0u);
    if (on) {
        w[0] = *reinterpret_cast<const uint4*>(block + at);
        w[1] = *reinterpret_cast<const uint4*>(block + kvb_value_offset(D) + at);
        scale = *reinterpret_cast<const uint2*>(block + kvb_scale_offset(D));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        void* out = k ? a.v_out : a.k_out;
        if (out == nullptr) continue;
        const float s = kvb_pow2(kvb_exponent(k ? scale.y : scale.x));
        const unsigned int word[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            float2 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 y = kvb_values((word[2 * p + (e >> 1)] >> (16 * (e & 1))) & 0xFFFFu);
                x[e] = make_float2(y.x * s, y.y * s);
            }
            store8<DT, VEC>(out, row * D + 16 * c + 8 * p, x);
        }
    }
}

// ---- the accepted path ------------------------------------------------------------------------------

// grid: (sequence, group of heads of all layers), as in the 4-bit cache; a warp moves the keys or the values of one head,
// target page by target page.  A page's scale becomes the largest of its own and those its new entries come from; entries
// that stay follow it.  Places behind the path are left as they are.  A chain of loads that depend on one another (parents, path,
// table, scales, codes); heads of all layers go side by side.  Measured: one path in 16 layers of 8 heads of 128 channels 6 us,
// 128 paths in 4 layers of 4 heads 9 us.
template <int D>
__global__ void __launch_bounds__(kCommitThreads) kvb_commit_kernel(const KvCommitArgs a) {
    __shared__ int s_node[AASD_KV_MAX_NODES];
    __shared__ int s_path[AASD_KV_MAX_NODES];
    __shared__ int s_len, s_bad;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const int cached = a.cached_len[b];
    const KvPath path = kv_accepted_path(a, b, cached, s_node, s_path, s_len, s_bad);
    if (path.from >= path.len) return;
    constexpr int WORDS = D / 8;                                 // 8-byte words of an entry's half
    constexpr int PER = WORDS < 32 ? 32 / WORDS : 1;             // entries that a warp fetches at a time
    constexpr int NB = 4;                                        // such fetches under way together
    static_assert(WORDS <= 32, "a lane per word");
    const int64_t items = (int64_t)a.p.n_layers * a.p.n_kv_heads * 2, hb = kvb_head_bytes(D);
    for (int64_t it = (int64_t)blockIdx.y * (kCommitThreads / 32) + (tid >> 5); it < items; it += (int64_t)gridDim.y * (kCommitThreads / 32)) {
        const int half = (int)(it & 1);
        const int64_t lh = it >> 1;
        const int layer = (int)(lh / a.p.n_kv_heads), head = (int)(lh % a.p.n_kv_heads);
        uint8_t* pool = a.pages + (int64_t)layer * a.p.layer_stride;
        const auto block_of = [&](int slot) { return pool + ((int64_t)(slot / kPage) * a.p.n_kv_heads + head) * hb; };
        const auto scale_of = [&](int slot) { return reinterpret_cast<unsigned int*>(block_of(slot) + kvb_scale_offset(D)) + half; };
        const auto word_of = [&](int slot, int w) {
            return reinterpret_cast<u64*>(block_of(slot) + (half ? kvb_value_offset(D) : 0) + kvb_chunk_offset(D, slot % kPage, w >> 1) + 8 * (w & 1));
        };
        for (int i0 = path.from; i0 < path.len;) {
            const int dst0 = kv_commit_slot(a, b, cached, i0);
            const int n = min(path.len - i0, kPage - dst0 % kPage);   // entries that this page takes
            if (!AASD_IN_RANGE(dst0 >= 0 && dst0 / kPage < a.p.n_pages && layer < a.p.n_layers, a.state)) return;
            const int own = kvb_exponent(*scale_of(dst0));
            int e = own;
            for (int i = lane; i < n; i += 32) e = max(e, kvb_exponent(*scale_of(s_node[i0 + i])));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) e = max(e, __shfl_xor_sync(0xFFFFFFFFu, e, o));
            if (e > own) {
                // what stays: cached entries and the path's first ones
                const float f = e - own > 126 ? 0.f : kvb_pow2(own - e);
                const int stay = dst0 % kPage;
                for (int k = lane; k < stay * WORDS; k += 32) {
                    u64* at = word_of(dst0 - stay + k / WORDS, k % WORDS);
                    *at = kvb_rescale(*at, f);
                }
            }
            for (int k0 = 0; k0 < n; k0 += NB * PER) {
                u64 x[NB];
#pragma unroll
                for (int q = 0; q < NB; ++q) {
                    const int k = k0 + q * PER + lane / WORDS;
                    x[q] = 0;
                    if (k < n && lane / WORDS < PER) {
                        const int src = s_node[i0 + k], from = kvb_exponent(*scale_of(src));
                        x[q] = *word_of(src, lane % WORDS);
                        if (from < e) x[q] = kvb_rescale(x[q], e - from > 126 ? 0.f : kvb_pow2(from - e));
                    }
                }
                __syncwarp();   // every lane has its loads before the first store
#pragma unroll
                for (int q = 0; q < NB; ++q) {
                    const int k = k0 + q * PER + lane / WORDS;
                    if (k < n && lane / WORDS < PER) *word_of(dst0 + k, lane % WORDS) = x[q];
                }
                __syncwarp();
            }
            if (e > own && lane == 0) *scale_of(dst0) = (unsigned int)(e + 127) << 23;
            __syncwarp();
            i0 += n;
        }
    }
}
#endif

}  // namespace aasd
