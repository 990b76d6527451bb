// Attention of a step's new tokens over the paged 4-bit cache.
//
// The rows of a key/value head are the queries of its group of query heads for every new token:
// row = i * G + g for token i and query head h * G + g.  A code c stands for s c + m with the
// token's own scale and minimum, so
//     q . k_t     = s_t (q . c_t) + m_t sum(q)
//     sum p_t v_t = sum (p_t s_t) c_t + sum p_t m_t
// and the matrix products run on the bare codes.  A code needs no conversion to get there: the
// 16 bits 0x000c are the fp16 number c 2^-24 and 0x00c0 are c 2^-20 (both exact), so one AND per
// two codes makes a tensor-core operand, and the powers of two join the factors above.
#pragma once

#include <cuda_fp16.h>

#include <type_traits>

#include "aasd_kv.cuh"
#include "aasd_stream.cuh"

namespace aasd {

// A partial result: the part of a segment (one row tile of one head of one sequence) whose pages
// one warp, or one CTA, has been through.
struct KvPiece {
    int seg;            // unit of the segment's first page, -1: no piece
    int pages;          // of the segment
    int h, row0, n;     // head, first row of the tile, rows in use
    int first;          // token row of the sequence's first new token
};

// What the tile kernel leaves per CTA: the segment that it began and others go on with, how many
// CTAs hold parts of it (0: there is none), and (the same from every CTA) whether there are rows to
// clear: 1 padding, 2 all.
struct KvTileOpen {
    KvPiece piece;
    int parts, padding;
};

struct KvAttendArgs {
    const void* q;
    const uint8_t* pages;
    const int32_t* block_table;
    const int32_t* cached_len;
    const int32_t* kv_len;
    const int32_t* tok_offsets;   // packed rows
    const int32_t* node_parent;   // may be NULL
    aasd_kv_attend_params p;
    aasd_kv_attend_out o;
    float scale_log2;             // scale * log2 e
    int q_vec, out_vec;           // rows of q / out start on 16-byte boundaries
    DeviceState* state;
    unsigned int* tickets;        // scratch, zero between calls
    float* cta_parts;             // scratch: partial results of segments that several CTAs share
    KvTileOpen* tile_open;        // scratch, one per CTA of the tile kernel
    float* warp_parts;            // scratch: a warp's first piece, when it goes on to another segment
    unsigned int wait_limit;      // polls after which a wait inside the kernels gives up (kWaitLimit)
    int withhold_page;            // testing aid (aasd_debug_withhold_tile): the first CTA's page of this number never arrives; -1: none
};

// Bounded wait (see mbar_wait).  The call's limit is looked at every 256 polls, off the path of waits that end.
__device__ __forceinline__ bool kv_wait(const KvAttendArgs& a, u64* bar, unsigned int parity, volatile int* abort_flag) {
#pragma unroll 1
    for (unsigned int it = 0; it < kWaitLimit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 255u) == 255u && (*abort_flag || it > a.wait_limit)) break;
    }
    return false;
}

constexpr int kKvMaxCtas = 160;        // CTAs of a launch (one per SM)
constexpr float kKvNothing = -3.0e38f; // running maximum of a row that has seen nothing (below any sum of products)
constexpr float kKvHidden = -3.3e38f;  // exponent of a key that the row does not see

// ---- what there is to do ---------------------------------------------------------------------------

struct KvSeq {
    int cached, fresh;        // cached tokens; new tokens in the cache
    int first;                // token row of the first new one
    int rows;                 // token rows, padding included
    int pages;                // pages that hold them
    int tiles;                // row tiles of a key/value head
};

// tile_rows: rows of a tile.  PAGE: tokens of what is counted as a page (a kernel may take pages in parts).
template <int PAGE = kPage>
__device__ __forceinline__ KvSeq kv_load_seq(const KvAttendArgs& a, int b, int tile_rows) {
    KvSeq s;
    s.cached = a.cached_len[b];
    const long long fresh = (long long)a.kv_len[b] - s.cached;
    long long first, rows;
    if (a.p.rows_per_seq > 0) {
        first = (long long)b * a.p.rows_per_seq;
        rows = a.p.rows_per_seq;
    } else {
        first = a.tok_offsets[b];
        rows = (long long)a.tok_offsets[b + 1] - first;
    }
    const bool inside = first >= 0 && rows >= 0 && first + rows <= a.p.n_tokens;
    s.first = inside ? (int)first : 0;
    s.rows = inside ? (int)rows : 0;
    s.fresh = s.cached < 0 || fresh < 0 ? 0 : (int)(fresh < s.rows ? fresh : s.rows);
    const long long pages = ((long long)s.cached + s.fresh + PAGE - 1) / PAGE, most = (long long)a.p.max_pages * (kPage / PAGE);
    s.pages = s.fresh == 0 ? 0 : (int)(pages < most ? pages : most);
    const long long n = (long long)s.fresh * (a.p.n_q_heads / a.p.n_kv_heads);
    s.tiles = (int)((n + tile_rows - 1) / tile_rows);
    return s;
}
// Work is counted in pages: a segment (one row tile of one head of one sequence) is kSegCost + its
// pages, the first for loading the queries and handing the result on, which take a warp about as
// long as a page.  Page p of the segment is unit kSegCost + p of it.
constexpr int kSegCost = 1;
__device__ __forceinline__ long long kv_units(const KvAttendArgs& a, const KvSeq& s) {
    return s.pages == 0 ? 0 : (long long)(s.pages + kSegCost) * s.tiles * a.p.n_kv_heads;
}

// A place in the list of all units: sequence by sequence, head by head, tile by tile, page by page.
template <int PAGE = kPage>
struct KvCursor {
    int b, h, tile, pg;
    int unit;                 // of page pg
    KvSeq s;
    const int32_t* table;     // the sequence's row of the block table
    // To the first page at or behind unit u, which is unit rem of sequence b_.
    __device__ __forceinline__ void seek(const KvAttendArgs& a, int b_, const KvSeq& s_, int rem, int u) {
        b = b_;
        s = s_;
        unit = u;
        const int seg = rem / (s.pages + kSegCost);
        unit -= rem;                                           // (of the sequence's first unit)
        rem -= seg * (s.pages + kSegCost);
        pg = rem < kSegCost ? 0 : rem - kSegCost;
        unit += seg * (s.pages + kSegCost) + kSegCost + pg;
        h = seg / s.tiles;
        tile = seg - h * s.tiles;
        table = a.block_table + (long long)b * a.p.max_pages;
    }
    __device__ __forceinline__ void next_segment(const KvAttendArgs& a, int tile_rows) {
        pg = 0;
        unit += kSegCost;
        if (++tile < s.tiles) return;
        tile = 0;
        if (++h < a.p.n_kv_heads) return;
        h = 0;
#pragma unroll 1
        do {
            if (++b >= a.p.n_seqs) return;   // (past the last unit: never looked at)
            s = kv_load_seq<PAGE>(a, b, tile_rows);
        } while (s.pages == 0 || s.tiles == 0);
        table = a.block_table + (long long)b * a.p.max_pages;
    }
};

// `total` units in `n` shares that differ by one unit at most, the larger ones first.
struct KvShares {
    int each, more;           // units of a small share; shares with one more
    KvShares() = default;
    __device__ __forceinline__ KvShares(int total, int n) {
        each = (int)((unsigned int)total / (unsigned int)n);
        more = total - each * n;
    }
    __device__ __forceinline__ int first(int share) const { return each * share + min(share, more); }
    __device__ __forceinline__ int owner(int unit) const {
        const int big = (each + 1) * more;
        return unit < big ? (int)((unsigned int)unit / (unsigned int)(each + 1)) : more + (int)((unsigned int)(unit - big) / (unsigned int)each);
    }
};

// All units of a call: what the threads of a CTA have added up.  Units are counted in 31 bits (137 G keys).
__device__ __forceinline__ int kv_total(const KvAttendArgs& a, long long total) {
    if (total <= 0x7FFFFFFFLL) return (int)total;
    raise(a.state, AASD_STATUS_BAD_OFFSETS);
    return 0;
}

// One row tile of one head of one sequence, as a warp works on it.
struct KvSegment {
    int cached, fresh, first; // see KvSeq
    int pages;
    int h, row0;              // head, first row of the tile
    int pg;                   // the warp's first page of it
    int unit;                 // of page 0
};

// Bit j of the result: place 64 pg + j of a sequence (a cached token or a new one) is seen by its new
// token i.  cached, fresh, first: see KvSeq.
__device__ __forceinline__ u64 kv_seen(const KvAttendArgs& a, int cached, int fresh, int first, int pg, int i) {
    if (i >= fresh) return 0ull;
    const int before = cached - pg * kPage;                       // cached tokens of this page
    u64 seen = before >= kPage ? ~0ull : before <= 0 ? 0ull : (1ull << before) - 1ull;
    if (a.node_parent == nullptr) {
        const int upto = before + i + 1;                          // causal
        return upto >= kPage ? ~0ull : upto <= 0 ? 0ull : (1ull << upto) - 1ull;
    }
    int x = i;
#pragma unroll 1
    while (x >= 0) {
        const int j = before + x;
        if (j < 0) break;                                         // ancestors only get smaller
        if (j < kPage) seen |= 1ull << j;
        const int p = a.node_parent[first + x];
        if (p >= x || p < AASD_NONE) {
            raise(a.state, AASD_STATUS_BAD_OFFSETS);
            break;
        }
        x = p;
    }
    return seen;
}

// ---- tensor-core and packing primitives --------------------------------------------------------------

__device__ __forceinline__ void mma_16816(float (&c)[4], unsigned int a0, unsigned int a1, unsigned int a2, unsigned int a3,
                                          unsigned int b0, unsigned int b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned int transpose_8x8(unsigned int x) {
    unsigned int y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ unsigned int pack_half(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned int*>(&h);
}
// What rounding to fp16 left out of a and b.
__device__ __forceinline__ unsigned int pack_rest(float a, float b, unsigned int h) {
    const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return pack_half(a - r.x, b - r.y);
}
// Two codes of a word as fp16 numbers: those in bits 0-3 and 16-19 (HIGH = false) or 4-7 and 20-23.
// CENTRED = false: c 2^-24, or c 2^-20 for the high ones.  CENTRED: c - 8, one operation more, for
// fp32 queries: sums of c itself are several times the result that is left when the minimum's part
// is added, and fp32 results would show it.
template <bool CENTRED, bool HIGH>
__device__ __forceinline__ unsigned int codes(unsigned int w) {
    constexpr unsigned int mask = HIGH ? 0x00F000F0u : 0x000F000Fu;
    if constexpr (!CENTRED) {
        return w & mask;
    } else {
        const unsigned int b = (w & mask) | 0x64006400u;            // 1024 + c, or 1024 + 16 c
        __half2 h = *reinterpret_cast<const __half2*>(&b);
        h = HIGH ? __hfma2(h, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hsub2(h, __float2half2_rn(1032.f));
        return *reinterpret_cast<const unsigned int*>(&h);
    }
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }   // -126 <= e <= 127

template <int DT>
__device__ __forceinline__ void store4(void* base, long long i, float4 x, bool vec) {
    if constexpr (DT == AASD_F32) {
        float* p = static_cast<float*>(base) + i;
        if (vec) *reinterpret_cast<float4*>(p) = x;
        else { p[0] = x.x; p[1] = x.y; p[2] = x.z; p[3] = x.w; }
    } else {
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + i;
        if (vec) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
        else {
            p[0] = __float2bfloat16_rn(x.x);
            p[1] = __float2bfloat16_rn(x.y);
            p[2] = __float2bfloat16_rn(x.z);
            p[3] = __float2bfloat16_rn(x.w);
        }
    }
}

// ---- rows that see nothing ---------------------------------------------------------------------------

// Whether sequence b has rows without a placed token, or rows lie outside the sequences (found with b = 0).
__device__ __forceinline__ bool kv_has_padding(const KvAttendArgs& a, const KvSeq& s, int b) {
    if (a.p.rows_per_seq > 0) return s.fresh != a.p.rows_per_seq;
    return s.fresh != (long long)a.tok_offsets[b + 1] - a.tok_offsets[b] ||
           (b == 0 && (a.tok_offsets[0] != 0 || a.tok_offsets[a.p.n_seqs] != a.p.n_tokens));
}
// Zeros (and an lse of -inf) for the token rows that hold no placed token.  The warps of the whole grid
// share them: each sequence's padding over `share` warps, then the rows outside every sequence over
// all (by one warp, 20000 rows of 32 heads of 128 channels took 22 ms behind a call of 0.37 ms).
// A sequence whose rows pass n_tokens (aasd_kv_plan leaves it out) has none placed: those of its rows
// that exist are cleared.  total: all units of the call; where there are none (or more than can be
// counted) no row is worked on.  Calls without padding skip this.
template <int DT>
__device__ __forceinline__ void kv_clear_rows(const KvAttendArgs& a, int D, int total, int warp, int warps) {
    const int lane = threadIdx.x & 31;
    const int Hq = a.p.n_q_heads, B = a.p.n_seqs;
    const bool padded = a.p.rows_per_seq > 0;
    const int share = B > 0 && B < warps ? warps / B : 1;
    const int rounds = B > 0 ? (B * share + warps - 1) / warps : 0;
#pragma unroll 1
    for (int r = 0; r < (padded ? rounds : rounds + 2); ++r) {
        long long lo = 0, hi = 0;
        int part = warp, parts = warps;
        if (r < rounds) {
            const int item = warp + r * warps, b = item / share;
            if (b >= B) continue;
            part = item - b * share;
            parts = share;
            // (not KvSeq's first and rows, which are none where they do not all exist)
            lo = padded ? (long long)b * a.p.rows_per_seq : a.tok_offsets[b];
            hi = padded ? lo + a.p.rows_per_seq : a.tok_offsets[b + 1];
            lo += total > 0 ? kv_load_seq(a, b, 8).fresh : 0;
        } else if (r == rounds) {
            lo = B > 0 ? a.tok_offsets[B] : 0;
            hi = a.p.n_tokens;
        } else if (B > 0) {
            hi = a.tok_offsets[0];
        }
        lo = lo < 0 ? 0 : lo;
        hi = hi < a.p.n_tokens ? hi : a.p.n_tokens;
        const long long e1 = hi * Hq * D;
#pragma unroll 1
        for (long long e = lo * Hq * D + part * 128 + lane * 4; e < e1; e += parts * 128) store4<DT>(a.o.out, e, make_float4(0.f, 0.f, 0.f, 0.f), a.out_vec);
        if (a.o.lse)
#pragma unroll 1
            for (long long e = lo * Hq + part * 32 + lane; e < hi * Hq; e += parts * 32) a.o.lse[e] = -CUDART_INF_F;
    }
}

// ---- a row's result ----------------------------------------------------------------------------------

// From the row's denominator l and, in base 2, what it is relative to: a factor of the sums, and the lse.  A row that sees nothing (l = 0)
// gives zeros and -inf; a denominator that is NaN (a query that is not finite) goes on into both.
__device__ __forceinline__ float kv_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float kv_lse(float m, float l) { return l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * (float)kLn2; }

// ---- joining ---------------------------------------------------------------------------------------------

// Row r of a segment from its parts, one warp.  Part k lies at base + 2 k stride, the first one stride further;
// a part is rows of D sums, then the rows' maxima, then their denominators.  The weights are found lane
// by lane, the channels summed as independent loads.
template <int DT, int D>
__device__ __forceinline__ void kv_join_row(const KvAttendArgs& a, const KvPiece& pc, int r, const float* base, int stride, int rows, int parts, int G,
                                            int lane) {
    float M = kKvNothing;
#pragma unroll 1
    for (int k = lane; k < parts; k += 32) M = fmaxf(M, __ldcg(base + (long long)(2 * k + (k == 0)) * stride + rows * D + r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
#pragma unroll 1
    for (int cb = 0; cb < D; cb += 128) {
        const int ch = cb + lane * 4;
        const bool on = ch < D;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        float L = 0.f, f = 0.f;
#pragma unroll 1
        for (int k0 = 0; k0 < parts; k0 += 8) {
            if ((k0 & 31) == 0) {
                const int k = k0 + lane;
                const float* from = base + (long long)(2 * k + (k == 0)) * stride + rows * D + r;
                f = k < parts ? ex2_approx(__ldcg(from) - M) : 0.f;
                if (k < parts) L = fmaf(__ldcg(from + rows), f, L);
            }
            float4 x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int k = k0 + q;
                x[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (on && k < parts) x[q] = __ldcg(reinterpret_cast<const float4*>(base + (long long)(2 * k + (k == 0)) * stride + r * D + ch));
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float fk = __shfl_sync(0xFFFFFFFFu, f, (k0 + q) & 31);
                o.x = fmaf(x[q].x, fk, o.x);
                o.y = fmaf(x[q].y, fk, o.y);
                o.z = fmaf(x[q].z, fk, o.z);
                o.w = fmaf(x[q].w, fk, o.w);
            }
        }
#pragma unroll
        for (int q = 16; q > 0; q >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, q);
        if (!on) continue;
        const float inv = kv_inverse(L);
        const int row = pc.row0 + r;
        const long long head = ((long long)pc.first + row / G) * a.p.n_q_heads + pc.h * G + row % G;
        if (!AASD_IN_RANGE(parts <= kKvMaxCtas && head < a.p.n_tokens * a.p.n_q_heads, a.state)) continue;
        store4<DT>(a.o.out, head * D + ch, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), a.out_vec);
        if (a.o.lse != nullptr && ch == 0) a.o.lse[head] = kv_lse(M, L);
    }
}

// ---- few rows per head: the keys split over all warps -----------------------------------------------

// W warps per CTA, each with a ring of S blocks of its own that lane 0 fills with one bulk copy per
// block: 100 to 200 KB per SM are on their way at any time (memory wants about 40).  Twelve warps
// where their registers allow it (168 each): the chains of a page's products and exponentials leave
// issue slots that only other warps fill.
//
// The list of all pages is cut into equal shares, one per warp, whatever sequences they belong to;
// pieces of a segment are joined first in the CTA, then by the last CTA that delivers one.
// Measured (bf16, 128 channels): 256 sequences of 100 to 4000 tokens, 28 query and 4 key heads, 66 us, two
// thirds of the copy rate (start-up 10 us, joining 5); one sequence of 16384 tokens 16 us, which is
// the chain plan of the share - table - page - product - join - join and not its 18 MB (2.7 us).
template <int DT, int D, int NT>
struct KvSplitShape {
    static constexpr int W = D == 256 ? 4 : DT == AASD_BF16 && NT == 1 ? 12 : 8;
    static constexpr int S = D == 64 ? (W == 12 ? 4 : 5) : W == 12 ? 2 : 3;
    static constexpr int kBlock = kv_head_bytes(D);
    static constexpr int kThreads = W * 32;
};

template <int DT, int D, int NT>
struct KvSplitShared {
    using Sh = KvSplitShape<DT, D, NT>;
    static constexpr int R = 8 * NT;
    alignas(128) unsigned char ring[Sh::W][Sh::S][Sh::kBlock];
    int base[Sh::kThreads];
    long long scan[Sh::W];
    KvSegment seg[Sh::W][Sh::S + 1];   // of the blocks on their way, and the one being worked on
    KvPiece piece[2 * Sh::W];
    float m[2 * Sh::W][R], l[2 * Sh::W][R];
    u64 full[Sh::W][Sh::S];
    int abort_flag, last[2], padding;
};

// Joining the pieces of a CTA's W warps: a piece lies in its warp's first ring block (the last one of the share), or in the warp's
// scratch; rows are TS floats apart.
template <int DT, int D, int W, int R, int TS, class Shared>
__device__ __forceinline__ void kv_split_join(const KvAttendArgs& a, Shared& sh, const KvShares& shares) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
    const int G = a.p.n_q_heads / a.p.n_kv_heads;
    // Every warp finds the groups of pieces that belong together (lane k looks
    // at piece k) and the warps share the groups' rows; a row's weights are found lane by lane, its
    // channels summed as independent loads.
    static_assert(2 * W <= 32, "a lane per piece");
    constexpr int kPart = R * D + 2 * R;
    const int U0 = shares.first(c * W), U1 = shares.first(c * W + W);
    const int seg = lane < 2 * W ? sh.piece[lane].seg : -1;
    const unsigned int valid = __ballot_sync(0xFFFFFFFFu, seg >= 0);
    const unsigned int below = valid & ((1u << lane) - 1u);
    const int previous = __shfl_sync(0xFFFFFFFFu, seg, below ? 31 - __clz(below) : 0);
    unsigned int starts = __ballot_sync(0xFFFFFFFFu, seg >= 0 && (below == 0 || previous != seg));
    auto finish_row = [&](const KvPiece& pc, int r, float M, float L, float4 o, int ch) {
        const float inv = kv_inverse(L);
        const int row = pc.row0 + r;
        const long long head = ((long long)pc.first + row / G) * a.p.n_q_heads + pc.h * G + row % G;
        if (!AASD_IN_RANGE(head < a.p.n_tokens * a.p.n_q_heads, a.state)) return;
        store4<DT>(a.o.out, head * D + ch, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), a.out_vec);
        if (a.o.lse != nullptr && ch == 0) a.o.lse[head] = kv_lse(M, L);
    };
    int open[2] = {-1, -1};        // first pieces of the groups that other CTAs hold parts of: begun before this CTA, in it
    // rows r0 .. r0 + RB of the group of pieces `group`
    auto join_rows = [&](auto rb, const KvPiece& pc, unsigned int group, bool complete, float* part, int r0) {
        constexpr int RB = decltype(rb)::value;
        const bool in = (group >> lane) & 1u;
        const int own = lane < 2 * W ? lane : 0;
        float M[RB], L[RB], f[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            const int r = min(r0 + i, pc.n - 1);
            const float m = in ? sh.m[own][r] : kKvNothing;
            M[i] = m;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) M[i] = fmaxf(M[i], __shfl_xor_sync(0xFFFFFFFFu, M[i], o));
            f[i] = in ? ex2_approx(m - M[i]) : 0.f;
            L[i] = in ? sh.l[own][r] * f[i] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) L[i] += __shfl_xor_sync(0xFFFFFFFFu, L[i], o);
        }
        for (int cb = 0; cb < D; cb += 128) {
            const int ch = cb + lane * 4;
            const bool on = ch < D;
            float4 o[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            unsigned int left = group;
#pragma unroll 1
            while (left) {
                constexpr int NB = RB == 1 ? 4 : 1;   // pieces whose loads are under way together
                int k[NB];
                float4 x[NB][RB];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    k[b] = left ? __ffs(left) - 1 : -1;
                    left &= left - 1;
                    const float* from = (k[b] & 1) ? reinterpret_cast<const float*>(sh.ring[k[b] >> 1][0])
                                                   : a.warp_parts + (long long)(c * W + (k[b] >> 1)) * (R * TS);
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        x[b][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (on && k[b] >= 0) x[b][i] = *reinterpret_cast<const float4*>(from + min(r0 + i, pc.n - 1) * TS + ch);
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (NB > 1 && k[b] < 0) break;
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        const float fk = __shfl_sync(0xFFFFFFFFu, f[i], k[b]);
                        o[i].x = fmaf(x[b][i].x, fk, o[i].x);
                        o[i].y = fmaf(x[b][i].y, fk, o[i].y);
                        o[i].z = fmaf(x[b][i].z, fk, o[i].z);
                        o[i].w = fmaf(x[b][i].w, fk, o[i].w);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const int r = r0 + i;
                if (!on || r >= pc.n) continue;
                if (complete) {
                    finish_row(pc, r, M[i], L[i], o[i], ch);
                } else {
                    *reinterpret_cast<float4*>(part + r * D + ch) = o[i];
                    if (ch == 0) {
                        part[R * D + r] = M[i];
                        part[R * D + R + r] = L[i];
                    }
                }
            }
        }
    };
    // few rows: one per warp, else four at a time
    const bool few = __reduce_add_sync(0xFFFFFFFFu, (starts >> lane) & 1u ? (unsigned int)sh.piece[lane].n : 0u) <= (unsigned int)W;
    int done = 0;                              // row batches dealt with so far, modulo W
    while (starts) {
        const int p = __ffs(starts) - 1;
        starts &= starts - 1;
        const unsigned int group = valid & ~((1u << p) - 1u) & (starts ? (1u << (__ffs(starts) - 1)) - 1u : 0xFFFFFFFFu);
        const KvPiece pc = sh.piece[p];
        const bool complete = pc.seg >= U0 && pc.seg + pc.pages <= U1;
        const int which = pc.seg < U0 ? 0 : 1;   // scratch slot of this CTA
        if (!complete) open[which] = p;
        float* part = a.cta_parts + (long long)(c * 2 + which) * kPart;
        const int batches = few ? pc.n : (pc.n + 3) / 4;
        int k = warp - done;
        k += k < 0 ? W : 0;
        done = (done + batches) % W;
        for (; k < batches; k += W) {
            if (few) join_rows(std::integral_constant<int, 1>(), pc, group, complete, part, k);
            else join_rows(std::integral_constant<int, 4>(), pc, group, complete, part, 4 * k);
        }
    }
    // the last CTA that delivers a part of a segment joins them all
    if (open[0] >= 0 || open[1] >= 0) {
        __syncthreads();
        if (tid < 2) {
            int last = 0;
            if (open[tid] >= 0) {
                const KvPiece pc = sh.piece[open[tid]];
                const int c0 = shares.owner(pc.seg) / W, c1 = shares.owner(pc.seg + pc.pages - 1) / W;
                last = take_ticket(a.tickets + c0) == (unsigned int)(c1 - c0);
                if (last) a.tickets[c0] = 0;
            }
            sh.last[tid] = last;
        }
        __syncthreads();
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!sh.last[which]) continue;
            const KvPiece pc = sh.piece[open[which]];
            const int c0 = shares.owner(pc.seg) / W;
            const int parts = (shares.owner(pc.seg + pc.pages - 1) / W - c0) + 1;
            const float* base = a.cta_parts + (long long)c0 * 2 * kPart;   // part k: 2 k, the first one's 1
            for (int r = warp; r < pc.n; r += W) kv_join_row<DT, D>(a, pc, r, base, kPart, R, parts, G, lane);
        }
    }
}

// DT: type of the queries.  bf16 values fit an fp16 number scaled by the row's own power of two;
// fp32 queries and their probabilities travel as two fp16 numbers each (22 bits).
// NT: row tiles of eight that share the codes of a page.
template <int DT, int D, int NT>
__global__ void __launch_bounds__(KvSplitShape<DT, D, NT>::kThreads, 1) kv_attend_split_kernel(const KvAttendArgs a) {
    using Sh = KvSplitShape<DT, D, NT>;
    using Shared = KvSplitShared<DT, D, NT>;
    constexpr int W = Sh::W, S = Sh::S, R = 8 * NT, H = D / 2;
    constexpr int TS = D + 4;                       // floats between the rows of a warp's piece: its stores meet every bank once
    constexpr int NP = DT == AASD_F32 ? 2 : 1;      // fp16 numbers per query element and probability
    constexpr bool CEN = NP == 2;                   // codes are centred (see codes())
    constexpr int kC = CEN ? 0 : 24;                // the operands hold the codes times 2^-kC
    constexpr float kHigh = CEN ? 1.f : 0.0625f;    // undoes the high codes' factor
    constexpr int KW = H / 16;                      // words of a token's keys per lane
    constexpr int MQ = H / 16;                      // channel tiles of each half
    // Probabilities are scaled to at most 2^kP before they are rounded to fp16, so that small ones
    // keep their bits; the running maximum may lag by 2^kLazy before everything is rescaled.
    constexpr float kLazy = DT == AASD_F32 ? 0.f : 4.f;
    constexpr int kP = DT == AASD_F32 ? 14 : 10;
    static_assert(R * TS * 4 <= S * Sh::kBlock, "a piece fits its warp's ring");
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw);
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, j = lane & 3;
    if (tid == 0) {
#pragma unroll 1
        for (int i = 0; i < W * S; ++i) mbar_init(&sh.full[0][0] + i, blockIdx.x == 0 && i == a.withhold_page ? 2 : 1);   // (the second arrival never comes)
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 2 * W; i += Sh::kThreads) sh.piece[i].seg = -1;
    pdl_wait();
    const int B = a.p.n_seqs, G = a.p.n_q_heads / a.p.n_kv_heads;
    // every thread adds up the units of its strip of sequences
    const int strip = (B + Sh::kThreads - 1) / Sh::kThreads;
    long long mine = 0;
    bool padding = B == 0;
#pragma unroll 1
    for (int b = tid * strip; b < min(B, (tid + 1) * strip); ++b) {
        const KvSeq s = kv_load_seq(a, b, R);
        mine += kv_units(a, s);
        padding = padding || kv_has_padding(a, s, b);
        if (s.fresh > 0 && (long long)s.cached + s.fresh > (long long)a.p.max_pages * kPage) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    long long sum;
    const long long before = block_scan<Sh::kThreads>(mine, sh.scan, sum);
    sh.base[tid] = (int)before;
    sh.padding = __syncthreads_or(padding);   // (every thread writes the same)
    const int total = kv_total(a, sum);
    // CTAs at work: as many as leave every warp a page
    const int c = blockIdx.x, active = min((total + W - 1) / W, (int)gridDim.x);
    const bool works = c < active;
    const KvShares shares(total, works ? active * W : 1);
    const int u0 = works ? shares.first(c * W + warp) : 0, u1 = works ? shares.first(c * W + warp + 1) : 0;
    volatile int* abort_flag = &sh.abort_flag;
    u64* full = sh.full[warp];

    if (u0 < u1) {
        KvCursor<> ahead;
        {
            int lo = 0, hi = (B + strip - 1) / strip;
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh.base[mid] <= u0) lo = mid;
                else hi = mid;
            }
            int rem = u0 - sh.base[lo], b = lo * strip;
            KvSeq s = kv_load_seq(a, b, R);
#pragma unroll 1
            for (int n; rem >= (n = (int)kv_units(a, s)); s = kv_load_seq(a, ++b, R)) rem -= n;
            ahead.seek(a, b, s, rem, u0);
        }
        const unsigned int page_stride = (unsigned int)a.p.n_kv_heads * Sh::kBlock;
        unsigned int missing = 0;   // bit s: stage s holds no block (the table names no page)
        int seg_in = 0;             // where the next segment's description goes
        bool begins = true;         // the next block is the first of a segment
        int issued = 0;             // blocks asked for so far
        // a segment's queries are wanted when the blocks in front of its own are done
        auto prefetch_queries = [&]() {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int row = ahead.tile * R + 8 * nt + g;
                if (row < ahead.s.fresh * G) {
                    constexpr int es = DT == AASD_F32 ? 4 : 2;
                    const char* q0 = static_cast<const char*>(a.q) + ((long long)(ahead.s.first + row / G) * a.p.q_stride +
                                                                      (long long)(ahead.h * G + row % G) * D + (H / 4) * j) * es;
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(q0));
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(q0 + H * es));
                }
            }
        };
        int ids = 0, ids_b = -1, ids_at = 0;   // lane k: the table's entry ids_at + k of sequence ids_b
        auto issue = [&](int stage) {
            if (ids_b != ahead.b || (unsigned int)(ahead.pg - ids_at) >= 32u) {
                ids_b = ahead.b;
                ids_at = ahead.pg;
                ids = ids_at + lane < ahead.s.pages ? ahead.table[ids_at + lane] : -1;
            }
            const int page = __shfl_sync(0xFFFFFFFFu, ids, ahead.pg - ids_at);
            const bool ok = page >= 0 && page < a.p.n_pages &&
                            AASD_IN_RANGE(ahead.b < B && ahead.h < a.p.n_kv_heads && ahead.pg < ahead.s.pages && ahead.pg < a.p.max_pages, a.state);
            missing = (missing & ~(1u << stage)) | (ok ? 0u : 1u << stage);
            if (lane == 0) {
                if (ok) {
                    mbar_arrive_expect_tx(&full[stage], Sh::kBlock);
                    bulk_copy_g2s(sh.ring[warp][stage], a.pages + (u64)(unsigned int)page * page_stride + (u64)(ahead.h * Sh::kBlock),
                                  Sh::kBlock, &full[stage]);
                } else {
                    raise(a.state, AASD_STATUS_BAD_OFFSETS);
                    mbar_arrive(&full[stage]);
                }
            }
            if (begins) {
                begins = false;
                if (lane == 0) sh.seg[warp][seg_in] = KvSegment{ahead.s.cached, ahead.s.fresh, ahead.s.first, ahead.s.pages, ahead.h, ahead.tile * R, ahead.pg, ahead.unit - ahead.pg};
                if (++seg_in > S) seg_in = 0;
                if (issued > 0) prefetch_queries();
            }
            ++ahead.unit;
            if (++ahead.pg == ahead.s.pages) {
                ahead.next_segment(a, R);
                begins = true;
            }
        };
        if (ahead.unit < u1) prefetch_queries();   // (in front of the copies, which would hold them up)
#pragma unroll 1
        for (int s = 0; s < S && ahead.unit < u1; ++s, ++issued) issue(s);
        __syncwarp();

        unsigned int qf[NP][NT][D / 16][2];   // query operands
        float rfac[NT][2], qsum[NT][2];       // per column: what scales the codes' products, and the sum of q, in base 2
        float mref[NT][2], l[NT][2], mv[NT][2];
        float oacc[NT][2][MQ][4];             // [tile][half][channel tile][fragment]
        int ev = 0;                           // exponent field that the probabilities are scaled by
        bool fresh_segment = true;
        int stage = 0, seg_out = -1, pg = 0, last_pg = 0, open_to = 0, end = 0;
        unsigned int phase = 0;

#pragma unroll 1
        for (int u = 0; u < issued; ++u) {
            if (fresh_segment) {
                fresh_segment = false;
                seg_out = seg_out == S ? 0 : seg_out + 1;
                const KvSegment at = sh.seg[warp][seg_out];
                pg = at.pg;
                last_pg = at.pages - 1;
                // places up to which every row of the tile sees everything
                open_to = a.node_parent != nullptr ? at.cached : at.cached + at.row0 / G + 1;
                end = at.cached + at.fresh;
                ev = 64;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    // lane (g, j): row 8 nt + g, channels (H / 4) j .. of each half
                    const int row = at.row0 + 8 * nt + g;
                    const bool valid = row < at.fresh * G && AASD_IN_RANGE(row >= 0 && at.first + row / G < a.p.n_tokens && at.h < a.p.n_kv_heads, a.state);
                    const long long tok = at.first + (valid ? row / G : 0);
                    const long long q0 = tok * a.p.q_stride + (long long)(at.h * G + (valid ? row % G : 0)) * D + (H / 4) * j;
                    float top = 0.f, sum = 0.f;
                    float x[2][H / 4];
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int k = 0; k < H / 4; k += 8) {
                            float y[8];
                            if (a.q_vec) load8<DT, true>(a.q, q0 + half * H + k, y);
                            else load8<DT, false>(a.q, q0 + half * H + k, y);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                x[half][k + i] = valid ? y[i] : 0.f;
                                top = fmaxf(top, fabsf(x[half][k + i]));
                                sum += x[half][k + i];
                            }
                        }
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
                    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
                    // the row's largest element becomes 2^14 .. 2^15
                    int e = (int)(__float_as_uint(top) >> 23) - 127;
                    e = e < -100 ? -100 : e > 100 ? 100 : e;
                    const float up = pow2f(14 - e);
#pragma unroll
                    for (int w = 0; w < KW; ++w)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const float f = half ? up * kHigh : up;
                                const float p = x[half][4 * w + r] * f, q = x[half][4 * w + r + 2] * f;
                                const unsigned int hi = pack_half(p, q);
                                qf[0][nt][2 * w + half][r] = hi;
                                if (NP == 2) qf[NP - 1][nt][2 * w + half][r] = pack_rest(p, q, hi);
                            }
                    const float rf = a.scale_log2 * pow2f(e + kC - 14);   // of the codes and of the row
                    sum *= a.scale_log2;
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        rfac[nt][col] = __shfl_sync(0xFFFFFFFFu, rf, (2 * j + col) * 4);
                        qsum[nt][col] = __shfl_sync(0xFFFFFFFFu, sum, (2 * j + col) * 4);
                        mref[nt][col] = kKvNothing;
                        l[nt][col] = mv[nt][col] = 0.f;
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int q = 0; q < MQ; ++q)
#pragma unroll
                            for (int i = 0; i < 4; ++i) oacc[nt][half][q][i] = 0.f;
                }
            }
            // (the lanes of a warp go on, or give up, together)
            if (!__all_sync(0xFFFFFFFFu, kv_wait(a, &full[stage], phase, abort_flag))) {
                give_up(abort_flag, a.state);
                break;
            }
            if (!(missing & (1u << stage))) {
                const unsigned char* st = sh.ring[warp][stage];
                // S^T: tokens are the rows of the product, queries its columns.  Row g (and g + 8) of token
                // tile mt is token 16 (g / 2) + 4 mt + 2 (g % 2) (and the next): the order in which a lane
                // finds the values of its tokens in 16 consecutive bytes below.
                const int t0 = 16 * (g >> 1) + 2 * (g & 1);
                float x[NT][4][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[nt][mt][i] = 0.f;
                // (the token tiles take turns, so that products into the same registers stand apart)
                constexpr int KB = KW < 4 ? KW : 4;   // words fetched at a time
#pragma unroll
                for (int wb = 0; wb < KW; wb += KB) {
                    unsigned int k0[4][KB], k1[4][KB];
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
                        const unsigned char* kp = st + (t0 + 4 * mt) * H + (H / 4) * j + 4 * wb;
                        if constexpr (KB == 2) {
                            const uint2 p = *reinterpret_cast<const uint2*>(kp), q = *reinterpret_cast<const uint2*>(kp + H);
                            k0[mt][0] = p.x; k0[mt][1] = p.y; k1[mt][0] = q.x; k1[mt][1] = q.y;
                        } else {
                            const uint4 p = lds16(kp), q = lds16(kp + H);
                            k0[mt][0] = p.x; k0[mt][1] = p.y; k0[mt][2] = p.z; k0[mt][3] = p.w;
                            k1[mt][0] = q.x; k1[mt][1] = q.y; k1[mt][2] = q.z; k1[mt][3] = q.w;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < KB; ++w)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int mt = 0; mt < 4; ++mt) {
                                const unsigned int a0 = half ? codes<CEN, true>(k0[mt][w]) : codes<CEN, false>(k0[mt][w]);
                                const unsigned int a1 = half ? codes<CEN, true>(k1[mt][w]) : codes<CEN, false>(k1[mt][w]);
                                const unsigned int a2 = half ? codes<CEN, true>(k0[mt][w] >> 8) : codes<CEN, false>(k0[mt][w] >> 8);
                                const unsigned int a3 = half ? codes<CEN, true>(k1[mt][w] >> 8) : codes<CEN, false>(k1[mt][w] >> 8);
                                const int ks = 2 * (wb + w) + half;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int np = 0; np < NP; ++np) mma_16816(x[nt][mt], a0, a1, a2, a3, qf[np][nt][ks][0], qf[np][nt][ks][1]);
                            }
                }
                // scales, masks, running maximum
                uint2 vm[4];
                const bool masked = (pg + 1) * kPage > open_to;
                const int live = end - pg * kPage;
                float mx[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = kKvHidden;
                unsigned int vmax = 0;
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
                    const int t = t0 + 4 * mt;
                    uint2 km = *reinterpret_cast<const uint2*>(st + kv_key_meta_offset(D) + 4 * t);
                    vm[mt] = *reinterpret_cast<const uint2*>(st + kv_value_meta_offset(D) + 4 * t);
                    if (masked) {   // places past the end hold anything
                        if (t >= live) km.x = vm[mt].x = 0;
                        if (t + 1 >= live) km.y = vm[mt].y = 0;
                    }
                    vmax = max(vmax, max(vm[mt].x & 0xFFFFu, vm[mt].y & 0xFFFFu));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const unsigned int m = i < 2 ? km.x : km.y;
                            const float mn = CEN ? fmaf(8.f, meta_scale(m), meta_min(m)) : meta_min(m);
                            x[nt][mt][i] = fmaf(meta_scale(m), x[nt][mt][i] * rfac[nt][i & 1], mn * qsum[nt][i & 1]);
                        }
                }
                if (masked) {
                    // (lane r finds out what row r sees)
                    const KvSegment at = sh.seg[warp][seg_out];
                    const u64 mine = kv_seen(a, at.cached, at.fresh, at.first, pg, (at.row0 + (lane & (R - 1))) / G);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int col = 0; col < 2; ++col) {
                            const u64 seen = __shfl_sync(0xFFFFFFFFu, mine, 8 * nt + 2 * j + col);
#pragma unroll
                            for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                                for (int f = 0; f < 2; ++f)
                                    if (!((seen >> (t0 + 4 * mt + f)) & 1ull)) x[nt][mt][2 * f + col] = kKvHidden;
                        }
                }
                bool grow = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        float m = kKvHidden;
#pragma unroll
                        for (int mt = 0; mt < 4; ++mt) m = fmaxf(m, fmaxf(x[nt][mt][col], x[nt][mt][2 + col]));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                        mx[nt][col] = m;
                        grow = grow || m > mref[nt][col] + kLazy;
                    }
                const int ep = (int)(__reduce_max_sync(0xFFFFFFFFu, vmax) >> 7);   // exponent field of the largest value scale
                if (__any_sync(0xFFFFFFFFu, grow || ep > ev)) {
                    const int en = max(ev, min(ep, 250));
                    const float shift = en - ev > 126 ? 0.f : pow2f(ev - en);
                    ev = en;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int col = 0; col < 2; ++col) {
                            const float mn = fmaxf(mref[nt][col], mx[nt][col]);
                            const float f = ex2_approx(mref[nt][col] - mn);
                            mref[nt][col] = mn;
                            l[nt][col] *= f;
                            mv[nt][col] *= f;
#pragma unroll
                            for (int half = 0; half < 2; ++half)
#pragma unroll
                                for (int q = 0; q < MQ; ++q) {
                                    oacc[nt][half][q][col] *= f * shift;
                                    oacc[nt][half][q][2 + col] *= f * shift;
                                }
                        }
                }
                const float vup = pow2f(kP - (ev - 127));
                // probabilities, as the second operand of the next product
                unsigned int pb[NP][NT][4][2];
#pragma unroll
                for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const unsigned int m = f ? vm[mt].y : vm[mt].x;
                        const float sv = meta_scale(m) * vup, mn = CEN ? fmaf(8.f, meta_scale(m), meta_min(m)) : meta_min(m);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float p[2];
#pragma unroll
                            for (int col = 0; col < 2; ++col) {
                                p[col] = ex2_approx(x[nt][mt][2 * f + col] - mref[nt][col]);
                                l[nt][col] += p[col];
                                mv[nt][col] = fmaf(p[col], mn, mv[nt][col]);
                                p[col] *= sv;
                            }
                            const unsigned int hi = pack_half(p[0], p[1]);
                            pb[0][nt][mt][f] = transpose_8x8(hi);
                            if (NP == 2) pb[NP - 1][nt][mt][f] = transpose_8x8(pack_rest(p[0], p[1], hi));
                        }
                    }
                // O^T: channels are the rows; a lane's 16 bytes of a channel are its tokens in order
#pragma unroll
                for (int qb = 0; qb < MQ; qb += 2) {
                    unsigned int w0[2][4], w1[2][4];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const unsigned char* vp = st + kv_value_offset(D) + (16 * (qb + q) + g) * kPage + 16 * j;
                        const uint4 v0 = lds16(vp), v1 = lds16(vp + 8 * kPage);
                        w0[q][0] = v0.x; w0[q][1] = v0.y; w0[q][2] = v0.z; w0[q][3] = v0.w;
                        w1[q][0] = v1.x; w1[q][1] = v1.y; w1[q][2] = v1.z; w1[q][3] = v1.w;
                    }
                    float part[NP == 2 ? NT : 1][2][2][4];
                    if (NP == 2) {   // fp32: a page's sum is added in full precision
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) part[nt][0][0][i] = part[nt][0][1][i] = part[nt][1][0][i] = part[nt][1][1][i] = 0.f;
                    }
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const unsigned int a0 = half ? codes<CEN, true>(w0[q][kt]) : codes<CEN, false>(w0[q][kt]);
                                const unsigned int a1 = half ? codes<CEN, true>(w1[q][kt]) : codes<CEN, false>(w1[q][kt]);
                                const unsigned int a2 = half ? codes<CEN, true>(w0[q][kt] >> 8) : codes<CEN, false>(w0[q][kt] >> 8);
                                const unsigned int a3 = half ? codes<CEN, true>(w1[q][kt] >> 8) : codes<CEN, false>(w1[q][kt] >> 8);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    if (NP == 2) {
                                        mma_16816(part[nt][half][q], a0, a1, a2, a3, pb[0][nt][kt][0], pb[0][nt][kt][1]);
                                        mma_16816(part[nt][half][q], a0, a1, a2, a3, pb[NP - 1][nt][kt][0], pb[NP - 1][nt][kt][1]);
                                    } else {
                                        mma_16816(oacc[nt][half][qb + q], a0, a1, a2, a3, pb[0][nt][kt][0], pb[0][nt][kt][1]);
                                    }
                                }
                            }
                    if (NP == 2) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int q = 0; q < 2; ++q)
#pragma unroll
                                for (int half = 0; half < 2; ++half)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) oacc[nt][half][qb + q][i] += part[nt][half][q][i];
                    }
                }
            }
            __syncwarp();   // the stage has been read by every lane
            if (ahead.unit < u1) {
                issue(stage);
                ++issued;
                __syncwarp();   // (a segment's description may have been written)
            }
            if (++stage == S) {
                stage = 0;
                phase ^= 1u;
            }
            const bool seg_end = pg == last_pg;
            ++pg;
            const bool tail = u == issued - 1;   // (blocks are asked for at least one ahead)
            if (seg_end || tail) {
                // the piece is done
                fresh_segment = true;
                const KvSegment at = sh.seg[warp][seg_out];
                const bool complete = at.pg == 0 && seg_end;
                const float unscale = pow2f((ev - 127) - kP), back = pow2f(kC);
                const int n = min(R, at.fresh * G - at.row0);
                const int slot = 2 * warp + (tail ? 1 : 0);
                float* to = tail ? reinterpret_cast<float*>(sh.ring[warp][0]) : a.warp_parts + (long long)(c * W + warp) * (R * TS);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        float ls = l[nt][col], ms = mv[nt][col];
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) {
                            ls += __shfl_xor_sync(0xFFFFFFFFu, ls, o);
                            ms += __shfl_xor_sync(0xFFFFFFFFu, ms, o);
                        }
                        const int r = 8 * nt + 2 * j + col;
                        const int row = at.row0 + r;
                        const float inv = complete ? kv_inverse(ls) : 1.f;
                        const long long head = ((long long)at.first + row / G) * a.p.n_q_heads + at.h * G + row % G;
                        if (g == 0) {
                            if (!complete) {
                                sh.m[slot][r] = mref[nt][col];
                                sh.l[slot][r] = ls;
                            } else if (a.o.lse != nullptr && r < n) {
                                a.o.lse[head] = kv_lse(mref[nt][col], ls);
                            }
                        }
                        if (r < n && AASD_IN_RANGE(c < kKvMaxCtas && head < a.p.n_tokens * a.p.n_q_heads, a.state)) {
#pragma unroll
                            for (int half = 0; half < 2; ++half)
#pragma unroll
                                for (int q = 0; q < MQ; ++q)
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        const int ch = half * H + 16 * q + 8 * i + g;
                                        const float o = fmaf(oacc[nt][half][q][2 * i + col] * (half ? back * kHigh : back), unscale, ms) * inv;
                                        if (!complete) to[r * TS + ch] = o;
                                        else if (DT == AASD_F32) static_cast<float*>(a.o.out)[head * D + ch] = o;
                                        else static_cast<__nv_bfloat16*>(a.o.out)[head * D + ch] = __float2bfloat16_rn(o);
                                    }
                        }
                    }
                if (!complete && lane == 0) sh.piece[slot] = KvPiece{at.unit, at.pages, at.h, at.row0, n, at.first};
            }
        }
        if (*abort_flag) {   // nothing may be on its way into this CTA's shared memory when it leaves
            for (int s = 0; s < S; ++s)
                for (unsigned int it = 0; it < a.wait_limit && s < issued && !mbar_try_wait(&full[s], ((unsigned int)((issued - 1 - s) / S)) & 1u); ++it) {}
        }
    }
    __syncthreads();
    if (works && !*abort_flag) kv_split_join<DT, D, Sh::W, R, TS>(a, sh, shares);
    if (sh.padding || total == 0) kv_clear_rows<DT>(a, D, total, (int)(blockIdx.x * W + warp), (int)(gridDim.x * W));
}

}  // namespace aasd
