// Attention of a step's new tokens over the paged 8-bit cache.
//
// Rows and the list of work are those of the 4-bit kernels (aasd_kv_attend.cuh).  A code is turned into the fp16 number that it
// stands for (exact, one conversion for two); the scales are the page's, so they multiply sums: the keys' the exponents
// of the softmax, the values' the probabilities.
#pragma once

#include "aasd_kv_attend.cuh"
#include "aasd_kvb.cuh"

namespace aasd {

// Two codes (the low 16 bits, or the high ones) as fp16 numbers.
template <bool HIGH>
__device__ __forceinline__ unsigned int kvb_halves(unsigned int w) {
    unsigned int h;
    if (HIGH) asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;}" : "=r"(h) : "r"(w));
    else asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;}" : "=r"(h) : "r"(w));
    return h;
}

// ---- few rows per head: the keys split over all warps -----------------------------------------------

// As the 4-bit kernel: W warps per CTA, each with a ring of S blocks that lane 0 fills by bulk copies, equal shares of the list of
// work.  A block is a part of a page (32 tokens of 128 channels), so that twelve warps have two of them each: 200 KB per
// SM are on their way.  (mma.sync: sixteen rows would leave a tcgen05 tile mostly empty.)
//
// Bound by memory with a batch, by the chain share - table - block - products - joins with one sequence.  Measured (bf16, 128
// channels, one token each): 256 sequences of 100 to 4000 tokens, 28 query and 4 key heads, 101 us, 541 MB at 5.3 TB/s, 82 % of the copy
// rate; one sequence of 16384 tokens, 32 and 8 heads, 18 us, where its 34 MB alone take 5.  fp32 queries come here with any number of
// rows and go over the pages once for every 16 of them (8 with 256 channels), two products each: 32 trees of 33 over 3800 tokens
// 645 us, 2 x 2048 tokens of a prompt 1820, ten and nine times what the tiles take with bf16.
template <int DT, int D, int NT>
struct KvbSplitShape {
    static constexpr int TB = D == 64 ? 64 : D == 128 ? 32 : 16;       // tokens of a block
    static constexpr int W = DT == AASD_BF16 && NT == 1 && D < 256 ? 12 : 8;
    static constexpr int S = W == 12 ? 2 : 3;
    static constexpr int kHalf = TB * D;                               // bytes of its keys, and of its values
    static constexpr int kBlock = 2 * kHalf + 128;                     // (the scales are 16 bytes)
    static constexpr int kThreads = W * 32;
};

template <int DT, int D, int NT>
struct KvbSplitShared {
    using Sh = KvbSplitShape<DT, D, NT>;
    static constexpr int R = 8 * NT;
    alignas(128) unsigned char ring[Sh::W][Sh::S][Sh::kBlock];
    int base[Sh::kThreads];
    KvSeq seq[Sh::kThreads];           // batches up to the number of threads: what the scan has loaded
    long long scan[Sh::W];
    KvSegment seg[Sh::W][Sh::S + 1];   // of the blocks on their way, and the one being worked on
    KvPiece piece[2 * Sh::W];
    float m[2 * Sh::W][R], l[2 * Sh::W][R];
    u64 full[Sh::W][Sh::S];
    int abort_flag, last[2], padding;
};

// Byte of token t's 16-byte chunk in a block (see kvb_chunk_offset; t counted from the block's first token, a multiple of 16).
template <int D, int TB>
__device__ __forceinline__ int kvb_block_offset(int t, int chunk) {
    return D == 64 ? t * 64 + ((chunk ^ ((t >> 1) & 3)) << 4) : (chunk >> 3) * (TB * 128) + t * 128 + (((chunk & 7) ^ (t & 7)) << 4);
}

// DT: type of the queries.  bf16 values fit an fp16 number scaled by the row's own power of two;
// fp32 queries and their probabilities travel as two fp16 numbers each (22 bits).
// NT: row tiles of eight that share the codes of a block.
template <int DT, int D, int NT>
__global__ void __launch_bounds__(KvbSplitShape<DT, D, NT>::kThreads, 1) kvb_attend_split_kernel(const KvAttendArgs a) {
    using Sh = KvbSplitShape<DT, D, NT>;
    using Shared = KvbSplitShared<DT, D, NT>;
    constexpr int W = Sh::W, S = Sh::S, R = 8 * NT, TB = Sh::TB;
    constexpr int TS = D + 4;                       // floats between the rows of a warp's piece
    constexpr int NP = DT == AASD_F32 ? 2 : 1;      // fp16 numbers per query element and probability
    constexpr int C = D / 64;                       // 16-byte chunks of a key that a lane has: j, j + 4, ..
    constexpr int CW = D == 64 ? 2 : 4;             // words of a value chunk that a lane has
    constexpr int CP = D == 256 ? 2 : 1;            // such chunks: g, g + 8
    constexpr int MT = TB / 16, MQ = D / 16;        // token tiles of a block, channel tiles
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
        const KvSeq s = kv_load_seq<TB>(a, b, R);
        if (strip == 1) sh.seq[b] = s;
        mine += kv_units(a, s);
        padding = padding || kv_has_padding(a, s, b);
        if (s.fresh > 0 && (long long)s.cached + s.fresh > (long long)a.p.max_pages * kPage) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    long long sum;
    const long long before = block_scan<Sh::kThreads>(mine, sh.scan, sum);
    sh.base[tid] = (int)before;
    sh.padding = __syncthreads_or(padding);   // (every thread writes the same)
    const int total = kv_total(a, sum);
    // CTAs at work: as many as leave every warp a block
    const int c = blockIdx.x, active = min((total + W - 1) / W, (int)gridDim.x);
    const bool works = c < active;
    const KvShares shares(total, works ? active * W : 1);
    const int u0 = works ? shares.first(c * W + warp) : 0, u1 = works ? shares.first(c * W + warp + 1) : 0;
    volatile int* abort_flag = &sh.abort_flag;
    u64* full = sh.full[warp];

    if (u0 < u1) {
        KvCursor<TB> ahead;
        {
            int lo = 0, hi = (B + strip - 1) / strip;
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh.base[mid] <= u0) lo = mid;
                else hi = mid;
            }
            int rem = u0 - sh.base[lo], b = lo * strip;
            const auto load = [&](int k) { return strip == 1 ? sh.seq[k] : kv_load_seq<TB>(a, k, R); };
            KvSeq s = load(b);
#pragma unroll 1
            for (int n; rem >= (n = (int)kv_units(a, s)); s = load(++b)) rem -= n;
            ahead.seek(a, b, s, rem, u0);
        }
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
                                                                      (long long)(ahead.h * G + row % G) * D + (D / 4) * j) * es;
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(q0));
                }
            }
        };
        int ids = 0, ids_b = -1, ids_at = 0;   // lane k: the table's entry ids_at + k of sequence ids_b
        auto issue = [&](int stage) {
            constexpr int PB = kPage / TB;      // blocks of a page
            const int pg = ahead.pg / PB, part = ahead.pg % PB;
            if (ids_b != ahead.b || (unsigned int)(pg - ids_at) >= 32u) {
                ids_b = ahead.b;
                ids_at = pg;
                ids = (ids_at + lane) * PB < ahead.s.pages ? ahead.table[ids_at + lane] : -1;
            }
            const int page = __shfl_sync(0xFFFFFFFFu, ids, pg - ids_at);
            const bool ok = page >= 0 && page < a.p.n_pages &&
                            AASD_IN_RANGE(ahead.b < B && ahead.h < a.p.n_kv_heads && ahead.pg < ahead.s.pages && pg < a.p.max_pages, a.state);
            missing = (missing & ~(1u << stage)) | (ok ? 0u : 1u << stage);
            if (lane == 0) {
                if (ok) {
                    const uint8_t* from = a.pages + ((u64)(unsigned int)page * (unsigned int)a.p.n_kv_heads + (unsigned int)ahead.h) * kvb_head_bytes(D);
                    unsigned char* to = sh.ring[warp][stage];
                    mbar_arrive_expect_tx(&full[stage], 2 * Sh::kHalf + 16);
                    if constexpr (TB == kPage) {
                        bulk_copy_g2s(to, from, 2 * Sh::kHalf + 16, &full[stage]);
                    } else {
                        // (a panel of 128 channels is 64 tokens; a block's part of each)
                        constexpr int panels = D / 128, bytes = TB * 128;
#pragma unroll
                        for (int k = 0; k < 2 * panels; ++k) bulk_copy_g2s(to + k * bytes, from + k * (kPage * 128) + part * bytes, bytes, &full[stage]);
                        bulk_copy_g2s(to + 2 * Sh::kHalf, from + kvb_scale_offset(D), 16, &full[stage]);
                    }
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
        float rfac[NT][2];                    // per column: what scales the codes' products, in base 2
        float mref[NT][2], l[NT][2];
        float oacc[NT][MQ][4];                // [tile][channel tile][fragment]
        int ev = 0;                           // exponent field that the probabilities are scaled by
        bool fresh_segment = true;
        int stage = 0, seg_out = -1, pg = 0, last_pg = 0, open_to = 0, end = 0;
        unsigned int phase = 0;
        // Row r of a token tile (of its first eight, the others are 8 further) is token tk(r): with 128 channels the two rows that are read
        // together lie in different halves of the swizzle.
        const auto tk = [](int r) { return D == 64 ? r : ((r & 1) << 2) | (r >> 1); };
        // The values of tokens tk(2j) and tk(2j + 1) are fetched in an order that keeps eight neighbouring lanes on different banks.
        const bool turned = D == 64 ? (j & 1) != 0 : (g & 1) != 0;
        const int ta = turned ? tk(2 * j + 1) : tk(2 * j), tb = turned ? tk(2 * j) : tk(2 * j + 1);
        const unsigned int sel0 = turned ? 0x1504u : 0x5140u, sel1 = turned ? 0x3726u : 0x7362u;

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
                    // lane (g, j): row 8 nt + g, channels of the chunks j, j + 4, ..
                    const int row = at.row0 + 8 * nt + g;
                    const bool valid = row < at.fresh * G && AASD_IN_RANGE(row >= 0 && at.first + row / G < a.p.n_tokens && at.h < a.p.n_kv_heads, a.state);
                    const long long tok = at.first + (valid ? row / G : 0);
                    const long long q0 = tok * a.p.q_stride + (long long)(at.h * G + (valid ? row % G : 0)) * D + 16 * j;
                    float top = 0.f;
                    float x[C][16];
#pragma unroll
                    for (int k = 0; k < C; ++k)
#pragma unroll
                        for (int h = 0; h < 16; h += 8) {
                            float y[8];
                            if (a.q_vec) load8<DT, true>(a.q, q0 + 64 * k + h, y);
                            else load8<DT, false>(a.q, q0 + 64 * k + h, y);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                x[k][h + i] = valid ? y[i] : 0.f;
                                top = fmaxf(top, fabsf(x[k][h + i]));
                            }
                        }
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    // the row's largest element becomes 2^14 .. 2^15
                    int e = (int)(__float_as_uint(top) >> 23) - 127;
                    e = max(e, -112);
                    const float up = kvb_pow2(14 - e);
#pragma unroll
                    for (int k = 0; k < C; ++k)
#pragma unroll
                        for (int w = 0; w < 4; ++w)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const float p = x[k][4 * w + 2 * r] * up, q = x[k][4 * w + 2 * r + 1] * up;
                                const unsigned int hi = pack_half(p, q);
                                qf[0][nt][4 * k + w][r] = hi;
                                if (NP == 2) qf[NP - 1][nt][4 * k + w][r] = pack_rest(p, q, hi);
                            }
                    // (a row with an infinity becomes NaN, as one with a NaN is)
                    const float rf = top < CUDART_INF_F ? a.scale_log2 * kvb_pow2(e - 14) : CUDART_NAN_F;
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        rfac[nt][col] = __shfl_sync(0xFFFFFFFFu, rf, (2 * j + col) * 4);
                        mref[nt][col] = kKvNothing;
                        l[nt][col] = 0.f;
                    }
#pragma unroll
                    for (int q = 0; q < MQ; ++q)
#pragma unroll
                        for (int i = 0; i < 4; ++i) oacc[nt][q][i] = 0.f;
                }
            }
            // (the lanes of a warp go on, or give up, together)
            if (!__all_sync(0xFFFFFFFFu, kv_wait(a, &full[stage], phase, abort_flag))) {
                give_up(abort_flag, a.state);
                break;
            }
            if (!(missing & (1u << stage))) {
                const unsigned char* st = sh.ring[warp][stage];
                // S^T: tokens are the rows of the product, queries its columns.
                float x[NT][MT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[nt][mt][i] = 0.f;
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    uint4 k0[MT], k1[MT];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        k0[mt] = lds16(st + kvb_block_offset<D, TB>(16 * mt + tk(g), j + 4 * k));
                        k1[mt] = lds16(st + kvb_block_offset<D, TB>(16 * mt + 8 + tk(g), j + 4 * k));
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            const unsigned int w0 = w == 0 ? k0[mt].x : w == 1 ? k0[mt].y : w == 2 ? k0[mt].z : k0[mt].w;
                            const unsigned int w1 = w == 0 ? k1[mt].x : w == 1 ? k1[mt].y : w == 2 ? k1[mt].z : k1[mt].w;
                            const unsigned int a0 = kvb_halves<false>(w0), a1 = kvb_halves<false>(w1), a2 = kvb_halves<true>(w0), a3 = kvb_halves<true>(w1);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int np = 0; np < NP; ++np) mma_16816(x[nt][mt], a0, a1, a2, a3, qf[np][nt][4 * k + w][0], qf[np][nt][4 * k + w][1]);
                        }
                }
                // scales, masks, running maximum
                const uint2 scale = *reinterpret_cast<const uint2*>(st + 2 * Sh::kHalf);
                const float sk = kvb_pow2(kvb_exponent(scale.x));
                const bool masked = (pg + 1) * TB > open_to;
                const int live = end - pg * TB;
                float mx[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mx[nt][0] = mx[nt][1] = kKvHidden;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[nt][mt][i] *= rfac[nt][i & 1] * sk;
                }
                if (masked) {
                    // (lane r finds out what row r sees)
                    const KvSegment at = sh.seg[warp][seg_out];
                    const u64 mine = kv_seen(a, at.cached, at.fresh, at.first, pg * TB / kPage, (at.row0 + (lane & (R - 1))) / G) >> (pg * TB % kPage);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int col = 0; col < 2; ++col) {
                            const u64 seen = __shfl_sync(0xFFFFFFFFu, mine, 8 * nt + 2 * j + col) >> tk(g);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int f = 0; f < 2; ++f)
                                    if (!((seen >> (16 * mt + 8 * f)) & 1ull)) x[nt][mt][2 * f + col] = kKvHidden;
                        }
                }
                bool grow = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        float m = kKvHidden;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) m = fmaxf(m, fmaxf(x[nt][mt][col], x[nt][mt][2 + col]));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                        mx[nt][col] = m;
                        grow = grow || m > mref[nt][col] + kLazy;
                    }
                const int ep = kvb_exponent(scale.y) + 127;   // exponent field of the values' scale
                if (__any_sync(0xFFFFFFFFu, grow || ep > ev)) {
                    const int en = max(ev, ep);
                    const float shift = en - ev > 126 ? 0.f : kvb_pow2(ev - en);
                    ev = en;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int col = 0; col < 2; ++col) {
                            const float mn = fmaxf(mref[nt][col], mx[nt][col]);
                            const float f = ex2_approx(mref[nt][col] - mn);
                            mref[nt][col] = mn;
                            l[nt][col] *= f;
#pragma unroll
                            for (int q = 0; q < MQ; ++q) {
                                oacc[nt][q][col] *= f * shift;
                                oacc[nt][q][2 + col] *= f * shift;
                            }
                        }
                }
                const float sv = ev - ep > 120 ? 0.f : kvb_pow2(ep - ev + kP);
                // probabilities, as the second operand of the next product
                unsigned int pb[NP][NT][MT][2];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int f = 0; f < 2; ++f)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float p[2];
#pragma unroll
                            for (int col = 0; col < 2; ++col) {
                                p[col] = ex2_approx(x[nt][mt][2 * f + col] - mref[nt][col]);
                                l[nt][col] += p[col];
                                p[col] *= sv;
                            }
                            const unsigned int hi = pack_half(p[0], p[1]);
                            pb[0][nt][mt][f] = transpose_8x8(hi);
                            if (NP == 2) pb[NP - 1][nt][mt][f] = transpose_8x8(pack_rest(p[0], p[1], hi));
                        }
                // O^T: channels are the rows.  Row g of channel tile q is channel 2 q of the lane's chunk, row g + 8 the next one.
#pragma unroll
                for (int cp = 0; cp < CP; ++cp) {
                    float part[NP == 2 ? NT : 1][NP == 2 ? 2 * CW : 1][4];
                    if (NP == 2) {   // fp32: a block's sum is added in full precision
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int q = 0; q < 2 * CW; ++q)
#pragma unroll
                                for (int i = 0; i < 4; ++i) part[nt][q][i] = 0.f;
                    }
#pragma unroll
                    for (int kt = 0; kt < MT; ++kt) {
                        unsigned int v[4][CW];   // tokens ta, tb, ta + 8, tb + 8
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int t = 16 * kt + (k & 1 ? tb : ta) + (k & 2 ? 8 : 0);
                            const unsigned char* at = st + Sh::kHalf + (D == 64 ? kvb_block_offset<D, TB>(t, g >> 1) + 8 * (g & 1) : kvb_block_offset<D, TB>(t, g + 8 * cp));
                            if constexpr (CW == 2) {
                                const uint2 y = *reinterpret_cast<const uint2*>(at);
                                v[k][0] = y.x; v[k][1] = y.y;
                            } else {
                                const uint4 y = lds16(at);
                                v[k][0] = y.x; v[k][1] = y.y; v[k][2] = y.z; v[k][3] = y.w;
                            }
                            if (masked && t >= live) {   // places past the end hold anything
#pragma unroll
                                for (int w = 0; w < CW; ++w) v[k][w] = 0u;
                            }
                        }
#pragma unroll
                        for (int w = 0; w < CW; ++w)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const unsigned int y0 = __byte_perm(v[0][w], v[1][w], h ? sel1 : sel0), y1 = __byte_perm(v[2][w], v[3][w], h ? sel1 : sel0);
                                const unsigned int a0 = kvb_halves<false>(y0), a1 = kvb_halves<true>(y0), a2 = kvb_halves<false>(y1), a3 = kvb_halves<true>(y1);
                                const int q = 2 * w + h;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    if (NP == 2) {
                                        mma_16816(part[nt][NP == 2 ? q : 0], a0, a1, a2, a3, pb[0][nt][kt][0], pb[0][nt][kt][1]);
                                        mma_16816(part[nt][NP == 2 ? q : 0], a0, a1, a2, a3, pb[NP - 1][nt][kt][0], pb[NP - 1][nt][kt][1]);
                                    } else {
                                        mma_16816(oacc[nt][cp * 2 * CW + q], a0, a1, a2, a3, pb[0][nt][kt][0], pb[0][nt][kt][1]);
                                    }
                                }
                            }
                    }
                    if (NP == 2) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int q = 0; q < 2 * CW; ++q)
#pragma unroll
                                for (int i = 0; i < 4; ++i) oacc[nt][cp * 2 * CW + q][i] += part[nt][NP == 2 ? q : 0][i];
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
                const int n = min(R, at.fresh * G - at.row0);
                const int slot = 2 * warp + (tail ? 1 : 0);
                const float unscale = kvb_pow2(ev - 127), back = kvb_pow2(-kP);
                float* to = tail ? reinterpret_cast<float*>(sh.ring[warp][0]) : a.warp_parts + (long long)(c * W + warp) * (R * TS);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        float ls = l[nt][col];
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) ls += __shfl_xor_sync(0xFFFFFFFFu, ls, o);
                        const int r = 8 * nt + 2 * j + col;
                        const int row = at.row0 + r;
                        const float f = back * (complete ? kv_inverse(ls) : 1.f);
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
                            // (channels 2 q and 2 q + 1 of the lane's chunk are tile q's)
#pragma unroll
                            for (int q = 0; q < MQ; q += 2) {
                                const int ch = (D == 64 ? 8 * g : 16 * g + 128 * (q / 8)) + 2 * (q % 8);
                                const float4 o = make_float4(oacc[nt][q][col] * f * unscale, oacc[nt][q][2 + col] * f * unscale, oacc[nt][q + 1][col] * f * unscale,
                                                             oacc[nt][q + 1][2 + col] * f * unscale);
                                if (!complete) *reinterpret_cast<float4*>(to + r * TS + ch) = o;
                                else store4<DT>(a.o.out, head * D + ch, o, a.out_vec);
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
