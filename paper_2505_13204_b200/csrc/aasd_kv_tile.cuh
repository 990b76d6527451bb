// Attention over the paged 4-bit cache for many rows per key/value head (draft trees, chunks of a
// prompt): tiles of 128 rows on the fifth-generation tensor cores.
//
// One persistent CTA per SM; its warps have roles:
//   walker      goes through the CTA's share of the work and hands it out piece by piece;
//   loader      brings pages (packed blocks) in by bulk copies;
//   unpackers   (4 warps) turn a page's codes into fp16 operands in shared memory, K-major rows of 128
//               bytes in the 128-byte swizzle;
//   two issuers, one thread each: tcgen05.mma of S = Q K^T (both operands in shared memory) and
//               O += P V (P in tensor memory) for one softmax group, a page (64 tokens) at a time;
//   two softmax groups of 4 warps, 32 rows each: S to registers, probabilities back as P.
// The two groups work on two row tiles of the same pages (PAIR), or, where a segment has no more
// than 128 rows, on alternate pages of one tile, joined at the end.  A group has two S buffers, so
// that the next page's products are there when it is done with one.
//
// Keys stay bare codes (as bf16 numbers, like the queries, which are copied as they are), whose scale
// and minimum are applied to S.  Values are expanded here, relative to the largest exponent of the
// segment's pages so far (so that values of any size fit fp16), and rounded to 11 bits like the
// probabilities: a value is used for 128 rows, and scaling the probabilities instead, with a sum of
// the minima beside them, costs the softmax groups, which pace the kernel, a third more instructions.
//
// Tensor memory (512 columns): two S buffers of each group, whose first halves P takes over, and O.
//
// Measured (32 query and 8 key heads of 128 channels): 2 chunks of 2048 tokens over ~1000 cached ones 222 us, 617
// TFLOP/s; 32 trees of 33 nodes over ~3800 174 us; 64 new tokens over 131072 176 us, 782 TFLOP/s.  A pair of
// tiles takes some 2400 cycles per page, of which the tensor cores work 1300 and the exponentials 1000, and no unit is
// busy for more than 40 % of the time (issue slots 47 %): the roles wait for one another.  Which of them sets
// the pace is not known: with the exponentials left out it took 5 % less, with cheaper unpacking of values
// no less, and the single tile, where a softmax group has the time of two pages for each, is a sixth faster
// per page.  A piece costs 15000 cycles beside its pages (queries in, result out), about six pages.
#pragma once

#include "aasd_kv_attend.cuh"

namespace aasd {

constexpr int kTileThreads = 512;      // 8 softmax warps, 4 unpackers, two issuers, loader, walker
// Registers per thread: a launch of 512 threads has 128 for each; the softmax groups, which hold a
// row of S, take what the others give up (2 x 184 + 2 x 72 = 4 x 128).
constexpr int kTileLaunchRegs = 128, kTileSoftmaxRegs = 184, kTileOtherRegs = 72;
static_assert(2 * kTileSoftmaxRegs + 2 * kTileOtherRegs <= 4 * kTileLaunchRegs, "the shares add up to the launch's registers");
constexpr int kTileRows = 128;
constexpr int kTileRaw = 4, kTileKeys = 3, kTileValues = 4, kTileMeta = 6;   // ring depths, in pages
constexpr int kTilePieces = 8;
// the probabilities' power of two (see the split kernel): the maximum may lag by what is left of fp16's range
constexpr float kTileP = 7.f;
// Exponents from which products are scaled in an operation of their own.  Below, the scaling is fused with the
// subtraction of the rounded maximum: what its rounding left out, at most 2^-5 here, is a factor that the row's
// probabilities and their sum share.  At 2^28 that factor would leave fp16's range.
constexpr float kTileLarge = 1048576.f;

// ---- the list of work ---------------------------------------------------------------------------------

// Pages that a row tile looks at: those up to its last query's own token, or all (trees).
__device__ __forceinline__ int kv_tile_pages(const KvAttendArgs& a, int cached, int fresh, int pages, int tile, int R, int G) {
    if (a.node_parent != nullptr) return pages;
    const int last = (int)min((long long)fresh * G, (long long)(tile + 1) * R) - 1;
    return min(pages, (int)(((unsigned int)cached + (unsigned int)(last / G) + kPage) / kPage));
}
// Loading the queries and handing the result on takes about as long as six pages (2 chunks of 2048 tokens: 264 us
// with 2, 247 with 4, 233 with 6, 238 with 9, when it was chosen).
constexpr int kTileSegCost = 6;
// Units of one head of a sequence.
__device__ __forceinline__ long long kv_tile_head_units(const KvAttendArgs& a, const KvSeq& s, int R, int G) {
    if (s.pages == 0) return 0;
    if (a.node_parent != nullptr) return (long long)s.tiles * (s.pages + kTileSegCost);
    long long n = 0;
#pragma unroll 1
    for (int t = 0; t < s.tiles; ++t) n += kv_tile_pages(a, s.cached, s.fresh, s.pages, t, R, G) + kTileSegCost;
    return n;
}

// A piece: the run of pages of one segment that falls into a CTA's share.  One lane walks the share and
// hands the pieces to the other roles through a ring.
struct KvTilePiece {
    int b, h, tile;
    int pg, np, pages;        // first page, pages of the piece (0: the share is done), pages of the segment
    int cached, fresh, first; // see KvSeq
    int seg;                  // unit of the segment's first page
};

template <int D, bool PAIR>
struct KvTileShared {
    static constexpr int R = PAIR ? 2 * kTileRows : kTileRows;
    alignas(1024) unsigned char queries[PAIR ? 2 : 1][kTileRows * D * 2];
    unsigned char keys[kTileKeys][kPage * D * 2];
    unsigned char values[kTileValues][kPage * D * 2];
    alignas(128) unsigned char raw[kTileRaw][kv_head_bytes(D)];
    float4 kmeta[kTileMeta][kPage / 2];   // token pairs: the keys' scales, and minima
    uint4 vmeta[4][kPage / 4];         // per unpacking warp, four tokens each: scales of 0 and 2, 1 and 3, minima likewise
    int ev[kTileMeta];                 // exponent field that a page's values are relative to; -1: page hidden
    int raw_missing[kTileRaw];
    float row_q[PAIR ? 2 : 1][kTileRows];         // sums of the rows' queries
    float exchange_m[kTileRows], exchange_l[kTileRows], exchange_up[kTileRows];   // between the groups, where they share a tile
    int base[kTileThreads];
    long long scan[kTileThreads / 32];
    KvTilePiece piece[kTilePieces];
    KvShares shares;
    KvPiece open;                      // the segment that begins in this CTA and ends in another
    u64 piece_full[kTilePieces], piece_empty[kTilePieces];
    u64 raw_full[kTileRaw], raw_empty[kTileRaw];
    u64 full[kTileMeta];               // a page is unpacked: keys, values and their scales
    u64 k_empty[kTileKeys], v_empty[kTileValues], m_empty[kTileMeta];
    u64 q_full[2], s_full[2][2], p_full[2][2], o_done[2][2], x_full, x_empty, r_full, drain[2];
    unsigned int tmem;
    int abort_flag, padding;
};

// ---- tcgen05 ----------------------------------------------------------------------------------------

__device__ __forceinline__ void tc_alloc(unsigned int* where, unsigned int columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tc_free(unsigned int base, unsigned int columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(u64* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// D (fp32, tensor memory) (+)= A (fp16, tensor memory) B (fp16, shared memory)
__device__ __forceinline__ void tc_mma(unsigned int d, unsigned int a, u64 b, unsigned int idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u)
        : "memory");
}
// ... with A in shared memory
__device__ __forceinline__ void tc_mma_ss(unsigned int d, u64 a, u64 b, unsigned int idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u)
        : "memory");
}
// fp32 result, fp16 or bf16 operands, both K-major, M = 128
__host__ __device__ constexpr unsigned int tc_idesc(int n, bool bf16) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// Rows of 128 bytes in the 128-byte swizzle, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ u64 tc_desc(unsigned int addr) {
    return (u64)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// 64 columns of 16 lanes (rows): thread (g = lane / 4, j = lane % 4) has columns 8 k + 2 j and the next of rows
// g (x[4 k], x[4 k + 1]) and g + 8 (x[4 k + 2], x[4 k + 3]).  Loads have arrived when the statement is done.
__device__ __forceinline__ void tc_load(unsigned int addr, float (&x)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
        : "r"(addr) : "memory");
}
// ... of 32 lanes: rows g and g + 8, then g + 16 and g + 24
__device__ __forceinline__ void tc_load(unsigned int addr, float (&x)[2][32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%64];\n\t"
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%65];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(x[0][0]), "=f"(x[0][1]), "=f"(x[0][2]), "=f"(x[0][3]), "=f"(x[0][4]), "=f"(x[0][5]), "=f"(x[0][6]), "=f"(x[0][7]), "=f"(x[0][8]), "=f"(x[0][9]), "=f"(x[0][10]), "=f"(x[0][11]), "=f"(x[0][12]), "=f"(x[0][13]), "=f"(x[0][14]), "=f"(x[0][15]), "=f"(x[0][16]), "=f"(x[0][17]), "=f"(x[0][18]), "=f"(x[0][19]), "=f"(x[0][20]), "=f"(x[0][21]), "=f"(x[0][22]), "=f"(x[0][23]), "=f"(x[0][24]), "=f"(x[0][25]), "=f"(x[0][26]), "=f"(x[0][27]), "=f"(x[0][28]), "=f"(x[0][29]), "=f"(x[0][30]), "=f"(x[0][31]), "=f"(x[1][0]), "=f"(x[1][1]), "=f"(x[1][2]), "=f"(x[1][3]), "=f"(x[1][4]), "=f"(x[1][5]), "=f"(x[1][6]), "=f"(x[1][7]), "=f"(x[1][8]), "=f"(x[1][9]), "=f"(x[1][10]), "=f"(x[1][11]), "=f"(x[1][12]), "=f"(x[1][13]), "=f"(x[1][14]), "=f"(x[1][15]), "=f"(x[1][16]), "=f"(x[1][17]), "=f"(x[1][18]), "=f"(x[1][19]), "=f"(x[1][20]), "=f"(x[1][21]), "=f"(x[1][22]), "=f"(x[1][23]), "=f"(x[1][24]), "=f"(x[1][25]), "=f"(x[1][26]), "=f"(x[1][27]), "=f"(x[1][28]), "=f"(x[1][29]), "=f"(x[1][30]), "=f"(x[1][31])
        : "r"(addr), "r"(addr + (16u << 16)) : "memory");
}
__device__ __forceinline__ void tc_store(unsigned int addr, const float (&x)[32]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "f"(x[8]), "f"(x[9]), "f"(x[10]), "f"(x[11]), "f"(x[12]), "f"(x[13]), "f"(x[14]), "f"(x[15]), "f"(x[16]), "f"(x[17]), "f"(x[18]), "f"(x[19]), "f"(x[20]), "f"(x[21]), "f"(x[22]), "f"(x[23]), "f"(x[24]), "f"(x[25]), "f"(x[26]), "f"(x[27]), "f"(x[28]), "f"(x[29]), "f"(x[30]), "f"(x[31]) : "memory");
}
// 32 columns of 16 lanes, a 32-bit cell each: column 4 k + j of rows g (x[2 k]) and g + 8 (x[2 k + 1]).
__device__ __forceinline__ void tc_store_cells(unsigned int addr, const unsigned int (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
__device__ __forceinline__ void tc_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ __half2 as_half2(unsigned int x) { return *reinterpret_cast<const __half2*>(&x); }
// Values of two codes of a word (those in bits 0-3 and 16-19, or 4-7 and 20-23).
// Two codes of a word as bf16 numbers: 128 + c, less 128 (both exact).
template <bool HIGH>
__device__ __forceinline__ unsigned int bf16_codes(unsigned int w) {
    const unsigned int b = ((HIGH ? w >> 4 : w) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 c = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&b), __float2bfloat162_rn(128.f));
    return *reinterpret_cast<const unsigned int*>(&c);
}
template <bool HIGH>
__device__ __forceinline__ unsigned int expand(unsigned int w, __half2 scale, __half2 minimum) {
    const unsigned int b = (w & (HIGH ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;     // 1024 + c, or 1024 + 16 c
    const __half2 c = HIGH ? __hfma2(as_half2(b), __float2half2_rn(0.0625f), __float2half2_rn(-64.f)) : __hsub2(as_half2(b), __float2half2_rn(1024.f));
    const __half2 v = __hfma2(c, scale, minimum);
    return *reinterpret_cast<const unsigned int*>(&v);
}
// Column of S (row of the key operand) of a page's token: the two inner ones of every four change
// places, so that neighbouring columns are the tokens whose codes leave a word of the values together.
__device__ __forceinline__ int tile_place(int t) { return (t & ~3) | ((t & 1) << 1) | ((t >> 1) & 1); }
__device__ __forceinline__ u64 tile_places(u64 tokens) {
    return (tokens & 0x9999999999999999ull) | ((tokens & 0x2222222222222222ull) << 1) | ((tokens & 0x4444444444444444ull) >> 1);
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// O of a warp's 32 rows times a factor per row (fo[q]: row g + 8 q).
template <int D>
__device__ __forceinline__ void tile_scale_o(unsigned int col_o, const float (&fo)[4]) {
#pragma unroll 1
    for (int cb = 0; cb < D; cb += 64)
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const float f0 = half ? fo[2] : fo[0], f1 = half ? fo[3] : fo[1];
            float o[32];
            tc_load(col_o + cb + ((unsigned int)(16 * half) << 16), o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] *= (k >> 1) & 1 ? f1 : f0;
            tc_store(col_o + cb + ((unsigned int)(16 * half) << 16), o);
        }
    tc_wait_store();   // (a page may scale O twice)
}

// The walker's one thread: goes through the CTA's share of the work and hands it out piece by piece.  False: a wait has given up.
template <class Shared, class Wait>
__device__ __forceinline__ bool kv_tile_walk(const KvAttendArgs& a, Shared& sh, int total, int strip, int R, int G, const Wait& wait_one) {
    const int B = a.p.n_seqs, c = blockIdx.x;
    bool ok = true;
    const KvShares shares(total, min((int)gridDim.x, max(total, 1)));
    sh.shares = shares;
    KvTilePiece w{};
    int left = 0;            // units of the share from page w.pg on
    KvSeq q{};
    if (c < total) {
        // the share's first unit: its sequence, head, tile and page
        const int u0 = shares.first(c);
        int lo = 0, hi = (B + strip - 1) / strip;
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sh.base[mid] <= u0) lo = mid;
            else hi = mid;
        }
        int rem = u0 - sh.base[lo], per_head;
        w.b = lo * strip - 1;
#pragma unroll 1
        do {
            q = kv_load_seq(a, ++w.b, R);
            per_head = (int)kv_tile_head_units(a, q, R, G);
            rem -= per_head * a.p.n_kv_heads;
        } while (rem >= 0);
        rem += per_head * a.p.n_kv_heads;
        w.h = rem / per_head;
        rem -= w.h * per_head;
        w.tile = -1;
#pragma unroll 1
        do {
            w.pages = kv_tile_pages(a, q.cached, q.fresh, q.pages, ++w.tile, R, G);
            rem -= w.pages + kTileSegCost;
        } while (rem >= 0);
        rem += w.pages;              // of the first page, counted from page 0
        w.pg = max(rem, 0);
        left = shares.first(c + 1) - u0 - (w.pg - rem);
        w.seg = u0 - rem;
    }
#pragma unroll 1
    for (int k = 0; ok; ++k) {
        ok = wait_one(&sh.piece_empty[k % kTilePieces], ((k / kTilePieces) & 1) ^ 1);
        if (!ok) break;
        w.np = max(0, min(w.pages - w.pg, left));
        w.cached = q.cached;
        w.fresh = q.fresh;
        w.first = q.first;
        sh.piece[k % kTilePieces] = w;
        mbar_arrive(&sh.piece_full[k % kTilePieces]);
        if (w.np == 0) break;
        left -= w.pages - w.pg + kTileSegCost;
        w.seg += w.pages + kTileSegCost;
        w.pg = 0;
        if (++w.tile == q.tiles) {
            w.tile = 0;
            if (++w.h == a.p.n_kv_heads) {
                w.h = 0;
#pragma unroll 1
                do {
                    if (++w.b >= B) {
                        left = 0;
                        break;
                    }
                    q = kv_load_seq(a, w.b, R);
                } while (q.pages == 0 || q.tiles == 0);
            }
        }
        if (left > 0) w.pages = kv_tile_pages(a, q.cached, q.fresh, q.pages, w.tile, R, G);
    }
    return ok;
}

// ---- the kernel ---------------------------------------------------------------------------------------

template <int D, bool PAIR>
__global__ void __launch_bounds__(kTileThreads, 1) kv_attend_tile_kernel(const KvAttendArgs a) {
    using Shared = KvTileShared<D, PAIR>;
    constexpr int R = Shared::R, H = D / 2;
    constexpr unsigned int kColS = 0, kColO = 256, kStep = 128;    // first columns of group 0's S and O; group 1's are kStep behind
    constexpr unsigned int kIdescS = tc_idesc(kPage, true), kIdescO = tc_idesc(D, false);
    extern __shared__ unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
#pragma unroll 1
        for (int i = 0; i < kTilePieces; ++i) {
            mbar_init(&sh.piece_full[i], 1);
            mbar_init(&sh.piece_empty[i], 8 + 4 + 2 + 1);
        }
#pragma unroll 1
        for (int i = 0; i < kTileRaw; ++i) {
            mbar_init(&sh.raw_full[i], blockIdx.x == 0 && i == a.withhold_page ? 2 : 1);   // (testing aid: the second arrival never comes)
            mbar_init(&sh.raw_empty[i], 4);
        }
#pragma unroll 1
        for (int i = 0; i < kTileKeys; ++i) {
            mbar_init(&sh.k_empty[i], PAIR ? 2 : 1);
        }
#pragma unroll 1
        for (int i = 0; i < kTileValues; ++i) {
            mbar_init(&sh.v_empty[i], PAIR ? 2 : 1);
        }
#pragma unroll 1
        for (int i = 0; i < kTileMeta; ++i) {
            mbar_init(&sh.full[i], 4);
            mbar_init(&sh.m_empty[i], PAIR ? 8 : 4);
        }
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_full[i], 4);
            for (int b = 0; b < 2; ++b) {
                mbar_init(&sh.s_full[i][b], 1);
                mbar_init(&sh.p_full[i][b], 4);
                mbar_init(&sh.o_done[i][b], 1);
            }
            mbar_init(&sh.drain[i], 1);
        }
        mbar_init(&sh.x_full, 4);
        mbar_init(&sh.x_empty, 4);
        mbar_init(&sh.r_full, 4);
        sh.abort_flag = 0;
        sh.open.seg = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tc_alloc(&sh.tmem, 512);
    pdl_wait();
    const int B = a.p.n_seqs, G = a.p.n_q_heads / a.p.n_kv_heads;
    const int strip = (B + kTileThreads - 1) / kTileThreads;
    long long mine = 0;
    bool padding = B == 0;
#pragma unroll 1
    for (int b = tid * strip; b < min(B, (tid + 1) * strip); ++b) {
        const KvSeq s = kv_load_seq(a, b, R);
        mine += kv_tile_head_units(a, s, R, G) * a.p.n_kv_heads;
        padding = padding || kv_has_padding(a, s, b);
        if (s.fresh > 0 && (long long)s.cached + s.fresh > (long long)a.p.max_pages * kPage) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    tc_fence_before();
    long long sum;
    sh.base[tid] = (int)block_scan<kTileThreads>(mine, sh.scan, sum);
    if (tid == 0) sh.padding = 0;
    __syncthreads();
    if (padding) sh.padding = 1;
    __syncthreads();
    tc_fence_after();
    const unsigned int tm = sh.tmem;
    volatile int* abort_flag = &sh.abort_flag;
    const int c = blockIdx.x, total = kv_total(a, sum);
    // Waits are bounded; a role that gives up says so when it leaves, and the others find out in theirs.
    const auto wait_one = [&](u64* bar, unsigned int parity) { return kv_wait(a, bar, parity, abort_flag); };
    // (the lanes of a warp go on, or give up, together)
    const auto together = [](bool on) { return __all_sync(0xFFFFFFFFu, on) != 0; };
    const auto wait = [&](u64* bar, unsigned int parity) { return together(wait_one(bar, parity)); };
    bool ok = true;

    if (warp >= 12) {
        fewer_registers<kTileOtherRegs>();
        if (warp == 15) {
            // ---- walker
            if (lane == 0) {
                ok = kv_tile_walk(a, sh, total, strip, R, G, wait_one);
            }
            __syncwarp();
        } else if (warp == 13) {
            // ---- loader
            int n = 0;
#pragma unroll 1
            for (int k = 0;; ++k) {
                ok = wait(&sh.piece_full[k % kTilePieces], (k / kTilePieces) & 1);
                if (!ok) break;
                const KvTilePiece& w = sh.piece[k % kTilePieces];
                const int np = w.np, pg = w.pg;
                if (np == 0) break;
                const bool inside = AASD_IN_RANGE(w.b < B && w.h < a.p.n_kv_heads && pg + np <= a.p.max_pages, a.state);
                const int32_t* table = a.block_table + (long long)w.b * a.p.max_pages + pg;
                const uint8_t* head = a.pages + (long long)w.h * kv_head_bytes(D);
                const u64 stride = (u64)a.p.n_kv_heads * kv_head_bytes(D);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.piece_empty[k % kTilePieces]);
                int ids = 0;
#pragma unroll 1
                for (int i = 0; i < np; ++i, ++n) {
                    if ((i & 31) == 0) ids = i + lane < np && inside ? table[i + lane] : -1;
                    const int page = __shfl_sync(0xFFFFFFFFu, ids, i & 31);
                    const int slot = n % kTileRaw;
                    ok = wait(&sh.raw_empty[slot], ((n / kTileRaw) & 1) ^ 1);
                    if (!ok) break;
                    if (lane == 0) {
                        const bool there = page >= 0 && page < a.p.n_pages;
                        sh.raw_missing[slot] = !there;
                        if (there) {
                            mbar_arrive_expect_tx(&sh.raw_full[slot], kv_head_bytes(D));
                            bulk_copy_g2s(sh.raw[slot], head + (u64)(unsigned int)page * stride, kv_head_bytes(D), &sh.raw_full[slot]);
                        } else {
                            raise(a.state, AASD_STATUS_BAD_OFFSETS);
                            mbar_arrive(&sh.raw_full[slot]);
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
            }
            // nothing may be on its way into this CTA's shared memory when it leaves
#pragma unroll 1
            for (int k = max(0, n - kTileRaw); k < n; ++k)
#pragma unroll 1
                for (unsigned int it = 0; it < a.wait_limit && !mbar_try_wait(&sh.raw_full[k % kTileRaw], (k / kTileRaw) & 1); ++it) {}
        } else {
            // ---- issuers: warp 12 for group 0, warp 14 for group 1
            if (lane == 0) {
                const int x = (warp - 12) >> 1;
                // A piece's pages of the group: all, or every other page of the share.  The keys' products run up to two
                // pages ahead, but not into the next piece: its queries come when this one's last page is in O.
                int n0 = 0, taken = 0;   // pages of the share before the piece; of the group so far
#pragma unroll 1
                for (int k = 0;; ++k) {
                    ok = wait_one(&sh.piece_full[k % kTilePieces], (k / kTilePieces) & 1);
                    if (!ok) break;
                    const int np = sh.piece[k % kTilePieces].np;
                    if (np == 0) break;
                    mbar_arrive(&sh.piece_empty[k % kTilePieces]);
                    ok = wait_one(&sh.q_full[x], k & 1);
                    if (!ok) break;
                    const u64 q = tc_desc(smem_u32(sh.queries[PAIR ? x : 0]));
                    const int first = PAIR ? 0 : (n0 ^ x) & 1, step = PAIR ? 1 : 2;
                    int ahead = first, asked = taken;
#pragma unroll 1
                    for (int i = first; i < np; i += step, ++taken) {
#pragma unroll 1
                        for (; ahead < np && asked < taken + 2; ahead += step, ++asked) {
                            const int n = n0 + ahead, slot = n % kTileKeys, buf = asked & 1;
                            ok = wait_one(&sh.full[n % kTileMeta], (n / kTileMeta) & 1);
                            if (!ok) break;
                            tc_fence_after();
                            const u64 keys = tc_desc(smem_u32(sh.keys[slot]));
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)   // (descriptors count 16 bytes; a panel is 64 channels of all rows)
                                tc_mma_ss(tm + kColS + x * kStep + buf * 64, q + (ks / 4) * (kTileRows * 8) + (ks % 4) * 2,
                                          keys + (ks / 4) * (kPage * 8) + (ks % 4) * 2, kIdescS, ks > 0);
                            tc_commit(&sh.s_full[x][buf]);
                            tc_commit(&sh.k_empty[slot]);
                        }
                        const int n = n0 + i, slot = n % kTileValues, buf = taken & 1;
                        ok = ok && wait_one(&sh.p_full[x][buf], (taken >> 1) & 1);   // (the page's values came with its keys)
                        if (!ok) break;
                        tc_fence_after();
                        const u64 v = tc_desc(smem_u32(sh.values[slot]));
#pragma unroll
                        for (int ks = 0; ks < kPage / 16; ++ks)
                            tc_mma(tm + kColO + x * kStep, tm + kColS + x * kStep + buf * 64 + ks * 8, v + ks * 2, kIdescO, i > first || ks > 0);
                        tc_commit(&sh.v_empty[slot]);
                        tc_commit(&sh.o_done[x][buf]);
                    }
                    if (!ok) break;
                    n0 += np;
                }
                // products in flight read this CTA's shared memory
                tc_commit(&sh.drain[x]);
#pragma unroll 1
                for (unsigned int it = 0; it < a.wait_limit && !mbar_try_wait(&sh.drain[x], 0); ++it) {}
            }
            __syncwarp();
        }
    } else if (warp >= 8) {
        // ---- unpackers
        fewer_registers<kTileOtherRegs>();
        const int u = tid - 256, uw = warp - 8;
        int n = 0;
#pragma unroll 1
        for (int k = 0;; ++k) {
            ok = wait(&sh.piece_full[k % kTilePieces], (k / kTilePieces) & 1);
            if (!ok) break;
            const KvTilePiece& piece = sh.piece[k % kTilePieces];
            const int np = piece.np, end = piece.cached + piece.fresh - piece.pg * kPage;   // places from the first page's on
            __syncwarp();
            if (np == 0) break;
            if (lane == 0) mbar_arrive(&sh.piece_empty[k % kTilePieces]);
            int ev = 64;
#pragma unroll 1
            for (int i = 0; i < np; ++i, ++n) {
                const int slot = n % kTileRaw, mslot = n % kTileMeta, kslot = n % kTileKeys, vslot = n % kTileValues;
                ok = together(wait_one(&sh.raw_full[slot], (n / kTileRaw) & 1) && wait_one(&sh.k_empty[kslot], ((n / kTileKeys) & 1) ^ 1) &&
                              wait_one(&sh.v_empty[vslot], ((n / kTileValues) & 1) ^ 1) && wait_one(&sh.m_empty[mslot], ((n / kTileMeta) & 1) ^ 1));
                if (!ok) break;
                const unsigned char* raw = sh.raw[slot];
                const bool missing = sh.raw_missing[slot] != 0;
                const int left = missing ? 0 : end - i * kPage;   // places in use
                // Everything is fetched first.  Keys: half a token's row per thread (word k of a token: channels 4k .. of each
                // half).  Values: a channel's 64 codes, and those of the channel H above it, per TPR threads.
                constexpr int NW = H / 8;                        // words of keys per thread
                constexpr int TPR = 128 / H, NP = 8 / TPR;       // threads per row of values; 16-byte pieces per thread and half
                const int t = u >> 1, khalf = u & 1, r = u / TPR, vpart = u % TPR;
                unsigned int kw[NW], vw[2 * NP];
                const uint2 vm = *reinterpret_cast<const uint2*>(raw + kv_value_meta_offset(D) + 8 * lane);
                const uint4 four = lds16(raw + kv_value_meta_offset(D) + 16 * (lane & 15));
                const unsigned int key_meta = *reinterpret_cast<const unsigned int*>(raw + kv_key_meta_offset(D) + 4 * (u & (kPage - 1)));
#pragma unroll
                for (int k = 0; k < NW; k += 4) {
                    const uint4 q = lds16(raw + t * H + khalf * (H / 2) + 4 * k);
                    kw[k] = q.x; kw[k + 1] = q.y; kw[k + 2] = q.z; kw[k + 3] = q.w;
                }
#pragma unroll
                for (int k = 0; k < 2 * NP; k += 4) {
                    const uint4 q = lds16(raw + kv_value_offset(D) + r * kPage + vpart * (kPage / TPR) + 4 * k);
                    vw[k] = q.x; vw[k + 1] = q.y; vw[k + 2] = q.z; vw[k + 3] = q.w;
                }
                // largest value of the page (every warp for itself): codes run from the minimum to 15 scales above it
                auto reach = [](unsigned int m) { return fmaxf(fabsf(meta_min(m)), fabsf(fmaf(15.f, meta_scale(m), meta_min(m)))); };
                float vt = 2 * lane < left ? reach(vm.x) : 0.f;
                if (2 * lane + 1 < left) vt = fmaxf(vt, reach(vm.y));
                // (an exponent field, held to a range in which the factors below are normal numbers)
                ev = max(ev, min(250, (int)(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(vt)) >> 23)));
                // the values' table: lane q < 16 has tokens 4q .. 4q + 3, in the order in which their codes leave a word
                if (lane < kPage / 4) {
                    const float norm = pow2f(127 - ev);
                    const unsigned int m0 = 4 * lane < left ? four.x : 0u, m1 = 4 * lane + 1 < left ? four.y : 0u,
                                       m2 = 4 * lane + 2 < left ? four.z : 0u, m3 = 4 * lane + 3 < left ? four.w : 0u;
                    sh.vmeta[uw][lane] = make_uint4(pack_half(meta_scale(m0) * norm, meta_scale(m2) * norm), pack_half(meta_scale(m1) * norm, meta_scale(m3) * norm),
                                                    pack_half(meta_min(m0) * norm, meta_min(m2) * norm), pack_half(meta_min(m1) * norm, meta_min(m3) * norm));
                }
                if (u < kPage) {
                    const unsigned int km = u < left ? key_meta : 0u;
                    const int at = tile_place(u);
                    float* kq = reinterpret_cast<float*>(&sh.kmeta[mslot][at >> 1]);
                    kq[at & 1] = meta_scale(km);
                    kq[2 + (at & 1)] = meta_min(km);
                    if (u == 0) sh.ev[mslot] = missing ? -1 : ev;
                }
                {
                    // Keys: word k becomes 16-byte piece k of the token's row; the two threads of a token take their pieces
                    // in orders that keep eight neighbouring threads on eight different pieces.
                    const int at = tile_place(t);
                    unsigned char* to = sh.keys[kslot] + at * 128;
#pragma unroll
                    for (int k = 0; k < NW; ++k) {
                        const int kk = NW == 8 ? k ^ (khalf * 4) : k;
                        const unsigned int x = NW == 8 ? (khalf ? kw[k ^ 4] : kw[k]) : kw[k], y = x >> 8;
                        const int piece = khalf * NW + kk;       // of the token's H / 4
                        *reinterpret_cast<uint4*>(to + (piece >> 3) * (kPage * 128) + (((piece & 7) ^ (at & 7)) << 4)) =
                            make_uint4(bf16_codes<false>(x), bf16_codes<false>(y), bf16_codes<true>(x), bf16_codes<true>(y));
                    }
                }
                __syncwarp();   // (the table)
                // values: 8 tokens of a channel are a 16-byte piece
                unsigned char* lo = sh.values[vslot] + r * 128;
                unsigned char* hi = lo + H * 128;            // (H is a multiple of 8: the same swizzle)
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const unsigned int x0 = vw[2 * k], x1 = vw[2 * k + 1], y0 = x0 >> 8, y1 = x1 >> 8;
                    const uint4 q0 = sh.vmeta[uw][2 * (vpart * NP + k)], q1 = sh.vmeta[uw][2 * (vpart * NP + k) + 1];
                    const __half2 s0 = as_half2(q0.x), s1 = as_half2(q0.y), m0 = as_half2(q0.z), m1 = as_half2(q0.w);
                    const __half2 s2 = as_half2(q1.x), s3 = as_half2(q1.y), m2 = as_half2(q1.z), m3 = as_half2(q1.w);
                    const int at = ((vpart * NP + k) ^ (r & 7)) << 4;
                    *reinterpret_cast<uint4*>(lo + at) =
                        make_uint4(expand<false>(x0, s0, m0), expand<false>(y0, s1, m1), expand<false>(x1, s2, m2), expand<false>(y1, s3, m3));
                    *reinterpret_cast<uint4*>(hi + at) =
                        make_uint4(expand<true>(x0, s0, m0), expand<true>(y0, s1, m1), expand<true>(x1, s2, m2), expand<true>(y1, s3, m3));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.full[mslot]);
                    mbar_arrive(&sh.raw_empty[slot]);
                }
            }
            if (!ok) break;
        }
    } else {
        // ---- softmax: thread (g, j) of a warp has rows g, g + 8, g + 16, g + 24 of the warp's 32 and two columns of every eight
        more_registers<kTileSoftmaxRegs>();
        const int x = warp >> 2, g = lane >> 2, j = lane & 3, row_base = (warp & 3) * 32;   // (of the group's 128 rows)
        const unsigned int lanes = (unsigned int)row_base << 16;
        const unsigned int col_s = tm + kColS + x * kStep + lanes, col_o = tm + kColO + x * kStep + lanes;
        const float rf = fmaxf(a.scale_log2, 1e-37f);   // (never 0: what is hidden is -inf times it)
        int n0 = 0, taken = 0;    // pages of the share before the piece; of the group so far
        // All pages taken so far are in O.  (Not waited for with every page: a barrier for every other page keeps the
        // phases apart, since S of a page comes after O of the page two before it.)
        const auto o_complete = [&]() {
            const bool done = wait(&sh.o_done[x][(taken - 1) & 1], ((taken - 1) >> 1) & 1);
            tc_fence_after();
            return done;
        };
#pragma unroll 1
        for (int piece = 0;; ++piece) {
            ok = wait(&sh.piece_full[piece % kTilePieces], (piece / kTilePieces) & 1);
            if (!ok) break;
            const KvTilePiece w = sh.piece[piece % kTilePieces];
            __syncwarp();
            const int np = w.np;
            if (np == 0) break;
            if (lane == 0) mbar_arrive(&sh.piece_empty[piece % kTilePieces]);
            const int row0 = w.tile * R + (PAIR ? x * kTileRows : 0) + row_base;   // of the warp's first row, among the head's
            const int rows_here = AASD_IN_RANGE(w.first + w.fresh <= a.p.n_tokens && w.h < a.p.n_kv_heads, a.state) ? w.fresh * G : 0;   // rows of the head
            const int own_row = max(min(row0 + lane, rows_here - 1), 0);   // the lane's row: what the warp wants to know of its 32 rows
            const int token = own_row / G, member = own_row - token * G;
            if (PAIR || x == 0) {
                // The rows' queries, channels in the order of the keys' words, and their sums; D / 8 lanes fetch a row together.
                constexpr int LR = D / 8, RI = 32 / LR;        // lanes per row, rows per step
                const int part = lane % LR;                    // eight channels: of the low half, then of the high one
                const long long at = ((long long)w.first + token) * a.p.q_stride + (long long)(w.h * G + member) * D;   // of the lane's row
                unsigned char* to = sh.queries[PAIR ? x : 0];
#pragma unroll 1
                for (int rb = 0; rb < 32; rb += 8 * RI) {
                    Raw8<AASD_BF16, true> raw[8];
                    // (all on their way before the first is looked at; rows past the last one repeat it, and become zero)
                    if (a.q_vec) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) raw[k].load(a.q, __shfl_sync(0xFFFFFFFFu, at, rb + k * RI + lane / LR) + part * 8);
                    } else {
#pragma unroll 1
                        for (int k = 0; k < 8; ++k) {
                            Raw8<AASD_BF16, false> slow;
                            slow.load(a.q, __shfl_sync(0xFFFFFFFFu, at, rb + k * RI + lane / LR) + part * 8);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (i == k) raw[i].a = slow.a;
                        }
                    }
                    float sum[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = row_base + rb + k * RI + lane / LR;
                        if (row0 + rb + k * RI + lane / LR >= rows_here) raw[k].clear();
                        float2 y[4];
                        raw[k].unpack(y);
                        sum[k] = ((y[0].x + y[0].y) + (y[1].x + y[1].y)) + ((y[2].x + y[2].y) + (y[3].x + y[3].y));
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int piece = 2 * (part % (LR / 2)) + q;
                            const unsigned int c01 = q ? raw[k].a.z : raw[k].a.x, c23 = q ? raw[k].a.w : raw[k].a.y;
                            *reinterpret_cast<uint2*>(to + r * 128 + (piece >> 3) * (kTileRows * 128) + (((piece & 7) ^ (r & 7)) << 4) +
                                                      (part >= LR / 2 ? 8 : 0)) = make_uint2(__byte_perm(c01, c23, 0x5410), __byte_perm(c01, c23, 0x7632));
                        }
                    }
#pragma unroll
                    for (int o = 1; o < LR; o <<= 1)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], o);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (part == 0) sh.row_q[PAIR ? x : 0][row_base + rb + k * RI + lane / LR] = sum[k];
                }
                fence_async_smem();
                __syncwarp();
            }
            if (!PAIR) {
                // one set of queries for both groups
                if (x == 0) {
                    if (lane == 0) mbar_arrive(&sh.r_full);
                } else {
                    ok = wait(&sh.r_full, piece & 1);
                    if (!ok) break;
                }
            }
            if (lane == 0) mbar_arrive(&sh.q_full[x]);
            float qf[4], mref[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qf[i] = sh.row_q[PAIR ? x : 0][row_base + g + 8 * i];
                mref[i] = kKvNothing;
                l[i] = 0.f;
            }
            // sixteen rows at a time are left out where the head has none of them (their probabilities are anything, and so
            // is what becomes of them)
            const int halves = min(2, (rows_here - row0 + 15) >> 4);
            // places up to which every row of the warp sees everything
            const int open_to = a.node_parent != nullptr ? w.cached : w.cached + row0 / G + 1;
            int ev = 64;
            bool first = true, large = false;
#pragma unroll 1
            for (int i = PAIR ? 0 : (n0 ^ x) & 1; i < np; i += PAIR ? 1 : 2) {
                const int n = n0 + i, mslot = n % kTileMeta, pg = w.pg + i, buf = taken & 1;
                const unsigned int col = col_s + buf * 64;
                ok = together(wait_one(&sh.full[mslot], (n / kTileMeta) & 1) && wait_one(&sh.s_full[x][buf], (taken >> 1) & 1));
                if (!ok) break;
                if (halves > 0) {
                    tc_fence_after();
                    float s[2][32];   // rows g and g + 8; g + 16 and g + 24
                    if (halves == 2) {
                        tc_load(col, s);
                    } else {
                        tc_load(col, s[0]);
#pragma unroll
                        for (int k = 0; k < 32; ++k) s[1][k] = 0.f;
                    }
                    const int evn = sh.ev[mslot];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float4 m = sh.kmeta[mslot][4 * k + j];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {   // row g + 8 q
                            float& s0 = s[q >> 1][4 * k + 2 * (q & 1)];
                            float& s1 = s[q >> 1][4 * k + 2 * (q & 1) + 1];
                            const float2 y = __ffma2_rn(make_float2(m.z, m.w), make_float2(qf[q], qf[q]), __fmul2_rn(make_float2(s0, s1), make_float2(m.x, m.y)));
                            s0 = y.x;
                            s1 = y.y;
                        }
                    }
                    if (evn < 0 || (pg + 1) * kPage > open_to) {   // what a row does not see becomes -inf (lane r finds out for row r)
                        const u64 mine = evn < 0 || row0 + lane >= rows_here ? 0ull : tile_places(kv_seen(a, w.cached, w.fresh, w.first, pg, token));
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const u64 seen = __shfl_sync(0xFFFFFFFFu, mine, g + 8 * q) >> (2 * j);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const unsigned int two = (unsigned int)(seen >> (8 * k));
                                if (!(two & 1u)) s[q >> 1][4 * k + 2 * (q & 1)] = -CUDART_INF_F;
                                if (!(two & 2u)) s[q >> 1][4 * k + 2 * (q & 1) + 1] = -CUDART_INF_F;
                            }
                        }
                    }
                    // Probabilities with the maximum as it stands; only where a thread's sum of them leaves fp16's range (by a
                    // new maximum at least 2^5 above it), on the first page, and with large products, is the maximum looked for
                    // and this done again.
                    float ls[4];
                    bool again = first || large;
                    float rr = rf;             // what S is still to be multiplied by
#pragma unroll 1
                    for (;;) {
                        if (again) {
                            float fo[4], m[4], top = 0.f;
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                m[q] = -CUDART_INF_F;
#pragma unroll
                                for (int k = 0; k < 8; ++k) m[q] = fmaxf(m[q], fmaxf(s[q >> 1][4 * k + 2 * (q & 1)], s[q >> 1][4 * k + 2 * (q & 1) + 1]));
                                m[q] = fmaxf(m[q], __shfl_xor_sync(0xFFFFFFFFu, m[q], 1));
                                m[q] = fmaxf(m[q], __shfl_xor_sync(0xFFFFFFFFu, m[q], 2));
                                m[q] *= rf;
                                if (m[q] > -CUDART_INF_F) top = fmaxf(top, fabsf(m[q]));
                            }
                            large = large || __any_sync(0xFFFFFFFFu, top >= kTileLarge);
                            if (large) {
                                rr = 1.f;
#pragma unroll
                                for (int half = 0; half < 2; ++half)
#pragma unroll
                                    for (int k = 0; k < 32; ++k) s[half][k] *= rf;
                            }
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float mn = fmaxf(mref[q], m[q]);
                                fo[q] = ex2_approx(mref[q] - mn);
                                mref[q] = mn;
                                l[q] *= fo[q];
                            }
                            if (!first) {
                                ok = o_complete();
                                if (!ok) break;
                                tile_scale_o<D>(col_o, fo);
                            }
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (half >= halves) {
                                ls[2] = ls[3] = 0.f;
                                break;
                            }
                            unsigned int pk[16];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int q = 2 * half + e;
                                const float2 ff = make_float2(rr, rr), mm = make_float2(kTileP - mref[q], kTileP - mref[q]);
                                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    float2 p = __ffma2_rn(make_float2(s[half][4 * k + 2 * e], s[half][4 * k + 2 * e + 1]), ff, mm);
                                    p = make_float2(ex2_approx(p.x), ex2_approx(p.y));
                                    sum = __fadd2_rn(sum, p);
                                    pk[2 * k + e] = pack_half(p.x, p.y);
                                }
                                ls[q] = sum.x + sum.y;
                            }
                            tc_store_cells(col + ((unsigned int)(16 * half) << 16), pk);
                        }
                        if (again || __all_sync(0xFFFFFFFFu, fmaxf(fmaxf(ls[0], ls[1]), fmaxf(ls[2], ls[3])) < 65504.f)) break;
                        again = true;
                    }
                    if (!ok) break;
                    if (evn > ev) {
                        // values of this page are relative to a larger exponent than O
                        if (!first) {
                            ok = o_complete();
                            if (!ok) break;
                            const float f = evn - ev > 126 ? 0.f : pow2f(ev - evn);
                            const float fo[4] = {f, f, f, f};
                            tile_scale_o<D>(col_o, fo);
                        }
                        ev = evn;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) l[q] += ls[q];
                }
                first = false;
                ++taken;
                tc_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.p_full[x][buf]);
                    mbar_arrive(&sh.m_empty[mslot]);
                }
            }
            if (!ok) break;
            // the result of the piece
            const bool any = !first;
            if (any) {
                ok = o_complete();
                if (!ok) break;
            }
            const bool complete = w.pg == 0 && np == w.pages;
            const int which = w.pg > 0 ? 0 : 1;
            const int rows = AASD_IN_RANGE(c < kKvMaxCtas, a.state) ? min(R, rows_here - w.tile * R) : 0;
            constexpr int kPart = R * D + 2 * R;
            float* part = a.cta_parts + (long long)(c * 2 + which) * kPart;
            float own[4], other[4];        // factors of this group's O, and of the other's
            const float unscale = any ? pow2f(ev - 127) : 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                l[q] += __shfl_xor_sync(0xFFFFFFFFu, l[q], 1);
                l[q] += __shfl_xor_sync(0xFFFFFFFFu, l[q], 2);
                mref[q] -= kTileP;         // (l and O carry the probabilities' power of two)
                own[q] = unscale;
                other[q] = 0.f;
            }
            if (!PAIR) {
                // group 0 reads both groups' O (the same lanes of tensor memory)
                if (x == 1) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (j == 0) {
                            const int r = row_base + g + 8 * q;
                            sh.exchange_m[r] = mref[q];
                            sh.exchange_l[r] = l[q];
                            sh.exchange_up[r] = unscale;
                        }
                    }
                    __syncwarp();
                    tc_fence_before();
                    if (lane == 0) mbar_arrive(&sh.x_full);
                    ok = wait(&sh.x_empty, piece & 1);
                    if (!ok) break;
                } else {
                    ok = wait(&sh.x_full, piece & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int r = row_base + g + 8 * q;
                        const float om = sh.exchange_m[r], mn = fmaxf(mref[q], om), of = ex2_approx(om - mn), f = ex2_approx(mref[q] - mn);
                        l[q] = l[q] * f + sh.exchange_l[r] * of;
                        own[q] *= f;
                        other[q] = sh.exchange_up[r] * of;
                        mref[q] = mn;
                    }
                }
            }
            if (PAIR || x == 0) {
                const bool any1 = !PAIR && sh.exchange_up[row_base] != 0.f;   // (the same for every row)
                // the results go through the places of the warp's own queries, which have been used
                const auto stage = [&](int lr, int piece) {
                    return sh.queries[PAIR ? x : 0] + (row_base + lr) * 128 + (piece >> 3) * (kTileRows * 128) + (((piece & 7) ^ (lr & 7)) << 4);
                };
                if (complete) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float inv = kv_inverse(l[q]);
                        own[q] *= inv;
                        other[q] *= inv;
                    }
                }
#pragma unroll 1
                for (int cb = 0; cb < D; cb += 64) {
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {      // rows g, g + 8; g + 16, g + 24
                        const float f0 = half ? own[2] : own[0], f1 = half ? own[3] : own[1];
                        float o[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = 0.f;
                        if (any) {
                            tc_load(col_o + cb + ((unsigned int)(16 * half) << 16), o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] *= (k >> 1) & 1 ? f1 : f0;
                        }
                        if (any1) {
                            const float g0 = half ? other[2] : other[0], g1 = half ? other[3] : other[1];
                            float y[32];
                            tc_load(col_o + kStep + cb + ((unsigned int)(16 * half) << 16), y);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = fmaf(y[k], (k >> 1) & 1 ? g1 : g0, o[k]);
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int lr = g + 16 * half + 8 * e, ch = cb + 8 * k + 2 * j;
                                const float2 v = make_float2(o[4 * k + 2 * e], o[4 * k + 2 * e + 1]);
                                if (complete) {
                                    *reinterpret_cast<unsigned int*>(stage(lr, ch >> 3) + 4 * j) = pack_bf16(v.x, v.y);
                                } else if ((PAIR ? x * kTileRows : 0) + row_base + lr < rows) {
                                    *reinterpret_cast<float2*>(part + ((PAIR ? x * kTileRows : 0) + row_base + lr) * D + ch) = v;
                                }
                            }
                    }
                }
                if (complete) {
                    __syncwarp();
                    constexpr int LR = D / 8, RI = 32 / LR;     // lanes per row, rows per step
                    const long long own_head = ((long long)w.first + token) * a.p.n_q_heads + w.h * G + member;
#pragma unroll 4
                    for (int rb = 0; rb < 32; rb += RI) {
                        const int lr = rb + lane / LR;
                        const long long head = __shfl_sync(0xFFFFFFFFu, own_head, lr);
                        if (row0 + lr < rows_here) {
                            const uint4 v = lds16(stage(lr, lane % LR));
                            if (a.out_vec) {
                                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o.out) + head * D + (lane % LR) * 8) = v;
                            } else {
                                unsigned short* to = static_cast<unsigned short*>(a.o.out) + head * D + (lane % LR) * 8;
                                const unsigned int u4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 8; ++e) to[e] = (unsigned short)(u4[e >> 1] >> (16 * (e & 1)));
                            }
                        }
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = (PAIR ? x * kTileRows : 0) + row_base + g + 8 * q, row = row0 + g + 8 * q;
                    if (j == 0 && row < rows_here) {
                        if (!complete) {
                            part[R * D + r] = mref[q];
                            part[R * D + R + r] = l[q];
                        } else if (a.o.lse != nullptr) {
                            a.o.lse[((long long)w.first + row / G) * a.p.n_q_heads + w.h * G + row % G] = kv_lse(mref[q], l[q]);
                        }
                    }
                }
                if (!complete && which == 1 && tid == 0) sh.open = KvPiece{w.seg, w.pages, w.h, w.tile * R, rows, w.first};
            }
            if (!PAIR && x == 0) {   // group 1 may go on
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.x_empty);
            }
            tc_fence_before();
            n0 += np;
        }
        if (!ok) tc_wait_store();   // (a group that gave up may have stores on their way to the memory that is freed below)
        // the segment that this CTA begins and others go on with, and rows to clear: the joining kernel's work
        if (tid == 0) {
            KvTileOpen o{sh.open, 0, total == 0 ? 2 : sh.padding ? 1 : 0};
            if (sh.open.seg >= 0 && ok && !*abort_flag) o.parts = sh.shares.owner(sh.open.seg + sh.open.pages - 1) - c + 1;
            a.tile_open[c] = o;
        }
    }
    if (!ok) give_up(abort_flag, a.state);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tc_free(tm, 512);
}

constexpr int kTileJoinThreads = 256, kTileJoinCtas = 2;   // a CTA's threads; CTAs per SM (with 4, and 64 registers, loads spill: 2 us more)
constexpr int kTileJoinRows = 4;

// Rows r0 .. r0 + 3 of a segment of at most eight parts, one warp: as kv_join_row, eight lanes finding a row's weights, with the
// first two parts' sums under way meanwhile.
template <int D>
__device__ __forceinline__ void kv_join_rows(const KvAttendArgs& a, const KvPiece& pc, int r0, const float* base, int stride, int rows, int parts, int G, int lane) {
    constexpr int NR = kTileJoinRows;
    const auto part = [&](int k) { return base + (long long)(2 * k + (k == 0)) * stride; };
    const int own = min(r0 + (lane >> 3), pc.n - 1), k = lane & 7;
    const bool mine = k < parts;
    const float m = mine ? __ldcg(part(k) + rows * D + own) : kKvNothing, l = mine ? __ldcg(part(k) + rows * D + rows + own) : 0.f;
    const bool on = lane * 4 < D;
    float4 x[NR][2];
    const auto load = [&](int k0, int ch) {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                x[i][q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (on && k0 + q < parts && r0 + i < pc.n) x[i][q] = __ldcg(reinterpret_cast<const float4*>(part(k0 + q) + (r0 + i) * D + ch));
            }
    };
    load(0, lane * 4);
    float M = fmaxf(kKvNothing, m);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
    const float f = mine ? ex2_approx(m - M) : 0.f;
    float L = mine ? fmaf(l, f, 0.f) : 0.f;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, o);
#pragma unroll 1
    for (int ch = lane * 4;;) {
        float4 o[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int k0 = 0;;) {
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float fk = __shfl_sync(0xFFFFFFFFu, f, 8 * i + ((k0 + q) & 7));
                    o[i].x = fmaf(x[i][q].x, fk, o[i].x);
                    o[i].y = fmaf(x[i][q].y, fk, o[i].y);
                    o[i].z = fmaf(x[i][q].z, fk, o[i].z);
                    o[i].w = fmaf(x[i][q].w, fk, o[i].w);
                }
            k0 += 2;
            if (k0 >= parts) break;
            load(k0, ch);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float Li = __shfl_sync(0xFFFFFFFFu, L, 8 * i), Mi = __shfl_sync(0xFFFFFFFFu, M, 8 * i);
            if (!on || r0 + i >= pc.n) continue;
            const float inv = kv_inverse(Li);
            const int row = pc.row0 + r0 + i;
            const long long head = ((long long)pc.first + row / G) * a.p.n_q_heads + pc.h * G + row % G;
            if (!AASD_IN_RANGE(head < a.p.n_tokens * a.p.n_q_heads, a.state)) continue;
            store4<AASD_BF16>(a.o.out, head * D + ch, make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), a.out_vec);
            if (a.o.lse != nullptr && ch == 0) a.o.lse[head] = kv_lse(Mi, Li);
        }
        if (D <= 128) break;
        ch += 128;
        if (ch >= D) break;
        load(0, ch);
    }
}

// Joins the parts of the segments that several CTAs of the tile kernel went through.  Every warp of the launch takes its turn
// at the list of their rows: four at a time, or one where there are more than eight parts.  It adds 6 to 14 us to a call's kernel
// (39 MB of parts where every CTA of a device has cut segments at both ends).  A block for every eight rows that a CTA's segment
// could have, most of which left at once, added 12 to 18; left to the last CTA that delivers a part, one
// sequence of 64k tokens with 64 new ones waited 100 us for 19 parts of 256 rows.  The warps also clear the rows that no
// tile has.  grid: (CTAs of the tile kernel, kTileJoinCtas).
template <int D, bool PAIR>
__global__ void __launch_bounds__(kTileJoinThreads, kTileJoinCtas) kv_tile_join_kernel(const KvAttendArgs a) {
    constexpr int R = PAIR ? 2 * kTileRows : kTileRows, kPart = R * D + 2 * R;
    static_assert(kKvMaxCtas <= kTileJoinThreads, "a thread for each CTA's segment");
    __shared__ int s_first[kTileJoinThreads];
    __shared__ long long s_warp[kTileJoinThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, ctas = (int)gridDim.x;
    const int warp = (int)(blockIdx.y * gridDim.x + blockIdx.x) * (kTileJoinThreads / 32) + (tid >> 5), warps = (int)(gridDim.x * gridDim.y) * (kTileJoinThreads / 32);
    int items = 0;
    if (tid < ctas) {
        const int parts = a.tile_open[tid].parts, n = a.tile_open[tid].piece.n;
        if (parts > 0) items = parts > 8 ? n : (n + kTileJoinRows - 1) / kTileJoinRows;
    }
    const int padding = a.tile_open[0].padding;
    long long total;
    s_first[tid] = (int)block_scan<kTileJoinThreads>(items, s_warp, total);
    __syncthreads();
    if (padding != 0) kv_clear_rows<AASD_BF16>(a, D, 2 - padding, warp, warps);
    const int G = a.p.n_q_heads / a.p.n_kv_heads;
#pragma unroll 1
    for (int i = warp; i < (int)total; i += warps) {
        const int c = last_not_above(s_first, ctas, i), at = i - s_first[c];
        const KvTileOpen open = a.tile_open[c];
        const float* base = a.cta_parts + (long long)c * 2 * kPart;   // part k: 2 k, the first one's 1
        if (open.parts > 8) kv_join_row<AASD_BF16, D>(a, open.piece, at, base, kPart, R, open.parts, G, lane);
        else kv_join_rows<D>(a, open.piece, at * kTileJoinRows, base, kPart, R, open.parts, G, lane);
    }
}

}  // namespace aasd
