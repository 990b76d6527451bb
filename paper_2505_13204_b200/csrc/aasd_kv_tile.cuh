// Attention over the paged 4-bit cache for many rows per key/value head (draft trees, chunks of a
// prompt): tiles of 128 rows on the fifth-generation tensor cores.
//
// One persistent CTA per SM; its warps have roles:
//   loader      brings pages (packed blocks) in by bulk copies;
//   unpackers   (4 warps) turn a page's codes into fp16 operands in shared memory, K-major rows of 128
//               bytes in the 128-byte swizzle;
//   two issuers, one thread each: tcgen05.mma of S = Q K^T (both operands in shared memory) and
//               O += P V (P in tensor memory) for one softmax group, a page (64 tokens) at a time;
//   two softmax groups of 4 warps, a thread per row: S to registers, probabilities back as P.
// The two groups work on two row tiles of the same pages (PAIR), or, where a segment has no more
// than 128 rows, on alternate pages of one tile, joined at the end.  A group has two S buffers, so
// that the next page's products are there when it is done with one.
//
// Keys stay bare codes, whose scale and minimum are applied to S (exactly: see aasd_kv_attend.cuh).
// Values are expanded here, relative to the largest exponent of the segment's pages so far (so that
// values of any size fit fp16), and rounded to 11 bits like the probabilities: a value is used for 128
// rows, and scaling the probabilities instead, with a sum of the minima beside them, costs the
// softmax groups, which pace the kernel, a third more instructions.
//
// Tensor memory (512 columns): two S buffers of each group, whose first halves P takes over, and O.
#pragma once

#include "aasd_kv_attend.cuh"

namespace aasd {

constexpr int kTileThreads = 512;      // 8 softmax warps, 4 unpackers; issuer, loader and two that fill their group of four
// Registers per thread: a launch of 512 threads has 128 for each; the softmax groups, which hold a
// row of S, take what the others give up (2 x 184 + 2 x 72 = 4 x 128).
constexpr int kTileLaunchRegs = 128, kTileSoftmaxRegs = 184, kTileOtherRegs = 72;
static_assert(2 * kTileSoftmaxRegs + 2 * kTileOtherRegs <= 4 * kTileLaunchRegs, "the shares add up to the launch's registers");
constexpr int kTileRows = 128;
constexpr int kTileRaw = 4, kTileKeys = 3, kTileValues = 4, kTileMeta = 6;   // ring depths, in pages
// the probabilities' power of two and the running maximum's lag (see the split kernel)
constexpr float kTileP = 7.f, kTileLazy = 8.f;

// ---- the list of work ---------------------------------------------------------------------------------

// Pages that a row tile looks at: those up to its last query's own token, or all (trees).
__device__ __forceinline__ int kv_tile_pages(const KvAttendArgs& a, int cached, int fresh, int pages, int tile, int R, int G) {
    if (a.node_parent != nullptr) return pages;
    const int last = (int)min((long long)fresh * G, (long long)(tile + 1) * R) - 1;
    return min(pages, (int)(((unsigned int)cached + (unsigned int)(last / G) + kPage) / kPage));
}
// Loading the queries into tensor memory and the result out of it takes about as long as two pages.
constexpr int kTileSegCost = 2;
// Units of one head of a sequence.
__device__ __forceinline__ long long kv_tile_head_units(const KvAttendArgs& a, const KvSeq& s, int R, int G) {
    if (s.pages == 0) return 0;
    if (a.node_parent != nullptr) return (long long)s.tiles * (s.pages + kTileSegCost);
    long long n = 0;
    for (int t = 0; t < s.tiles; ++t) n += kv_tile_pages(a, s.cached, s.fresh, s.pages, t, R, G) + kTileSegCost;
    return n;
}

// One CTA's way through its share; every role walks it for itself.  A piece is the run of pages of
// one segment that falls into the share.
struct KvTileWalk {
    int b, h, tile;
    int pg, pages;            // next page, and how many the segment has
    int left;                 // units of the share from page pg on
    int cached, fresh, first, seq_pages, tiles;   // see KvSeq
    __device__ __forceinline__ bool live() const { return left > 0; }
    __device__ __forceinline__ int piece_pages() const { return min(pages - pg, left); }
    __device__ __forceinline__ int tile_pages(const KvAttendArgs& a, int R, int G) const {
        return kv_tile_pages(a, cached, fresh, seq_pages, tile, R, G);
    }
    __device__ __forceinline__ void take(const KvSeq& s) {
        cached = s.cached;
        fresh = s.fresh;
        first = s.first;
        seq_pages = s.pages;
        tiles = s.tiles;
    }
    __device__ __forceinline__ void next(const KvAttendArgs& a, int R, int G) {
        left -= pages - pg + kTileSegCost;
        if (left <= 0) return;
        pg = 0;
        if (++tile == tiles) {
            tile = 0;
            if (++h == a.p.n_kv_heads) {
                h = 0;
                do {
                    if (++b >= a.p.n_seqs) {
                        left = 0;
                        return;
                    }
                    take(kv_load_seq(a, b, R));
                } while (seq_pages == 0 || tiles == 0);
            }
        }
        pages = tile_pages(a, R, G);
    }
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
    float exchange_m[kTileRows], exchange_l[kTileRows], exchange_up[kTileRows];   // between the groups, where they share a tile
    long long base[kTileThreads];
    long long scan[kTileThreads / 32];
    KvTileWalk start;                  // the CTA's share of the work: where it begins, and the unit behind its last one
    long long end;
    KvShares shares;
    KvPiece open[2];                   // segments that other CTAs hold parts of: begun before this CTA, in it
    u64 raw_full[kTileRaw], raw_empty[kTileRaw];
    u64 k_full[kTileKeys], k_empty[kTileKeys], v_full[kTileValues], v_empty[kTileValues];
    u64 m_full[kTileMeta], m_empty[kTileMeta];
    u64 q_full[2], s_full[2][2], p_full[2][2], o_done[2], x_full, x_empty, r_full, drain[2];
    unsigned int tmem;
    int abort_flag, last[2];
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
// fp32 result, fp16 operands, both K-major, M = 128
__host__ __device__ constexpr unsigned int tc_idesc(int n) { return (1u << 4) | ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24); }
// Rows of 128 bytes in the 128-byte swizzle, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ u64 tc_desc(unsigned int addr) {
    return (u64)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Columns of a warp's 32 lanes; the values have arrived when the statement is done.
__device__ __forceinline__ void tc_load32(unsigned int addr, float (&x)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_load64(unsigned int addr, float (&x)[64]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31]), "=f"(x[32]), "=f"(x[33]), "=f"(x[34]), "=f"(x[35]), "=f"(x[36]), "=f"(x[37]), "=f"(x[38]), "=f"(x[39]), "=f"(x[40]), "=f"(x[41]), "=f"(x[42]), "=f"(x[43]), "=f"(x[44]), "=f"(x[45]), "=f"(x[46]), "=f"(x[47]), "=f"(x[48]), "=f"(x[49]), "=f"(x[50]), "=f"(x[51]), "=f"(x[52]), "=f"(x[53]), "=f"(x[54]), "=f"(x[55]), "=f"(x[56]), "=f"(x[57]), "=f"(x[58]), "=f"(x[59]), "=f"(x[60]), "=f"(x[61]), "=f"(x[62]), "=f"(x[63])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_store8(unsigned int addr, unsigned int x0, unsigned int x1, unsigned int x2, unsigned int x3, unsigned int x4,
                                          unsigned int x5, unsigned int x6, unsigned int x7) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(x0), "r"(x1), "r"(x2), "r"(x3), "r"(x4),
                 "r"(x5), "r"(x6), "r"(x7)
                 : "memory");
}
__device__ __forceinline__ void tc_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ __half2 as_half2(unsigned int x) { return *reinterpret_cast<const __half2*>(&x); }
// Values of two codes of a word (those in bits 0-3 and 16-19, or 4-7 and 20-23).
template <bool HIGH>
__device__ __forceinline__ unsigned int expand(unsigned int w, __half2 scale, __half2 minimum) {
    const unsigned int b = (w & (HIGH ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;     // 1024 + c, or 1024 + 16 c
    const __half2 c = HIGH ? __hfma2(as_half2(b), __float2half2_rn(0.0625f), __float2half2_rn(-64.f)) : __hsub2(as_half2(b), __float2half2_rn(1024.f));
    const __half2 v = __hfma2(c, scale, minimum);
    return *reinterpret_cast<const unsigned int*>(&v);
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }   // the eight softmax warps
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- the kernel ---------------------------------------------------------------------------------------

template <int D, bool PAIR>
__global__ void __launch_bounds__(kTileThreads, 1) kv_attend_tile_kernel(const KvAttendArgs a) {
    using Shared = KvTileShared<D, PAIR>;
    constexpr int R = Shared::R, H = D / 2;
    constexpr unsigned int kColS = 0, kColO = 256, kStep = 128;    // first columns of group 0's S and O; group 1's are kStep behind
    constexpr unsigned int kIdescS = tc_idesc(kPage), kIdescO = tc_idesc(D);
    extern __shared__ unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < kTileRaw; ++i) {
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], 4);
        }
        for (int i = 0; i < kTileKeys; ++i) {
            mbar_init(&sh.k_full[i], 4);
            mbar_init(&sh.k_empty[i], PAIR ? 2 : 1);
        }
        for (int i = 0; i < kTileValues; ++i) {
            mbar_init(&sh.v_full[i], 4);
            mbar_init(&sh.v_empty[i], PAIR ? 2 : 1);
        }
        for (int i = 0; i < kTileMeta; ++i) {
            mbar_init(&sh.m_full[i], 4);
            mbar_init(&sh.m_empty[i], PAIR ? 8 : 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_full[i], 4);
            for (int b = 0; b < 2; ++b) {
                mbar_init(&sh.s_full[i][b], 1);
                mbar_init(&sh.p_full[i][b], 4);
            }
            mbar_init(&sh.o_done[i], 1);
            mbar_init(&sh.drain[i], 1);
            sh.open[i].seg = -1;
        }
        mbar_init(&sh.x_full, 4);
        mbar_init(&sh.x_empty, 4);
        mbar_init(&sh.r_full, 4);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tc_alloc(&sh.tmem, 512);
    pdl_wait();
    const int B = a.p.n_seqs, G = a.p.n_q_heads / a.p.n_kv_heads;
    const int strip = (B + kTileThreads - 1) / kTileThreads;
    long long mine = 0;
    for (int b = tid * strip; b < min(B, (tid + 1) * strip); ++b) {
        const KvSeq s = kv_load_seq(a, b, R);
        mine += kv_tile_head_units(a, s, R, G) * a.p.n_kv_heads;
        if (s.fresh > 0 && (long long)s.cached + s.fresh > (long long)a.p.max_pages * kPage) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    tc_fence_before();
    long long total;
    sh.base[tid] = block_scan<kTileThreads>(mine, sh.scan, total);
    __syncthreads();
    tc_fence_after();
    const unsigned int tm = sh.tmem;
    volatile int* abort_flag = &sh.abort_flag;
    const long long c = blockIdx.x;
    const bool works = c < total;
    if (tid == 0) {
        const KvShares shares(total, works ? min((long long)gridDim.x, total) : 1);
        KvTileWalk start{};
        long long u1 = 0;
        if (works) {
            const long long u0 = shares.first(c);
            u1 = shares.first(c + 1);
            int lo = 0, hi = (B + strip - 1) / strip;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh.base[mid] <= u0) lo = mid;
                else hi = mid;
            }
            long long rem = u0 - sh.base[lo];
            int b = lo * strip;
            KvSeq s = kv_load_seq(a, b, R);
            long long per_head = kv_tile_head_units(a, s, R, G);
            while (rem >= per_head * a.p.n_kv_heads) {
                rem -= per_head * a.p.n_kv_heads;
                s = kv_load_seq(a, ++b, R);
                per_head = kv_tile_head_units(a, s, R, G);
            }
            start.b = b;
            start.take(s);
            start.h = (int)(rem / per_head);
            rem -= start.h * per_head;
            start.pages = start.tile_pages(a, R, G);
            if (a.node_parent != nullptr) {
                start.tile = (int)(rem / (s.pages + kTileSegCost));
                rem -= (long long)start.tile * (s.pages + kTileSegCost);
            } else {
                while (rem >= start.pages + kTileSegCost) {
                    rem -= start.pages + kTileSegCost;
                    ++start.tile;
                    start.pages = start.tile_pages(a, R, G);
                }
            }
            const int lead = rem < kTileSegCost ? kTileSegCost - (int)rem : 0;
            start.pg = lead > 0 ? 0 : (int)rem - kTileSegCost;
            start.left = (int)min(u1 - u0, (long long)0x7FFFFFFF) - lead;
        }
        sh.start = start;
        sh.end = u1;
        sh.shares = shares;
    }
    __syncthreads();
    const auto wait_one = [&](u64* bar, unsigned int parity) {
        if (mbar_wait(bar, parity, abort_flag, kWaitLimit)) return true;
        give_up(abort_flag, a.state);
        return false;
    };
    // (the lanes of a warp go on, or give up, together)
    const auto wait = [&](u64* bar, unsigned int parity) { return __all_sync(0xFFFFFFFFu, wait_one(bar, parity)) != 0; };

    if (warp >= 12) {
        fewer_registers<kTileOtherRegs>();
        if (warp == 13) {
            // ---- loader
            int n = 0;
            bool ok = true;
            for (KvTileWalk w = sh.start; ok && w.live(); w.next(a, R, G)) {
                const int np = w.piece_pages();
                const int32_t* table = a.block_table + (long long)w.b * a.p.max_pages;
                int ids = 0;
                for (int i = 0; i < np; ++i, ++n) {
                    if ((i & 31) == 0) ids = i + lane < np ? table[w.pg + i + lane] : -1;
                    const int page = __shfl_sync(0xFFFFFFFFu, ids, i & 31);
                    const int slot = n % kTileRaw;
                    ok = wait(&sh.raw_empty[slot], ((n / kTileRaw) & 1) ^ 1);
                    if (!ok) break;
                    if (lane == 0) {
                        const bool there = page >= 0 && page < a.p.n_pages;
                        sh.raw_missing[slot] = !there;
                        if (there) {
                            mbar_arrive_expect_tx(&sh.raw_full[slot], kv_head_bytes(D));
                            bulk_copy_g2s(sh.raw[slot], a.pages + ((long long)page * a.p.n_kv_heads + w.h) * kv_head_bytes(D), kv_head_bytes(D),
                                          &sh.raw_full[slot]);
                        } else {
                            raise(a.state, AASD_STATUS_BAD_OFFSETS);
                            mbar_arrive(&sh.raw_full[slot]);
                        }
                    }
                    __syncwarp();
                }
            }
            if (*abort_flag)   // nothing may be on its way into this CTA's shared memory when it leaves
                for (int k = max(0, n - kTileRaw); k < n; ++k)
                    for (unsigned int it = 0; it < kWaitLimit && !mbar_try_wait(&sh.raw_full[k % kTileRaw], (k / kTileRaw) & 1); ++it) {}
        } else if (warp == 12 || warp == 14) {
            // ---- issuers: warp 12 for group 0, warp 14 for group 1
            if (lane == 0) {
                const int x = (warp - 12) >> 1;
                // The group's pages: all of a piece, or every other page of the share.
                struct Pages {
                    KvTileWalk w;
                    int np, i, n, j, piece;   // pages of the piece, page in it, page of the share, of the group, piece of the share
                    bool first;               // of the group in this piece
                };
                auto skip = [&](Pages& p) {   // one page on, into the next piece if need be
                    ++p.n;
                    if (++p.i == p.np) {
                        p.i = 0;
                        ++p.piece;
                        p.first = true;
                        p.w.next(a, R, G);
                        if (p.w.live()) p.np = p.w.piece_pages();
                    }
                };
                auto begin = [&]() {
                    Pages p{sh.start, sh.start.piece_pages(), 0, 0, 0, 0, true};
                    if (!PAIR && x == 1 && p.w.live()) skip(p);
                    return p;
                };
                auto step = [&](Pages& p) {
                    p.first = false;
                    ++p.j;
                    skip(p);
                    if (!PAIR && p.w.live()) skip(p);
                };
                bool ok = true;
                int asked = 0;           // pieces whose queries have been waited for
                auto multiply_keys = [&](Pages& p) {
                    const int slot = p.n % kTileKeys, buf = p.j & 1;
                    while (ok && asked <= p.piece) {
                        ok = wait_one(&sh.q_full[x], asked & 1);
                        ++asked;
                    }
                    ok = ok && wait_one(&sh.k_full[slot], (p.n / kTileKeys) & 1);
                    if (!ok) return;
                    tc_fence_after();
                    const u64 q = tc_desc(smem_u32(sh.queries[PAIR ? x : 0])), k = tc_desc(smem_u32(sh.keys[slot]));
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)   // (descriptors count 16 bytes; a panel is 64 channels of all rows)
                        tc_mma_ss(tm + kColS + x * kStep + buf * 64, q + (ks / 4) * (kTileRows * 8) + (ks % 4) * 2,
                                  k + (ks / 4) * (kPage * 8) + (ks % 4) * 2, kIdescS, ks > 0);
                    tc_commit(&sh.s_full[x][buf]);
                    tc_commit(&sh.k_empty[slot]);
                    step(p);
                };
                Pages keys = begin(), vals = begin();
                while (ok && vals.w.live()) {
                    // (not into the next piece: its queries come when this one's last page is in O)
                    while (ok && keys.w.live() && keys.piece == vals.piece && keys.j < vals.j + 2) multiply_keys(keys);
                    const int slot = vals.n % kTileValues, buf = vals.j & 1;
                    ok = ok && wait_one(&sh.v_full[slot], (vals.n / kTileValues) & 1) && wait_one(&sh.p_full[x][buf], (vals.j >> 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const u64 v = tc_desc(smem_u32(sh.values[slot]));
#pragma unroll
                    for (int ks = 0; ks < kPage / 16; ++ks)
                        tc_mma(tm + kColO + x * kStep, tm + kColS + x * kStep + buf * 64 + ks * 8, v + ks * 2, kIdescO, !vals.first || ks > 0);
                    tc_commit(&sh.v_empty[slot]);
                    tc_commit(&sh.o_done[x]);
                    step(vals);
                }
                // products in flight read this CTA's shared memory
                tc_commit(&sh.drain[x]);
                for (unsigned int it = 0; it < kWaitLimit && !mbar_try_wait(&sh.drain[x], 0); ++it) {}
            }
            __syncwarp();
        }
    } else if (warp >= 8) {
        // ---- unpackers
        fewer_registers<kTileOtherRegs>();
        const int u = tid - 256, uw = warp - 8;
        int n = 0;
        bool ok = true;
        for (KvTileWalk w = sh.start; ok && w.live(); w.next(a, R, G)) {
            const int np = w.piece_pages();
            int ev = 64;
            for (int i = 0; i < np; ++i, ++n) {
                const int slot = n % kTileRaw, mslot = n % kTileMeta, kslot = n % kTileKeys, vslot = n % kTileValues;
                ok = wait(&sh.raw_full[slot], (n / kTileRaw) & 1) && wait(&sh.m_empty[mslot], ((n / kTileMeta) & 1) ^ 1) &&
                     wait(&sh.k_empty[kslot], ((n / kTileKeys) & 1) ^ 1);
                if (!ok) break;
                const unsigned char* raw = sh.raw[slot];
                const bool missing = sh.raw_missing[slot] != 0;
                const int left = missing ? 0 : w.cached + w.fresh - (w.pg + i) * kPage;   // places in use
                // largest value of the page (every warp for itself): codes run from the minimum to 15 scales above it
                const uint2 vm = *reinterpret_cast<const uint2*>(raw + kv_value_meta_offset(D) + 8 * lane);
                auto reach = [](unsigned int m) { return fmaxf(fabsf(meta_min(m)), fabsf(fmaf(15.f, meta_scale(m), meta_min(m)))); };
                float vt = 2 * lane < left ? reach(vm.x) : 0.f;
                if (2 * lane + 1 < left) vt = fmaxf(vt, reach(vm.y));
                // (an exponent field, held to a range in which the factors below are normal numbers)
                ev = max(ev, min(250, (int)(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(vt)) >> 23)));
                if (u < kPage) {
                    const unsigned int km = u < left ? *reinterpret_cast<const unsigned int*>(raw + kv_key_meta_offset(D) + 4 * u) : 0u;
                    float* kq = reinterpret_cast<float*>(&sh.kmeta[mslot][u >> 1]);
                    kq[u & 1] = meta_scale(km);
                    kq[2 + (u & 1)] = meta_min(km);
                    if (u == 0) sh.ev[mslot] = missing ? -1 : ev;
                }
                {
                    // keys: half a token's row per thread.  Word k of a token (channels 4k .. of each half) becomes
                    // 16-byte piece k of its row; the two threads of a token take their pieces in orders that keep
                    // eight neighbouring threads on eight different pieces.
                    constexpr int NW = H / 8;                       // words per thread: a token's H / 4, halved
                    const int t = u >> 1, part = u & 1;
                    const unsigned char* from = raw + t * H + part * (H / 2);
                    unsigned int wd[NW];
#pragma unroll
                    for (int k = 0; k < NW; k += 4) {
                        const uint4 q = lds16(from + 4 * k);
                        wd[k] = q.x; wd[k + 1] = q.y; wd[k + 2] = q.z; wd[k + 3] = q.w;
                    }
                    unsigned char* to = sh.keys[kslot] + t * 128;
#pragma unroll
                    for (int k = 0; k < NW; ++k) {
                        const int kk = NW == 8 ? k ^ (part * 4) : k;
                        const unsigned int x = NW == 8 ? (part ? wd[k ^ 4] : wd[k]) : wd[k], y = x >> 8;
                        const int piece = part * NW + kk;        // of the token's H / 4
                        *reinterpret_cast<uint4*>(to + (piece >> 3) * (kPage * 128) + (((piece & 7) ^ (t & 7)) << 4)) =
                            make_uint4(x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u);
                    }
                }
                // the values' table: lane q < 16 has tokens 4q .. 4q + 3, in the order in which their codes leave a word
                const float norm = pow2f(127 - ev);
                if (lane < kPage / 4) {
                    const uint4 m = lds16(raw + kv_value_meta_offset(D) + 16 * lane);
                    const unsigned int m0 = 4 * lane < left ? m.x : 0u, m1 = 4 * lane + 1 < left ? m.y : 0u, m2 = 4 * lane + 2 < left ? m.z : 0u,
                                       m3 = 4 * lane + 3 < left ? m.w : 0u;
                    sh.vmeta[uw][lane] = make_uint4(pack_half(meta_scale(m0) * norm, meta_scale(m2) * norm), pack_half(meta_scale(m1) * norm, meta_scale(m3) * norm),
                                                    pack_half(meta_min(m0) * norm, meta_min(m2) * norm), pack_half(meta_min(m1) * norm, meta_min(m3) * norm));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.k_full[kslot]);
                    mbar_arrive(&sh.m_full[mslot]);
                }
                // values: rows of channels; 8 tokens of a channel are a 16-byte piece
                ok = wait(&sh.v_empty[vslot], ((n / kTileValues) & 1) ^ 1);
                if (!ok) break;
                constexpr int TPR = 128 / H;                 // threads per channel-pair row
                constexpr int NP = 8 / TPR;                  // pieces per thread and half
                const int r = u / TPR, part = u % TPR;
                const unsigned char* from = raw + kv_value_offset(D) + r * kPage + part * (kPage / TPR);
                unsigned int wd[2 * NP];
#pragma unroll
                for (int k = 0; k < 2 * NP; k += 4) {
                    const uint4 q = lds16(from + 4 * k);
                    wd[k] = q.x; wd[k + 1] = q.y; wd[k + 2] = q.z; wd[k + 3] = q.w;
                }
                unsigned char* lo = sh.values[vslot] + r * 128;
                unsigned char* hi = lo + H * 128;            // (H is a multiple of 8: the same swizzle)
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const unsigned int x0 = wd[2 * k], x1 = wd[2 * k + 1], y0 = x0 >> 8, y1 = x1 >> 8;
                    const uint4 q0 = sh.vmeta[uw][2 * (part * NP + k)], q1 = sh.vmeta[uw][2 * (part * NP + k) + 1];
                    const __half2 s0 = as_half2(q0.x), s1 = as_half2(q0.y), m0 = as_half2(q0.z), m1 = as_half2(q0.w);
                    const __half2 s2 = as_half2(q1.x), s3 = as_half2(q1.y), m2 = as_half2(q1.z), m3 = as_half2(q1.w);
                    const int at = ((part * NP + k) ^ (r & 7)) << 4;
                    *reinterpret_cast<uint4*>(lo + at) =
                        make_uint4(expand<false>(x0, s0, m0), expand<false>(y0, s1, m1), expand<false>(x1, s2, m2), expand<false>(y1, s3, m3));
                    *reinterpret_cast<uint4*>(hi + at) =
                        make_uint4(expand<true>(x0, s0, m0), expand<true>(y0, s1, m1), expand<true>(x1, s2, m2), expand<true>(y1, s3, m3));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.v_full[vslot]);
                    mbar_arrive(&sh.raw_empty[slot]);
                }
            }
        }
    } else {
        // ---- softmax: thread = row
        more_registers<kTileSoftmaxRegs>();
        const int x = warp >> 2, row_in = tid & 127;
        const unsigned int lanes = (unsigned int)(warp & 3) << 21;         // the warp's lanes in an address: 32 (warp % 4) << 16
        const unsigned int col_s = tm + kColS + x * kStep + lanes, col_o = tm + kColO + x * kStep + lanes;
        int n0 = 0, taken = 0, added = 0, pieces = 0;    // pages before the piece; pages taken; pages known to be in O; pieces done
        bool ok = true;
        for (KvTileWalk w = sh.start; ok && w.live(); w.next(a, R, G)) {
            const int np = w.piece_pages();
            const int row = w.tile * R + (PAIR ? x * kTileRows : 0) + row_in;
            const bool valid = row < w.fresh * G;
            const int tok = valid ? row / G : 0;
            const long long head = ((long long)w.first + tok) * a.p.n_q_heads + w.h * G + (valid ? row - tok * G : 0);
            float rfac = 1.f, qfac = 0.f;  // exponent (base 2) of a product = rfac * (scale * S + minimum * qfac)
            if (PAIR || x == 0) {
                // the row's queries as fp16 numbers, its largest element 2^14 .. 2^15, channels in the order of the keys' words
                const long long q0 = ((long long)w.first + tok) * a.p.q_stride + (head - ((long long)w.first + tok) * a.p.n_q_heads) * D;
                float top = 0.f, sum = 0.f;
#pragma unroll 4
                for (int k = 0; k < D; k += 8) {
                    float y[8];
                    if (a.q_vec) load8<AASD_BF16, true>(a.q, q0 + k, y);
                    else load8<AASD_BF16, false>(a.q, q0 + k, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        top = fmaxf(top, fabsf(y[e]));
                        sum += y[e];
                    }
                }
                int e = (int)(__float_as_uint(top) >> 23) - 127;
                e = e < -100 ? -100 : e > 100 ? 100 : e;
                const float up = valid ? pow2f(14 - e) : 0.f;
                rfac = fmaxf(a.scale_log2 * pow2f(e + 10), 1e-37f);   // (never 0: what is hidden is -inf times it)
                qfac = valid ? sum * pow2f(-10 - e) : 0.f;
                unsigned char* to = sh.queries[PAIR ? x : 0] + row_in * 128;
#pragma unroll 4
                for (int cb = 0; cb < H; cb += 8) {       // eight channels of each half are two 16-byte pieces
                    float lo[8], hi[8];
                    if (a.q_vec) {
                        load8<AASD_BF16, true>(a.q, q0 + cb, lo);
                        load8<AASD_BF16, true>(a.q, q0 + H + cb, hi);
                    } else {
                        load8<AASD_BF16, false>(a.q, q0 + cb, lo);
                        load8<AASD_BF16, false>(a.q, q0 + H + cb, hi);
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        lo[q] = valid ? lo[q] * up : 0.f;
                        hi[q] = valid ? hi[q] * (up * 0.0625f) : 0.f;
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int piece = cb / 4 + q;
                        *reinterpret_cast<uint4*>(to + (piece >> 3) * (kTileRows * 128) + (((piece & 7) ^ (row_in & 7)) << 4)) =
                            make_uint4(pack_half(lo[4 * q], lo[4 * q + 2]), pack_half(lo[4 * q + 1], lo[4 * q + 3]), pack_half(hi[4 * q], hi[4 * q + 2]),
                                       pack_half(hi[4 * q + 1], hi[4 * q + 3]));
                    }
                }
                fence_async_smem();
                if (!PAIR) {
                    sh.exchange_up[row_in] = rfac;
                    sh.exchange_m[row_in] = qfac;
                }
            }
            if (!PAIR) {
                // one set of queries for both groups
                if (x == 0) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.r_full);
                } else {
                    ok = wait(&sh.r_full, pieces & 1);
                    if (!ok) break;
                    rfac = sh.exchange_up[row_in];
                    qfac = sh.exchange_m[row_in];
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.q_full[x]);
            float mref = kKvNothing, l = 0.f;
            int ev = 64;
            bool first = true;
            float s[64];
            for (int i = PAIR ? 0 : (n0 ^ x) & 1; i < np; i += PAIR ? 1 : 2) {
                const int n = n0 + i, mslot = n % kTileMeta, pg = w.pg + i, buf = taken & 1;
                const unsigned int col = col_s + buf * 64;
                ok = wait(&sh.m_full[mslot], (n / kTileMeta) & 1) && wait(&sh.s_full[x][buf], (taken >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                tc_load64(col, s);
                const int evn = sh.ev[mslot];
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const float4 m = sh.kmeta[mslot][k];
                    const float2 y = __ffma2_rn(make_float2(m.z, m.w), make_float2(qfac, qfac),
                                                __fmul2_rn(make_float2(s[2 * k], s[2 * k + 1]), make_float2(m.x, m.y)));
                    s[2 * k] = y.x;
                    s[2 * k + 1] = y.y;
                }
                if (evn < 0 || (pg + 1) * kPage > w.cached) {   // what the row does not see becomes -inf
                    const u64 seen = evn < 0 || !valid ? 0ull : kv_seen(a, w.cached, w.fresh, w.first, pg, tok);
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (!((seen >> k) & 1ull)) s[k] = -CUDART_INF_F;
                }
                float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
                for (int k = 4; k < 64; k += 4) {
                    m0 = fmaxf(m0, s[k]);
                    m1 = fmaxf(m1, s[k + 1]);
                    m2 = fmaxf(m2, s[k + 2]);
                    m3 = fmaxf(m3, s[k + 3]);
                }
                const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * rfac;
                // (the page before is in O: the issuer's products of it ran during the steps above)
                if (added < taken) {
                    ok = wait(&sh.o_done[x], added & 1);
                    ++added;
                    if (!ok) break;
                }
                const int en = max(ev, evn);
                if (__any_sync(0xFFFFFFFFu, top > mref + kTileLazy || en > ev)) {
                    const float mn = fmaxf(mref, top);
                    const float f = ex2_approx(mref - mn);
                    mref = mn;
                    l *= f;
                    if (!first) {
                        tc_fence_after();
                        const float fo = en - ev > 126 ? 0.f : f * pow2f(ev - en);
#pragma unroll
                        for (int cb = 0; cb < D; cb += 32) {
                            float o[32];
                            tc_load32(col_o + cb, o);
#pragma unroll
                            for (int k = 0; k < 32; k += 8)
                                tc_store8(col_o + cb + k, __float_as_uint(o[k] * fo), __float_as_uint(o[k + 1] * fo), __float_as_uint(o[k + 2] * fo),
                                          __float_as_uint(o[k + 3] * fo), __float_as_uint(o[k + 4] * fo), __float_as_uint(o[k + 5] * fo),
                                          __float_as_uint(o[k + 6] * fo), __float_as_uint(o[k + 7] * fo));
                        }
                    }
                    ev = en;
                }
                first = false;
                // probabilities, to 32 columns in the order of the values' words
                const float2 ff = make_float2(rfac, rfac), mm = make_float2(kTileP - mref, kTileP - mref);
                float2 l0 = make_float2(0.f, 0.f), l1 = make_float2(0.f, 0.f);
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) {             // sixteen tokens are eight columns
                    unsigned int pk[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int t = 16 * kb + 4 * k;
                        float2 p = __ffma2_rn(make_float2(s[t], s[t + 1]), ff, mm), q = __ffma2_rn(make_float2(s[t + 2], s[t + 3]), ff, mm);
                        p = make_float2(ex2_approx(p.x), ex2_approx(p.y));
                        q = make_float2(ex2_approx(q.x), ex2_approx(q.y));
                        l0 = __fadd2_rn(l0, p);
                        l1 = __fadd2_rn(l1, q);
                        pk[2 * k] = pack_half(p.x, q.x);
                        pk[2 * k + 1] = pack_half(p.y, q.y);
                    }
                    tc_store8(col + 8 * kb, pk[0], pk[1], pk[2], pk[3], pk[4], pk[5], pk[6], pk[7]);
                }
                l += (l0.x + l0.y) + (l1.x + l1.y);
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
                ok = wait(&sh.o_done[x], added & 1);
                ++added;
                if (!ok) break;
                tc_fence_after();
            }
            float unscale = pow2f(ev - 127);
            mref -= kTileP;                // (l and O carry the probabilities' power of two)
            const bool complete = w.pg == 0 && np == w.pages;
            const int which = w.pg > 0 ? 0 : 1;
            const int rows = min(R, w.fresh * G - w.tile * R);
            constexpr int kPart = R * D + 2 * R;
            const int r = (PAIR ? x * kTileRows : 0) + row_in;
            float* part = a.cta_parts + (c * 2 + which) * kPart;
            float other = 0.f;             // factor of the other group's O
            if (!PAIR) {
                // group 0 reads both groups' O (the same lanes of tensor memory)
                if (x == 1) {
                    sh.exchange_m[row_in] = mref;
                    sh.exchange_l[row_in] = l;
                    sh.exchange_up[row_in] = any ? unscale : 0.f;
                    __syncwarp();
                    tc_fence_before();
                    if (lane == 0) mbar_arrive(&sh.x_full);
                    ok = wait(&sh.x_empty, pieces & 1);
                    if (!ok) break;
                } else {
                    ok = wait(&sh.x_full, pieces & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const float om = sh.exchange_m[row_in], mn = fmaxf(mref, om), of = ex2_approx(om - mn), own = ex2_approx(mref - mn);
                    l = l * own + sh.exchange_l[row_in] * of;
                    unscale *= own;
                    other = sh.exchange_up[row_in] * of;
                    mref = mn;
                }
            }
            if (PAIR || x == 0) {
                const bool any1 = !PAIR && __any_sync(0xFFFFFFFFu, sh.exchange_up[row_in] != 0.f);   // (the same for every row)
                const float inv = complete ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
#pragma unroll
                for (int cb = 0; cb < D; cb += 32) {
                    float o[32];
                    if (any) {
                        tc_load32(col_o + cb, o);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] *= unscale;
                    if (!PAIR && any1) {
                        float y[32];
                        tc_load32(col_o + kStep + cb, y);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = fmaf(y[k], other, o[k]);
                    }
                    if (r < rows) {
                        if (complete) {
#pragma unroll
                            for (int k = 0; k < 32; k += 8) {
                                float y[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q) y[q] = o[k + q] * inv;
                                if (a.out_vec) store8<AASD_BF16, true>(a.o.out, head * D + cb + k, y);
                                else store8<AASD_BF16, false>(a.o.out, head * D + cb + k, y);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(part + r * D + cb + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                        }
                    }
                }
                if (r < rows) {
                    if (complete) {
                        if (a.o.lse != nullptr) a.o.lse[head] = l > 0.f ? (mref + log2f(l)) * (float)kLn2 : -CUDART_INF_F;
                    } else {
                        part[R * D + r] = mref;
                        part[R * D + R + r] = l;
                    }
                }
                if (!complete && tid == 0) sh.open[which] = KvPiece{sh.end - w.left - w.pg, w.pages, w.h, w.tile * R, rows, w.first};
            }
            if (!PAIR && x == 0) {   // group 1 may go on
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.x_empty);
            }
            ++pieces;
            tc_fence_before();
            n0 += np;
        }
        softmax_sync();
        if (works && !*abort_flag && (sh.open[0].seg >= 0 || sh.open[1].seg >= 0)) {
            // the last CTA that delivers a part of a segment joins them all
            if (tid < 2) {
                int last = 0;
                if (sh.open[tid].seg >= 0) {
                    const KvPiece pc = sh.open[tid];
                    const long long c0 = sh.shares.owner(pc.seg), c1 = sh.shares.owner(pc.seg + pc.pages - 1);
                    last = take_ticket(a.tickets + c0) == (unsigned int)(c1 - c0);
                    if (last) a.tickets[c0] = 0;
                }
                sh.last[tid] = last;
            }
            softmax_sync();
            constexpr int kPart = R * D + 2 * R;
            constexpr int RB = 8;             // rows that a warp has under way together
#pragma unroll 1
            for (int which = 0; which < 2; ++which) {
                if (!sh.last[which]) continue;
                const KvPiece pc = sh.open[which];
                const long long c0 = sh.shares.owner(pc.seg);
                const int parts = (int)(sh.shares.owner(pc.seg + pc.pages - 1) - c0) + 1;
                const float* base = a.cta_parts + c0 * 2 * kPart;   // part k: 2 k, the first one's 1
                for (int r0 = warp * RB; r0 < pc.n; r0 += 8 * RB) {
                    float M[RB], L[RB];
                    float4 o[RB];
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        M[i] = kKvNothing;
                        L[i] = 0.f;
                        o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    const int ch = lane * 4;
                    for (int k = 0; k < parts; ++k) {
                        const float* from = base + (2 * k + (k == 0)) * kPart;
                        float4 y[RB];
                        float m[RB], ll[RB];
#pragma unroll
                        for (int i = 0; i < RB; ++i) {
                            const int r = min(r0 + i, pc.n - 1);
                            m[i] = __ldcg(from + R * D + r);
                            ll[i] = __ldcg(from + R * D + R + r);
                            y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (ch < D) y[i] = __ldcg(reinterpret_cast<const float4*>(from + r * D + ch));
                        }
#pragma unroll
                        for (int i = 0; i < RB; ++i) {
                            const float mn = fmaxf(M[i], m[i]), f0 = ex2_approx(M[i] - mn), f1 = ex2_approx(m[i] - mn);
                            M[i] = mn;
                            L[i] = fmaf(L[i], f0, ll[i] * f1);
                            o[i].x = fmaf(o[i].x, f0, y[i].x * f1);
                            o[i].y = fmaf(o[i].y, f0, y[i].y * f1);
                            o[i].z = fmaf(o[i].z, f0, y[i].z * f1);
                            o[i].w = fmaf(o[i].w, f0, y[i].w * f1);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        const int r = r0 + i;
                        if (r >= pc.n || ch >= D) continue;
                        const float inv = L[i] > 0.f ? 1.f / L[i] : 0.f;
                        const int row = pc.row0 + r;
                        const long long head = ((long long)pc.first + row / G) * a.p.n_q_heads + pc.h * G + row % G;
                        store4<AASD_BF16>(a.o.out, head * D + ch, make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), a.out_vec);
                        if (a.o.lse != nullptr && ch == 0) a.o.lse[head] = L[i] > 0.f ? (M[i] + log2f(L[i])) * (float)kLn2 : -CUDART_INF_F;
                    }
                }
            }
        }
        kv_clear_rows<AASD_BF16>(a, D, (int)(blockIdx.x * 8 + warp), (int)(gridDim.x * 8));
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tc_free(tm, 512);
}

}  // namespace aasd
