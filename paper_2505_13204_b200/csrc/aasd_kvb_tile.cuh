// Attention over the paged 8-bit cache for many rows per key/value head (draft trees, chunks of a prompt): tiles of 128
// rows on the fifth-generation tensor cores.
//
// One persistent CTA per SM takes its share of the list of work as in the 4-bit kernel (aasd_kv_tile.cuh: walker, pieces, joining).
// Its warps have roles:
//   walker, loader   as there; the loader brings a page's codes in as they lie, and its scales apart;
//   unpackers        (4 warps) turn the values' codes into fp16 numbers, token by token: an operand whose rows run along K;
//   two issuers      a warp each: tcgen05.mma of S = Q K^T (e4m3, the keys as they came, both operands in shared memory)
//                    and O += P V (fp16, P in tensor memory) for one softmax group, a page at a time;
//   softmax          two groups of 8 warps, 16 rows each: S to registers, probabilities back as P.
// The two groups work on two row tiles of the same pages (PAIR), or, where a segment has no more than 128 rows, on
// alternate pages of one tile, joined at the end.  With 256 channels there is one group.  A group has two S buffers, so that the next page's products are there
// when it is done with one.
//
// A bf16 query is two e4m3 numbers (eight bits), multiplied one after the other.  A page's scale of the keys is a factor of S that
// all its columns share; that of its values goes into the exponents of the probabilities, relative to the largest
// of the pages so far, which O is relative to.
//
// Tensor memory (512 columns): two S buffers of each group, whose first halves P takes over, and O; with 256 channels the queries.
//
// A page and group of 128 rows cost 384 cycles of S products (64 columns from shared memory, twice) and 256 of PV, 1259 for both
// groups with the shared memory that they contend for; two issuers, unpackers and loader alone go at 1390 a page.  With
// the softmax warps it is about 2300, and they are what bounds it: 512 cycles of exponentials, 330 until S is in registers, the
// rest scaling, sums, packing and storing of P.  Measured: 2 x 2048 tokens of a prompt (32 over 8 heads of 128, bf16) 175 to 219
// us from GPU to GPU, 627 to 785 TFLOP/s; 32 draft trees of 33 over about 3800 tokens 158 to 162 us; 64 tokens over 65536 98 to 102 us.  Eight warps of 32 rows
// took 236 us for the first (fewer waits, but half as many warps to hide them), exponentials in turns of the two groups 233.
// With 256 channels (16 over 4 heads): the same prompt behind 1000 tokens 200 us, 677 TFLOP/s, 32 trees 151 us, 64 tokens
// over 65536 97 us.  There the queries lie in the tensor memory that is left: from shared memory their reads took 512 cycles a page
// (trees 166 us, 64 tokens 102).  A page takes about 1900 cycles, 1580 of them one softmax warp's from S to P; eight unpackers,
// three or four pages under way instead of two gave nothing.
#pragma once

#include "aasd_kv_tile.cuh"
#include "aasd_kvb_attend.cuh"

namespace aasd {

// What depends on the channels.  256 of them leave room for one group: O takes half of tensor memory, a page 32 KB and its values
// in fp16 as much.
template <int D>
struct KvbTileShape {
    static constexpr int kGroups = D == 256 ? 1 : 2;
    static constexpr int kSoftmax = 8 * kGroups;                           // softmax warps
    static constexpr int kThreads = 32 * (kSoftmax + 8);                   // and 4 unpackers, two issuers (one without work in a single group), loader, walker
    static constexpr int kRaw = D == 256 ? 2 : 5, kValues = D == 256 ? 2 : 4;   // ring depths, in pages
    // Registers per thread: the softmax warps take what the others give up of the launch's (fewer threads have enough).  The compiler
    // knows the launch's only, and spills: 68 bytes stored and 168 loaded (128 channels, one tile), 20 and 68 (two tiles), 56 and 132, 32 and 104
    // (64 channels), 12 and 20 (256).
    static constexpr int kLaunchRegs = D == 256 ? 128 : 80, kSoftmaxRegs = D == 256 ? 128 : 96, kOtherRegs = D == 256 ? 128 : 48;
    static_assert(kSoftmax * kSoftmaxRegs + 8 * kOtherRegs <= (kSoftmax + 8) * kLaunchRegs, "the shares add up to the launch's registers");
};
constexpr int kByteScales = 8;                                             // ring depth of the scales, in pages
// Where a page's scale of the values is this much below the largest (in powers of two), the row's maximum is looked for: fp16's
// range says nothing about probabilities that were scaled down so far.
constexpr int kByteFar = 30;
// The most that probabilities are scaled down by.  With the maximum known they are 2^(kTileP - 40) at most, which fp16 rounds to zero
// as it does everything smaller, so that O loses nothing more; their sum, which is scaled back, keeps weights down to 2^-93.
constexpr int kByteDown = 40;

template <int D, bool PAIR>
struct KvbTileShared {
    using Shape = KvbTileShape<D>;
    static constexpr int kRaw = Shape::kRaw, kValues = Shape::kValues, kThreads = Shape::kThreads;
    static constexpr int R = PAIR ? 2 * kTileRows : kTileRows;
    alignas(1024) unsigned char queries[PAIR ? 2 : 1][kTileRows * D * 2];   // panels of 128 bytes per row, a query's first numbers, then its second ones (D = 64: the halves of one; D = 256: on their way to tensor memory)
    alignas(1024) unsigned char raw[kRaw][2 * kPage * D];
    alignas(1024) unsigned char values[kValues][kPage * D * 2];
    alignas(16) uint4 scale[kByteScales];         // as they lie in the page
    int missing[kByteScales], raw_missing[kRaw];
    float row_q[PAIR ? 2 : 1][kTileRows];         // what the rows' queries were divided by, times the scale of the products
    float exchange_m[kTileRows], exchange_l[kTileRows], exchange_up[kTileRows];   // between the groups, where they share a tile
    int base[kThreads];
    long long scan[kThreads / 32];
    KvTilePiece piece[kTilePieces];
    KvShares shares;
    KvPiece open;                      // the segment that begins in this CTA and ends in another
    u64 piece_full[kTilePieces], piece_empty[kTilePieces];
    u64 raw_full[kRaw], raw_empty[kRaw];
    u64 scale_empty[kByteScales];
    u64 v_full[kValues], v_empty[kValues];
    u64 q_full[2], s_full[2][2], p_full[2][2], o_done[2][2], x_full, x_empty, r_full, drain[2];
    unsigned int tmem;
    int abort_flag, padding;
};

// A place in a ring of N slots, and the parity of its round.
template <int N>
struct KvRing {
    int slot = 0;
    unsigned int round = 0;
    __device__ __forceinline__ void next() {
        if (++slot == N) {
            slot = 0;
            round ^= 1u;
        }
    }
    __device__ __forceinline__ void next(int k) {
        for (; k > 0; --k) next();
    }
};

// The issuers run as whole warps, whose values the compiler can see to be the same in every lane and keep in uniform registers,
// where the tensor-core instructions want them; a lane is elected for each.  Eight products take 118 cycles to
// issue so, and 410 from one thread inside a branch: the roles other than softmax then go at 2125 cycles a page, not 1390.
__device__ __forceinline__ bool elect_one() {
    unsigned int on;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(on));
    return on != 0;
}
// D (fp32, tensor memory) (+)= A B, e4m3 both, in shared memory.  Operands: low and high words of their descriptors.
__device__ __forceinline__ void tc_mma_bytes(unsigned int d, unsigned int a, unsigned int a_high, unsigned int b, unsigned int b_high, unsigned int idesc, bool add) {
    if (elect_one())
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %6, 0;\n\tmov.b64 x, {%1, %2};\n\tmov.b64 y, {%3, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], x, y, %5, p;\n\t}" ::"r"(d),
            "r"(a), "r"(a_high), "r"(b), "r"(b_high), "r"(idesc), "r"(add ? 1u : 0u)
            : "memory");
}
// ... with A in tensor memory, four numbers in a cell
__device__ __forceinline__ void tc_mma_bytes(unsigned int d, unsigned int a, unsigned int b, unsigned int b_high, unsigned int idesc, bool add) {
    if (elect_one())
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 y, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], y, %4, p;\n\t}" ::"r"(d),
            "r"(a), "r"(b), "r"(b_high), "r"(idesc), "r"(add ? 1u : 0u)
            : "memory");
}
// ... A B, fp16 both, A in tensor memory
__device__ __forceinline__ void tc_mma_halves(unsigned int d, unsigned int a, unsigned int b, unsigned int b_high, unsigned int idesc, bool add) {
    if (elect_one())
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 y, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n\t}" ::"r"(d),
            "r"(a), "r"(b), "r"(b_high), "r"(idesc), "r"(add ? 1u : 0u)
            : "memory");
}
__device__ __forceinline__ void tc_commit_one(unsigned int bar) {
    if (elect_one()) asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// (e4m3 is type 0 of its kind, as fp16 is of the other: tc_idesc(n, false) describes both.)
constexpr unsigned int kTcRowsB = 1u << 16;   // the second operand's rows run along K
// Rows of 64 bytes in the 64-byte swizzle, groups of eight rows 512 bytes apart.
__device__ __forceinline__ u64 tc_desc_64(unsigned int addr) {
    return (u64)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (32ull << 32) | (1ull << 46) | (4ull << 61);
}
// An operand whose rows (128 bytes, 64 fp16 numbers, in the 128-byte swizzle) run along K: groups of eight rows 1024 bytes
// apart, panels of 64 numbers kPage rows apart.
__device__ __forceinline__ u64 tc_desc_rows(unsigned int addr) {
    return (u64)((addr & 0x3FFFFu) >> 4) | ((u64)(kPage * 128 / 16) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// 32 columns of 16 lanes: half of what tc_load and tc_store move, in half the registers.
__device__ __forceinline__ void tc_load(unsigned int addr, float (&x)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_store(unsigned int addr, const float (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "f"(x[8]), "f"(x[9]), "f"(x[10]), "f"(x[11]), "f"(x[12]), "f"(x[13]), "f"(x[14]), "f"(x[15]) : "memory");
}
// O of a warp's rows times a factor for each of a thread's two.
template <int D>
__device__ __forceinline__ void kvb_scale_o(unsigned int col_o, const float (&fo)[2]) {
#pragma unroll 1
    for (int cb = 0; cb < D; cb += 32) {
        float o[16];
        tc_load(col_o + cb, o);
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] *= fo[(k >> 1) & 1];
        tc_store(col_o + cb, o);
    }
    tc_wait_store();   // (a page may scale O twice)
}

template <int D, bool PAIR>
__global__ void __launch_bounds__(KvbTileShape<D>::kThreads, 1) kvb_attend_tile_kernel(const KvAttendArgs a) {
    using Shape = KvbTileShape<D>;
    using Shared = KvbTileShared<D, PAIR>;
    static_assert(!PAIR || Shape::kGroups == 2, "a tile for each group");
    constexpr int kByteSoftmax = Shape::kSoftmax, kByteTileThreads = Shape::kThreads, kByteRaw = Shape::kRaw, kByteValues = Shape::kValues;
    constexpr bool ALT = !PAIR && Shape::kGroups == 2;             // the groups take alternate pages
    constexpr int R = Shared::R, STEP = ALT ? 2 : 1;               // pages from one of a group to its next
    constexpr unsigned int kColS = 0, kColQ = 128, kColO = 256, kStep = 128;    // first columns of group 0's S and O; group 1's are kStep behind
    constexpr unsigned int kIdescS = tc_idesc(kPage, false), kIdescO = tc_idesc(D, false) | kTcRowsB;
    extern __shared__ unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
#pragma unroll 1
        for (int i = 0; i < kTilePieces; ++i) {
            mbar_init(&sh.piece_full[i], 1);
            mbar_init(&sh.piece_empty[i], kByteSoftmax + 4 + Shape::kGroups + 1);
        }
#pragma unroll 1
        for (int i = 0; i < kByteRaw; ++i) {
            mbar_init(&sh.raw_full[i], blockIdx.x == 0 && i == a.withhold_page ? 2 : 1);   // (testing aid: the second arrival never comes)
            mbar_init(&sh.raw_empty[i], 4 + (PAIR ? 2 : 1));
        }
#pragma unroll 1
        for (int i = 0; i < kByteScales; ++i) {
            mbar_init(&sh.scale_empty[i], PAIR ? 16 : 8);
        }
#pragma unroll 1
        for (int i = 0; i < kByteValues; ++i) {
            mbar_init(&sh.v_full[i], 4);
            mbar_init(&sh.v_empty[i], PAIR ? 2 : 1);
        }
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_full[i], 8);
            for (int b = 0; b < 2; ++b) {
                mbar_init(&sh.s_full[i][b], 2);    // the products' end, and the issuer's word
                mbar_init(&sh.p_full[i][b], 8);
                mbar_init(&sh.o_done[i][b], 1);
            }
            mbar_init(&sh.drain[i], 1);
        }
        mbar_init(&sh.x_full, 8);
        mbar_init(&sh.x_empty, 8);
        mbar_init(&sh.r_full, 8);
        sh.abort_flag = 0;
        sh.open.seg = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kByteSoftmax + 4) tc_alloc(&sh.tmem, 512);
    pdl_wait();
    const int B = a.p.n_seqs, G = a.p.n_q_heads / a.p.n_kv_heads;
    const int strip = (B + kByteTileThreads - 1) / kByteTileThreads;
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
    sh.base[tid] = (int)block_scan<kByteTileThreads>(mine, sh.scan, sum);
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
    // (The lanes of a warp go on, or give up, together.  What is there already costs one look.)
    const auto together = [](bool on) { return __all_sync(0xFFFFFFFFu, on) != 0; };
    const auto wait = [&](u64* bar, unsigned int parity) { return together(mbar_try_wait(bar, parity)) || together(wait_one(bar, parity)); };
    bool ok = true;

    if (warp >= kByteSoftmax + 4) {
        if (Shape::kOtherRegs < Shape::kLaunchRegs) fewer_registers<Shape::kOtherRegs>();
        if (warp == kByteSoftmax + 7) {
            // ---- walker
            if (lane == 0) ok = kv_tile_walk(a, sh, total, strip, R, G, wait_one);
            __syncwarp();
        } else if (warp == kByteSoftmax + 5) {
            // ---- loader
            KvRing<kByteRaw> raw;
            KvRing<kByteScales> sc;
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
                const uint8_t* head = a.pages + (long long)w.h * kvb_head_bytes(D);
                const u64 stride = (u64)a.p.n_kv_heads * kvb_head_bytes(D);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.piece_empty[k % kTilePieces]);
                int ids = 0;
#pragma unroll 1
                for (int i = 0; i < np; ++i, ++n, raw.next(), sc.next()) {
                    if ((i & 31) == 0) ids = i + lane < np && inside ? table[i + lane] : -1;
                    const int page = __shfl_sync(0xFFFFFFFFu, ids, i & 31);
                    ok = wait(&sh.raw_empty[raw.slot], raw.round ^ 1u) && wait(&sh.scale_empty[sc.slot], sc.round ^ 1u);
                    if (!ok) break;
                    if (lane == 0) {
                        const bool there = page >= 0 && page < a.p.n_pages;
                        sh.raw_missing[raw.slot] = sh.missing[sc.slot] = !there;
                        if (there) {
                            const uint8_t* from = head + (u64)(unsigned int)page * stride;
                            mbar_arrive_expect_tx(&sh.raw_full[raw.slot], 2 * kPage * D + 16);
                            bulk_copy_g2s(sh.raw[raw.slot], from, 2 * kPage * D, &sh.raw_full[raw.slot]);
                            bulk_copy_g2s(&sh.scale[sc.slot], from + kvb_scale_offset(D), 16, &sh.raw_full[raw.slot]);
                        } else {
                            raise(a.state, AASD_STATUS_BAD_OFFSETS);
                            mbar_arrive(&sh.raw_full[raw.slot]);
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
            }
            // nothing may be on its way into this CTA's shared memory when it leaves
#pragma unroll 1
            for (int k = max(0, n - kByteRaw); k < n; ++k)
#pragma unroll 1
                for (unsigned int it = 0; it < a.wait_limit && !mbar_try_wait(&sh.raw_full[k % kByteRaw], (k / kByteRaw) & 1); ++it) {}
        } else if (Shape::kGroups == 2 || warp == kByteSoftmax + 4) {
            // ---- issuers, one for each group
            const int x = __shfl_sync(0xFFFFFFFFu, (warp - kByteSoftmax - 4) >> 1, 0);
            const unsigned int tmem = __shfl_sync(0xFFFFFFFFu, tm, 0) + x * kStep;
            const auto low = [](u64 desc) { return (unsigned int)desc; };
            const auto high = [](u64 desc) { return (unsigned int)(desc >> 32); };
            const unsigned int q0 = low(tc_desc(smem_u32(sh.queries[0]))) + (PAIR ? x * (kTileRows * D * 2 / 16) : 0), q_high = high(tc_desc(0));
            const unsigned int k0 = low(D == 64 ? tc_desc_64(smem_u32(sh.raw[0])) : tc_desc(smem_u32(sh.raw[0]))), k_high = high(D == 64 ? tc_desc_64(0) : tc_desc(0));
            const unsigned int v0 = low(tc_desc_rows(smem_u32(sh.values[0]))), v_high = high(tc_desc_rows(0));
            // A piece's pages of the group: all, or every other page of the share.  The keys' products run up to two
            // pages ahead, but not into the next piece: its queries come when this one's last page is in O.
            KvRing<kByteRaw> raw;
            KvRing<kByteValues> val;
            if (ALT && x == 1) {
                raw.next();
                val.next();
            }
            int n0 = 0, taken = 0;   // pages of the share before the piece; of the group so far
#pragma unroll 1
            for (int k = 0;; ++k) {
                ok = wait(&sh.piece_full[k % kTilePieces], (k / kTilePieces) & 1);
                if (!ok) break;
                const int np = __shfl_sync(0xFFFFFFFFu, sh.piece[k % kTilePieces].np, 0);
                if (np == 0) break;
                if (elect_one()) mbar_arrive(&sh.piece_empty[k % kTilePieces]);
                ok = wait(&sh.q_full[x], k & 1);
                if (!ok) break;
                const int first = ALT ? (n0 ^ x) & 1 : 0;
                int ahead = first, asked = taken;
#pragma unroll 1
                for (int i = first; i < np; i += STEP, ++taken) {
#pragma unroll 1
                    for (; ahead < np && asked < taken + 2; ahead += STEP, ++asked) {
                        const unsigned int buf = asked & 1;
                        ok = wait(&sh.raw_full[raw.slot], raw.round);
                        if (!ok) break;
                        tc_fence_after();
                        const unsigned int keys = k0 + raw.slot * (2 * kPage * D / 16), to = tmem + kColS + buf * 64;
#pragma unroll
                        for (int ks = 0; ks < 2 * (D / 32); ++ks) {   // (the queries' first numbers, then their second ones; descriptors count 16 bytes)
                            const int second = ks / (D / 32), j = ks % (D / 32), panel = j / 4;
                            if (D == 256)
                                tc_mma_bytes(to, tmem + kColQ + ks * 8, keys + panel * (kPage * 8) + (j % 4) * 2, k_high, kIdescS, ks > 0);
                            else
                                tc_mma_bytes(to, q0 + (D == 64 ? second * 4 : (second * (D / 128) + panel) * (kTileRows * 8)) + (j % 4) * 2, q_high,
                                             keys + panel * (kPage * 8) + (j % 4) * 2, k_high, kIdescS, ks > 0);
                        }
                        tc_commit_one(smem_u32(&sh.s_full[x][buf]));
                        tc_commit_one(smem_u32(&sh.raw_empty[raw.slot]));
                        // (the softmax warps look at no other barrier: what came with the page's codes is theirs too)
                        if (elect_one()) mbar_arrive(&sh.s_full[x][buf]);
                        raw.next(STEP);
                    }
                    const unsigned int buf = taken & 1;
                    ok = ok && wait(&sh.v_full[val.slot], val.round) && wait(&sh.p_full[x][buf], (taken >> 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const unsigned int v = v0 + val.slot * (kPage * D * 2 / 16);
#pragma unroll
                    for (int ks = 0; ks < kPage / 16; ++ks)   // (16 rows are 2048 bytes)
                        tc_mma_halves(tmem + kColO, tmem + kColS + buf * 64 + ks * 8, v + ks * 128, v_high, kIdescO, i > first || ks > 0);
                    tc_commit_one(smem_u32(&sh.v_empty[val.slot]));
                    tc_commit_one(smem_u32(&sh.o_done[x][buf]));
                    val.next(STEP);
                }
                if (!ok) break;
                n0 += np;
            }
            // products in flight read this CTA's shared memory
            tc_commit_one(smem_u32(&sh.drain[x]));
#pragma unroll 1
            for (unsigned int it = 0; it < a.wait_limit && !mbar_try_wait(&sh.drain[x], 0); ++it) {}
            __syncwarp();
        }
    } else if (warp >= kByteSoftmax) {
        // ---- unpackers: a lane takes 16 channels of a token at a time, and eight neighbouring lanes write to eight different chunks
        if (Shape::kOtherRegs < Shape::kLaunchRegs) fewer_registers<Shape::kOtherRegs>();
        constexpr int C = D / 16, TS = 128 / C;      // chunks of a token; tokens at a time
        const int u = tid - 32 * kByteSoftmax, chunk = u % C, t0 = u / C;
        // (t % 8 is the same for all of a lane's tokens: one address, 128 TS bytes apart)
        static_assert(TS % 8 == 0, "the swizzle repeats");
        const int from = kvb_value_offset(D) + kvb_chunk_offset(D, t0, chunk);
        const int panel = chunk >> 2, second = panel & 1;   // (neighbouring panels' lanes store their halves in turn)
        const int to0 = panel * (kPage * 128) + t0 * 128 + (((2 * (chunk & 3) + second) ^ (t0 & 7)) << 4);
        const int to1 = panel * (kPage * 128) + t0 * 128 + (((2 * (chunk & 3) + 1 - second) ^ (t0 & 7)) << 4);
        KvRing<kByteRaw> raw;
        KvRing<kByteValues> val;
#pragma unroll 1
        for (int k = 0;; ++k) {
            ok = wait(&sh.piece_full[k % kTilePieces], (k / kTilePieces) & 1);
            if (!ok) break;
            const KvTilePiece& piece = sh.piece[k % kTilePieces];
            const int np = piece.np, end = piece.cached + piece.fresh - piece.pg * kPage;   // places from the first page's on
            __syncwarp();
            if (np == 0) break;
            if (lane == 0) mbar_arrive(&sh.piece_empty[k % kTilePieces]);
#pragma unroll 1
            for (int i = 0; i < np; ++i, raw.next(), val.next()) {
                ok = wait(&sh.raw_full[raw.slot], raw.round) && wait(&sh.v_empty[val.slot], val.round ^ 1u);
                if (!ok) break;
                const unsigned char* src = sh.raw[raw.slot] + from;
                unsigned char* to = sh.values[val.slot];
                const int left = sh.raw_missing[raw.slot] ? 0 : end - i * kPage;   // places in use; others hold anything
                uint4 w[kPage / TS];
#pragma unroll
                for (int m = 0; m < kPage / TS; ++m) w[m] = lds16(src + m * (TS * (D == 64 ? 64 : 128)));
                if (left < kPage) {
#pragma unroll
                    for (int m = 0; m < kPage / TS; ++m)
                        if (t0 + m * TS >= left) w[m] = make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int m = 0; m < kPage / TS; ++m) {
                    const uint4 lo = make_uint4(kvb_halves<false>(w[m].x), kvb_halves<true>(w[m].x), kvb_halves<false>(w[m].y), kvb_halves<true>(w[m].y));
                    const uint4 hi = make_uint4(kvb_halves<false>(w[m].z), kvb_halves<true>(w[m].z), kvb_halves<false>(w[m].w), kvb_halves<true>(w[m].w));
                    *reinterpret_cast<uint4*>(to + to0 + m * (TS * 128)) = second ? hi : lo;
                    *reinterpret_cast<uint4*>(to + to1 + m * (TS * 128)) = second ? lo : hi;
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.v_full[val.slot]);
                    mbar_arrive(&sh.raw_empty[raw.slot]);
                }
            }
            if (!ok) break;
        }
    } else {
        // ---- softmax: thread (g, j) of a warp has rows g and g + 8 of the warp's 16 and two columns of every eight
        if (Shape::kSoftmaxRegs > Shape::kLaunchRegs) more_registers<Shape::kSoftmaxRegs>();
        constexpr int Q = 2;                         // rows of a thread
        // (of the group's 128 rows; a warp reaches the 32 lanes of tensor memory that its number gives it)
        const int x = warp / (8), g = lane >> 2, j = lane & 3, row_base = (warp & 3) * 32 + ((warp >> 2) & 1) * 16;
        const unsigned int lanes = (unsigned int)row_base << 16;
        const unsigned int col_s = tm + kColS + x * kStep + lanes, col_o = tm + kColO + x * kStep + lanes;
        static_assert((kByteScales & (kByteScales - 1)) == 0, "a slot is a page's number, cut off");
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
            const KvTilePiece& w = sh.piece[piece % kTilePieces];   // (given back when its result is out)
            const int np = w.np;
            if (np == 0) break;
            const int row0 = w.tile * R + (PAIR ? x * kTileRows : 0) + row_base;   // of the warp's first row, among the head's
            const int rows_here = AASD_IN_RANGE(w.first + w.fresh <= a.p.n_tokens && w.h < a.p.n_kv_heads, a.state) ? w.fresh * G : 0;   // rows of the head
            // the lane's row: what the warp wants to know of its 16 rows
            const auto own_row = [&]() { return max(min(row0 + (lane & 15), rows_here - 1), 0); };
            constexpr int LR = D / 8, RI = 32 / LR, NL = 4;    // lanes per row, rows per step, steps at a time
            if (PAIR || x == 0) {
                // The rows' queries, each as two e4m3 numbers, the row's largest element between 2^7 and 2^8: eight bits from 2^-2 on,
                // smaller ones are off by 2^-10 at most.  A row that is not finite becomes NaN.
                const int part = lane % LR;                    // eight channels
                const int token = own_row() / G, member = own_row() - token * G;
                const long long at = ((long long)w.first + token) * a.p.q_stride + (long long)(w.h * G + member) * D;   // of the lane's row
                unsigned char* to = sh.queries[PAIR ? x : 0];
#pragma unroll 1
                for (int rb = 0; rb < 16; rb += NL * RI) {
                    Raw8<AASD_BF16, true> raw[NL];
                    // (all on their way before the first is looked at; rows past the last one repeat it, and become zero)
                    if (a.q_vec) {
#pragma unroll
                        for (int k = 0; k < NL; ++k) raw[k].load(a.q, __shfl_sync(0xFFFFFFFFu, at, rb + k * RI + lane / LR) + part * 8);
                    } else {
#pragma unroll 1
                        for (int k = 0; k < NL; ++k) {
                            Raw8<AASD_BF16, false> slow;
                            slow.load(a.q, __shfl_sync(0xFFFFFFFFu, at, rb + k * RI + lane / LR) + part * 8);
#pragma unroll
                            for (int i = 0; i < NL; ++i)
                                if (i == k) raw[i].a = slow.a;
                        }
                    }
                    unsigned int top[NL];
#pragma unroll
                    for (int k = 0; k < NL; ++k) {
                        if (row0 + rb + k * RI + lane / LR >= rows_here) raw[k].clear();
                        float2 y[4];
                        raw[k].unpack(y);
                        top[k] = 0u;
#pragma unroll
                        for (int q = 0; q < 4; ++q)   // (as bits: NaN is above everything)
                            top[k] = max(top[k], max(__float_as_uint(fabsf(y[q].x)), __float_as_uint(fabsf(y[q].y))));
                    }
#pragma unroll
                    for (int o = 1; o < LR; o <<= 1)
#pragma unroll
                        for (int k = 0; k < NL; ++k) top[k] = max(top[k], __shfl_xor_sync(0xFFFFFFFFu, top[k], o));
#pragma unroll
                    for (int k = 0; k < NL; ++k) {
                        const int r = row_base + rb + k * RI + lane / LR;
                        const int e = max(-119, min(127, (int)(top[k] >> 23) - 127));
                        const float up = kvb_pow2(7 - e);
                        float2 y[4];
                        raw[k].unpack(y);
                        unsigned int hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float2 z = make_float2(y[q].x * up, y[q].y * up);
                            const unsigned int h = kvb_codes(z);
                            const float2 v = kvb_values(h);
                            hi[q >> 1] |= h << (16 * (q & 1));
                            lo[q >> 1] |= kvb_codes(make_float2(z.x - v.x, z.y - v.y)) << (16 * (q & 1));
                        }
                        if (top[k] >= 0x7F800000u) hi[0] = hi[1] = 0x7F7F7F7Fu;
                        const int chunk = part >> 1;     // of 16 channels
                        unsigned char* row = to + r * 128 + 8 * (part & 1) + (chunk >> 3) * (kTileRows * 128);
                        const int at16 = ((chunk & 7) ^ (r & 7)) << 4;
                        *reinterpret_cast<uint2*>(row + at16) = make_uint2(hi[0], hi[1]);
                        *reinterpret_cast<uint2*>(row + (D == 64 ? ((chunk + 4) ^ (r & 7)) << 4 : D / 128 * (kTileRows * 128) + at16)) = make_uint2(lo[0], lo[1]);
                        if (part == 0) sh.row_q[PAIR ? x : 0][r] = a.scale_log2 * kvb_pow2(e - 7);
                    }
                }
                if (D == 256) {
                    // .. and on to tensor memory: thread (g, j) has eight channels of every 32
                    __syncwarp();
#pragma unroll 1
                    for (int cb = 0; cb < 2 * D / 4; cb += 32) {   // 32 cells of four channels
                        float x[16];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int r = row_base + g + 8 * e, byte = 4 * cb + 32 * k + 8 * j;
                                const float2 v = *reinterpret_cast<const float2*>(to + (byte >> 7) * (kTileRows * 128) + r * 128 + ((((byte >> 4) & 7) ^ (r & 7)) << 4) + (byte & 8));
                                x[4 * k + 2 * e] = v.x;
                                x[4 * k + 2 * e + 1] = v.y;
                            }
                        tc_store(tm + lanes + kColQ + cb, x);
                    }
                    tc_wait_store();
                    tc_fence_before();
                } else {
                    fence_async_smem();
                }
                __syncwarp();
            }
            if (ALT) {
                // one set of queries for both groups
                if (x == 0) {
                    if (lane == 0) mbar_arrive(&sh.r_full);
                } else {
                    ok = wait(&sh.r_full, piece & 1);
                    if (!ok) break;
                }
            }
            if (lane == 0) mbar_arrive(&sh.q_full[x]);
            float qf[Q], mref[Q], l[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                qf[q] = sh.row_q[PAIR ? x : 0][row_base + g + 8 * q];
                mref[q] = kKvNothing;
                l[q] = 0.f;
            }
            // a warp whose rows the head does not have leaves them out (their probabilities are anything, and so is what becomes
            // of them)
            const bool busy = row0 < rows_here;
            // places up to which every row of the warp sees everything
            const int open_to = a.node_parent != nullptr ? w.cached : w.cached + row0 / G + 1;
            int ev = 64;              // exponent field that O is relative to
            bool first = true, large = false;
            const int first_pg = w.pg;
#pragma unroll 1
            for (int i = ALT ? (n0 ^ x) & 1 : 0; i < np; i += STEP) {
                const int pg = first_pg + i, buf = taken & 1, slot = (n0 + i) & (kByteScales - 1);
                const unsigned int col = col_s + buf * 64;
                ok = wait(&sh.s_full[x][buf], (taken >> 1) & 1);   // (the page's scales came with its codes)
                if (!ok) break;
                if (busy) {
                    tc_fence_after();
                    const uint2 scale = *reinterpret_cast<const uint2*>(&sh.scale[slot]);
                    const bool missing = sh.missing[slot] != 0;
                    float s[32];          // rows g (s[4 k], s[4 k + 1]) and g + 8
                    tc_load(col, s);
                    const int ep = missing ? 0 : (int)(kvb_scale_bits(scale.y) >> 23);
                    const float ks = __uint_as_float(kvb_scale_bits(scale.x));   // (anything where the page is missing)
                    float ff[Q];          // what S is to be multiplied by (never 0: what is hidden is -inf times it)
#pragma unroll
                    for (int q = 0; q < Q; ++q) ff[q] = fmaxf(qf[q] * ks, 1e-37f);
                    if (missing || (pg + 1) * kPage > open_to) {   // what a row does not see becomes -inf (lane r finds out for row r)
                        const u64 mine = missing || row0 + (lane & 15) >= rows_here ? 0ull : kv_seen(a, w.cached, w.fresh, w.first, pg, own_row() / G);
#pragma unroll
                        for (int q = 0; q < Q; ++q) {
                            const u64 seen = __shfl_sync(0xFFFFFFFFu, mine, g + 8 * q) >> (2 * j);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const unsigned int two = (unsigned int)(seen >> (8 * k));
                                if (!(two & 1u)) s[4 * k + 2 * q] = -CUDART_INF_F;
                                if (!(two & 2u)) s[4 * k + 2 * q + 1] = -CUDART_INF_F;
                            }
                        }
                    }
                    if (ep > ev) {
                        // values of this page are relative to a larger exponent than O
                        if (!first) {
                            ok = o_complete();
                            if (!ok) break;
                            const float f = ep - ev > 126 ? 0.f : kvb_pow2(ev - ep);
                            float fo[Q];
#pragma unroll
                            for (float& y : fo) y = f;
                            kvb_scale_o<D>(col_o, fo);
                        }
                        ev = ep;
                    }
                    const int down = missing ? 0 : min(ev - ep, kByteDown);
                    const float shift = kTileP - (float)down;
                    // Probabilities with the maximum as it stands; only where a thread's sum of them leaves fp16's range (by a
                    // new maximum at least 2^5 above it), on the first page, and with large products, is the maximum looked for
                    // and this done again.
                    float ls[Q];
                    bool again = first || large || down > kByteFar;
#pragma unroll 1
                    for (;;) {
                        if (again) {
                            float fo[Q], m[Q], top = 0.f;
#pragma unroll
                            for (int q = 0; q < Q; ++q) {
                                m[q] = -CUDART_INF_F;
#pragma unroll
                                for (int k = 0; k < 8; ++k) m[q] = fmaxf(m[q], fmaxf(s[4 * k + 2 * q], s[4 * k + 2 * q + 1]));
                                m[q] = fmaxf(m[q], __shfl_xor_sync(0xFFFFFFFFu, m[q], 1));
                                m[q] = fmaxf(m[q], __shfl_xor_sync(0xFFFFFFFFu, m[q], 2));
                                m[q] *= ff[q];
                                if (m[q] > -CUDART_INF_F) top = fmaxf(top, fabsf(m[q]));
                            }
                            large = large || __any_sync(0xFFFFFFFFu, top >= kTileLarge);
                            if (large) {
#pragma unroll
                                for (int k = 0; k < 32; ++k) s[k] *= ff[(k >> 1) & 1];
                                for (float& y : ff) y = 1.f;
                            }
#pragma unroll
                            for (int q = 0; q < Q; ++q) {
                                const float mn = fmaxf(mref[q], m[q]);
                                fo[q] = ex2_approx(mref[q] - mn);
                                mref[q] = mn;
                                l[q] *= fo[q];
                            }
                            if (!first) {
                                ok = o_complete();
                                if (!ok) break;
                                kvb_scale_o<D>(col_o, fo);
                            }
                        }
                        unsigned int pk[16];
#pragma unroll
                        for (int q = 0; q < Q; ++q) {
                            const float2 fq = make_float2(ff[q], ff[q]), mm = make_float2(shift - mref[q], shift - mref[q]);
                            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                float2 p = __ffma2_rn(make_float2(s[4 * k + 2 * q], s[4 * k + 2 * q + 1]), fq, mm);
                                p = make_float2(ex2_approx(p.x), ex2_approx(p.y));
                                sum = __fadd2_rn(sum, p);
                                pk[2 * k + q] = pack_half(p.x, p.y);
                            }
                            ls[q] = sum.x + sum.y;
                        }
                        tc_store_cells(col, pk);
                        if (again || __all_sync(0xFFFFFFFFu, fmaxf(ls[0], ls[1]) < 65504.f)) break;
                        again = true;
                    }
                    if (!ok) break;
                    const float back = kvb_pow2(down);   // (the probabilities were scaled down by so much)
#pragma unroll
                    for (int q = 0; q < Q; ++q) l[q] = fmaf(ls[q], back, l[q]);
                }
                first = false;
                ++taken;
                tc_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.p_full[x][buf]);
                    mbar_arrive(&sh.scale_empty[slot]);
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
            float own[Q], other[Q];        // factors of this group's O, and of the other's
            const float unscale = any ? kvb_pow2(ev - 127) : 0.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                l[q] += __shfl_xor_sync(0xFFFFFFFFu, l[q], 1);
                l[q] += __shfl_xor_sync(0xFFFFFFFFu, l[q], 2);
                mref[q] -= kTileP;         // (l and O carry the probabilities' power of two)
                own[q] = unscale;
                other[q] = 0.f;
            }
            if (ALT) {
                // group 0 reads both groups' O (the same lanes of tensor memory)
                if (x == 1) {
#pragma unroll
                    for (int q = 0; q < Q; ++q) {
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
                    for (int q = 0; q < Q; ++q) {
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
                const bool any1 = ALT && sh.exchange_up[row_base] != 0.f;   // (the same for every row)
                // the results go through the places of the warp's own queries, which have been used
                const auto stage = [&](int lr, int chunk) {
                    return sh.queries[PAIR ? x : 0] + (row_base + lr) * 128 + (chunk >> 3) * (kTileRows * 128) + (((chunk & 7) ^ (lr & 7)) << 4);
                };
                if (complete) {
#pragma unroll
                    for (int q = 0; q < Q; ++q) {
                        const float inv = kv_inverse(l[q]);
                        own[q] *= inv;
                        other[q] *= inv;
                    }
                }
#pragma unroll 1
                for (int cb = 0; cb < D; cb += 64) {
                    float o[32];                                // rows g, g + 8
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0.f;
                    if (any) {
                        tc_load(col_o + cb, o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] *= own[(k >> 1) & 1];
                    }
                    if (any1) {
                        float y[32];
                        tc_load(col_o + kStep + cb, y);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = fmaf(y[k], other[(k >> 1) & 1], o[k]);
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int lr = g + 8 * e, ch = cb + 8 * k + 2 * j;
                            const float2 v = make_float2(o[4 * k + 2 * e], o[4 * k + 2 * e + 1]);
                            if (complete) {
                                *reinterpret_cast<unsigned int*>(stage(lr, ch >> 3) + 4 * j) = pack_bf16(v.x, v.y);
                            } else if ((PAIR ? x * kTileRows : 0) + row_base + lr < rows) {
                                *reinterpret_cast<float2*>(part + ((PAIR ? x * kTileRows : 0) + row_base + lr) * D + ch) = v;
                            }
                        }
                }
                if (complete) {
                    __syncwarp();
                    const int token = own_row() / G, member = own_row() - token * G;
                    const long long own_head = ((long long)w.first + token) * a.p.n_q_heads + w.h * G + member;
#pragma unroll 4
                    for (int rb = 0; rb < 16; rb += RI) {
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
                for (int q = 0; q < Q; ++q) {
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
            if (ALT && x == 0) {   // group 1 may go on
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.x_empty);
            }
            tc_fence_before();
            n0 += np;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.piece_empty[piece % kTilePieces]);
        }
        if (!ok) {   // (a group that gave up may have loads or stores under way in the memory that is freed below)
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tc_wait_store();
        }
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
    if (warp == kByteSoftmax + 4) tc_free(tm, 512);
}

}  // namespace aasd
