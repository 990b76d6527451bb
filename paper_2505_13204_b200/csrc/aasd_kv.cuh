// The paged 4-bit cache: layout, quantiser, and the kernels that keep it (page tables, norm +
// rotation + store, moving an accepted path, reading entries back).  Attention over it is in
// aasd_kv_attend.cuh.
#pragma once

#include <cuda_bf16.h>

#include "aasd_device.cuh"

namespace aasd {

constexpr int kPage = AASD_KV_PAGE;       // tokens of a page
constexpr float kKvTiny = 8.673617379884035e-19f;   // 2^-60: smallest scale, so that its reciprocal is finite

// Offsets inside one head's block of a page (see include/aasd.h).
__host__ __device__ constexpr int kv_head_bytes(int D) { return kPage * D + 2 * kPage * 4; }
__host__ __device__ constexpr int kv_value_offset(int D) { return kPage * D / 2; }
__host__ __device__ constexpr int kv_key_meta_offset(int D) { return kPage * D; }
__host__ __device__ constexpr int kv_value_meta_offset(int D) { return kPage * D + kPage * 4; }

__device__ __forceinline__ void raise(DeviceState* state, unsigned int bits) { atomicOr(&state->status, bits); }

__device__ __forceinline__ float bf16_round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
__device__ __forceinline__ float meta_scale(unsigned int m) { return __uint_as_float(m << 16); }
__device__ __forceinline__ float meta_min(unsigned int m) { return __uint_as_float(m & 0xFFFF0000u); }

// Scale and minimum of a row, from its extremes (every operation in fp32, rounded to nearest:
// the stored bytes are a function of the inputs alone).
struct KvQuant {
    float m, inv;
    unsigned int meta;
};
__device__ __forceinline__ KvQuant kv_quantiser(float lo, float hi, bool bad) {
    KvQuant z;
    float m = bf16_round(lo);
    float s = bf16_round(__fmul_rn(__fsub_rn(hi, m), 1.0f / 15.0f));
    s = fmaxf(s, kKvTiny);
    if (bad) {
        m = 0.f;
        s = kKvTiny;
    }
    z.m = m;
    z.inv = __frcp_rn(s);
    z.meta = (__float_as_uint(m) & 0xFFFF0000u) | (__float_as_uint(s) >> 16);
    return z;
}
// Codes of eight channels of each half of a row, a byte per pair.  Adding 1.5 * 2^23 to a value in 0..15
// rounds it to the nearest whole number (ties to even) and leaves that in the low bits.  (NaN
// cannot reach this: such rows are zeroed.)
__device__ __forceinline__ unsigned long long kv_row_codes(const float2 (&x)[4], const float2 (&y)[4], const KvQuant& z, bool bad) {
    const float2 m = make_float2(-z.m, -z.m), inv = make_float2(z.inv, z.inv), magic = make_float2(12582912.f, 12582912.f);
    unsigned int word[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float2 a = __fmul2_rn(__fadd2_rn(x[e], m), inv), b = __fmul2_rn(__fadd2_rn(y[e], m), inv);
        a = make_float2(fminf(fmaxf(a.x, 0.f), 15.f), fminf(fmaxf(a.y, 0.f), 15.f));
        b = make_float2(fminf(fmaxf(b.x, 0.f), 15.f), fminf(fmaxf(b.y, 0.f), 15.f));
        a = __fadd2_rn(a, magic);
        b = __fadd2_rn(b, magic);
        const unsigned int c0 = (__float_as_uint(a.x) & 15u) | ((__float_as_uint(b.x) & 15u) << 4);
        const unsigned int c1 = (__float_as_uint(a.y) & 15u) | ((__float_as_uint(b.y) & 15u) << 4);
        word[e >> 1] |= (c0 | (c1 << 8)) << (16 * (e & 1));
    }
    return bad ? 0ull : (unsigned long long)word[0] | ((unsigned long long)word[1] << 32);
}

// Eight consecutive elements as fp32; `vec`: the address is 16-byte aligned.
template <int DT, bool VEC>
__device__ __forceinline__ void load8(const void* base, int64_t i, float (&x)[8]) {
    if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Elt<DT>::load(base, i + e);
    } else if constexpr (DT == AASD_F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
        const float4 a = __ldg(p), b = __ldg(p + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(base) + i));
        Elt<AASD_BF16>::unpack(q, x);
    }
}
// The same eight elements as they come from memory, so that many can be under way in few registers.
template <int DT, bool VEC>
struct Raw8 {
    uint4 a, b;   // (bf16: a alone)
    __device__ __forceinline__ void clear() { a = b = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const void* base, int64_t i) {
        if constexpr (!VEC) {
            float x[8];
            load8<DT, false>(base, i, x);
            if constexpr (DT == AASD_F32) {
                a = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
                b = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
            } else {   // (bf16 values as fp32 hold their bits in the upper half)
                a.x = (__float_as_uint(x[0]) >> 16) | __float_as_uint(x[1]);
                a.y = (__float_as_uint(x[2]) >> 16) | __float_as_uint(x[3]);
                a.z = (__float_as_uint(x[4]) >> 16) | __float_as_uint(x[5]);
                a.w = (__float_as_uint(x[6]) >> 16) | __float_as_uint(x[7]);
            }
        } else if constexpr (DT == AASD_F32) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + i);
            a = __ldg(p);
            b = __ldg(p + 1);
        } else {
            a = __ldg(reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(base) + i));
        }
    }
    __device__ __forceinline__ void unpack(float2 (&x)[4]) const {
        if constexpr (DT == AASD_F32) {
            x[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
            x[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
            x[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
            x[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
        } else {
            const unsigned int w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u));
        }
    }
};
__device__ __forceinline__ unsigned int pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned int*>(&h);
}
// Stores to the library's own [.. x D] outputs, whose rows are 16-byte aligned when the base is.
template <int DT, bool VEC>
__device__ __forceinline__ void store8(void* base, int64_t i, const float (&x)[8]) {
    if constexpr (DT == AASD_F32) {
        float* p = static_cast<float*>(base) + i;
        if constexpr (VEC) {
            reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = x[e];
        }
    } else {
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + i;
        if constexpr (VEC) {
            *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                                                      pack_bf16(x[6], x[7]));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = __float2bfloat16_rn(x[e]);
        }
    }
}

template <int DT, bool VEC>
__device__ __forceinline__ void store8(void* base, int64_t i, const float2 (&x)[4]) {
    const float y[8] = {x[0].x, x[0].y, x[1].x, x[1].y, x[2].x, x[2].y, x[3].x, x[3].y};
    store8<DT, VEC>(base, i, y);
}

// ---- page tables, slots and positions -----------------------------------------------------------

struct KvPlanArgs {
    const int32_t* cached_len;
    const int32_t* n_new;
    const int32_t* node_depth;   // may be NULL
    aasd_kv_plan_params p;
    aasd_kv_plan_state s;
    aasd_kv_plan_out o;
    DeviceState* state;
    int tokens_inline;           // the planning CTA also writes the token arrays
};

// Exclusive scan over the CTA of one value per thread; `total` is the sum.
template <int NT>
__device__ __forceinline__ long long block_scan(long long v, long long* s_warp, long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();   // s_warp may still be read from the scan before
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const long long t = s_warp[w];
        if (w < warp) before += t;
        all += t;
    }
    total = all;
    return before + x - v;
}

// Index of the last entry of first[0..n) that is <= r (first[0] <= r).
__device__ __forceinline__ int last_not_above(const int* first, int n, int r) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Slot and position of token row t, place i of sequence b.
__device__ __forceinline__ void kv_place_token(const KvPlanArgs& a, int64_t t, int b, int64_t i, int& slot, int& pos) {
    slot = pos = AASD_NONE;
    if (b < 0) return;
    const int cached = a.cached_len[b];
    const int64_t at = (int64_t)cached + i;
    if (i < 0 || at >= a.o.kv_len[b]) return;
    if (!AASD_IN_RANGE(b < a.p.n_seqs && at >= 0 && at / kPage < a.p.max_pages && t < a.p.n_tokens, a.state)) return;
    const int page = a.s.block_table[(int64_t)b * a.p.max_pages + at / kPage];
    if (page < 0 || page >= a.p.n_pages) {
        raise(a.state, AASD_STATUS_BAD_OFFSETS);
        return;
    }
    slot = page * kPage + (int)(at % kPage);
    pos = a.node_depth ? cached + a.node_depth[t] : (int)at;
}

#ifdef AASD_KV_TU
constexpr int kPlanThreads = 256, kPlanThreadsMany = 1024;   // of batches up to 256 sequences, and larger ones

// One CTA: the books of all sequences (NT at a time) by prefix sums, the pages moved
// by all threads together (a thread finds its page's sequence by bisection of the sums), so one
// long sequence that ends or arrives costs no more than many short ones.  Latency-bound: four
// scans and three trips to memory (4 trees of 9 nodes 3.4 us, 256 sequences of one token 3.7; 256 arriving
// prompts of 1000 tokens 14 us with the token arrays' launch, which waits while this CTA hands
// out 4096 pages; a launch alone is 2 us).
template <int NT>
__global__ void __launch_bounds__(NT) kv_plan_kernel(const KvPlanArgs a) {
    __shared__ long long s_warp[NT / 32];
    __shared__ int s_first[NT + 1], s_at[NT];
    __shared__ int s_off[NT + 1];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x;
    const int B = a.p.n_seqs, P = a.p.max_pages;
    unsigned int bits = 0;
    long long n_free = a.s.n_free[0];
    if (n_free < 0 || n_free > a.p.n_pages) {
        bits |= AASD_STATUS_BAD_OFFSETS;
        n_free = n_free < 0 ? 0 : a.p.n_pages;
    }
    struct Seq {
        int cached, fresh, held;
        long long need;
        bool bad;
    };
    auto load = [&](int b) {
        Seq q{0, 0, 0, 0, false};
        if (b < B) {
            q.cached = a.cached_len[b];
            q.fresh = a.n_new[b];
            q.held = a.s.seq_pages[b];
            q.bad = q.cached < 0 || q.fresh < 0 || q.held < 0 || q.held > P || (long long)q.held * kPage < q.cached ||
                    (a.p.rows_per_seq > 0 && q.fresh > a.p.rows_per_seq);
            if (q.fresh < 0) q.fresh = 0;
            q.need = q.bad ? q.held : ((long long)q.cached + q.fresh + kPage - 1) / kPage;
        }
        return q;
    };
    // pages past their sequence's need go back on the stack
    for (int base = 0; base < B; base += NT) {
        const Seq q = load(base + tid);
        if (q.bad) bits |= AASD_STATUS_BAD_OFFSETS;
        const int back = q.held > q.need ? (int)(q.held - q.need) : 0;
        long long total;
        const long long first = block_scan<NT>(back, s_warp, total);
        if (total == 0) continue;
        s_first[tid] = (int)first;
        s_at[tid] = (int)q.need;
        __syncthreads();
        for (int r = tid; r < (int)total; r += NT) {
            const int k = last_not_above(s_first, NT, r);
            if (!AASD_IN_RANGE(base + k < B && s_at[k] >= 0 && s_at[k] + (r - s_first[k]) < P, a.state)) continue;
            int32_t* entry = a.s.block_table + (int64_t)(base + k) * P + s_at[k] + (r - s_first[k]);
            const int page = *entry;
            *entry = AASD_NONE;
            if (page < 0 || page >= a.p.n_pages) bits |= AASD_STATUS_BAD_OFFSETS;
            const long long to = n_free + r;
            if (to < a.p.n_pages) a.s.free_pages[to] = page;
            else bits |= AASD_STATUS_BAD_OFFSETS;
        }
        n_free += total;
        if (n_free > a.p.n_pages) n_free = a.p.n_pages;
        __syncthreads();
    }
    // missing pages come off it, sequence by sequence
    long long asked = 0, taken = 0, row0 = 0;
    for (int base = 0; base < B; base += NT) {
        const int b = base + tid;
        const Seq q = load(b);
        const int held = q.held > q.need ? (int)q.need : q.held;
        long long fresh_total, want_total;
        const long long off = row0 + block_scan<NT>(q.fresh, s_warp, fresh_total);
        const bool fits = !q.bad && q.need <= P && (a.p.rows_per_seq > 0 || off + q.fresh <= a.p.n_tokens);
        const int want = fits && q.need > held ? (int)(q.need - held) : 0;
        const long long first = block_scan<NT>(want, s_warp, want_total);
        const bool served = fits && (want == 0 || asked + first + want <= n_free);
        if (b < B) {
            if (!served && !q.bad) bits |= AASD_STATUS_KV_FULL;
            a.s.seq_pages[b] = served ? held + want : held;
            a.o.kv_len[b] = served ? q.cached + q.fresh : q.cached;
            if (a.o.tok_offsets) {
                const long long at = a.p.rows_per_seq > 0 ? (long long)b * a.p.rows_per_seq : off;
                a.o.tok_offsets[b] = (int32_t)(at > 0x7FFFFFFFLL ? 0x7FFFFFFFLL : at);
            }
        }
        s_off[tid] = (int)(off > 0x7FFFFFFFLL ? 0x7FFFFFFFLL : off);
        s_first[tid] = (int)first;
        s_at[tid] = held;
        // the sequences that get what they ask for are the first ones of those that ask
        long long got;
        block_scan<NT>(served ? want : 0, s_warp, got);   // (also the barrier for the arrays above)
        for (int r0 = tid; r0 < (int)got; r0 += 4 * NT) {
            int page[4];   // (four loads under way before the first store)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = r0 + e * NT;
                const bool there = r < (int)got && AASD_IN_RANGE(n_free - 1 - (asked + r) >= 0 && n_free <= a.p.n_pages, a.state);
                page[e] = there ? a.s.free_pages[n_free - 1 - (asked + r)] : 0;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = r0 + e * NT;
                if (r >= (int)got) break;
                const int k = last_not_above(s_first, NT, r);
                if (!AASD_IN_RANGE(n_free - 1 - (asked + r) >= 0 && base + k < B && s_at[k] >= 0 && s_at[k] + (r - s_first[k]) < P, a.state)) continue;
                a.s.free_pages[n_free - 1 - (asked + r)] = AASD_NONE;
                if (page[e] < 0 || page[e] >= a.p.n_pages) bits |= AASD_STATUS_BAD_OFFSETS;
                a.s.block_table[(int64_t)(base + k) * P + s_at[k] + (r - s_first[k])] = page[e];
            }
        }
        asked += want_total;
        taken += got;
        row0 += fresh_total;
        __syncthreads();
    }
    if (tid == 0) {
        a.s.n_free[0] = (int32_t)(n_free - taken);
        if (a.o.tok_offsets) {
            const long long at = a.p.rows_per_seq > 0 ? (long long)B * a.p.rows_per_seq : row0;
            a.o.tok_offsets[B] = (int32_t)(at > 0x7FFFFFFFLL ? 0x7FFFFFFFLL : at);
        }
    }
    if (a.tokens_inline) {   // one round of sequences: their offsets are still in shared memory
        __syncthreads();
        for (int64_t t = tid; t < a.p.n_tokens; t += NT) {
            int b;
            int64_t i;
            if (a.p.rows_per_seq > 0) {
                b = (int)(t / a.p.rows_per_seq);
                i = t - (int64_t)b * a.p.rows_per_seq;
            } else {
                b = t < row0 ? last_not_above(s_off, B, (int)t) : -1;
                i = b < 0 ? 0 : t - s_off[b];
            }
            int slot, pos;
            kv_place_token(a, t, b, i, slot, pos);
            a.o.slot_map[t] = slot;
            a.o.positions[t] = pos;
        }
    }
    if (bits) raise(a.state, bits);
}

// Token arrays of large steps: four tokens per thread.  A CTA's 1024 tokens belong to few
// sequences, which its first warp finds by bisection of the offsets, a 32nd of the range at a time.
__global__ void __launch_bounds__(256) kv_tokens_kernel(const KvPlanArgs a) {
    __shared__ int s_b;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t c0 = (int64_t)blockIdx.x * 1024, t0 = c0 + threadIdx.x * 4;
    const int B = a.p.n_seqs;
    int b;
    if (a.p.rows_per_seq > 0) {
        b = (int)(t0 / a.p.rows_per_seq);
    } else {
        if (threadIdx.x < 32) {
            int lo = 0, n = B + 1;                            // the last offset <= c0 is among [lo, lo + n)
            while (n > 1) {
                const int step = (n + 31) / 32, at = lo + (int)threadIdx.x * step;
                const unsigned int below = __ballot_sync(0xFFFFFFFFu, at < lo + n && a.o.tok_offsets[at] <= c0);
                const int k = below ? 31 - __clz(below) : 0;
                n = min(step, lo + n - (lo + k * step));
                lo += k * step;
            }
            if (threadIdx.x == 0) s_b = lo;
        }
        __syncthreads();
        b = s_b;
        while (b < B && t0 >= a.o.tok_offsets[b + 1]) ++b;
    }
    if (t0 >= a.p.n_tokens) return;
    int slot[4], pos[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t t = t0 + e;
        int64_t first = 0;
        if (a.p.rows_per_seq > 0) {
            if (t >= (int64_t)(b + 1) * a.p.rows_per_seq) ++b;
            first = (int64_t)b * a.p.rows_per_seq;
        } else {
            while (b < B && t >= a.o.tok_offsets[b + 1]) ++b;   // (sequences without new tokens are passed over)
            if (b < B) first = a.o.tok_offsets[b];
        }
        kv_place_token(a, t, b < B ? b : -1, t - first, slot[e], pos[e]);
    }
    if (t0 + 4 <= a.p.n_tokens && ((uintptr_t)a.o.slot_map % 16) == 0 && ((uintptr_t)a.o.positions % 16) == 0) {
        *reinterpret_cast<int4*>(a.o.slot_map + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        *reinterpret_cast<int4*>(a.o.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t0 + e < a.p.n_tokens) {
                a.o.slot_map[t0 + e] = slot[e];
                a.o.positions[t0 + e] = pos[e];
            }
    }
}
#endif

// ---- norm, rotation, store -----------------------------------------------------------------------

struct KvWriteArgs {
    const void *q, *k, *v, *q_weight, *k_weight;
    const float* cos_sin;
    const int32_t* positions;
    const int32_t* slot_map;
    int64_t n_tokens;
    aasd_kv_write_params p;
    uint8_t* pages;
    void *q_out, *k_out;
    DeviceState* state;
    unsigned int value_blocks;   // CTAs that store values; the others take queries and keys
    float2 minus_zero;           // see mul2_rounded
};

// A product rounded by itself.  The assembler makes one fused multiply-add, which rounds once, of a
// packed product and the packed sum behind it, whatever their rounding modes say (scalar ones are left
// alone).  a * b + (-0) is the rounded product, as fast, and stays as it is as long as -0 is a number
// that the compiler does not know: a launch argument.
__device__ __forceinline__ float2 mul2_rounded(float2 a, float2 b, float2 minus_zero) { return __ffma2_rn(a, b, minus_zero); }

#ifdef AASD_KV_TU
// A CTA either takes query and key rows or stores values; both kinds share the launch.
//
// Query and key rows: D / 16 lanes share a row, a lane holds eight channels of each half, so that both
// members of a rotated pair, and both halves of a stored byte, are its own.  One row each: four rows of
// a token per lane, with the cosines, weights and a reciprocal root shared, were slower at every size
// (64 tokens 4.6 us instead of 2.7, 512 tokens 7.0 instead of 6.3, 4096 tokens 34.4 instead of 30.0; 32 query and 8 key
// heads of 128 channels, which take 2.5, 5.8 and 27.4 us as the kernel stands).  4096 tokens: 89 MB at half the
// copy rate; seven of ten issue slots are used, so that it is the instructions that bound it.  The norm's sum follows the order of the definition: halves, then
// neighbours (three steps inside the lane, the others across lanes by butterfly; a sum does not
// ask which operand is first), each operation rounded by itself.
//
// Values: a CTA takes kValueTokens tokens of one head.  Their codes meet in shared memory, and lane t
// of a warp stores the bytes of token t: neighbouring tokens, which lie in neighbouring bytes, in one
// go (byte by byte from the rows' own lanes, 4096 tokens took 62 us in all).
constexpr int kValueTokens = 32;
constexpr int kWriteThreads = 256;

// What a row's lanes know about its token.
__device__ __forceinline__ unsigned int kv_write_token(const KvWriteArgs& a, int64_t t, bool store, int& pos, int& slot) {
    unsigned int bits = 0;
    pos = a.positions[t];
    slot = store ? a.slot_map[t] : AASD_NONE;
    if (pos < AASD_NONE || (a.p.rotary_dim > 0 && pos >= a.p.max_positions)) {
        bits |= AASD_STATUS_ID_RANGE;
        pos = AASD_NONE;
    }
    if (slot < AASD_NONE || slot / kPage >= a.p.n_pages) {
        bits |= AASD_STATUS_ID_RANGE;
        slot = AASD_NONE;
    }
    if (pos == AASD_NONE) slot = AASD_NONE;
    return bits;
}
// Quantiser of a row spread over L lanes; every lane of the warp takes part.
template <int L>
__device__ __forceinline__ KvQuant kv_row_quantiser(const float2 (&x)[4], const float2 (&y)[4], bool& bad) {
    float lo = x[0].x, hi = x[0].x;
    float2 sick = make_float2(0.f, 0.f);   // NaN as soon as one value is NaN or infinite
    const float2 zero = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lo = fminf(lo, fminf(fminf(x[e].x, x[e].y), fminf(y[e].x, y[e].y)));
        hi = fmaxf(hi, fmaxf(fmaxf(x[e].x, x[e].y), fmaxf(y[e].x, y[e].y)));
        sick = __ffma2_rn(x[e], zero, sick);
        sick = __ffma2_rn(y[e], zero, sick);
    }
    float s = sick.x + sick.y;
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
        s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    }
    const float m = bf16_round(lo);
    bad = s != 0.f || !(hi - m <= 3.3e38f) || !(fabsf(m) <= 3.4e38f);
    return kv_quantiser(lo, hi, bad);
}

// FULL: all D channels are rotated, in halves (the usual form); otherwise whatever the parameters say.
template <int DT, int D, bool VEC, bool FULL>
__global__ void __launch_bounds__(kWriteThreads) kv_write_kernel(const KvWriteArgs a) {
    constexpr int L = D / 16;              // lanes of a row
    constexpr int H = D / 2;
    // rows in passage: partial rotation (a float per channel), or the values' codes (rows padded to 8 bytes more)
    constexpr int kRows = kWriteThreads / L, kPitch = H + 8;
    __shared__ alignas(16) unsigned char s_mem[!FULL && kRows * D * 4 > kValueTokens * kPitch ? kRows * D * 4 : kValueTokens * kPitch];
    __shared__ int s_slot[kValueTokens];
    pdl_launch_dependents();
    pdl_wait();
    const int hq = a.p.n_q_heads, hkv = a.p.n_kv_heads;
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    unsigned int bits = 0;
    if (blockIdx.x < a.value_blocks) {
        // ---- values
        const int64_t t0 = (int64_t)(blockIdx.x / hkv) * kValueTokens;
        const int head = (int)(blockIdx.x % hkv);
        for (int k = group; k < kValueTokens; k += kRows) {
            const int64_t t = t0 + k;
            const bool live = t < a.n_tokens;
            // (the row does not wait for its slot)
            Raw8<DT, VEC> rx, ry;
            rx.clear();
            ry.clear();
            if (live) {
                const int64_t at = t * a.p.v_stride + (int64_t)head * D + 8 * l;
                rx.load(a.v, at);
                ry.load(a.v, at + H);
            }
            int pos, slot = AASD_NONE;
            if (live) bits |= kv_write_token(a, t, true, pos, slot);
            float2 x[4], y[4];
            rx.unpack(x);
            ry.unpack(y);
            bool bad;
            const KvQuant z = kv_row_quantiser<L>(x, y, bad);
            if (slot != AASD_NONE && bad) bits |= AASD_STATUS_BAD_ROW;
            *reinterpret_cast<unsigned long long*>(s_mem + k * kPitch + 8 * l) = kv_row_codes(x, y, z, bad);
            if (l == 0) {
                s_slot[k] = slot;
                if (slot != AASD_NONE) {
                    uint8_t* block = a.pages + ((int64_t)(slot / kPage) * hkv + head) * kv_head_bytes(D);
                    reinterpret_cast<unsigned int*>(block + kv_value_meta_offset(D))[slot % kPage] = z.meta;
                }
            }
        }
        __syncthreads();
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        static_assert(kValueTokens == 32, "a lane per token");
        const int slot = s_slot[lane];
        if (slot != AASD_NONE && AASD_IN_RANGE(slot / kPage < a.p.n_pages && head < hkv, a.state)) {
            uint8_t* col = a.pages + ((int64_t)(slot / kPage) * hkv + head) * kv_head_bytes(D) + kv_value_offset(D) + slot % kPage;
            constexpr int kWordsPerWarp = H / 4 / (kWriteThreads / 32);   // 1, 2 or 4 words of four channel pairs
#pragma unroll
            for (int w = 0; w < kWordsPerWarp; ++w) {
                const int i = (warp * kWordsPerWarp + w) * 4;
                const unsigned int b = *reinterpret_cast<const unsigned int*>(s_mem + lane * kPitch + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) col[(i + e) * kPage] = (uint8_t)(b >> (8 * e));
            }
        }
        if (bits) raise(a.state, bits);
        return;
    }
    // ---- queries and keys
    float* s_rows = reinterpret_cast<float*>(s_mem);
    const int heads = hq + hkv;
    const int64_t g = ((int64_t)(blockIdx.x - a.value_blocks) * kWriteThreads + threadIdx.x) / L;
    const bool live = g < a.n_tokens * heads;
    const int64_t t = live ? g / heads : 0;
    const int h = live ? (int)(g - t * heads) : 0;
    // (the row does not wait for its token's position)
    Raw8<DT, VEC> rx, ry;           // channels 8l .. and D/2 + 8l ..
    rx.clear();
    ry.clear();
    if (live) {
        const void* src = h < hq ? a.q : a.k;
        const int64_t at = h < hq ? t * a.p.q_stride + (int64_t)h * D + 8 * l : t * a.p.k_stride + (int64_t)(h - hq) * D + 8 * l;
        rx.load(src, at);
        ry.load(src, at + H);
    }
    int pos = AASD_NONE, slot = AASD_NONE;
    if (live) bits |= kv_write_token(a, t, hkv > 0, pos, slot);
    const bool used = live && pos != AASD_NONE;
    if (!used) {
        rx.clear();
        ry.clear();
    }
    // cosines and sines of the lane's pairs (the branches on the form of the rotation are the same for every lane)
    const int rot = FULL ? D : a.p.rotary_dim, half = rot / 2;
    const bool neighbours = !FULL && (a.p.flags & AASD_KV_ROPE_INTERLEAVED) != 0;
    const float* cs = a.cos_sin + (int64_t)(used ? pos : 0) * rot;
    float co[8], si[8];   // neighbours: pairs of the low half, then of the high half; else of channels 8l + e
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        co[e] = 1.f;
        si[e] = 0.f;
    }
    if (rot > 0 && used) {
        if (neighbours) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = (e < 4 ? 8 * l : H + 8 * l) + 2 * (e & 3);
                if (c < rot) {
                    co[e] = __ldg(cs + c / 2);
                    si[e] = __ldg(cs + half + c / 2);
                }
            }
        } else if (rot == D) {
            load8<AASD_F32, VEC>(cs, 8 * l, co);
            load8<AASD_F32, VEC>(cs, half + 8 * l, si);
        }
    }
    const bool key = h >= hq;
    float2 u[4], v[4];
    rx.unpack(u);
    ry.unpack(v);
    const float2 mz = a.minus_zero;
    // (the lanes of a row take the same way; shuffles stay among all lanes of the warp)
    if (a.q_weight != nullptr || a.k_weight != nullptr) {
        float s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 q = __fadd2_rn(mul2_rounded(u[e], u[e], mz), mul2_rounded(v[e], v[e], mz));
            s[e] = __fadd_rn(q.x, q.y);
        }
        float sum = __fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3]));
#pragma unroll
        for (int o = 1; o < L; o <<= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xFFFFFFFFu, sum, o));
        const float r = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.0f / D), a.p.eps)));
        const void* w = key ? a.k_weight : a.q_weight;
        if (used && w != nullptr) {
            Raw8<DT, VEC> g;
            float2 wx[4], wy[4];
            g.load(w, 8 * l);
            g.unpack(wx);
            g.load(w, H + 8 * l);
            g.unpack(wy);
            const float2 rr = make_float2(r, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u[e] = __fmul2_rn(__fmul2_rn(u[e], rr), wx[e]);
                v[e] = __fmul2_rn(__fmul2_rn(v[e], rr), wy[e]);
            }
        }
    }
    // (a - b is written a + (-b): the same rounding)
    if (!FULL && rot > 0 && neighbours) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            float2(&z)[4] = part ? v : u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (part * H + 8 * l + 2 * e < rot) {
                    const float c = co[4 * part + e], n = si[4 * part + e];
                    z[e] = __fadd2_rn(mul2_rounded(z[e], make_float2(c, c), mz), mul2_rounded(make_float2(z[e].y, z[e].x), make_float2(-n, n), mz));
                }
            }
        }
    } else if (FULL || rot == D) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 c = make_float2(co[2 * e], co[2 * e + 1]), n = make_float2(si[2 * e], si[2 * e + 1]);
            const float2 p = u[e], q = v[e];
            u[e] = __fadd2_rn(mul2_rounded(p, c, mz), mul2_rounded(q, make_float2(-n.x, -n.y), mz));
            v[e] = __fadd2_rn(mul2_rounded(q, c, mz), mul2_rounded(p, n, mz));
        }
    } else if (!FULL && rot > 0) {
        // a pair (c, c + half) inside the first rot channels: its members may be different lanes',
        // so the warp's rows pass through shared memory (partial rotation is the rare case)
        float* mine = s_rows + group * D;
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            *reinterpret_cast<float2*>(mine + 8 * l + 2 * e) = u[e];
            *reinterpret_cast<float2*>(mine + H + 8 * l + 2 * e) = v[e];
        }
        __syncwarp();
        if (used) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                float2(&z)[4] = part ? v : u;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float& x = e & 1 ? z[e >> 1].y : z[e >> 1].x;
                    const int c = part * H + 8 * l + e;
                    if (c < half) x = __fsub_rn(__fmul_rn(x, cs[c]), __fmul_rn(mine[c + half], cs[half + c]));
                    else if (c < rot) x = __fadd_rn(__fmul_rn(x, cs[c - half]), __fmul_rn(mine[c - half], cs[c]));
                }
            }
        }
    }
    if (live && h < hq) {
        const int64_t at = (t * hq + h) * D + 8 * l;
        store8<DT, VEC>(a.q_out, at, u);
        store8<DT, VEC>(a.q_out, at + H, v);
    }
    if (live && key && a.k_out != nullptr) {
        const int64_t at = (t * hkv + h - hq) * D + 8 * l;
        store8<DT, VEC>(a.k_out, at, u);
        store8<DT, VEC>(a.k_out, at + H, v);
    }
    if (__any_sync(0xFFFFFFFFu, used && key)) {
        bool bad;
        const KvQuant z = kv_row_quantiser<L>(u, v, bad);
        if (used && key && slot != AASD_NONE && AASD_IN_RANGE(slot / kPage < a.p.n_pages && h - hq < hkv, a.state)) {
            if (bad) bits |= AASD_STATUS_BAD_ROW;
            uint8_t* block = a.pages + ((int64_t)(slot / kPage) * hkv + h - hq) * kv_head_bytes(D);
            const int at = slot % kPage;
            *reinterpret_cast<unsigned long long*>(block + at * H + 8 * l) = kv_row_codes(u, v, z, bad);
            if (l == 0) reinterpret_cast<unsigned int*>(block + kv_key_meta_offset(D))[at] = z.meta;
        }
    }
    if (bits) raise(a.state, bits);
}

// ---- entries as values -----------------------------------------------------------------------------

struct KvReadArgs {
    const uint8_t* pages;
    const int32_t* slots;
    int64_t n;
    int n_pages, n_kv_heads;
    void *k_out, *v_out;
    DeviceState* state;
};

// A CTA takes kValueTokens slots of one head.  The values' bytes are fetched with a lane per slot, so
// that neighbouring slots are one access, and pass through shared memory; then D / 16 lanes turn out a
// row as in the writing kernel.  4096 slots of 8 heads of 128 channels take 7.8 us; their 21 MB would take
// 3.2, and six of ten issue slots are used.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(kWriteThreads) kv_read_kernel(const KvReadArgs a) {
    constexpr int L = D / 16, H = D / 2, kRows = kWriteThreads / L, kPitch = H + 8;
    __shared__ alignas(16) unsigned char s_code[kValueTokens * kPitch];
    __shared__ int s_slot[kValueTokens];
    pdl_launch_dependents();
    pdl_wait();
    const int hkv = a.n_kv_heads;
    const int64_t i0 = (int64_t)(blockIdx.x / hkv) * kValueTokens;
    const int head = (int)(blockIdx.x % hkv);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int slot = AASD_NONE;
    if (i0 + lane < a.n) {
        slot = a.slots[i0 + lane];
        if (slot < AASD_NONE || slot / kPage >= a.n_pages) {
            if (warp == 0) raise(a.state, AASD_STATUS_ID_RANGE);
            slot = AASD_NONE;
        }
    }
    if (warp == 0) s_slot[lane] = slot;
    if (a.v_out != nullptr) {
        constexpr int kWordsPerWarp = H / 4 / (kWriteThreads / 32);
        unsigned char b[kWordsPerWarp][4];
        const uint8_t* col = a.pages + ((int64_t)((slot < 0 ? 0 : slot) / kPage) * hkv + head) * kv_head_bytes(D) + kv_value_offset(D) + (slot < 0 ? 0 : slot) % kPage;
#pragma unroll
        for (int w = 0; w < kWordsPerWarp; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) b[w][e] = slot != AASD_NONE ? col[((warp * kWordsPerWarp + w) * 4 + e) * kPage] : (unsigned char)0;
#pragma unroll
        for (int w = 0; w < kWordsPerWarp; ++w)
            *reinterpret_cast<unsigned int*>(s_code + lane * kPitch + (warp * kWordsPerWarp + w) * 4) =
                b[w][0] | (b[w][1] << 8) | (b[w][2] << 16) | ((unsigned int)b[w][3] << 24);
    }
    __syncthreads();
    const int l = threadIdx.x % L;
    // rows: keys of all slots, then values
    for (int k = threadIdx.x / L; k < 2 * kValueTokens; k += kRows) {
        const int q = k % kValueTokens;
        const bool value = k >= kValueTokens;
        void* out = value ? a.v_out : a.k_out;
        if (out == nullptr || i0 + q >= a.n) continue;
        const int at = s_slot[q];
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
        if (at != AASD_NONE && AASD_IN_RANGE(at >= 0 && at / kPage < a.n_pages && head < hkv, a.state)) {
            const uint8_t* block = a.pages + ((int64_t)(at / kPage) * hkv + head) * kv_head_bytes(D);
            const int off = at % kPage;
            const unsigned long long bytes = value ? *reinterpret_cast<const unsigned long long*>(s_code + q * kPitch + 8 * l)
                                                   : *reinterpret_cast<const unsigned long long*>(block + off * H + 8 * l);
            const unsigned int meta = reinterpret_cast<const unsigned int*>(block + (value ? kv_value_meta_offset(D) : kv_key_meta_offset(D)))[off];
            const float s = meta_scale(meta), m = meta_min(meta);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned int b = (unsigned int)(bytes >> (8 * e)) & 255u;
                x[e] = __fadd_rn(__fmul_rn(s, (float)(b & 15u)), m);
                y[e] = __fadd_rn(__fmul_rn(s, (float)(b >> 4)), m);
            }
        }
        const int64_t to = ((i0 + q) * hkv + head) * D + 8 * l;
        store8<DT, VEC>(out, to, x);
        store8<DT, VEC>(out, to + H, y);
    }
}

// ---- the accepted path ------------------------------------------------------------------------------

struct KvCommitArgs {
    uint8_t* pages;
    const int32_t* block_table;
    const int32_t* cached_len;
    const int32_t* kv_len;
    const int32_t* tok_offsets;
    const int32_t* best_node;
    const int32_t* node_parent;
    aasd_kv_commit_params p;
    int32_t* new_len;
    DeviceState* state;
};

constexpr int kCommitThreads = 256;

// grid: (sequence, group of heads of all layers).  Every CTA reads its tree's parents into shared
// memory, walks the path there, turns it into (source slot, destination slot) pairs, and its
// warps move the entries of one head after another.  Path nodes are in ascending order and never
// in front of their depth, so a destination is a source of an earlier node at most: entries are
// moved in ascending order, a batch's loads before its stores.  A token's values are single bytes 64 apart,
// so a moved entry touches a 32-byte sector per byte of them: 256 paths of 8 layers (4 heads of 128
// channels) take 15.4 us, and one path of 16 layers 2.9 us, the chain of its dependent loads.
template <int D>
__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const KvCommitArgs a) {
    constexpr int H = D / 2, W = H / 4;        // W: 32-bit words of a token's keys
    __shared__ int s_node[AASD_KV_MAX_NODES];   // parents, then sources
    __shared__ int s_path[AASD_KV_MAX_NODES];   // leaf first
    __shared__ int s_len, s_bad;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int cached = a.cached_len[b];
    const int64_t first = a.p.rows_per_seq > 0 ? (int64_t)b * a.p.rows_per_seq : a.tok_offsets[b];
    const int n = a.kv_len[b] - cached;        // new tokens in the cache
    const int best = a.best_node[b];
    if (n <= 0 || best < 0 || best >= n || cached < 0 || n > AASD_KV_MAX_NODES ||
        (a.p.rows_per_seq > 0 && n > a.p.rows_per_seq)) {
        if (tid == 0 && blockIdx.y == 0) {
            a.new_len[b] = cached;
            if (n > AASD_KV_MAX_NODES || cached < 0 || (a.p.rows_per_seq > 0 && n > a.p.rows_per_seq))
                raise(a.state, AASD_STATUS_BAD_OFFSETS);
        }
        return;
    }
    if (!AASD_IN_RANGE(best < AASD_KV_MAX_NODES && first >= 0, a.state)) return;
    for (int i = tid; i <= best; i += kCommitThreads) s_node[i] = a.node_parent[first + i];
    if (tid == 0) s_bad = 0;
    __syncthreads();
    if (tid == 0) {
        int len = 0;
        for (int x = best; x >= 0; ++len) {
            s_path[len] = x;
            const int p = s_node[x];
            if (p >= x || p < AASD_NONE) {
                s_bad = 1;
                break;
            }
            x = p;
        }
        s_len = len;
    }
    __syncthreads();
    const int len = s_len;
    // the path is leaf first: entry i (depth i) is s_path[len - 1 - i]
    auto slot_of = [&](int place) {
        const int64_t at = (int64_t)cached + place;
        if (at / kPage >= a.p.max_pages) return -1;
        const int page = a.block_table[(int64_t)b * a.p.max_pages + at / kPage];
        return page < 0 || page >= a.p.n_pages ? -1 : page * kPage + (int)(at % kPage);
    };
    if (!s_bad)
        for (int i = tid; i < len; i += kCommitThreads) {
            const int src = slot_of(s_path[len - 1 - i]);
            if (src < 0 || slot_of(i) < 0) s_bad = 1;
            s_node[i] = src;     // (the parents have been read)
        }
    __syncthreads();
    const bool bad = s_bad != 0;
    if (tid == 0 && blockIdx.y == 0) {
        a.new_len[b] = bad ? cached : cached + len;
        if (bad) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    if (bad) return;
    int from = 0;                               // nodes that are where they belong already
    while (from < len && s_path[len - 1 - from] == from) ++from;
    if (from == len) return;
    const int lane = tid & 31;
    const int64_t items = (int64_t)a.p.n_layers * a.p.n_kv_heads;
    const int64_t hb = kv_head_bytes(D);
    for (int64_t it = (int64_t)blockIdx.y * (kCommitThreads / 32) + (tid >> 5); it < items;
         it += (int64_t)gridDim.y * (kCommitThreads / 32)) {
        const int layer = (int)(it / a.p.n_kv_heads), head = (int)(it % a.p.n_kv_heads);
        uint8_t* pool = a.pages + (int64_t)layer * a.p.layer_stride;
        constexpr int NB = 4;                                    // entries whose loads are under way together
        constexpr int KW = (W + 31) / 32, VW = (H + 31) / 32;    // words of keys, bytes of values per lane
        for (int i0 = from; i0 < len; i0 += NB) {
            unsigned int kw[NB][KW], meta[NB];
            uint8_t vb[NB][VW];
            int dst[NB];
            bool inside = true;   // (checked builds: every slot of the batch, by every lane alike)
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const int at = min(i0 + e, len - 1);
                inside = inside && AASD_IN_RANGE(s_node[at] >= 0 && s_node[at] / kPage < a.p.n_pages && slot_of(at) >= 0 && layer < a.p.n_layers, a.state);
            }
            if (!inside) break;
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const int src = s_node[min(i0 + e, len - 1)];
                dst[e] = slot_of(min(i0 + e, len - 1));
                const uint8_t* sb = pool + ((int64_t)(src / kPage) * a.p.n_kv_heads + head) * hb;
                const int so = src % kPage;
#pragma unroll
                for (int w = 0; w < KW; ++w)
                    kw[e][w] = lane + 32 * w < W ? reinterpret_cast<const unsigned int*>(sb + so * H)[lane + 32 * w] : 0u;
#pragma unroll
                for (int w = 0; w < VW; ++w) vb[e][w] = sb[kv_value_offset(D) + (lane + 32 * w) * kPage + so];
                meta[e] = reinterpret_cast<const unsigned int*>(sb + kv_key_meta_offset(D) + (lane & 1) * kPage * 4)[so];
            }
            __syncwarp();   // every lane has its loads before the first store
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                if (i0 + e >= len) break;
                uint8_t* db = pool + ((int64_t)(dst[e] / kPage) * a.p.n_kv_heads + head) * hb;
                const int to = dst[e] % kPage;
#pragma unroll
                for (int w = 0; w < KW; ++w)
                    if (lane + 32 * w < W) reinterpret_cast<unsigned int*>(db + to * H)[lane + 32 * w] = kw[e][w];
#pragma unroll
                for (int w = 0; w < VW; ++w) db[kv_value_offset(D) + (lane + 32 * w) * kPage + to] = vb[e][w];
                if (lane < 2) reinterpret_cast<unsigned int*>(db + kv_key_meta_offset(D) + lane * kPage * 4)[to] = meta[e];
            }
            __syncwarp();
        }
    }
}
#endif

}  // namespace aasd
