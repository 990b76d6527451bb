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
__device__ __forceinline__ unsigned int kv_code(float x, const KvQuant& z) {
    const float c = rintf(__fmul_rn(__fsub_rn(x, z.m), z.inv));
    return (unsigned int)fminf(fmaxf(c, 0.f), 15.f);   // (NaN cannot reach this: such rows are zeroed)
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
    const int page = a.s.block_table[(int64_t)b * a.p.max_pages + at / kPage];
    if (page < 0 || page >= a.p.n_pages) {
        raise(a.state, AASD_STATUS_BAD_OFFSETS);
        return;
    }
    slot = page * kPage + (int)(at % kPage);
    pos = a.node_depth ? cached + a.node_depth[t] : (int)at;
}

#ifdef AASD_KV_TU
constexpr int kPlanThreads = 256;

// One CTA: the books of all sequences (kPlanThreads at a time) by prefix sums, the pages moved
// by all threads together (a thread finds its page's sequence by bisection of the sums), so one
// long sequence that ends or arrives costs no more than many short ones.  Latency-bound: four
// scans and three trips to memory.
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const KvPlanArgs a) {
    constexpr int NT = kPlanThreads;
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
        for (int r = tid; r < (int)got; r += NT) {
            const int k = last_not_above(s_first, NT, r);
            const long long from = n_free - 1 - (asked + r);
            const int page = a.s.free_pages[from];
            a.s.free_pages[from] = AASD_NONE;
            if (page < 0 || page >= a.p.n_pages) bits |= AASD_STATUS_BAD_OFFSETS;
            a.s.block_table[(int64_t)(base + k) * P + s_at[k] + (r - s_first[k])] = page;
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

// Token arrays of large steps: four tokens per thread.
__global__ void __launch_bounds__(256) kv_tokens_kernel(const KvPlanArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int64_t t0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (t0 >= a.p.n_tokens) return;
    const int B = a.p.n_seqs;
    int b;
    if (a.p.rows_per_seq > 0) b = (int)(t0 / a.p.rows_per_seq);
    else b = t0 < a.o.tok_offsets[B] ? last_not_above(a.o.tok_offsets, B, (int)t0) : B;
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
};

#ifdef AASD_KV_TU
// D / 16 lanes share a head row: a lane holds eight channels of each half of the row, so that
// both members of a rotated pair, and both halves of a stored byte, are its own.
//
// The norm's sum follows the order of the definition: halves, then neighbours (three steps
// inside the lane, the others across lanes by butterfly; a sum does not ask which operand is
// first), each operation rounded by itself.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256) kv_write_kernel(const KvWriteArgs a) {
    constexpr int L = D / 16;              // lanes of a row
    constexpr int H = D / 2;
    __shared__ float s_rows[256 / L * D];
    pdl_launch_dependents();
    pdl_wait();
    const int hq = a.p.n_q_heads, hkv = a.p.n_kv_heads;
    const int heads = hq + 2 * hkv;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int l = threadIdx.x % L;
    const bool live = row < a.n_tokens * heads;
    const int64_t t = live ? row / heads : 0;
    const int h = live ? (int)(row - t * heads) : 0;
    const int kind = h < hq ? 0 : h < hq + hkv ? 1 : 2;   // query, key, value
    const int head = kind == 0 ? h : kind == 1 ? h - hq : h - hq - hkv;
    float x[8], y[8];   // channels 8l + e and D/2 + 8l + e
    int pos = AASD_NONE, slot = AASD_NONE;
    unsigned int bits = 0;
    if (live) {
        pos = a.positions[t];
        slot = kind > 0 ? a.slot_map[t] : AASD_NONE;
        if (pos < AASD_NONE || (a.p.rotary_dim > 0 && pos >= a.p.max_positions)) {
            bits |= AASD_STATUS_ID_RANGE;
            pos = AASD_NONE;
        }
        if (slot < AASD_NONE || slot / kPage >= a.p.n_pages) {
            bits |= AASD_STATUS_ID_RANGE;
            slot = AASD_NONE;
        }
        if (pos == AASD_NONE) slot = AASD_NONE;
    }
    const bool used = live && pos != AASD_NONE;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
    if (used && AASD_IN_RANGE(t < a.n_tokens && head >= 0 && head < (kind == 0 ? hq : hkv), a.state)) {
        const void* src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const int64_t at = t * (kind == 0 ? a.p.q_stride : kind == 1 ? a.p.k_stride : a.p.v_stride) + (int64_t)head * D + 8 * l;
        load8<DT, VEC>(src, at, x);
        load8<DT, VEC>(src, at + H, y);
    }
    const void* w = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
    // (the lanes of a row take the same way; shuffles stay among all lanes of the warp)
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = __fadd_rn(__fmul_rn(x[e], x[e]), __fmul_rn(y[e], y[e]));
    float sum = __fadd_rn(__fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3])), __fadd_rn(__fadd_rn(s[4], s[5]), __fadd_rn(s[6], s[7])));
#pragma unroll
    for (int o = 1; o < L; o <<= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xFFFFFFFFu, sum, o));
    if (used && w != nullptr) {
        const float r = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.0f / D), a.p.eps)));
        float wx[8], wy[8];
        load8<DT, VEC>(w, 8 * l, wx);
        load8<DT, VEC>(w, H + 8 * l, wy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __fmul_rn(__fmul_rn(x[e], r), wx[e]);
            y[e] = __fmul_rn(__fmul_rn(y[e], r), wy[e]);
        }
    }
    // (the branches on the form of the rotation are the same for every lane of the launch)
    const int rot = a.p.rotary_dim, half = rot / 2;
    const bool turn = used && kind < 2 && AASD_IN_RANGE(rot == 0 || (pos >= 0 && pos < a.p.max_positions), a.state);
    const float* cs = a.cos_sin + (int64_t)(turn ? pos : 0) * rot;
    if (rot > 0 && (a.p.flags & AASD_KV_ROPE_INTERLEAVED)) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            float(&z)[8] = part ? y : x;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const int c = part * H + 8 * l + e;
                if (turn && c < rot) {
                    const float co = cs[c / 2], si = cs[half + c / 2];
                    const float p = z[e], q = z[e + 1];
                    z[e] = __fsub_rn(__fmul_rn(p, co), __fmul_rn(q, si));
                    z[e + 1] = __fadd_rn(__fmul_rn(q, co), __fmul_rn(p, si));
                }
            }
        }
    } else if (rot == D) {
        if (turn) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float co = cs[8 * l + e], si = cs[half + 8 * l + e];
                const float p = x[e], q = y[e];
                x[e] = __fsub_rn(__fmul_rn(p, co), __fmul_rn(q, si));
                y[e] = __fadd_rn(__fmul_rn(q, co), __fmul_rn(p, si));
            }
        }
    } else if (rot > 0) {
        // a pair (c, c + half) inside the first rot channels: its members may be different lanes',
        // so the warp's rows pass through shared memory (partial rotation is the rare case)
        float* mine = s_rows + (threadIdx.x / L) * D;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mine[8 * l + e] = x[e];
            mine[H + 8 * l + e] = y[e];
        }
        __syncwarp();
        if (turn) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                float(&z)[8] = part ? y : x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = part * H + 8 * l + e;
                    if (c < half) z[e] = __fsub_rn(__fmul_rn(z[e], cs[c]), __fmul_rn(mine[c + half], cs[half + c]));
                    else if (c < rot) z[e] = __fadd_rn(__fmul_rn(z[e], cs[c - half]), __fmul_rn(mine[c - half], cs[c]));
                }
            }
        }
    }
    if (live && kind == 0 && AASD_IN_RANGE(a.q_out != nullptr && head < hq, a.state)) {
        const int64_t at = (t * hq + head) * D + 8 * l;
        store8<DT, VEC>(a.q_out, at, x);
        store8<DT, VEC>(a.q_out, at + H, y);
    }
    if (live && kind == 1 && a.k_out != nullptr) {
        const int64_t at = (t * hkv + head) * D + 8 * l;
        store8<DT, VEC>(a.k_out, at, x);
        store8<DT, VEC>(a.k_out, at + H, y);
    }
    float lo = x[0], hi = x[0], sick = 0.f;   // sick: NaN or infinite as soon as one value is
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, fminf(x[e], y[e]));
        hi = fmaxf(hi, fmaxf(x[e], y[e]));
        sick += x[e] * 0.f + y[e] * 0.f;
    }
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
        sick += __shfl_xor_sync(0xFFFFFFFFu, sick, o);
    }
    if (live && kind > 0 && slot != AASD_NONE) {
        const bool bad = sick != 0.f || !(hi - bf16_round(lo) <= 3.3e38f) || !(fabsf(bf16_round(lo)) <= 3.4e38f);
        if (bad) bits |= AASD_STATUS_BAD_ROW;
        const KvQuant z = kv_quantiser(lo, hi, bad);
        unsigned long long bytes = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned int b = bad ? 0u : kv_code(x[e], z) | (kv_code(y[e], z) << 4);
            bytes |= (unsigned long long)b << (8 * e);
        }
        uint8_t* block = a.pages + ((int64_t)(slot / kPage) * hkv + head) * kv_head_bytes(D);
        const int at = slot % kPage;
        if (!AASD_IN_RANGE(slot >= 0 && slot / kPage < a.p.n_pages && head >= 0 && head < hkv, a.state)) {
        } else if (kind == 1) {
            *reinterpret_cast<unsigned long long*>(block + at * H + 8 * l) = bytes;
            if (l == 0) reinterpret_cast<unsigned int*>(block + kv_key_meta_offset(D))[at] = z.meta;
        } else {
            uint8_t* col = block + kv_value_offset(D) + at;
#pragma unroll
            for (int e = 0; e < 8; ++e) col[(8 * l + e) * kPage] = (uint8_t)(bytes >> (8 * e));
            if (l == 0) reinterpret_cast<unsigned int*>(block + kv_value_meta_offset(D))[at] = z.meta;
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

// Lanes as in the writing kernel: one row (slot, head, key or value) per D / 16 lanes.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvReadArgs a) {
    constexpr int L = D / 16, H = D / 2;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int l = threadIdx.x % L;
    const int heads = 2 * a.n_kv_heads;
    if (row >= a.n * heads) return;
    const int64_t i = row / heads;
    const int h = (int)(row - i * heads);
    const bool value = h >= a.n_kv_heads;
    const int head = value ? h - a.n_kv_heads : h;
    void* out = value ? a.v_out : a.k_out;
    if (out == nullptr) return;
    int slot = a.slots[i];
    if (slot < AASD_NONE || slot / kPage >= a.n_pages) {
        raise(a.state, AASD_STATUS_ID_RANGE);
        slot = AASD_NONE;
    }
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
    if (slot != AASD_NONE) {
        const uint8_t* block = a.pages + ((int64_t)(slot / kPage) * a.n_kv_heads + head) * kv_head_bytes(D);
        const int at = slot % kPage;
        unsigned long long bytes = 0;
        unsigned int meta;
        if (!value) {
            bytes = *reinterpret_cast<const unsigned long long*>(block + at * H + 8 * l);
            meta = reinterpret_cast<const unsigned int*>(block + kv_key_meta_offset(D))[at];
        } else {
            const uint8_t* col = block + kv_value_offset(D) + at;
#pragma unroll
            for (int e = 0; e < 8; ++e) bytes |= (unsigned long long)col[(8 * l + e) * kPage] << (8 * e);
            meta = reinterpret_cast<const unsigned int*>(block + kv_value_meta_offset(D))[at];
        }
        const float s = meta_scale(meta), m = meta_min(meta);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned int b = (unsigned int)(bytes >> (8 * e)) & 255u;
            x[e] = __fadd_rn(__fmul_rn(s, (float)(b & 15u)), m);
            y[e] = __fadd_rn(__fmul_rn(s, (float)(b >> 4)), m);
        }
    }
    const int64_t to = (i * a.n_kv_heads + head) * D + 8 * l;
    store8<DT, VEC>(out, to, x);
    store8<DT, VEC>(out, to + H, y);
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
// moved in ascending order, a batch's loads before its stores.
template <int D>
__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const KvCommitArgs a) {
    constexpr int H = D / 2, W = H / 4;        // W: 32-bit words of a token's keys
    __shared__ int s_node[AASD_KV_MAX_NODES];   // parents, then sources
    __shared__ int s_path[AASD_KV_MAX_NODES];
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
        for (int i = from; i < len; ++i) {
            const int src = s_node[i], dst = slot_of(i);
            if (src == dst) continue;
            const uint8_t* sb = pool + ((int64_t)(src / kPage) * a.p.n_kv_heads + head) * hb;
            uint8_t* db = pool + ((int64_t)(dst / kPage) * a.p.n_kv_heads + head) * hb;
            const int so = src % kPage, to = dst % kPage;
            for (int w = lane; w < W; w += 32)
                reinterpret_cast<unsigned int*>(db + to * H)[w] = reinterpret_cast<const unsigned int*>(sb + so * H)[w];
            for (int r = lane; r < H; r += 32)
                db[kv_value_offset(D) + r * kPage + to] = sb[kv_value_offset(D) + r * kPage + so];
            if (lane < 2) {
                const int off = kv_key_meta_offset(D) + lane * kPage * 4;
                reinterpret_cast<unsigned int*>(db + off)[to] = reinterpret_cast<const unsigned int*>(sb + off)[so];
            }
            __syncwarp();
        }
    }
}
#endif

}  // namespace aasd
