// Attention of a step's new tokens over the paged 4-bit cache.
#pragma once

#include "aasd_kv.cuh"

namespace aasd {

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
    DeviceState* state;
};

// Where a token row belongs: its sequence and place among the new tokens.
__device__ __forceinline__ void kv_row_owner(const KvAttendArgs& a, int64_t t, int& b, int64_t& i) {
    if (a.p.rows_per_seq > 0) {
        b = (int)(t / a.p.rows_per_seq);
        i = t - (int64_t)b * a.p.rows_per_seq;
        return;
    }
    int lo = 0, hi = a.p.n_seqs;
    if (t < a.tok_offsets[0] || t >= a.tok_offsets[hi]) {
        b = -1;
        i = 0;
        return;
    }
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.tok_offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    b = lo;
    i = t - a.tok_offsets[lo];
}

// One warp per (token row, query head), one key after the other.
template <int DT, int D>
__global__ void __launch_bounds__(256) kv_attend_kernel(const KvAttendArgs a) {
    constexpr int H = D / 2, C = H / 32;   // a lane's pairs: channels lane + 32 c and H + lane + 32 c
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (row >= a.p.n_tokens * a.p.n_q_heads) return;
    const int64_t t = row / a.p.n_q_heads;
    const int h = (int)(row - t * a.p.n_q_heads);
    const int head = h / (a.p.n_q_heads / a.p.n_kv_heads);
    int b;
    int64_t i;
    kv_row_owner(a, t, b, i);
    float qx[C], qy[C], ox[C], oy[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        qx[c] = Elt<DT>::load(a.q, t * a.p.q_stride + (int64_t)h * D + lane + 32 * c);
        qy[c] = Elt<DT>::load(a.q, t * a.p.q_stride + (int64_t)h * D + H + lane + 32 * c);
        ox[c] = oy[c] = 0.f;
    }
    float m = -CUDART_INF_F, l = 0.f;
    auto visit = [&](int64_t at) {
        const int64_t pg = at / kPage;
        const int page = pg < a.p.max_pages ? a.block_table[(int64_t)b * a.p.max_pages + pg] : -1;
        if (page < 0 || page >= a.p.n_pages) {
            raise(a.state, AASD_STATUS_BAD_OFFSETS);
            return;
        }
        const uint8_t* block = a.pages + ((int64_t)page * a.p.n_kv_heads + head) * kv_head_bytes(D);
        const int off = (int)(at % kPage);
        const unsigned int km = reinterpret_cast<const unsigned int*>(block + kv_key_meta_offset(D))[off];
        const unsigned int vm = reinterpret_cast<const unsigned int*>(block + kv_value_meta_offset(D))[off];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const unsigned int w = block[off * H + lane + 32 * c];
            s += qx[c] * (meta_scale(km) * (float)(w & 15u) + meta_min(km)) + qy[c] * (meta_scale(km) * (float)(w >> 4) + meta_min(km));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        s *= a.scale_log2;
        const float nm = fmaxf(m, s);
        const float keep = exp2f(m - nm), p = exp2f(s - nm);
        m = nm;
        l = l * keep + p;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const unsigned int w = block[kv_value_offset(D) + (lane + 32 * c) * kPage + off];
            ox[c] = ox[c] * keep + p * (meta_scale(vm) * (float)(w & 15u) + meta_min(vm));
            oy[c] = oy[c] * keep + p * (meta_scale(vm) * (float)(w >> 4) + meta_min(vm));
        }
    };
    if (b >= 0) {
        const int cached = a.cached_len[b];
        const int64_t fresh = (int64_t)a.kv_len[b] - cached;
        if (i < fresh) {
            for (int64_t at = 0; at < cached; ++at) visit(at);
            if (a.node_parent == nullptr) {
                for (int64_t j = 0; j <= i; ++j) visit(cached + j);
            } else {
                int64_t x = i;
                while (x >= 0) {
                    visit(cached + x);
                    const int p = a.node_parent[t - i + x];
                    if (p >= x || p < AASD_NONE) {
                        raise(a.state, AASD_STATUS_BAD_OFFSETS);
                        break;
                    }
                    x = p;
                }
            }
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t at = row * D + lane + 32 * c;
        if (DT == AASD_F32) {
            static_cast<float*>(a.o.out)[at] = ox[c] * inv;
            static_cast<float*>(a.o.out)[at + H] = oy[c] * inv;
        } else {
            static_cast<__nv_bfloat16*>(a.o.out)[at] = __float2bfloat16_rn(ox[c] * inv);
            static_cast<__nv_bfloat16*>(a.o.out)[at + H] = __float2bfloat16_rn(oy[c] * inv);
        }
    }
    if (a.o.lse != nullptr && lane == 0) a.o.lse[row] = l > 0.f ? (m + log2f(l)) * (float)kLn2 : -CUDART_INF_F;
}

}  // namespace aasd
