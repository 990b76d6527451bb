// Attention of a step's new tokens over the paged 8-bit cache.
#pragma once

#include "aasd_kv_attend.cuh"
#include "aasd_kvb.cuh"

namespace aasd {

// A CTA takes one token row and query head, a warp every fourth page, the lanes the channels.
template <int DT, int D>
__global__ void __launch_bounds__(128) kvb_attend_plain_kernel(const KvAttendArgs a) {
    constexpr int C = D / 32;
    __shared__ float s_q[D], s_o[4][D], s_m[4], s_l[4];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.p.n_q_heads / a.p.n_kv_heads;
    const long long row = blockIdx.x, tok = row / a.p.n_q_heads;
    const int head = (int)(row % a.p.n_q_heads), h = head / G;
    int b = -1;
    if (a.p.rows_per_seq > 0) b = (int)(tok / a.p.rows_per_seq);
    else
        for (int k = 0; k < a.p.n_seqs; ++k)
            if (a.tok_offsets[k] <= tok && tok < a.tok_offsets[k + 1]) b = k;
    KvSeq s{};
    int i = 0;
    if (b >= 0) {
        s = kv_load_seq(a, b, 8);
        i = (int)(tok - s.first);
        if (s.fresh > 0 && (long long)s.cached + s.fresh > (long long)a.p.max_pages * kPage) raise(a.state, AASD_STATUS_BAD_OFFSETS);
    }
    const bool there = b >= 0 && i < s.fresh;
    for (int d = tid; d < D; d += 128) s_q[d] = there ? Elt<DT>::load(a.q, tok * a.p.q_stride + (long long)head * D + d) * a.scale_log2 : 0.f;
    __syncthreads();
    float m = kKvNothing, l = 0.f, o[C];
    for (int c = 0; c < C; ++c) o[c] = 0.f;
    for (int pg = warp; there && pg < s.pages; pg += 4) {
        const u64 seen = kv_seen(a, s.cached, s.fresh, s.first, pg, i);
        const int page = a.block_table[(long long)b * a.p.max_pages + pg];
        if (page < 0 || page >= a.p.n_pages) {
            raise(a.state, AASD_STATUS_BAD_OFFSETS);
            continue;
        }
        const uint8_t* block = a.pages + ((long long)page * a.p.n_kv_heads + h) * kvb_head_bytes(D);
        const unsigned int* scale = reinterpret_cast<const unsigned int*>(block + kvb_scale_offset(D));
        const float sk = kvb_pow2(kvb_exponent(scale[0])), sv = kvb_pow2(kvb_exponent(scale[1]));
        for (int t = 0; t < kPage; ++t) {
            if (!((seen >> t) & 1ull)) continue;
            float x = 0.f;
            for (int c = 0; c < C; ++c) {
                const int d = 32 * c + lane;
                x = fmaf(kvb_values(block[kvb_chunk_offset(D, t, d / 16) + d % 16]).x, s_q[d], x);
            }
            for (int k = 16; k > 0; k >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, k);
            x *= sk;
            const float mn = fmaxf(m, x), f = ex2_approx(m - mn), p = ex2_approx(x - mn);
            m = mn;
            l = l * f + p;
            for (int c = 0; c < C; ++c) {
                const int d = 32 * c + lane;
                o[c] = fmaf(kvb_values(block[kvb_value_offset(D) + kvb_chunk_offset(D, t, d / 16) + d % 16]).x * sv, p, o[c] * f);
            }
        }
    }
    for (int c = 0; c < C; ++c) s_o[warp][32 * c + lane] = o[c];
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
    __syncthreads();
    const float M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float L = 0.f;
    for (int w = 0; w < 4; ++w) L += s_l[w] * ex2_approx(s_m[w] - M);
    for (int d = tid; d < D; d += 128) {
        float x = 0.f;
        for (int w = 0; w < 4; ++w) x = fmaf(s_o[w][d], ex2_approx(s_m[w] - M), x);
        x = L > 0.f ? x / L : 0.f;
        if (DT == AASD_F32) static_cast<float*>(a.o.out)[row * D + d] = x;
        else static_cast<__nv_bfloat16*>(a.o.out)[row * D + d] = __float2bfloat16_rn(x);
    }
    if (tid == 0 && a.o.lse != nullptr) a.o.lse[row] = L > 0.f ? (M + log2f(L)) * (float)kLn2 : -CUDART_INF_F;
}

}  // namespace aasd
