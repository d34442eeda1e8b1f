// Attention of the step's new tokens over the paged cache.  One warp per (token, query head):
// 32 keys at a time, online softmax with a running maximum and sum.
#pragma once
#include "attn_common.cuh"

namespace ead {

template <int FMT>
__device__ __forceinline__ float pool_value(const KvCacheView &c, const uint8_t *pool, const uint8_t *scale, int page,
                                            int head, int slot, int d)
{
    const int64_t at = pool_offset(c, page, head, slot) + d;
    if (FMT == kFmtBf16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(pool)[at]);
    return from_e4m3x2(pool[at]).x * scale_value(scale[scale_offset(c, page, head, slot) + d / kFmtBlock]);
}

template <int FMT>
__global__ void __launch_bounds__(128) ead_kv_attention_simple_kernel(AttnParams p)
{
    __shared__ float qs[4][128];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int hq = blockIdx.y, t = blockIdx.x * 4 + w;
    if (t >= p.batch.n_tokens) return;
    const KvCacheView &c = p.cache;
    const int D = c.head_dim, h = hq / p.group;
    const int b = find_sequence(p.batch.new_start, p.batch.B, t, lane);
    const int n_b = p.batch.new_start[b + 1] - p.batch.new_start[b];
    const int pos = p.batch.kv_len[b] - (p.batch.new_start[b + 1] - t);
    if (n_b * p.group <= p.few_rows) return;
    if (n_b > p.batch.max_new && lane == 0) flag_status(p.status, kStatusBadCount);
    for (int d = lane; d < D; d += 32)
        qs[w][d] = __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p.q)[t * p.q_stride + hq * D + d]) * p.scale_log2;
    __syncwarp();
    const int cap = p.batch.max_len;
    if (p.batch.kv_len[b] > cap && lane == 0) flag_status(p.status, kStatusBadPage);
    const int end = min(pos + 1, cap);
    const int lo = p.window ? max(0, pos - p.window + 1) : 0;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < end; j0 += 32) {
        if (j0 + 32 <= lo && j0 >= p.sinks) continue;
        const int j = j0 + lane;
        const bool seen = j < end && (j >= lo || j < p.sinks);
        int page = -1;
        float z = -INFINITY;
        if (seen) {
            page = find_page(c, p.batch, b, j);
            if (page < 0) flag_status(p.status, kStatusBadPage);
            z = 0.f;
            if (page >= 0)
                for (int d = 0; d < D; ++d)
                    z = fmaf(qs[w][d], pool_value<FMT>(c, c.k, c.k_scale, page, h, j & (c.page_size - 1), d), z);
        }
        float top = z;
#pragma unroll
        for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        const float m_new = fmaxf(m, top);
        const float f = m_new == -INFINITY ? 1.f : exp2f(m - m_new);
        const float e = seen ? exp2f(z - m_new) : 0.f;
        l = l * f + e;
        for (int i = 0; i < D / 32; ++i) o[i] *= f;
        for (int k = 0; k < 32; ++k) {
            const float pk = __shfl_sync(0xffffffffu, e, k);
            const int pg = __shfl_sync(0xffffffffu, page, k);
            if (pg < 0) continue;
            for (int i = 0; i < D / 32; ++i)
                o[i] = fmaf(pk, pool_value<FMT>(c, c.v, c.v_scale, pg, h, (j0 + k) & (c.page_size - 1), lane + 32 * i), o[i]);
        }
        m = m_new;
    }
#pragma unroll
    for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
    const float inv = end > 0 ? 1.f / l : 0.f;
    for (int i = 0; i < D / 32; ++i)
        reinterpret_cast<__nv_bfloat16 *>(p.out)[t * p.out_stride + hq * D + lane + 32 * i] = __float2bfloat16(o[i] * inv);
    if (p.lse && lane == 0) p.lse[static_cast<int64_t>(t) * p.heads_q + hq] = end > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace ead
