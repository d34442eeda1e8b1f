// Writing new tokens into the paged cache and reading tokens back.  Both move every byte once and
// compute next to nothing, so HBM bounds them at size and the launch bounds them at one step.
// One warp serves one token at a time: its row of 2 x heads x head_dim values is contiguous on the
// caller's side (except between k and v), its place is looked up once, and in passes of 512 values
// every lane moves 16 consecutive ones, which is one 16-byte store of codes and half a scale block.
#pragma once
#include "kv_format.cuh"
#include "ptx_sm100.cuh"

namespace ead {

constexpr int kKvThreads = 256;
constexpr int kKvLaneValues = 16;
constexpr int kKvPass = 32 * kKvLaneValues;       // values a warp moves per pass

struct KvMoveParams {
    KvCacheView cache;
    KvBatchView batch;
    uint8_t *rows_k, *rows_v;                     // caller's bf16 rows
    int64_t row_stride;                           // elements between tokens
    const int32_t *first;                         // reading: first position per sequence, or NULL
    uint32_t *status;
};

template <int FMT>
__global__ void __launch_bounds__(kKvThreads) ead_kv_write_kernel(KvMoveParams p)
{
    const int lane = threadIdx.x & 31;
    const int warp = (blockIdx.x * kKvThreads + threadIdx.x) >> 5, warps = (gridDim.x * kKvThreads) >> 5;
    const KvCacheView &c = p.cache;
    const int per_half = c.heads * c.head_dim, total = 2 * per_half;
    for (int t = warp; t < p.batch.n_tokens; t += warps) {
        const int b = find_sequence(p.batch.new_start, p.batch.B, t, lane);
        const int pos = __ldg(p.batch.kv_len + b) - (__ldg(p.batch.new_start + b + 1) - t);
        const int page = find_page(c, p.batch, b, pos);
        if (page < 0) {
            if (lane == 0) flag_status(p.status, kStatusBadPage);
            continue;
        }
        const int slot = pos & (c.page_size - 1);
        for (int base = 0; base < total; base += 2 * kKvPass) {      // two passes' loads in flight
            uint4 in[2][2];
            int off[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                off[u] = base + u * kKvPass + lane * kKvLaneValues;
                if (off[u] < total) {
                    const bool is_v = off[u] >= per_half;
                    const uint8_t *row = (is_v ? p.rows_v : p.rows_k) + 2 * (t * p.row_stride + off[u] - (is_v ? per_half : 0));
                    in[u][0] = __ldg(reinterpret_cast<const uint4 *>(row));
                    in[u][1] = __ldg(reinterpret_cast<const uint4 *>(row) + 1);
                } else {
                    in[u][0] = in[u][1] = make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool live = off[u] < total, is_v = off[u] >= per_half;
                const int x = off[u] - (is_v ? per_half : 0), head = x / c.head_dim, d = x - head * c.head_dim;
                const uint32_t w[8] = {in[u][0].x, in[u][0].y, in[u][0].z, in[u][0].w,
                                       in[u][1].x, in[u][1].y, in[u][1].z, in[u][1].w};
                uint8_t *pool = is_v ? c.v : c.k;
                if (FMT == kFmtBf16) {
                    if (live) {
                        uint4 *dst = reinterpret_cast<uint4 *>(pool + 2 * (pool_offset(c, page, head, slot) + d));
                        dst[0] = in[u][0];
                        dst[1] = in[u][1];
                    }
                } else {
                    uint32_t amax = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) amax = max(amax, max(abs_bits(bf16_lo(w[i])), abs_bits(bf16_hi(w[i]))));
                    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
                    const int byte = scale_byte(amax);
                    const float inv = inverse_scale(byte);
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o[i] = to_e4m3x2(bf16_lo(w[2 * i]) * inv, bf16_hi(w[2 * i]) * inv) |
                               to_e4m3x2(bf16_lo(w[2 * i + 1]) * inv, bf16_hi(w[2 * i + 1]) * inv) << 16;
                    if (live) {
                        *reinterpret_cast<uint4 *>(pool + pool_offset(c, page, head, slot) + d) =
                            make_uint4(o[0], o[1], o[2], o[3]);
                        if ((lane & 1) == 0)
                            (is_v ? c.v_scale : c.k_scale)[scale_offset(c, page, head, slot) + d / kFmtBlock] =
                                static_cast<uint8_t>(byte);
                    }
                }
            }
        }
    }
}

template <int FMT>
__global__ void __launch_bounds__(kKvThreads) ead_kv_read_kernel(KvMoveParams p)
{
    const int lane = threadIdx.x & 31;
    const int warp = (blockIdx.x * kKvThreads + threadIdx.x) >> 5, warps = (gridDim.x * kKvThreads) >> 5;
    const KvCacheView &c = p.cache;
    const int per_half = c.heads * c.head_dim, total = 2 * per_half;
    for (int t = warp; t < p.batch.n_tokens; t += warps) {
        const int b = find_sequence(p.batch.new_start, p.batch.B, t, lane);
        const int pos = (p.first ? __ldg(p.first + b) : 0) + t - __ldg(p.batch.new_start + b);
        const int page = find_page(c, p.batch, b, pos);
        if (page < 0 && lane == 0) flag_status(p.status, kStatusBadPage);
        const int slot = pos & (c.page_size - 1);
        for (int base = 0; base < total; base += 2 * kKvPass) {
            uint4 in[2][2];
            int byte[2];
            int off[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                off[u] = base + u * kKvPass + lane * kKvLaneValues;
                in[u][0] = in[u][1] = make_uint4(0, 0, 0, 0);
                byte[u] = 127;
                if (off[u] < total && page >= 0) {
                    const bool is_v = off[u] >= per_half;
                    const int x = off[u] - (is_v ? per_half : 0), head = x / c.head_dim, d = x - head * c.head_dim;
                    const uint8_t *pool = is_v ? c.v : c.k;
                    if (FMT == kFmtBf16) {
                        const uint4 *src = reinterpret_cast<const uint4 *>(pool + 2 * (pool_offset(c, page, head, slot) + d));
                        in[u][0] = __ldg(src);
                        in[u][1] = __ldg(src + 1);
                    } else {
                        in[u][0] = __ldg(reinterpret_cast<const uint4 *>(pool + pool_offset(c, page, head, slot) + d));
                        byte[u] = __ldg((is_v ? c.v_scale : c.k_scale) + scale_offset(c, page, head, slot) + d / kFmtBlock);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (off[u] >= total) continue;
                const bool is_v = off[u] >= per_half;
                uint4 *row = reinterpret_cast<uint4 *>((is_v ? p.rows_v : p.rows_k) +
                                                       2 * (t * p.row_stride + off[u] - (is_v ? per_half : 0)));
                if (FMT == kFmtBf16) {
                    row[0] = in[u][0];
                    row[1] = in[u][1];
                } else {
                    const float s = scale_value(byte[u]);
                    const uint32_t w[4] = {in[u][0].x, in[u][0].y, in[u][0].z, in[u][0].w};
                    uint32_t o[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 a = from_e4m3x2(w[i] & 0xffffu), e = from_e4m3x2(w[i] >> 16);
                        o[2 * i] = to_bf16x2(a.x * s, a.y * s);
                        o[2 * i + 1] = to_bf16x2(e.x * s, e.y * s);
                    }
                    row[0] = make_uint4(o[0], o[1], o[2], o[3]);
                    row[1] = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
        }
    }
}

}  // namespace ead
