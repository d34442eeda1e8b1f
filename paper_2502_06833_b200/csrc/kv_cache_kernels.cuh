// Writing new tokens into the paged cache and reading tokens back.  Both move every byte once and
// compute next to nothing, so HBM bounds them at size and the launch bounds them at one step.
// A warp moves one stretch of 512 of a token's 2 x heads x head_dim values, 16 consecutive ones per lane (one 16-byte
// store of codes, half a scale block), for a run of consecutive tokens: its lanes look up the places of all of
// them at once, so the chain new_start -> kv_len -> page table -> data costs its latency once per run.
//
// Measured, 8-bit cache, 8 heads of 128: write of 24 k tokens 31 us from a cold cache, 4.9 TB/s, 0.76 of the device's copy rate; read
// of 107 k tokens 115 us, 5.7 TB/s, 0.88; one step of 64 tokens (bf16) 2.9 us.  bf16, 8 heads of 128: write of 23 k tokens 33 us
// with the rows in L2, read of 55 k 78 us, 5.8 TB/s.  The write's bound at size is the chain of
// look-ups and loads before the first store: with half the instructions for the largest magnitude it took as long.
#pragma once
#include "kv_format.cuh"
#include "ptx_sm100.cuh"

namespace ead {

constexpr int kKvThreads = 256;
constexpr int kKvLaneValues = 16;
constexpr int kKvPass = 32 * kKvLaneValues;       // values a warp moves of a token

struct KvMoveParams {
    KvCacheView cache;
    KvBatchView batch;
    uint8_t *rows_k, *rows_v;                     // caller's bf16 rows
    int64_t row_stride;                           // elements between tokens
    const int32_t *first;                         // reading: first position per sequence, or NULL
    uint32_t *status;
};

// Data that is used once.
__device__ __forceinline__ uint4 load_once(const void *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// First token of this warp's run.  (A thread's index in the grid passes 32 bits from 2^27 tokens on, a warp's does not.)
__device__ __forceinline__ int first_token(int run) { return static_cast<int>(blockIdx.x * (kKvThreads / 32) + (threadIdx.x >> 5)) * run; }

// Page and slot of token t0 + lane for the lanes below n (page -1: no valid place).
template <bool WRITE>
__device__ __forceinline__ void find_places(const KvMoveParams &p, int t0, int n, int lane, int *page, int *slot)
{
    int b = find_sequence(p.batch.new_start, p.batch.B, t0, lane);
    const int t = t0 + lane;
    *page = -1;
    *slot = 0;
    if (lane < n) {
        while (b + 1 < p.batch.B && __ldg(p.batch.new_start + b + 1) <= t) ++b;
        const int begin = __ldg(p.batch.new_start + b), end = __ldg(p.batch.new_start + b + 1);
        const int pos = WRITE ? __ldg(p.batch.kv_len + b) - (end - t) : (p.first ? __ldg(p.first + b) : 0) + t - begin;
        // a token of no sequence, or of one that contradicts the host's bounds, has no place whatever the page table says
        const bool bad = begin < 0 || t < begin || t >= end || end > p.batch.n_tokens || end - begin > p.batch.max_new;
        *page = bad ? -1 : find_page(p.cache, p.batch, b, pos);
        *slot = pos & (p.cache.page_size - 1);
        if (*page < 0) flag_status(p.status, bad ? kStatusBadCount : kStatusBadPage);
    }
    __syncwarp();
}

// RUN tokens per warp, all their loads in flight before the first store.
template <int FMT, int RUN>
__global__ void __launch_bounds__(kKvThreads) ead_kv_write_kernel(KvMoveParams p)
{
    const int lane = threadIdx.x & 31;
    const int t0 = first_token(RUN), n = min(RUN, p.batch.n_tokens - t0);
    if (n <= 0) return;
    const KvCacheView &c = p.cache;
    const int per_half = c.heads * c.head_dim, off = blockIdx.y * kKvPass + lane * kKvLaneValues;
    const bool live = off < 2 * per_half, is_v = off >= per_half;
    const int x = off - (is_v ? per_half : 0), head = x / c.head_dim, d = x - head * c.head_dim;
    const uint8_t *const row0 = (is_v ? p.rows_v : p.rows_k) + 2 * (t0 * p.row_stride + x);
    uint8_t *const pool = is_v ? c.v : c.k, *const scales = is_v ? c.v_scale : c.k_scale;
    uint4 in[RUN][2];
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
        in[i][0] = in[i][1] = make_uint4(0, 0, 0, 0);
        if (live && i < n) {
            in[i][0] = load_once(row0 + 2 * i * p.row_stride);
            in[i][1] = load_once(row0 + 2 * i * p.row_stride + 16);
        }
    }
    int pages, slots;
    find_places<true>(p, t0, n, lane, &pages, &slots);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
        const int page = __shfl_sync(0xffffffffu, pages, i), slot = __shfl_sync(0xffffffffu, slots, i);
        if (FMT == kFmtBf16) {
            if (live && page >= 0) {
                uint4 *dst = reinterpret_cast<uint4 *>(pool + 2 * (pool_offset(c, page, head, slot) + d));
                dst[0] = in[i][0];
                dst[1] = in[i][1];
            }
        } else {
            const uint32_t w[8] = {in[i][0].x, in[i][0].y, in[i][0].z, in[i][0].w, in[i][1].x, in[i][1].y, in[i][1].z, in[i][1].w};
            uint32_t amax = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) amax = max(amax, max(abs_bits(bf16_lo(w[k])), abs_bits(bf16_hi(w[k]))));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            const int byte = scale_byte(amax);
            const float inv = inverse_scale(byte);
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[k] = to_e4m3x2(bf16_lo(w[2 * k]) * inv, bf16_hi(w[2 * k]) * inv) |
                       to_e4m3x2(bf16_lo(w[2 * k + 1]) * inv, bf16_hi(w[2 * k + 1]) * inv) << 16;
            if (live && page >= 0) {
                *reinterpret_cast<uint4 *>(pool + pool_offset(c, page, head, slot) + d) = make_uint4(o[0], o[1], o[2], o[3]);
                if ((lane & 1) == 0) scales[scale_offset(c, page, head, slot) + d / kFmtBlock] = static_cast<uint8_t>(byte);
            }
        }
    }
}

template <int FMT, int RUN>
__global__ void __launch_bounds__(kKvThreads) ead_kv_read_kernel(KvMoveParams p)
{
    const int lane = threadIdx.x & 31;
    const int t0 = first_token(RUN), n = min(RUN, p.batch.n_tokens - t0);
    if (n <= 0) return;
    const KvCacheView &c = p.cache;
    const int per_half = c.heads * c.head_dim, off = blockIdx.y * kKvPass + lane * kKvLaneValues;
    const bool live = off < 2 * per_half, is_v = off >= per_half;
    const int x = off - (is_v ? per_half : 0), head = x / c.head_dim, d = x - head * c.head_dim;
    uint8_t *const row0 = (is_v ? p.rows_v : p.rows_k) + 2 * (t0 * p.row_stride + x);
    const uint8_t *const pool = is_v ? c.v : c.k, *const scales = is_v ? c.v_scale : c.k_scale;
    int pages, slots;
    find_places<false>(p, t0, n, lane, &pages, &slots);
    uint4 in[RUN][FMT == kFmtBf16 ? 2 : 1];
    uint32_t byte[RUN];
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
        const int page = __shfl_sync(0xffffffffu, pages, i), slot = __shfl_sync(0xffffffffu, slots, i);
        in[i][0] = make_uint4(0, 0, 0, 0);         // no place: zeros
        if (FMT == kFmtBf16) in[i][FMT == kFmtBf16] = in[i][0];
        byte[i] = 127;
        if (live && page >= 0) {
            if (FMT == kFmtBf16) {
                const uint8_t *src = pool + 2 * (pool_offset(c, page, head, slot) + d);
                in[i][0] = load_once(src);
                in[i][FMT == kFmtBf16] = load_once(src + 16);
            } else {
                in[i][0] = load_once(pool + pool_offset(c, page, head, slot) + d);
                byte[i] = __ldg(scales + scale_offset(c, page, head, slot) + d / kFmtBlock);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
        if (!live || i >= n) continue;
        uint4 *const row = reinterpret_cast<uint4 *>(row0 + 2 * i * p.row_stride);
        if (FMT == kFmtBf16) {
            row[0] = in[i][0];
            row[1] = in[i][FMT == kFmtBf16];
        } else {
            const float s = scale_value(byte[i]);
            const uint32_t w[4] = {in[i][0].x, in[i][0].y, in[i][0].z, in[i][0].w};
            uint32_t o[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 a = from_e4m3x2(w[k] & 0xffffu), e = from_e4m3x2(w[k] >> 16);
                o[2 * k] = to_bf16x2(a.x * s, a.y * s);
                o[2 * k + 1] = to_bf16x2(e.x * s, e.y * s);
            }
            row[0] = make_uint4(o[0], o[1], o[2], o[3]);
            row[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

}  // namespace ead
