// Root-mean-square norm of every query and key head, and the position rotation, in one pass over a step's projections; the
// results go into tensors (dense) or, with the values, straight into the paged cache in its format:
//   y = x / sqrt(mean(x^2) + eps) * weight,   (a, b) -> (a cos - b sin, b cos + a sin),   angle = position * inv_freq[j]
// A lane holds 8 consecutive elements of a head, a head is 8 or 16 neighbouring lanes: the sum of squares and the partner of a pair
// in the other half of the head come by shuffles, and every element is read once and written once.  The angles of a
// token are computed once per block: the product in 64 bits, brought within half a turn before it is rounded to 32.
#pragma once
#include "quantise_kernel.cuh"

namespace ead {

constexpr int kRopeThreads = 256;
constexpr int kRopeRuns = 2;                      // runs of 32 x 8 elements per warp
constexpr int kRopeBlockValues = kRopeThreads * 8 * kRopeRuns;

struct RopeParams {
    KvCacheView cache;                            // !DENSE
    KvBatchView batch;                            // !DENSE
    const int32_t *positions;                     // DENSE
    const uint8_t *q, *k, *v;
    uint8_t *q_out, *k_out;                       // k_out: DENSE
    int64_t q_stride, kv_stride, q_out_stride, k_out_stride;   // elements between tokens
    const float *inv_freq;
    const uint8_t *q_weight, *k_weight;           // bf16 [dim] or NULL
    int32_t heads_q, heads_kv, dim, rot, interleaved;
    float eps;
    uint32_t *status;
};

// cos and sin of position * freq.
__device__ __forceinline__ float2 rotation(int position, float freq)
{
    double turns = static_cast<double>(position) * static_cast<double>(freq) * 0.15915494309189535;    // 1 / (2 pi)
    turns -= rint(turns);
    float2 cs;
    sincospif(static_cast<float>(2.0 * turns), &cs.y, &cs.x);
    return cs;
}

// One token per block row, blockIdx.y takes the next kRopeBlockValues of its values: all query heads, all key heads and, for the cache, all
// value heads.
template <int FMT, bool DENSE>
__global__ void __launch_bounds__(kRopeThreads) ead_rotate_kernel(RopeParams p)
{
    __shared__ float2 turn[64];
    __shared__ int place[3];                      // position, page, slot
    const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nq = p.heads_q * p.dim, nk = p.heads_kv * p.dim, total = nq + (DENSE ? 1 : 2) * nk;
    uint4 in[kRopeRuns];
    int at[kRopeRuns];
#pragma unroll
    for (int i = 0; i < kRopeRuns; ++i) {
        at[i] = ((blockIdx.y * kRopeRuns + i) * (kRopeThreads / 32) + warp) * 256 + lane * 8;
        in[i] = make_uint4(0, 0, 0, 0);
        if (at[i] < nq)
            in[i] = *reinterpret_cast<const uint4 *>(p.q + 2 * (t * p.q_stride + at[i]));
        else if (at[i] < total)
            in[i] = *reinterpret_cast<const uint4 *>((at[i] < nq + nk ? p.k : p.v) + 2 * (t * p.kv_stride + at[i] - nq - (at[i] < nq + nk ? 0 : nk)));
    }
    if (DENSE) {
        if (threadIdx.x == 0) place[0] = __ldg(p.positions + t);
    } else if (warp == 0) {
        const int b = find_sequence(p.batch.new_start, p.batch.B, t, lane);
        if (lane == 0) {
            const int begin = __ldg(p.batch.new_start + b), end = __ldg(p.batch.new_start + b + 1);
            const bool bad = begin < 0 || t < begin || t >= end || end > p.batch.n_tokens || end - begin > p.batch.max_new;
            const int cached = __ldg(p.batch.kv_len + b) - (end - t);
            const int page = bad ? -1 : find_page(p.cache, p.batch, b, cached);
            if (page < 0 && blockIdx.y == 0) flag_status(p.status, bad ? kStatusBadCount : kStatusBadPage);
            place[0] = p.positions ? __ldg(p.positions + t) : cached;
            place[1] = page;
            place[2] = cached & (p.cache.page_size - 1);
        }
    }
    __syncthreads();
    if (!DENSE && place[1] < 0) return;           // no place: nothing of the token is written
    if (threadIdx.x < p.rot / 2) turn[threadIdx.x] = rotation(place[0], __ldg(p.inv_freq + threadIdx.x));
    __syncthreads();
    const int per_head = p.dim >> 3, in_head = lane & (per_head - 1), e0 = in_head * 8, half = p.rot >> 1;
#pragma unroll
    for (int i = 0; i < kRopeRuns; ++i) {
        if (at[i] - lane * 8 >= total) break;     // the whole warp is past the end
        const bool is_q = at[i] < nq, is_v = at[i] >= nq + nk;
        float y[8];
        unpack8(in[i], y);
        const uint8_t *const weight = is_q ? p.q_weight : p.k_weight;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(y[k], y[k], sum);
        for (int o = 1; o < per_head; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (weight && !is_v) {
            const float r = rsqrtf(sum / static_cast<float>(p.dim) + p.eps);
            float w[8];
            unpack8(__ldg(reinterpret_cast<const uint4 *>(weight) + in_head), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = y[k] * r * w[k];
        }
        const bool low = e0 < half, turned = e0 < p.rot && !is_v;
        if (p.interleaved) {
            if (turned) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 cs = turn[e0 / 2 + k];
                    const float a = y[2 * k], b = y[2 * k + 1];
                    y[2 * k] = a * cs.x - b * cs.y;
                    y[2 * k + 1] = b * cs.x + a * cs.y;
                }
            }
        } else {
            const int partner = e0 < p.rot ? (low ? lane + (half >> 3) : lane - (half >> 3)) : lane;
            float other[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) other[k] = __shfl_sync(0xffffffffu, y[k], partner);
            if (turned) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 cs = turn[(low ? e0 : e0 - half) + k];
                    y[k] = y[k] * cs.x + (low ? -other[k] : other[k]) * cs.y;
                }
            }
        }
        const bool live = at[i] < total;
        if (is_q) {
            *reinterpret_cast<uint4 *>(p.q_out + 2 * (t * p.q_out_stride + at[i])) = pack8(y);
            if (DENSE || FMT == kFmtBf16) continue;
        }
        const int x = at[i] - nq - (is_v ? nk : 0);   // of a key or value
        if (DENSE) {
            if (live) *reinterpret_cast<uint4 *>(p.k_out + 2 * (t * p.k_out_stride + x)) = pack8(y);
            continue;
        }
        uint32_t amax = 0;
        if (FMT == kFmtE4m3) {                    // 4 lanes hold a block of 32 (lanes of a query take part in the exchange)
#pragma unroll
            for (int k = 0; k < 8; ++k) amax = max(amax, abs_bits(y[k]));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        }
        if (is_q || !live) continue;
        const int head = x / p.dim;
        const int64_t to = pool_offset(p.cache, place[1], head, place[2]) + e0;
        uint8_t *const pool = is_v ? p.cache.v : p.cache.k;
        if (FMT == kFmtBf16) {
            *reinterpret_cast<uint4 *>(pool + 2 * to) = pack8(y);
        } else {
            const int byte = scale_byte(amax);
            *reinterpret_cast<uint2 *>(pool + to) = to_e4m3x8(y, inverse_scale(byte));
            if ((lane & 3) == 0)
                (is_v ? p.cache.v_scale : p.cache.k_scale)[scale_offset(p.cache, place[1], head, place[2]) + (e0 >> 5)] = static_cast<uint8_t>(byte);
        }
    }
}

}  // namespace ead
