// Product of 8-bit activations with 8-bit weights, both with power-of-two scales:
//   out[t, n] = sum_k x[t, k] 2^(sx[t, k / block] - 127) w[n, k] 2^(sw[n / 128, k / 128] - 127) + bias[n]
// The tensor core takes the scales itself: tcgen05.mma kind::mxf8f6f4 multiplies every 32 values along K by one power of two
// per row of each operand, read from TMEM, at the rate of the plain 8-bit product; a coarser block repeats its byte.
//
// The weights are the M operand (128 features: exactly one row of scale blocks), the tokens the N operand, so one token costs an
// MMA of 16 columns and not of 128 rows.  A tile is 128 features x up to 240 tokens; two accumulators of 240 columns leave TMEM 32
// columns for two sets of scales, so the next tile's products run under this one's output.
//
// Whole rounds of tiles go to the SMs one each; what is left over is cut along K, every SM an equal stretch, and the
// last block of a tile to finish adds the parts in the order of K: the result does not depend on who comes last.
#pragma once
#include "attn_common.cuh"

namespace ead {

constexpr int kLinThreads = 256;                  // a loading warp, an MMA warp, two warps for scales, four for the output
constexpr int kLinM = 128, kLinK = 128;           // features and values along K of a stage
constexpr int kLinMaxTokens = 240;                // of a tile
constexpr int kLinMaxStages = 12;
constexpr int kLinScaleBytes = 512;               // scales of 128 rows x 4 blocks of 32
constexpr int kLinScaleStage = 3 * kLinScaleBytes;   // weights, then up to 256 tokens
constexpr int kLinScaleColumns = 12;              // the same in TMEM
constexpr int kLinOutBytes = 4096;                // 32 x 32 outputs of a warp
constexpr int kLinSmem = 232448 - 2048;           // beside it: static shared memory and what the system takes
constexpr int kLinMaxCtas = 160;
constexpr size_t kLinCounterBytes = 4096;
constexpr size_t kLinPartFloats = kLinM * kLinMaxTokens;
static_assert(2 * kLinMaxTokens + 2 * kLinScaleColumns <= 512, "TMEM");
static_assert(kLinMaxCtas * sizeof(uint32_t) <= kLinCounterBytes, "fewer tiles than blocks are cut");

struct LinearParams {
    const uint8_t *x_scale, *w_scale, *bias;
    uint8_t *out, *workspace;
    int64_t out_stride;
    int32_t T, N, kblocks;                        // kblocks: of 128
    int32_t x_scale_cols, w_scale_cols;
    int32_t tile_tokens, token_tiles, tiles;
    int32_t whole;                                // tiles in whole rounds
    int32_t rest_ctas;                            // blocks among which the others are cut
    int32_t stages;
    uint32_t *status;
    uint32_t wait_ns, wait_hint;
};

// The stretches of work of one block, in order.
struct LinSegment {
    int tile, k0, k1;
};
struct LinWork {
    int next, stride, whole;                      // whole tiles
    int64_t u, u1;                                // then units (tile, 128 values of K) of the rest
    __device__ __forceinline__ LinWork(const LinearParams &p) : next(blockIdx.x), stride(gridDim.x), whole(p.whole), u(0), u1(0)
    {
        if (static_cast<int>(blockIdx.x) < p.rest_ctas) {
            u = first_unit(p, blockIdx.x);
            u1 = first_unit(p, blockIdx.x + 1);
        }
    }
    static __device__ __forceinline__ int64_t rest_units(const LinearParams &p) { return static_cast<int64_t>(p.tiles - p.whole) * p.kblocks; }
    static __device__ __forceinline__ int64_t first_unit(const LinearParams &p, int cta) { return rest_units(p) * cta / p.rest_ctas; }
    static __device__ __forceinline__ int cta_of(const LinearParams &p, int64_t unit)
    {
        return static_cast<int>(((unit + 1) * p.rest_ctas - 1) / rest_units(p));
    }
    __device__ __forceinline__ bool get(const LinearParams &p, LinSegment &s)
    {
        if (next < whole) {
            s = LinSegment{next, 0, p.kblocks};
            next += stride;
            return true;
        }
        if (u >= u1) return false;
        const int tile = static_cast<int>(u / p.kblocks), k0 = static_cast<int>(u - static_cast<int64_t>(tile) * p.kblocks);
        const int n = static_cast<int>(min(u1 - u, static_cast<int64_t>(p.kblocks - k0)));
        s = LinSegment{whole + tile, k0, k0 + n};
        u += n;
        return true;
    }
};

// Shared-memory descriptor of an operand tile of 128-byte rows with the 128-byte swizzle (as for bf16: it counts bytes), and of a block of
// scales: 32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart.
__device__ __forceinline__ uint64_t scale_smem_desc(uint32_t saddr)
{
    const uint32_t lo = ((saddr >> 4) & 0x3FFFu) | (1u << 16);
    const uint32_t hi = (128u >> 4) | (1u << 14);
    return (static_cast<uint64_t>(hi) << 32) | lo;
}
// Scales of 128 rows from shared memory to 4 columns of TMEM (all four quadrants of lanes get them).
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t saddr)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(scale_smem_desc(saddr)) : "memory");
}
// Instruction descriptor of kind::mxf8f6f4: e4m3 operands (both K-major), scales of type ue8m0, M = 128, N a multiple of 16; `k`: which of
// the four scales of a row this instruction takes.
__device__ __forceinline__ uint32_t umma_idesc_mxf8(uint32_t n, uint32_t k)
{
    return (k << 4) | ((n >> 3) << 17) | (1u << 23) | ((128u >> 7) << 27) | (k << 29);
}
__device__ __forceinline__ void umma_mxf8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t a_scale, uint32_t b_scale,
                                          uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate)
        : "memory");
}

// The scale bytes of the four blocks of 32 in 128 values of one row; of blocks behind the last one 0 (their values are zeros).
template <int BLOCK>
__device__ __forceinline__ uint32_t row_scales(const uint8_t *scale, int cols, int kb)
{
    if (BLOCK == 128) return __ldg(scale + kb) * 0x01010101u;
    if ((cols & 3) == 0) return __ldg(reinterpret_cast<const uint32_t *>(scale) + kb);
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * kb + i < cols) v |= static_cast<uint32_t>(__ldg(scale + 4 * kb + i)) << (8 * i);
    return v;
}

// One warp's 32 features x up to 32 tokens, transposed through its own shared memory: rows of 32 features leave in 16-byte stores.
template <bool F32>
__device__ __forceinline__ void store_outputs(const LinearParams &p, uint8_t *buf, const float (&v)[32], int lane, int feature0, int64_t token0, int tokens)
{
    constexpr int kSize = F32 ? 4 : 2, kPer = 16 / kSize, kLanes = 32 / kPer;     // lanes of a row
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (F32)
            reinterpret_cast<float *>(buf)[j * 32 + lane] = v[j];
        else
            reinterpret_cast<__nv_bfloat16 *>(buf)[j * 32 + lane] = __float2bfloat16_rn(v[j]);
    }
    __syncwarp();
    const int f = feature0 + (lane % kLanes) * kPer;
#pragma unroll
    for (int i = 0; i < kLanes; ++i) {
        const int j = i * (32 / kLanes) + lane / kLanes;
        if (j >= tokens) break;
        const uint4 x = reinterpret_cast<const uint4 *>(buf)[j * kLanes + lane % kLanes];
        uint8_t *const to = p.out + kSize * ((token0 + j) * p.out_stride + f);
        if (f + kPer <= p.N) {
            *reinterpret_cast<uint4 *>(to) = x;
        } else {
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (f + e < p.N) {
                    if (F32)
                        reinterpret_cast<uint32_t *>(to)[e] = w[e];
                    else
                        reinterpret_cast<uint16_t *>(to)[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                }
        }
    }
}

template <int BLOCK, bool F32>
__global__ void __launch_bounds__(kLinThreads, 1)
    ead_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, LinearParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_bars[3 * kLinMaxStages + 5];
    __shared__ uint32_t s_tmem, s_gave_up;
    __shared__ int s_last, s_loads;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    const int S = p.stages, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t x_bytes = p.tile_tokens * kLinK, stage_bytes = kLinM * kLinK + x_bytes;
    const uint32_t scales = base + S * stage_bytes, out_smem = scales + S * kLinScaleStage;
    const uint32_t bar_tile = smem_u32(s_bars), bar_scale = bar_tile + 8 * kLinMaxStages, bar_empty = bar_scale + 8 * kLinMaxStages;
    const uint32_t bar_acc_full = bar_empty + 8 * kLinMaxStages, bar_acc_empty = bar_acc_full + 16, bar_last = bar_acc_empty + 16;
    const int chunks = (p.tile_tokens + 127) >> 7;
    if (tid == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(bar_tile + 8 * i, 1);
            mbar_init(bar_scale + 8 * i, 2);
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_acc_full + 8 * i, 1);
            mbar_init(bar_acc_empty + 8 * i, 4);
        }
        mbar_init(bar_last, 1);
        s_gave_up = 0;
        s_loads = 0;
        fence_mbar_init();
    }
    if (tid == 32) {
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmX);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&s_tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&s_tmem);
    // A wait that runs out makes every other role stop at its next one that does.
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_phase<true>(bar, parity, p, &s_gave_up); };
    auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    LinWork work(p);
    LinSegment g;
    uint32_t it = 0;                              // stages so far

    if (warp == 0) {
        // ------------------------------------------------------------- operand tiles
        bool go = true;
        while (go && work.get(p, g)) {
            const int feature0 = (g.tile / p.token_tiles) * kLinM, token0 = (g.tile % p.token_tiles) * p.tile_tokens;
            for (int kb = g.k0; kb < g.k1; ++kb, ++it) {
                const int st = it % S;
                if (!(go = warp_wait(bar_empty + 8 * st, ((it / S) & 1) ^ 1))) break;
                if (elect_one()) {
                    const uint32_t a = base + st * stage_bytes;
                    mbar_arrive_expect_tx(bar_tile + 8 * st, stage_bytes);
                    tma_load_2d(a, &tmW, kb * kLinK, feature0, bar_tile + 8 * st);
                    tma_load_2d(a + kLinM * kLinK, &tmX, kb * kLinK, token0, bar_tile + 8 * st);
                }
                __syncwarp();
            }
        }
        if (lane == 0) s_loads = it;
    } else if (warp == 1) {
        // ------------------------------------------------------------- products
        bool go = true;
        for (uint32_t n = 0; go && work.get(p, g); ++n) {
            const uint32_t acc = tmem + (n & 1) * kLinMaxTokens;
            if (!(go = warp_wait(bar_acc_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1))) break;
            for (int kb = g.k0; kb < g.k1; ++kb, ++it) {
                const int st = it % S;
                // the set of scales was used two stages ago
                if (it >= 2 && !(go = warp_wait(bar_empty + 8 * ((it - 2) % S), ((it - 2) / S) & 1))) break;
                if (!(go = warp_wait(bar_tile + 8 * st, (it / S) & 1) && warp_wait(bar_scale + 8 * st, (it / S) & 1))) break;
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t a = base + st * stage_bytes, sc = scales + st * kLinScaleStage;
                    const uint32_t ta = tmem + 2 * kLinMaxTokens + (it & 1) * kLinScaleColumns, tb = ta + 4;
                    copy_scales(ta, sc);
                    for (int c = 0; c < chunks; ++c) copy_scales(tb + 4 * c, sc + (1 + c) * kLinScaleBytes);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        umma_mxf8(acc, umma_smem_desc(a + 32 * k), umma_smem_desc(a + kLinM * kLinK + 32 * k), umma_idesc_mxf8(p.tile_tokens, k), ta, tb,
                                  kb > g.k0 || k > 0);
                    umma_commit(bar_empty + 8 * st);
                    if (kb + 1 == g.k1) umma_commit(bar_acc_full + 8 * (n & 1));
                }
                __syncwarp();
            }
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------- scales: 128 tokens a warp, the second warp the weights' too
        const int c = warp - 2;
        bool go = true;
        while (go && work.get(p, g)) {
            const int feature_tile = g.tile / p.token_tiles, token0 = (g.tile % p.token_tiles) * p.tile_tokens + c * 128 + lane;
            const int end = min(p.T, (g.tile % p.token_tiles + 1) * p.tile_tokens);
            for (int kb0 = g.k0; go && kb0 < g.k1; kb0 += 4) {
                uint32_t v[4][4], w[4];           // four stages' loads before the first wait
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = c == 1 && kb0 + i < g.k1 ? __ldg(p.w_scale + static_cast<int64_t>(feature_tile) * p.w_scale_cols + kb0 + i) * 0x01010101u : 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = token0 + 32 * j;
                        v[i][j] = t < end && kb0 + i < g.k1 ? row_scales<BLOCK>(p.x_scale + static_cast<int64_t>(t) * p.x_scale_cols, p.x_scale_cols, kb0 + i) : 0;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (kb0 + i >= g.k1) break;
                    const int st = it % S;
                    if (!(go = warp_wait(bar_empty + 8 * st, ((it / S) & 1) ^ 1))) break;
                    const uint32_t to = scales + st * kLinScaleStage + 16 * lane;
                    if (c < chunks) st_shared_16(to + (1 + c) * kLinScaleBytes, v[i][0], v[i][1], v[i][2], v[i][3]);
                    if (c == 1) st_shared_16(to, w[i], w[i], w[i], w[i]);
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_scale + 8 * st);
                    ++it;
                }
            }
        }
    } else {
        // ------------------------------------------------------------- output
        const int quadrant = warp - 4, row = quadrant * 32 + lane;
        uint8_t *const buf = smem_raw + (out_smem - raw) + quadrant * kLinOutBytes;
        float *const parts = reinterpret_cast<float *>(p.workspace + kLinCounterBytes);
        for (uint32_t n = 0; work.get(p, g); ++n) {
            const int feature0 = (g.tile / p.token_tiles) * kLinM + quadrant * 32, token0 = (g.tile % p.token_tiles) * p.tile_tokens;
            const int tokens = min(p.tile_tokens, p.T - token0);
            const bool part = g.k1 - g.k0 < p.kblocks;
            if (!named_all(1, 128, warp_wait(bar_acc_full + 8 * (n & 1), (n >> 1) & 1))) break;
            tc_fence_after_sync();
            const uint32_t acc = tmem + (n & 1) * kLinMaxTokens + (static_cast<uint32_t>(quadrant) << 21);
            const float bias = p.bias && feature0 + lane < p.N ? __uint_as_float(static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t *>(p.bias) + feature0 + lane)) << 16) : 0.f;
            // a block has at most two parts: of the tile that began in an earlier block (or with its stretch), and of the next one
            const int64_t tile_unit = static_cast<int64_t>(g.tile - p.whole) * p.kblocks;
            float *const mine = parts + (2 * blockIdx.x + (LinWork::first_unit(p, blockIdx.x) < tile_unit)) * kLinPartFloats + row;
            for (int c = 0; c < tokens; c += 32) {
                float v[32];
                tmem_ld_32cols(acc + c, v);
                if (part) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c + j < tokens) __stcg(mine + (c + j) * kLinM, v[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += bias;
                    store_outputs<F32>(p, buf, v, lane, feature0, token0 + c, tokens - c);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_acc_empty + 8 * (n & 1));
            if (!part) continue;
            fence_gpu();
            named_sync(1, 128);
            const int first = LinWork::cta_of(p, tile_unit), last = LinWork::cta_of(p, tile_unit + p.kblocks - 1);
            uint32_t *const counter = reinterpret_cast<uint32_t *>(p.workspace) + (g.tile - p.whole);
            if (tid == 128) s_last = atomicAdd(counter, 1u) == static_cast<uint32_t>(last - first);
            named_sync(1, 128);
            if (s_last) {
                fence_gpu();
                for (int c = 0; c < tokens; c += 32) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0.f;
                    for (int i = first; i <= last; ++i) {
                        const float *const from = parts + (2 * i + (LinWork::first_unit(p, i) < tile_unit)) * kLinPartFloats + row;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (c + j < tokens) v[j] += __ldcg(from + (c + j) * kLinM);
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += bias;
                    store_outputs<F32>(p, buf, v, lane, feature0, token0 + c, tokens - c);
                }
                if (tid == 128) *counter = 0;     // ready for the next call
            }
            named_sync(1, 128);                   // s_last may be written again
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (s_gave_up) {                              // nobody sets it any more: wait for loads and products under way
        if (warp == 0)
            for (int i = max(0, s_loads - S); i < s_loads; ++i) wait_own(bar_tile + 8 * (i % S), (i / S) & 1);
        if (warp == 1) {
            if (elect_one()) umma_commit(bar_last);
            __syncwarp();
            wait_own(bar_last, 0);
        }
        __syncthreads();
    }
    if (warp == 1) tmem_dealloc(tmem, 512);
}

}  // namespace ead
