// Product of 8-bit activations with 8-bit weights, both with power-of-two scales:
//   out[t, n] = sum_k x[t, k] 2^(sx[t, k / block] - 127) w[n, k] 2^(sw[n / 128, k / 128] - 127) + bias[n]
// The tensor core takes the scales itself: tcgen05.mma kind::mxf8f6f4 multiplies every 32 values along K by one power of two
// per row of each operand, read from TMEM, at the rate of the plain 8-bit product.
//
// The weights are the M operand (128 features: exactly one row of scale blocks), the tokens the N operand, so one token costs an
// MMA of 16 columns and not of 128 rows.  Two accumulators leave room in TMEM for the scales of two groups of 4 x 128 values of K:
// the next tile's products run under this one's output, the next group's scales come in under this one's products.
//
// Few tokens (PAIR = false): a tile is 128 features of one block.  Whole rounds of tiles go to the blocks one each; what is left over is
// cut along K among the blocks of a cluster, which add their parts up in the order of K through distributed shared memory.
// Many tokens (PAIR = true): two blocks share a tile of 256 features (cta_group::2), each holds its features' weights and half of the
// tokens: per product a third less passes through L2, which bounds the other form at size.
//
// What bounds it, measured.  4099 x 7168 x 5120: 111-114 us in short runs of a replayed graph, 2.64-2.70 PFLOP/s, 0.79-0.81 of twice the device's bf16
// burst rate, with the tensor pipe busy 80 % of the time; 130-135 us in calls one after another, whose clock the power limit sets: 2.23-2.31 PFLOP/s,
// 0.80-0.82 of twice the sustained rate.  A head of 152064 x 1536 for 61 tokens into 32 bits: 46-50 us either way, 5.4-5.9 TB/s, 0.83-0.90 of the copy rate.
// The sizes below take 0.1-0.4 us more in calls.
// 64 tokens x 7168 x 5120: 10.8 us: the 37 MB stream in 6 us, the rest is the way to the first product (2.5 us: launch, barriers, first loads from
// HBM) and from the last one (2.3 us: parts through the cluster, output).  347 x 5000 x 4128: 13.8 us: 33 stages of about 350 cycles for
// 256 cycles of products, which is what 24 KB in and 40 KB out of shared memory take, and the same two ends.  One token x 2048 x 1536: 4.3 us.
// A narrow output of a long sum is served worst where pairs begin, as they have no cut along K: 1536 x 8960, 160 tokens 10.5-13.8 us, 161 19.4, 200 19.2.
//
// Steps that mattered (us; 4099 tokens / 64 / 347): blocks of 128 x 240 with two sets of scales in TMEM and parts joined through global memory 252 / 34 / 50;
// pairs, groups of scales, clusters, one issuing thread 183 / 14.3 / 23; its loop unrolled, four warps for scales, parts fetched 32 at a time 131 / 11.5 / 17;
// setup under the end of the kernel before 131 / 10.7 / 16; tiles by measured cost 115; eight warps for scales 113 / - / 14.5; a row's scales of four stages in one
// load 111 / 10.8 / 13.8.  Tried and not kept: the first weights brought into L2 before the wait for the kernel before (64 tokens 11.2); a group's scales
// loaded before the last one's arrival (the arrival waits for the loads); parts sent to the block that adds them up instead of fetched by it (one token 7.2,
// 64 tokens 13.1: the barrier then waits for the remote stores).
#pragma once
#include "attn_common.cuh"

namespace ead {

constexpr int kLinM = 128, kLinK = 128;           // features and values along K of a stage
constexpr int kLinMaxStages = 12;
constexpr int kLinMaxGroups = 4;
constexpr int kLinScaleBytes = 512;               // scales of 128 rows x 4 blocks along K
constexpr int kLinOutBytes = 4096;                // 32 x 32 outputs of a warp
constexpr int kLinSmem = 232448 - 2048;           // beside it: static shared memory and what the system takes
constexpr int kLinMaxSplit = 8;                   // blocks of a cluster

// BLOCK: values of a token that share a scale.  With 128 the four bytes of a TMEM column serve four stages, with 32 one.
template <int BLOCK, bool PAIR>
struct LinLayout {
    // Pairs of warps that bring groups of scales in turns, and groups in shared memory.  A pair's group takes longest on its way (its arrival
    // crosses to the other block): four against two turns, 4099 x 7168 x 5120: 112 against 115 us, blocks of 32 124 against 153; a single block's
    // first group comes later the more of them load at a time: 64 tokens 10.9 us with two, 11.2 with four, 200 tokens 22.4 and 28.5.
    static constexpr int kTurns = PAIR ? 4 : 2, kGroups = PAIR ? 4 : 3;
    static constexpr int kThreads = 32 * (6 + 2 * kTurns);       // a loading warp, an MMA warp, the warps for scales, four for the output
    static_assert(kGroups <= kLinMaxGroups, "barriers");
    static constexpr int kTokenSets = BLOCK == 128 ? 1 : 4;                          // sets of token scales in a group
    static constexpr int kMaxTokens = BLOCK == 128 ? 240 : 208;                      // of a tile
    static constexpr int kGroupBytes = kLinScaleBytes * (1 + 2 * kTokenSets);        // weights, then up to 256 tokens per set
    static constexpr int kGroupColumns = 4 + 8 * kTokenSets;
    static_assert(2 * kMaxTokens + 2 * kGroupColumns <= 512, "TMEM");
    __host__ __device__ static constexpr int stage_bytes(int tile_tokens) { return kLinM * kLinK + (PAIR ? tile_tokens / 2 : tile_tokens) * kLinK; }
    __host__ __device__ static constexpr int fixed_bytes() { return 1024 + kGroups * kGroupBytes + 4 * kLinOutBytes; }
};

struct LinearParams {
    const uint8_t *x_scale, *w_scale, *bias;
    uint8_t *out;
    int64_t out_stride;
    int32_t T, N, kblocks;                        // kblocks: of 128
    int32_t x_scale_cols, w_scale_cols;
    int32_t tile_tokens, token_tiles;
    int32_t whole;                                // tiles that are served by one block (PAIR: by one pair) each
    int32_t rest;                                 // tiles behind them, one cluster each
    int32_t split;                                // blocks of a cluster (PAIR: 2)
    int32_t stages;
    int32_t wide;                                 // the output's rows are 16-byte aligned
    uint32_t *status;
    uint32_t wait_ns, wait_hint;
};

// ----------------------------------------------------------------- clusters
__device__ __forceinline__ int cluster_id()
{
    int i;
    asm("mov.u32 %0, %%clusterid.x;" : "=r"(i));
    return i;
}
__device__ __forceinline__ int cluster_rank()
{
    int i;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(i));
    return i;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Address in the shared memory of block `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void cluster_mbar_arrive(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ uint32_t cluster_ld_u32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_st(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ float cluster_ld(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// The stretches of work of one block, in order.
struct LinSegment {
    int tile, k0, k1;
};
template <bool PAIR>
struct LinWork {
    int next;
    // Row block of the weights and tile of tokens.  (With few tokens there is one tile of them.)
    static __device__ __forceinline__ int feature_tile(const LinearParams &p, const LinSegment &s, int rank) { return PAIR ? s.tile / p.token_tiles * 2 + rank : s.tile; }
    static __device__ __forceinline__ int token0(const LinearParams &p, const LinSegment &s) { return PAIR ? s.tile % p.token_tiles * p.tile_tokens : 0; }
    __device__ __forceinline__ LinWork() : next(PAIR ? blockIdx.x / 2 : blockIdx.x) {}
    __device__ __forceinline__ bool get(const LinearParams &p, LinSegment &s)
    {
        if (next < 0) return false;
        if (next < p.whole) {
            s = LinSegment{next, 0, p.kblocks};
            next += PAIR ? gridDim.x / 2 : gridDim.x;
            return true;
        }
        next = -1;
        if (PAIR) return false;
        const int cluster = cluster_id(), rank = cluster_rank();
        if (cluster >= p.rest) return false;
        s = LinSegment{p.whole + cluster, p.kblocks * rank / p.split, p.kblocks * (rank + 1) / p.split};     // (at most 2^23 x 8)
        return true;
    }
};

// Place in a ring of n barriers, and the parity of the phase that ends there next.  (Counted on: divisions by n in every stage were
// a third of the time of the warp that issues the products.)
struct LinRing {
    uint32_t i = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t n)
    {
        if (++i == n) {
            i = 0;
            phase ^= 1;
        }
    }
};

// Shared-memory descriptor of a block of scales: 32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart.  (An operand tile of
// 128-byte rows with the 128-byte swizzle has the descriptor of a bf16 one, which counts bytes.)
__device__ __forceinline__ uint64_t scale_smem_desc(uint32_t saddr)
{
    const uint32_t lo = ((saddr >> 4) & 0x3FFFu) | (1u << 16);
    const uint32_t hi = (128u >> 4) | (1u << 14);
    return (static_cast<uint64_t>(hi) << 32) | lo;
}
// Scales of 128 rows from shared memory to 4 columns of TMEM (all four quadrants of lanes get them); of a pair, each block from its own
// shared memory to its own TMEM.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t saddr)
{
    if (PAIR)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(scale_smem_desc(saddr)) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(scale_smem_desc(saddr)) : "memory");
}
// Instruction descriptor of kind::mxf8f6f4: e4m3 operands (both K-major), scales of type ue8m0, M = 128 (of a pair 256), N a multiple of 16;
// ka, kb: which of the four scales of a row of A and B this instruction takes.
template <bool PAIR>
__device__ __forceinline__ uint32_t umma_idesc_mxf8(uint32_t n, uint32_t ka, uint32_t kb)
{
    return (kb << 4) | ((n >> 3) << 17) | (1u << 23) | ((PAIR ? 2u : 1u) << 27) | (ka << 29);
}
template <bool PAIR>
__device__ __forceinline__ void umma_mxf8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t a_scale, uint32_t b_scale,
                                          uint32_t accumulate)
{
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate)
            : "memory");
}
// Arrives on the barrier (of a pair: on the one at this place in both blocks) when everything issued so far by this thread has completed.
template <bool PAIR>
__device__ __forceinline__ void lin_commit(uint32_t bar)
{
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"(static_cast<uint16_t>(3)) : "memory");
    else
        umma_commit(bar);
}
// The same on this block's barrier alone.
template <bool PAIR>
__device__ __forceinline__ void umma_commit_own(uint32_t bar)
{
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        umma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void lin_tmem_alloc(uint32_t result)
{
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(result) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tmem_alloc(result, 512);
        tmem_relinquish();
    }
}
template <bool PAIR>
__device__ __forceinline__ void lin_tmem_dealloc(uint32_t tmem)
{
    if (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else
        tmem_dealloc(tmem, 512);
}

// A tiled load of one block of a pair, counted on the leading block's barrier (bar: its address in this block's own window; the bit that
// tells the two blocks apart is cleared).
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const void *tmap, int32_t x, int32_t y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(bar & 0xFEFFFFFFu)
        : "memory");
}
// Counts bytes that nobody will bring.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// n (at most 4) consecutive bytes from any address, 0 behind them, by two aligned loads without a branch (a branch around a load keeps the next
// one from being issued under it).  p is the address of a byte that is there; a word is only read if it has one.
__device__ __forceinline__ uint32_t load_bytes(const uint8_t *p, int n)
{
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 3u;
    const uint32_t *const word = reinterpret_cast<const uint32_t *>(p - off);
    const uint32_t lo = ld_behind(word), hi = ld_behind(word + (static_cast<int>(off) + n > 4));
    return __funnelshift_r(lo, hi, 8 * off) & (n >= 4 ? 0xffffffffu : (1u << (8 * max(n, 0))) - 1);
}

// A group of scales on its way from global to shared memory: of 4 x 32 tokens for up to four stages, and of the weights.
template <int BLOCK, bool PAIR>
struct LinScales {
    static constexpr int kSets = LinLayout<BLOCK, PAIR>::kTokenSets;
    uint32_t v[kSets][4], w;
    // c: which 128 tokens of the tile.  What belongs to no token or stage may be anything: such rows and columns are not stored, and values behind a
    // row's end are zeros (their scales are not NaN: 0).
    __device__ __forceinline__ void load(const LinearParams &p, const LinSegment &g, int kb, int c, int lane, int rank)
    {
        const int first = LinWork<PAIR>::token0(p, g), last = min(p.T, first + p.tile_tokens) - 1, n = min(4, g.k1 - kb), cols = p.x_scale_cols;
        const int at = BLOCK == 128 ? kb : 4 * kb;
        const uint8_t *row[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) row[j] = p.x_scale + static_cast<int64_t>(min(first + c * 128 + 32 * j + lane, last)) * cols + at;
        const uint32_t odd = cols | at | static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p.x_scale));      // alignment of all rows' pieces
        if (BLOCK == 128) {                       // of four stages one byte each
            if ((odd & 3) == 0 && n == 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[0][j] = ld_behind(reinterpret_cast<const uint32_t *>(row[j]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[0][j] = load_bytes(row[j], n);
            }
        } else if ((odd & 15) == 0) {             // of four stages four bytes each
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 x = ld_behind(reinterpret_cast<const uint4 *>(row[j]));
                v[0][j] = x.x;
                v[kSets - 3][j] = x.y;
                v[kSets - 2][j] = x.z;
                v[kSets - 1][j] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSets; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int count = i < n ? min(4, cols - at - 4 * i) : 0;
                    v[i][j] = load_bytes(count > 0 ? row[j] + 4 * i : p.x_scale, count);
                }
        }
        const int feature_tile = min(LinWork<PAIR>::feature_tile(p, g, rank), (p.N - 1) / kLinM);
        w = c == 1 ? load_bytes(p.w_scale + static_cast<int64_t>(feature_tile) * p.w_scale_cols + kb, n) : 0;
    }
    __device__ __forceinline__ void store(uint32_t group, int c, int chunks, int lane) const
    {
        const uint32_t to = group + 16 * lane;
        if (c < chunks)
#pragma unroll
            for (int i = 0; i < kSets; ++i) st_shared_16(to + (1 + 2 * i + c) * kLinScaleBytes, v[i][0], v[i][1], v[i][2], v[i][3]);
        if (c == 1) st_shared_16(to, w, w, w, w);
    }
};

// One warp's 32 features x up to 32 tokens, transposed through its own shared memory: rows of 32 features leave in 16-byte stores.  (Where the
// output's rows are not aligned for that, an element per lane.)
template <bool F32>
__device__ __forceinline__ void store_outputs(const LinearParams &p, uint8_t *buf, const float (&v)[32], int lane, int feature0, int64_t token0, int tokens)
{
    constexpr int kSize = F32 ? 4 : 2, kPer = 16 / kSize, kLanes = 32 / kPer;     // lanes of a row
    if (!p.wide) {
        uint8_t *const to = p.out + kSize * (token0 * p.out_stride + feature0 + lane);
        if (feature0 + lane < p.N)
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                if (j >= tokens) break;
                if (F32)
                    *reinterpret_cast<float *>(to + kSize * j * p.out_stride) = v[j];
                else
                    *reinterpret_cast<__nv_bfloat16 *>(to + kSize * j * p.out_stride) = __float2bfloat16_rn(v[j]);
            }
        return;
    }
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

// Sums of the cluster's parts of one feature and up to 32 tokens, in the order of the blocks; `at`: the first one's place in each block's shared
// memory.  32 loads are on their way at a time.
template <int R>
__device__ __forceinline__ void add_parts(float (&v)[32], uint32_t at, int split, int tokens)
{
    constexpr int J = 32 / R;
    uint32_t from[R];
#pragma unroll
    for (int r = 0; r < R; ++r) from[r] = cluster_addr(at, min(r, split - 1));
#pragma unroll
    for (int j0 = 0; j0 < 32; j0 += J) {
        if (j0 >= tokens) break;
        float part[R][J];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < J; ++j) part[r][j] = r < split && j0 + j < tokens ? cluster_ld(from[r] + 4 * (j0 + j) * kLinM) : 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            v[j0 + j] = part[0][j];
#pragma unroll
            for (int r = 1; r < R; ++r) v[j0 + j] += part[r][j];
        }
    }
}

template <int BLOCK, bool F32, bool PAIR>
__global__ void __launch_bounds__(LinLayout<BLOCK, PAIR>::kThreads, 1)
    ead_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ LinearParams p)
{
    using L = LinLayout<BLOCK, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_bars[2 * kLinMaxStages + 2 * kLinMaxGroups + 5];
    __shared__ uint32_t s_tmem, s_gave_up, s_peer_gave_up;
    __shared__ int s_loads;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t S = p.stages;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank();
    const int pair_rank = PAIR ? rank : 0;
    const uint32_t stage_bytes = L::stage_bytes(p.tile_tokens);
    const uint32_t groups = base + S * stage_bytes, out_smem = groups + L::kGroups * L::kGroupBytes;
    // tile and empty per stage, scales and empty per group (of a pair, what comes in is counted in the leading block for both)
    const uint32_t bar_tile = smem_u32(s_bars), bar_empty = bar_tile + 8 * kLinMaxStages;
    const uint32_t bar_scale = bar_empty + 8 * kLinMaxStages, bar_scale_empty = bar_scale + 8 * kLinMaxGroups;
    const uint32_t bar_acc_full = bar_scale_empty + 8 * kLinMaxGroups, bar_acc_empty = bar_acc_full + 16, bar_last = bar_acc_empty + 16;
    const int chunks = (p.tile_tokens + 127) >> 7;
    if (tid == 0) {
        for (uint32_t i = 0; i < S; ++i) {
            mbar_init(bar_tile + 8 * i, 1);
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int i = 0; i < L::kGroups; ++i) {
            mbar_init(bar_scale + 8 * i, PAIR ? 4 : 2);
            mbar_init(bar_scale_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_acc_full + 8 * i, 1);
            mbar_init(bar_acc_empty + 8 * i, PAIR ? 8 : 4);
        }
        mbar_init(bar_last, 1);
        s_gave_up = s_peer_gave_up = 0;
        s_loads = 0;
        fence_mbar_init();
    }
    if (tid == 32) {
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmX);
    }
    if (warp == 1) lin_tmem_alloc<PAIR>(smem_u32(&s_tmem));
    tc_fence_before_sync();
    __syncthreads();
    if (PAIR) {                                   // the other block's barriers are there
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_after_sync();
    griddep_wait();                               // nothing above touches global memory: it runs under the end of the kernel before
    griddep_launch_dependents();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&s_tmem);
    // A wait that runs out makes every other role of the block stop at its next one that does.
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_phase<true>(bar, parity, p, &s_gave_up); };
    auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    LinWork<PAIR> work;
    LinSegment g;
    LinRing stage, group;

    if (warp == 0) {
        // ------------------------------------------------------------- operand tiles
        if (elect_one()) {
            const int x_rows = PAIR ? p.tile_tokens / 2 : p.tile_tokens;
            int loads = 0;
            bool go = true;
            while (go && work.get(p, g)) {
                const int feature0 = LinWork<PAIR>::feature_tile(p, g, pair_rank) * kLinM, token0 = LinWork<PAIR>::token0(p, g) + pair_rank * x_rows;
                for (int kb = g.k0; kb < g.k1; ++kb) {
                    if (!(go = wait(bar_empty + 8 * stage.i, stage.phase ^ 1))) break;
                    const uint32_t a = base + stage.i * stage_bytes, bar = bar_tile + 8 * stage.i;
                    if (PAIR) {
                        if (pair_rank == 0) mbar_arrive_expect_tx(bar, 2 * stage_bytes);
                        pair_load_2d(a, &tmW, kb * kLinK, feature0, bar);
                        pair_load_2d(a + kLinM * kLinK, &tmX, kb * kLinK, token0, bar);
                    } else {
                        mbar_arrive_expect_tx(bar, stage_bytes);
                        tma_load_2d(a, &tmW, kb * kLinK, feature0, bar);
                        tma_load_2d(a + kLinM * kLinK, &tmX, kb * kLinK, token0, bar);
                    }
                    stage.next(S);
                    ++loads;
                }
            }
            s_loads = loads;
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------- products (of a pair: by the leading block)
        if (pair_rank == 0 && elect_one()) {
            const uint32_t a0 = static_cast<uint32_t>(umma_smem_desc(base)), a_step = stage_bytes >> 4;
            const uint64_t desc_hi = umma_smem_desc(0) & 0xffffffff00000000ull;
            const uint32_t idesc = umma_idesc_mxf8<PAIR>(p.tile_tokens, 0, 0);
            uint32_t n_groups = 0;
            bool go = true;
            for (uint32_t n = 0; go && work.get(p, g); ++n) {
                const uint32_t acc = tmem + (n & 1) * L::kMaxTokens;
                go = wait(bar_acc_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1);
                for (int kb = g.k0; go && kb < g.k1; kb += 4) {
                    const uint32_t ta = tmem + 2 * L::kMaxTokens + (n_groups & 1) * L::kGroupColumns, tb = ta + 4;
                    // the columns were used two groups ago
                    if (n_groups >= 2)
                        go = group.i >= 2 ? wait(bar_scale_empty + 8 * (group.i - 2), group.phase) : wait(bar_scale_empty + 8 * (group.i + L::kGroups - 2), group.phase ^ 1);
                    go = go && wait(bar_scale + 8 * group.i, group.phase);
                    if (!go) break;
                    tc_fence_after_sync();
                    const uint32_t sc = groups + group.i * L::kGroupBytes;
                    copy_scales<PAIR>(ta, sc);
#pragma unroll
                    for (int i = 0; i < L::kTokenSets; ++i) {
                        copy_scales<PAIR>(tb + 8 * i, sc + (1 + 2 * i) * kLinScaleBytes);
                        if (chunks > 1) copy_scales<PAIR>(tb + 8 * i + 4, sc + (2 + 2 * i) * kLinScaleBytes);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) {    // unrolled: the way round a loop costs this thread 170 cycles
                        if (kb + static_cast<int>(j) >= g.k1) break;
                        go = go && wait(bar_tile + 8 * stage.i, stage.phase);
                        if (!go) break;
                        tc_fence_after_sync();
                        const uint32_t a = a0 + stage.i * a_step, b = a + (kLinM * kLinK >> 4);
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k)
                            umma_mxf8<PAIR>(acc, desc_hi | (a + 2 * k), desc_hi | (b + 2 * k), idesc + (j << 29) + ((BLOCK == 128 ? j : k) << 4), ta,
                                            BLOCK == 128 ? tb : tb + 8 * j, kb > g.k0 || j > 0 || k > 0);
                        lin_commit<PAIR>(bar_empty + 8 * stage.i);
                        stage.next(S);
                    }
                    lin_commit<PAIR>(bar_scale_empty + 8 * group.i);
                    group.next(L::kGroups);
                    ++n_groups;
                }
                if (go) lin_commit<PAIR>(bar_acc_full + 8 * (n & 1));
            }
        }
    } else if (warp < 2 + 2 * L::kTurns) {
        // ------------------------------------------------------------- scales: 128 tokens a warp, the second warp of two the weights' too; two
        // of these warps take every L::kTurns-th group (a group's way through one warp is longer than its products take)
        const int c = warp & 1, turn = (warp - 2) >> 1;
        uint32_t n_groups = 0;
        const uint32_t leader_scale = PAIR ? cluster_addr(bar_scale, 0) : 0;
        bool go = true;
        while (go && work.get(p, g))
            for (int kb = g.k0; kb < g.k1; kb += 4, group.next(L::kGroups), ++n_groups) {
                if (n_groups % L::kTurns != turn) continue;
                LinScales<BLOCK, PAIR> sc;        // (loads of the next group before this one's arrival would hold it up: it waits for them)
                sc.load(p, g, kb, c, lane, pair_rank);
                if (!(go = warp_wait(bar_scale_empty + 8 * group.i, group.phase ^ 1))) break;
                sc.store(groups + group.i * L::kGroupBytes, c, chunks, lane);
                fence_async_shared();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR)
                        cluster_mbar_arrive(leader_scale + 8 * group.i);
                    else
                        mbar_arrive(bar_scale + 8 * group.i);
                }
            }
    } else {
        // ------------------------------------------------------------- output
        const int quadrant = warp & 3, row = quadrant * 32 + lane;      // a warp reads the TMEM lanes of its place in four
        uint8_t *const buf = smem_raw + (out_smem - raw) + quadrant * kLinOutBytes;
        const uint32_t leader_acc_empty = PAIR ? cluster_addr(bar_acc_empty, 0) : 0;
        bool joins = false;
        int feature0 = 0, token0 = 0, tokens = 0;
        float bias = 0.f;
        for (uint32_t n = 0; work.get(p, g); ++n) {
            feature0 = LinWork<PAIR>::feature_tile(p, g, pair_rank) * kLinM + quadrant * 32;
            token0 = LinWork<PAIR>::token0(p, g);
            tokens = min(p.tile_tokens, p.T - token0);
            joins = !PAIR && p.split > 1 && g.tile >= p.whole;
            bias = p.bias && feature0 + lane < p.N ? __uint_as_float(static_cast<uint32_t>(ld_behind(reinterpret_cast<const uint16_t *>(p.bias) + feature0 + lane)) << 16) : 0.f;
            if (!warp_wait(bar_acc_full + 8 * (n & 1), (n >> 1) & 1)) break;
            tc_fence_after_sync();
            const uint32_t acc = tmem + (n & 1) * L::kMaxTokens + (static_cast<uint32_t>(quadrant) << 21);
            for (int c = 0; c < tokens; c += 32) {
                float v[32];
                tmem_ld_32cols(acc + c, v);
                if (joins) {                      // the last stretch of the block: the stages' place is free for it
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c + j < tokens) asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + 4 * ((c + j) * kLinM + row)), "f"(v[j]) : "memory");
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += bias;
                    store_outputs<F32>(p, buf, v, lane, feature0, token0 + c, tokens - c);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (PAIR)
                    cluster_mbar_arrive(leader_acc_empty + 8 * (n & 1));
                else
                    mbar_arrive(bar_acc_empty + 8 * (n & 1));
            }
        }
        if (!PAIR && p.split > 1 && p.rest) {
            __syncwarp();
            cluster_arrive();                     // (the other warps: below)
            cluster_wait();
            if (joins) {                          // every block adds up and stores its share of the tokens
                const int c0 = tokens * rank / p.split, c1 = tokens * (rank + 1) / p.split;
                for (int c = c0; c < c1; c += 32) {
                    float v[32];
                    const uint32_t at = base + 4 * (c * kLinM + row);
                    if (p.split <= 2)
                        add_parts<2>(v, at, p.split, c1 - c);
                    else if (p.split <= 4)
                        add_parts<4>(v, at, p.split, c1 - c);
                    else
                        add_parts<8>(v, at, p.split, c1 - c);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += bias;
                    store_outputs<F32>(p, buf, v, lane, feature0, token0 + c, c1 - c);
                }
            }
        }
    }
    __syncwarp();
    if (!PAIR && p.split > 1 && p.rest && warp < 2 + 2 * L::kTurns) {
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (PAIR) {                                   // neither block leaves, or ends the other way below, before the other one is done
        if (tid == 0 && s_gave_up) cluster_st(cluster_addr(smem_u32(&s_peer_gave_up), pair_rank ^ 1), 1u);
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (s_gave_up || s_peer_gave_up) {            // nobody sets it any more: wait for loads and products under way
        if (warp == 0 && lane == 0 && pair_rank == 0) {
            const int n = static_cast<int>(S), other = PAIR ? static_cast<int>(cluster_ld_u32(cluster_addr(smem_u32(&s_loads), 1))) : s_loads;
            for (int i = min(s_loads, other); i < max(s_loads, other); ++i) {      // stages that only one block of the pair has asked for
                if (i < s_loads)
                    mbar_complete_tx(bar_tile + 8 * (i % n), stage_bytes);
                else
                    mbar_arrive_expect_tx(bar_tile + 8 * (i % n), stage_bytes);
            }
            for (int i = max(0, max(s_loads, other) - n); i < max(s_loads, other); ++i) wait_own(bar_tile + 8 * (i % n), (i / n) & 1);
        }
        if (warp == 1 && pair_rank == 0) {
            if (elect_one()) umma_commit_own<PAIR>(bar_last);      // (the lane that issued the products)
            __syncwarp();
            wait_own(bar_last, 0);
        }
        __syncthreads();
        if (PAIR) {
            cluster_arrive();
            cluster_wait();
        }
    }
    if (!PAIR && p.split > 1) {                   // nobody leaves while the others may read its shared memory
        cluster_arrive_relaxed();
        cluster_wait();
    }
    if (warp == 1) lin_tmem_dealloc<PAIR>(tmem);
}

}  // namespace ead
