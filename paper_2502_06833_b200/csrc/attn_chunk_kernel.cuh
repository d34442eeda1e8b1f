// Attention for units of many packed rows (chunks of new tokens): tcgen05 MMAs with TMEM accumulators.
//
// A unit is up to two row tiles that share every key tile of 64 keys.  A row tile is as many whole tokens as fit into 128
// rows, all query heads of one cache head for each (consecutive rows are the heads of a token): one TMA box of the
// caller's [tokens, heads, head_dim] array.  Per key tile and row tile: S = Q K^T (TMEM),
// one thread per row turns S into probabilities P, which overwrite S as bf16 in TMEM, O += P V (TMEM).  Every row tile has two
// S buffers, so the scores of the next key tile are there when the softmax of this one ends: tensor core and softmax do not
// wait for each other's round trip.  (With 128-key tiles TMEM has room for one S per row tile,
// which exposes that trip: 508 us against 439 on the prompt chunks below, at the time.)  A unit of one row tile
// gives both turns to the same rows instead: even key tiles go to the first accumulator, odd ones
// to the second, and the two are joined at the end.
//
// Warps: 0-3 softmax and output of the first row tile, 4-7 of the second, 8 and 10 issue their MMAs (the instructions
// around the MMAs take longer than the MMAs: one warp for both row tiles took twice the time), 9 loads key and value
// tiles (TMA).  11 walks through the block's units, describes each to the others in shared memory and loads its query
// rows (TMA).  For an 8-bit cache, 12-15 turn codes into bf16 on their way into the MMA's operand tiles (as in the
// few-rows kernel).  Registers are dealt out by warpgroups, most of them to the softmax, which keeps a row's
// scores in them.
//
// What bounds it: at size the tensor core, whose operand reads take 2836 cycles per 256 rows x 128 keys (measured with the
// MMAs alone), and the exponentials, 2048 cycles of the special function units; together 3560.  Both row tiles'
// exponentials at once stall each other and then leave the units idle, so the two softmax warpgroups take turns at them
// (4054 cycles without).  Two chunks of 2041-2048 tokens over 6007-8192 keys, 8 cache heads of 4: 420-440 us,
// 980-1030 TFLOP/s, at the clock the power limit leaves in a long loop; 371-375 us, 1160 TFLOP/s, at full clock.  The same over an
// 8-bit cache: 475 us at full clock.  Short chunks are
// bound by the units' beginnings and ends (query rows in, output or part out: about 8 500 cycles each).
#pragma once
#include "attn_common.cuh"

namespace ead {

constexpr int kChunkMmaWarp = 8, kChunkLoadWarp = 9, kChunkUnitWarp = 11, kChunkFeedWarp = 12;
constexpr int kChunkKeys = 64;                    // keys per tile
constexpr int kChunkShift = 6;
constexpr int kChunkRows = 256;                   // rows per unit
constexpr size_t kChunkPartOffset = 4u << 20;     // the few-rows kernel's parts end below this

// Two bf16 rows of a register's codes, chosen by `pick`, times 2^-120 (see the few-rows kernel).
__device__ __forceinline__ uint32_t chunk_codes(uint32_t codes, uint32_t pick)
{
    const uint32_t w = __byte_perm(codes, 0, pick);
    return (w & 0x80008000u) | ((w >> 4) & 0x07F007F0u);
}

template <int FMT, int D>
struct ChunkLayout {
    static constexpr int kHalves = D / 64;                               // 128-byte lines per bf16 row
    static constexpr int kTileBytes = kChunkKeys * D * 2;                // a bf16 tile of keys or values
    static constexpr int kLine = kChunkKeys * 128;                       // ... of 64 dimensions of them
    static constexpr int kQTile = 128 * D * 2;                           // a tile of query rows
    static constexpr int kStages = D == 64 ? 16 : FMT == kFmtBf16 ? 10 : 8;   // at least 8: see the order of the MMAs
    static constexpr int kRawTile = FMT == kFmtE4m3 ? kChunkKeys * D : 0;
    static constexpr int kRawScale = FMT == kFmtE4m3 ? kChunkKeys * (D / kFmtBlock) : 0;
    static constexpr int kRaw = 3;                                       // stages of codes
    static constexpr int kRawBytes = kRaw * (kRawTile + kRawScale);
    static constexpr int kBars = 2 * kStages + 2 * kRaw + 20;
    static constexpr int kSmem = 1024 + 2 * kQTile + kStages * kTileBytes + kRawBytes + 8 * kBars;
    static constexpr int kWarps = FMT == kFmtBf16 ? 12 : 16, kThreads = 32 * kWarps;
    // registers per thread: two softmax warpgroups, MMA and loads, converters; together at most what the block is launched with
    static constexpr int kSoftmaxRegs = FMT == kFmtBf16 ? 200 : 152, kIssueRegs = 88, kFeedRegs = FMT == kFmtBf16 ? 0 : 120;
    static_assert(2 * kSoftmaxRegs + kIssueRegs + kFeedRegs <= (FMT == kFmtBf16 ? 3 * 168 : 4 * 128), "registers of the launch");
};

// ---- the string of tiles: units in the order (sequence, cache head, run of rows); a unit costs kChunkUnitCost (query rows
// in, output out: about 8 500 cycles against 1 780 per key tile of two row tiles), then 2 per tile of a two-tile unit,
// 1 of a one-tile unit; a tile belongs to the block in whose stretch it begins.  9, 12 and 16 differ by 1 % either way.
constexpr int kChunkUnitCost = 12;
struct ChunkCursor {
    int b, h, blk;                                // sequence, cache head, run of 256 rows
    int64_t begin;                                // the unit's place in the string
    SeqInfo s;
    int i0, tokens;                               // first new token of the unit, and how many
    int pa, pb;                                   // positions of its first and last token
    int cost;                                     // per tile
    KeyRange r;
    __host__ __device__ __forceinline__ int length() const { return kChunkUnitCost + cost * r.tiles; }
    // where the first tile begins
    __device__ __forceinline__ int64_t tiles_at() const { return begin + kChunkUnitCost; }
};
__host__ __device__ __forceinline__ int chunk_blocks(const AttnParams &p, const SeqInfo &s)
{
    const int per = 2 * p.tile_tokens;
    return s.n * p.group <= p.few_rows ? 0 : (s.n + per - 1) / per;   // the host has checked that the product fits
}
__host__ __device__ __forceinline__ void chunk_unit(const AttnParams &p, const SeqInfo &s, int blk, ChunkCursor *c)
{
    c->blk = blk;
    c->i0 = blk * 2 * p.tile_tokens;
    c->tokens = min(2 * p.tile_tokens, s.n - c->i0);
    c->pa = s.p0 + c->i0;
    c->pb = c->pa + c->tokens - 1;
    c->cost = c->tokens > p.tile_tokens ? 2 : 1;
    c->r = key_range(c->pa, c->pb, s.len, p.window, p.sinks, kChunkShift);
}
// Cost of a sequence's units `first`, `first + step`, ... for one cache head.  A unit's fits into 32 bits; the sum grows with the
// square of the prompt (1 M tokens with 32 query heads per cache head: 2^31).
__host__ __device__ __forceinline__ int64_t chunk_cost(const AttnParams &p, const SeqInfo &s, int first, int step)
{
    int64_t sum = 0;
    ChunkCursor u;
    for (int k = first, n = chunk_blocks(p, s); k < n; k += step) {
        chunk_unit(p, s, k, &u);
        sum += u.length();
    }
    return sum;
}
// Moves on to the next unit (the search ends with the batch, whatever its arrays hold).
__device__ __forceinline__ void chunk_next(const AttnParams &p, ChunkCursor *c)
{
    c->begin += c->length();
    int blk = c->blk + 1;
    if (blk >= chunk_blocks(p, c->s)) {
        blk = 0;
        if (++c->h >= p.cache.heads) {
            c->h = 0;
            while (c->b + 1 < p.batch.B) {
                c->s = seq_info(p.batch, ++c->b);
                if (chunk_blocks(p, c->s)) break;
            }
        }
    }
    chunk_unit(p, c->s, blk, c);
}
// The unit's tiles that begin within [g0, g1).
__device__ __forceinline__ void chunk_stretch(const ChunkCursor &c, int64_t g0, int64_t g1, int *ta, int *tb)
{
    const int64_t at = c.tiles_at(), a = (g0 - at + c.cost - 1) / c.cost, b = (g1 - at + c.cost - 1) / c.cost;
    *ta = g0 <= at ? 0 : static_cast<int>(a);
    *tb = b < c.r.tiles ? static_cast<int>(b) : c.r.tiles;
}

// Tiles so far only matter modulo the rings: a count that has grown past two periods goes on from the one before, so that it
// stays within 32 bits however long a block works.
constexpr int kChunkRingPeriod = 240;
__device__ __forceinline__ int ring_count(int tiles) { return tiles < 2 * kChunkRingPeriod ? tiles : kChunkRingPeriod + tiles % kChunkRingPeriod; }

// A block's part of a unit, as warp 11 describes it to the others.
struct ChunkUnit {
    int b, h, token0;                             // sequence, cache head, first row of the sequence in the step
    int i0, tokens;                               // first new token, tokens
    int p0, len;                                  // position of the sequence's first new token, keys in the cache
    int lo, hi, sink_tiles, first_tile;           // keys (KeyRange)
    int ta, nt;                                   // first tile, tiles
    int dual;                                     // two row tiles?
    int last;                                     // the block's last unit?
    int part;                                     // place of its result in the workspace (0, 1), or -1: the unit is this block's alone
    int first, blocks, first_part;                // blocks that hold a part of it; the first one's place
    __device__ __forceinline__ int base(int t) const
    {
        return (t < sink_tiles ? t : t - sink_tiles + first_tile) << kChunkShift;
    }
    __device__ __forceinline__ bool seen(int sinks, int j) const { return j < hi && (j >= lo || j < sinks); }
};

// ---- tensor memory
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
// Waits for every load of this thread; naming the registers keeps their uses behind it.
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                   "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                   "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                   "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
// Pairs of floats in one 64-bit register, two operations per instruction.
__device__ __forceinline__ uint64_t pack_f32x2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t pack_u32x2(uint32_t a, uint32_t b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Shared-memory writes of this thread become visible to the tensor core and to TMA.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem], A packed bf16.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Shared-memory descriptor from its low word: start address / 16 in bits 0-13 and leading offset / 16 in bits 16-29; 128-byte
// swizzle, 8-row groups 1024 bytes apart.  Tiles are rows of 64 elements.  Query rows and keys are contracted along the row
// (leading offset unused, 16 bytes).  Values are contracted along the ROW INDEX, their head dimension is the
// contiguous one: leading offset = next 64 elements of the head dimension, stride offset = next 8 keys.
__device__ __forceinline__ uint32_t umma_desc_hi(uint32_t next8) { return (next8 >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint64_t umma_desc_of(uint32_t lo) { return static_cast<uint64_t>(umma_desc_hi(1024)) << 32 | lo; }
// A tile of values in shared memory: box after box of 2^shift keys, in each the first 64 dimensions of its keys, then the
// next 64.  A step of 16 keys lies within one box, or is two boxes of 8.
template <int D>
struct ValueTile {
    int shift;
    uint32_t line, next8;                         // from 64 dimensions to the next 64, from 8 keys to the next 8
    __device__ __forceinline__ explicit ValueTile(int box_shift)
        : shift(box_shift), line(128u << box_shift), next8(box_shift == 3 ? 1024u * (D / 64) : 1024u) {}
    __device__ __forceinline__ uint32_t at(int key) const
    {
        return ((key >> shift) * (D / 64) << shift) * 128u + (key & ((1 << shift) - 1)) * 128u;
    }
};
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(p));
    return p != 0;
}
// 32 bytes to global memory, in one store if `wide` (the address is a multiple of 32 then).
__device__ __forceinline__ void store_32(uint8_t *dst, const uint32_t (&v)[8], bool wide)
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                     "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        reinterpret_cast<uint4 *>(dst)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4 *>(dst)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}
__device__ __forceinline__ void named_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// The same, and whether `ok` held for all of the barrier's threads.
__device__ __forceinline__ bool named_all(int id, int threads, bool ok)
{
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbar.red.and.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"(id), "r"(threads), "r"(static_cast<uint32_t>(ok)) : "memory");
    return all != 0;
}

template <int FMT, int D>
__global__ void __launch_bounds__(ChunkLayout<FMT, D>::kThreads, 1)
    ead_attn_chunk_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                          const __grid_constant__ CUtensorMap tmQ, AttnParams p,
                          int box_shift, int min_cost)
{
    using L = ChunkLayout<FMT, D>;
    constexpr int S = L::kStages, kChunkWarps = L::kWarps, kChunkThreads = L::kThreads;
    static_assert(kChunkRingPeriod % S == 0 && kChunkRingPeriod % L::kRaw == 0, "a period brings stages and phases back");
    extern __shared__ uint8_t smem_raw[];
    __shared__ int64_t s_scan[kChunkWarps];
    __shared__ int s_b, s_last;
    __shared__ ChunkUnit s_unit[2];
    __shared__ float s_stat[2][128];               // maxima and sums of a one-tile unit's second accumulator
    __shared__ int64_t s_before;
    __shared__ uint32_t s_tmem, s_gave_up;
    __shared__ int s_units, s_tiles;               // units whose query rows, tiles that have been asked for (written when a role stops)
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - raw);
    const uint32_t q_smem = base, ring = base + 2 * L::kQTile, rawk = ring + S * L::kTileBytes;
    const uint32_t raw_scale = rawk + L::kRaw * L::kRawTile;
    const uint32_t bars = rawk + L::kRawBytes;
    const uint32_t bar_full = bars, bar_empty = bars + 8 * S, bar_raw_full = bar_empty + 8 * S, bar_raw_empty = bar_raw_full + 8 * L::kRaw;
    // scores and probabilities: one barrier per row tile (16 bytes apart) and buffer
    const uint32_t bar_s = bar_raw_empty + 8 * L::kRaw, bar_p = bar_s + 32, bar_o = bar_p + 32, bar_v = bar_o + 16, bar_q_full = bar_v + 16, bar_q_empty = bar_q_full + 8;
    const uint32_t bar_u_full = bar_q_empty + 8, bar_u_empty = bar_u_full + 16, bar_last = bar_u_empty + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvCacheView &c = p.cache;

    if (tid == 32) {
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
        tma_prefetch_desc(&tmQ);
    }
    if (tid == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(bar_full + 8 * i, FMT == kFmtBf16 ? 1 : 128);
            mbar_init(bar_empty + 8 * i, 2);
        }
        for (int i = 0; i < L::kRaw; ++i) {
            mbar_init(bar_raw_full + 8 * i, 1);
            mbar_init(bar_raw_empty + 8 * i, 128);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(bar_s + 8 * i, 1);
            mbar_init(bar_p + 8 * i, 128);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_o + 8 * i, 1);
            mbar_init(bar_v + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_u_full + 8 * i, 1);
            mbar_init(bar_u_empty + 8 * i, kChunkWarps - 1);
            mbar_init(bar_last + 8 * i, 1);
        }
        s_gave_up = 0;
        mbar_init(bar_q_full, 1);
        mbar_init(bar_q_empty, 2);
        fence_mbar_init();
    }
    if (warp == kChunkMmaWarp) {
        tmem_alloc(smem_u32(&s_tmem), 512);
        tmem_relinquish();
    }

    // ---- the string: cost of one cache head of every sequence, and where this block's stretch begins
    int64_t *const s_cost = reinterpret_cast<int64_t *>(base_ptr);      // [B], in the query rows' place for now
    static_assert(kMaxBatch * sizeof(int64_t) <= 2 * L::kQTile, "the costs fit there");
    for (int b0 = warp * 32; b0 < p.batch.B; b0 += kChunkThreads) {
        const int b = b0 + lane;
        SeqInfo s{};
        int blocks = 0;
        int64_t cost = 0;
        if (b < p.batch.B) {
            bool bad;
            s = seq_info(p.batch, b, &bad);
            if (blockIdx.x == 0 && bad) flag_status(p.status, kStatusBadCount);
            blocks = chunk_blocks(p, s);
            if (blockIdx.x == 0 && blocks && s.p0 + s.n > p.batch.max_len) flag_status(p.status, kStatusBadPage);
        }
        unsigned many = __ballot_sync(0xffffffffu, blocks > 2);
        if (blocks <= 2) cost = chunk_cost(p, s, 0, 1);
        while (many) {                             // long chunks: the warp's lanes share the runs of one sequence
            const int src = __ffs(many) - 1;
            many &= many - 1;
            SeqInfo t;
            t.n = __shfl_sync(0xffffffffu, s.n, src);
            t.p0 = __shfl_sync(0xffffffffu, s.p0, src);
            t.len = __shfl_sync(0xffffffffu, s.len, src);
            t.token0 = 0;
            int64_t part = chunk_cost(p, t, lane, 32);
#pragma unroll
            for (int o = 16; o; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
            if (lane == src) cost = part;
        }
        if (b < p.batch.B) s_cost[b] = cost;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    const int per = (p.batch.B + kChunkThreads - 1) / kChunkThreads;
    const int b_lo = min(tid * per, p.batch.B), b_hi = min(b_lo + per, p.batch.B);
    int64_t mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += s_cost[b];
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) s_scan[warp] = upto;
    __syncthreads();
    int64_t total = 0, before = 0;
    for (int w = 0; w < kChunkWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    upto += before;
    const int64_t W = total * c.heads;
    const int64_t ctas = min(static_cast<int64_t>(gridDim.x), max(static_cast<int64_t>(1), W / min_cost));
    const bool idle = W == 0 || blockIdx.x >= ctas;
    const int64_t g0 = idle ? 0 : W * blockIdx.x / ctas, g1 = idle ? 0 : W * (blockIdx.x + 1) / ctas;
    if (!idle && mine > 0 && g0 >= (upto - mine) * c.heads && g0 < upto * c.heads) {
        int64_t at = upto - mine;
        for (int b = b_lo; b < b_hi; ++b) {
            if (g0 < (at + s_cost[b]) * c.heads) {
                s_b = b;
                s_before = at * c.heads;
                break;
            }
            at += s_cost[b];
        }
    }
    __syncthreads();
    ChunkCursor cur{};
    if (!idle) {
        cur.b = s_b;
        cur.s = seq_info(p.batch, cur.b);
        const int64_t cost = s_cost[cur.b];
        cur.h = static_cast<int>((g0 - s_before) / cost);
        cur.begin = s_before + static_cast<int64_t>(cur.h) * cost;
        chunk_unit(p, cur.s, 0, &cur);
        // the first unit with a tile that begins at g0 or later
        while (cur.tiles_at() + static_cast<int64_t>(cur.cost) * (cur.r.tiles - 1) < g0) chunk_next(p, &cur);
    }
    fence_async_shared();
    __syncthreads();                               // s_cost is done with; its place takes query rows now, by TMA

    // Every role takes the units one by one: waits for the description, works, releases it (one arrival per warp).
    // When a wait runs out, a warp that loads stops at its next wait that does, every other role walks through the unit
    // whose description it holds and stops (the softmax warps, which meet at barriers, all at the same one): nobody
    // reads a description that is not there.  What is under way then comes in before the block ends.  (A look at the block's
    // `gave_up` before every tile's load would end the loads sooner; it made the hand-over step 2 to 5 % slower.)
    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_phase(bar, parity, p, &s_gave_up); };
    auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    auto unit_wait = [&](int n) { return warp_wait(bar_u_full + 8 * (n & 1), (n >> 1) & 1); };
    auto unit_done = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_u_empty + 8 * (n & 1));
    };
    if (idle) {
        // nothing
    } else if (warp >= kChunkMmaWarp && warp < kChunkFeedWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::kIssueRegs));
        if (warp == kChunkUnitWarp) {
            // ============================================================ units
            int n = 0;
            for (;; ++n) {
                int ta, tb;
                chunk_stretch(cur, g0, g1, &ta, &tb);
                const int64_t at = cur.tiles_at(), end = at + static_cast<int64_t>(cur.cost) * cur.r.tiles;
                if (!warp_wait(bar_u_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1)) break;
                if (lane == 0) {
                    ChunkUnit &u = s_unit[n & 1];
                    u.b = cur.b; u.h = cur.h; u.token0 = cur.s.token0;
                    u.i0 = cur.i0; u.tokens = cur.tokens;
                    u.p0 = cur.s.p0; u.len = cur.s.len;
                    u.lo = cur.r.lo; u.hi = cur.r.hi; u.sink_tiles = cur.r.sink_tiles; u.first_tile = cur.r.first_tile;
                    u.ta = ta; u.nt = tb - ta;
                    u.dual = cur.cost == 2;
                    u.last = end + kChunkUnitCost >= g1;   // where the next unit's first tile would begin
                    u.part = ta == 0 && tb == cur.r.tiles ? -1 : at <= g0 ? 0 : 1;
                    // blocks in whose stretch its first and its last tile begin
                    u.first = static_cast<int>(((at + 1) * ctas - 1) / W);
                    u.blocks = static_cast<int>(((end - cur.cost + 1) * ctas - 1) / W) - u.first + 1;
                    u.first_part = at <= W * u.first / ctas ? 0 : 1;
                    mbar_arrive(bar_u_full + 8 * (n & 1));
                }
                // its query rows, when the unit before has done with theirs (rows of tokens behind the unit's come along)
                if (!warp_wait(bar_q_empty, (n & 1) ^ 1)) break;
                if (lane == 0) {
                    const uint32_t box = p.tile_tokens * p.group * 128;
                    mbar_arrive_expect_tx(bar_q_full, cur.cost * L::kHalves * box);
                    for (int x = 0; x < cur.cost * L::kHalves; ++x) {
                        const int tile = x / L::kHalves, hb = x - tile * L::kHalves;
                        tma_load_3d(q_smem + tile * L::kQTile + hb * (128 * 128), &tmQ, 64 * hb, cur.h * p.group,
                                    cur.s.token0 + cur.i0 + tile * p.tile_tokens, bar_q_full);
                    }
                }
                if (end + kChunkUnitCost >= g1) {
                    ++n;
                    break;
                }
                chunk_next(p, &cur);
            }
            if (lane == 0) s_units = n;
        } else if (warp == kChunkLoadWarp) {
            // ============================================================ key and value tiles
            const int boxes = kChunkKeys >> box_shift, box_keys = 1 << box_shift;     // at most 8
            int x = 0;                             // tiles asked for
            bool go = true;
            for (int n = 0;; ++n) {
                if (!unit_wait(n)) break;
                const ChunkUnit &u = s_unit[n & 1];
                const int ta = u.ta, nt = u.nt, last = u.last, b = u.b, h = u.h;
                KeyRange r;
                r.lo = u.lo; r.hi = u.hi; r.sink_tiles = u.sink_tiles; r.first_tile = u.first_tile; r.tiles = 0;
                unit_done(n);
                // this lane's box of a tile: its page as the table has it, or -2 if no query sees any of it
                auto look_up = [&](int k) {
                    const int at = r.base(k, kChunkShift) + lane * box_keys;
                    const bool any = lane < boxes && at < r.hi && (at + box_keys > r.lo || at < p.sinks);
                    return any ? max(__ldg(p.batch.page_table + static_cast<int64_t>(b) * p.batch.table_stride + (at >> c.page_shift)), -1) : -2;
                };
                int entry = look_up(ta);
                for (int k = ta; go && k < ta + nt; ++k) {
                    const int slot = (r.base(k, kChunkShift) + lane * box_keys) & (c.page_size - 1);
                    const int next = k + 1 < ta + nt ? look_up(k + 1) : -2;       // its latency runs under this tile's waits
                    int page = entry;
                    if (page != -2 && (page < 0 || page >= c.n_pages)) {
                        flag_status(p.status, kStatusBadPage);
                        page = c.n_pages;          // outside the pool: the copy delivers zeros
                    }
                    entry = next;
                    const int live = __popc(__ballot_sync(0xffffffffu, page >= 0));
                    const int good = __popc(__ballot_sync(0xffffffffu, page >= 0 && page < c.n_pages));
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!go) break;
                        const CUtensorMap *tm = kv ? &tmV : &tmK;
                        if (FMT == kFmtBf16) {
                            const int st = x % S;
                            const uint32_t bar = bar_full + 8 * st, dst = ring + st * L::kTileBytes + lane * box_keys * 128;
                            if (!(go = warp_wait(bar_empty + 8 * st, ((x / S) & 1) ^ 1))) break;
                            if (lane == 0) mbar_arrive_expect_tx(bar, live * box_keys * D * 2);
                            __syncwarp();
                            if (page >= 0) {
                                if (kv) {          // all lines of its keys in one box (see the value tiles' descriptor)
                                    tma_load_5d(dst + (L::kHalves - 1) * lane * box_keys * 128, tm, 0, slot, 0, h, page, bar);
                                } else {
#pragma unroll
                                    for (int hb = 0; hb < L::kHalves; ++hb)
                                        tma_load_5d(dst + hb * L::kLine, tm, 0, slot, hb, h, page, bar);
                                }
                            }
                        } else {
                            const int st = x % L::kRaw;
                            const uint32_t bar = bar_raw_full + 8 * st;
                            const uint32_t sc = raw_scale + st * L::kRawScale + lane * box_keys * (D / kFmtBlock);
                            const uint32_t sc_bytes = box_keys * (D / kFmtBlock);
                            if (!(go = warp_wait(bar_raw_empty + 8 * st, ((x / L::kRaw) & 1) ^ 1))) break;
                            if (page == c.n_pages)
                                for (uint32_t y = 0; y < sc_bytes; y += 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(sc + y), "r"(0) : "memory");
                            __syncwarp();
                            if (lane == 0) mbar_arrive_expect_tx(bar, live * box_keys * D + good * sc_bytes);
                            __syncwarp();
                            if (page >= 0) {
                                tma_load_5d(rawk + st * L::kRawTile + lane * box_keys * D, tm, 0, slot, 0, h, page, bar);
                                if (page < c.n_pages)
                                    bulk_load(sc, (kv ? c.v_scale : c.k_scale) + scale_offset(c, page, h, slot), sc_bytes, bar);
                            }
                        }
                        ++x;
                    }
                }
                if (last || !go) break;
                x = 2 * ring_count(x / 2);
            }
            if (lane == 0) s_tiles = x;
        } else {
            // ============================================================ MMAs
            // The whole warp walks through the loop, one lane issues.  It is chosen by elect.sync, not by its number: only then
            // does the compiler know that one lane is active, and eight 128 x 128 x 16 MMAs take 513 cycles to issue
            // instead of 663 (measured alone; the tensor core needs 512).
            const int w = __shfl_sync(0xffffffffu, (warp - kChunkMmaWarp) >> 1, 0);  // row tile
            const uint32_t id_qk = umma_idesc_bf16_m128(kChunkKeys), id_pv = umma_idesc_bf16_m128(D) | (1u << 16);
            const uint32_t q_lo = (q_smem >> 4) | (1u << 16), k_lo = (ring >> 4) | (1u << 16);
            const ValueTile<D> vt(FMT == kFmtBf16 ? box_shift : kChunkShift);
            const uint32_t v_lo = (ring >> 4) | (vt.line << (16 - 4)), v_hi = umma_desc_hi(vt.next8);
            const uint32_t t_s = tmem + w * 128, t_o = tmem + 256 + w * 128;
            int t = 0;
            uint32_t ns = 0, np = 0;               // scores issued and probabilities taken so far
            for (int n = 0;; ++n) {
                if (!unit_wait(n)) break;
                const ChunkUnit &u = s_unit[n & 1];
                const bool dual = __shfl_sync(0xffffffffu, u.dual, 0) != 0;
                const int nt = __shfl_sync(0xffffffffu, u.nt, 0), last = __shfl_sync(0xffffffffu, u.last, 0);
                unit_done(n);
                const int rounds = dual ? nt : (nt + 1 - w) >> 1;
                wait(bar_q_full, n & 1);
                const uint32_t a = q_lo + (dual ? w * (L::kQTile >> 4) : 0);
                auto scores = [&](int i) {         // S = Q K^T of the i-th tile
                    const int x = 2 * (t + (dual ? i : 2 * i + w)), st = x % S;
                    wait(bar_full + 8 * st, (x / S) & 1);
                    __syncwarp();
                    tc_fence_after_sync();
                    const uint32_t d = t_s + (ns & 1) * 64, b = k_lo + st * (L::kTileBytes >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            umma_bf16(d, umma_desc_of(a + (ks >> 2) * ((128 * 128) >> 4) + (ks & 3) * 2),
                                      umma_desc_of(b + (ks >> 2) * (L::kLine >> 4) + (ks & 3) * 2), id_qk, ks > 0);
                        umma_commit(bar_s + 16 * w + 8 * (ns & 1));
                        umma_commit(bar_empty + 8 * st);
                        if (!dual) umma_commit(bar_empty + 8 * st);              // for the row tile that is not there
                        if (i + 1 == rounds) umma_commit(bar_q_empty);           // the query rows' place is free after the last one
                    }
                    __syncwarp();
                    ++ns;
                };
                // Order: two tiles' scores ahead; a buffer's next scores are issued behind the product that reads its probabilities.
                // With one-tile units the keys of tile k + 4 are waited for while tile k's values are unread: 8 stages at least.
                if (rounds == 0 && elect_one()) mbar_arrive(bar_q_empty);
                for (int i = 0; i < 2; ++i)
                    if (i < rounds) scores(i);
                for (int i = 0; i < rounds; ++i) {
                    const int x = 2 * (t + (dual ? i : 2 * i + w)) + 1, st = x % S;
                    const uint32_t pr = t_s + (np & 1) * 64, b = v_lo + st * (L::kTileBytes >> 4);
                    wait(bar_full + 8 * st, (x / S) & 1);
                    wait(bar_p + 16 * w + 8 * (np & 1), (np >> 1) & 1);
                    __syncwarp();
                    tc_fence_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < kChunkKeys / 16; ++ks)
                            umma_bf16_ts(t_o, pr + ks * 8, static_cast<uint64_t>(v_hi) << 32 | (b + (vt.at(16 * ks) >> 4)), id_pv, i > 0 || ks > 0);
                        umma_commit(bar_v + 8 * w);
                        umma_commit(bar_empty + 8 * st);
                        if (!dual) umma_commit(bar_empty + 8 * st);
                        if (i + 1 == rounds) umma_commit(bar_o + 8 * w);
                    }
                    __syncwarp();
                    ++np;
                    if (i + 2 < rounds) scores(i + 2);
                }
                t = ring_count(t + nt);
                if (last) break;
            }
        }
    } else if (FMT == kFmtE4m3 && warp >= kChunkFeedWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(FMT == kFmtE4m3 ? L::kFeedRegs : 24));
        // ================================================================ codes to bf16
        const int ft = tid - kChunkFeedWarp * 32;  // 0 .. 127
        int t = 0;
        for (int n = 0;; ++n) {
            if (!unit_wait(n)) break;
            const ChunkUnit &un = s_unit[n & 1];
            const int last = un.last;
            {
                for (int k = un.ta, end = un.ta + un.nt; k < end; ++k, ++t)
                    for (int kv = 0; kv < 2; ++kv) {
                        // half a key per thread: threads 0-63 the first half of the dimensions, 64-127 the second
                        const int x = 2 * t + kv, st = x % S, rs = x % L::kRaw, key = ft & 63, part = ft >> 6;
                        wait(bar_raw_full + 8 * rs, (x / L::kRaw) & 1);
                        uint32_t w[D / 8], sc;
                        const uint32_t src = rawk + rs * L::kRawTile + key * D;
#pragma unroll
                        for (int c16 = 0; c16 < D / 32; ++c16) {
                            const int ch = part * (D / 32) + c16;
                            const uint32_t at = src + ((D == 128 ? ch ^ (key & 7) : ch ^ ((key >> 1) & 3)) << 4);
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(w[4 * c16]), "=r"(w[4 * c16 + 1]), "=r"(w[4 * c16 + 2]), "=r"(w[4 * c16 + 3]) : "r"(at) : "memory");
                        }
                        const uint32_t sa = raw_scale + rs * L::kRawScale + key * (D / kFmtBlock) + part * (D / 64);
                        if (D == 128)
                            asm volatile("{\n\t.reg .b16 h;\n\tld.shared.b16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(sc) : "r"(sa) : "memory");
                        else
                            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sc) : "r"(sa) : "memory");
                        // a key no query of the unit sees was perhaps not even loaded: zeros
                        const bool keep = un.seen(p.sinks, un.base(k) + key);
                        wait(bar_empty + 8 * st, ((x / S) & 1) ^ 1);
                        const uint32_t dst = ring + st * L::kTileBytes + key * 128;
#pragma unroll
                        for (int g = 0; g < D / 64; ++g) {
                            const uint32_t byte = (sc >> (8 * g)) & 0xffu;
                            const uint32_t f = ((min(byte, 134u) + 120u) << 7) * 0x10001u;       // see the few-rows kernel
                            const uint32_t f2 = ((byte == 255u ? 0x7FC0u : (byte > 134u ? byte - 7u : 127u) << 7)) * 0x10001u;
#pragma unroll
                            for (int u = 0; u < 4; ++u) {                 // 8 values: 16 bytes of bf16
                                uint32_t o[4];
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const uint32_t codes = w[8 * g + 2 * u + e];
                                    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[2 * e]) : "r"(chunk_codes(codes, 0x1404)), "r"(f));
                                    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[2 * e + 1]) : "r"(chunk_codes(codes, 0x3424)), "r"(f));
                                }
                                if (byte > 134u) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[e]) : "r"(o[e]), "r"(f2));
                                }
                                if (!keep) o[0] = o[1] = o[2] = o[3] = 0;
                                const int ch = part * (D / 16) + 4 * g + u;
                                const uint32_t at = dst + (ch >> 3) * L::kLine + (((ch & 7) ^ (key & 7)) << 4);
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                            }
                        }
                        fence_async_shared();
                        mbar_arrive(bar_full + 8 * st);
                        // not earlier: only the codes' use shows that their loads are done (released right after the loads, the
                        // next tile's copy overtook loads that the tensor core's own reads had held up)
                        mbar_arrive(bar_raw_empty + 8 * rs);
                    }
            }
            unit_done(n);
            if (last) break;
            t = ring_count(t);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::kSoftmaxRegs));
        // ================================================================ softmax and output
        const int w = warp >> 2, row = tid & 127;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;            // this warp's 32 lanes of tensor memory
        const uint32_t t_o = tmem + lanes + 256 + w * 128;
        int t = 0;
        uint32_t ns = 0;
        uint32_t outputs[2] = {0, 0};                  // finished outputs per accumulator
        // a thread writes a row: 32 bytes at a time, a whole sector each, if every row begins at one
        const bool whole_sectors = ((reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(2 * p.out_stride)) & 31) == 0;
        for (int n = 0;; ++n) {
            if (!named_all(1, 256, unit_wait(n))) break;
            const ChunkUnit &u = s_unit[n & 1];
            const bool dual = u.dual != 0;
            const int ta = u.ta, nt = u.nt, rounds = dual ? nt : (nt + 1 - w) >> 1;
            const int my_row = dual ? w * 128 + row : row;                       // row within the unit
            const int tile0 = dual ? w * p.tile_tokens : 0, tile1 = min(tile0 + p.tile_tokens, u.tokens);   // the row tile's tokens
            const int my_i = tile0 + row / p.group, gq = row - (my_i - tile0) * p.group;
            const int first_pos = u.p0 + u.i0, pos = first_pos + min(my_i, u.tokens - 1);
            // A tile needs no mask if its last key is no later than the row tile's first position (and in the cache), and its first
            // key is in the window of the row tile's last one, or all of it are sinks.
            const int no_later = min(first_pos + tile0, u.len - 1) - (kChunkKeys - 1);
            const int no_sooner = p.window ? first_pos + tile1 - p.window : -0x40000000;
            const int sink_tiles = u.sink_tiles, first_tile = u.first_tile - sink_tiles;
            float m = -INFINITY, l = 0.f;
            // Two-tile units: the row tiles take turns at the exponentials, so that one's run while the other waits for scores,
            // loads them and looks for their maximum.
            if (dual && w == 1) named_arrive(2, 256);
            for (int i = 0; i < rounds; ++i) {
                const int k = dual ? i : 2 * i + w;
                const int kt = ta + k, key0 = (kt < sink_tiles ? kt : kt + first_tile) << kChunkShift;
                const bool whole = key0 <= no_later && (key0 >= no_sooner || key0 + kChunkKeys <= p.sinks);
                if (FMT == kFmtBf16 && !whole) {
                    // values no query sees may be anything, and were perhaps not even loaded: zeros, so that 0 * NaN cannot arise
                    // (both row tiles' threads write them: each has its own product to come)
                    const bool clean = key0 + kChunkKeys <= u.hi && (key0 >= u.lo || key0 + kChunkKeys <= p.sinks);
                    if (!clean) {
                        const int x = 2 * (t + k) + 1, st = x % S;
                        wait(bar_full + 8 * st, (x / S) & 1);
                        if (row < kChunkKeys * L::kHalves && !u.seen(p.sinks, key0 + (row & 63))) {
                            const ValueTile<D> vt(box_shift);
                            const uint32_t dst = ring + st * L::kTileBytes + (row >> 6) * vt.line + vt.at(row & 63);
#pragma unroll
                            for (int ch = 0; ch < 8; ++ch)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + ch * 16), "r"(0) : "memory");
                        }
                        fence_async_shared();
                    }
                }
                const uint32_t t_s = tmem + lanes + w * 128 + (ns & 1) * 64, done = bar_p + 16 * w + 8 * (ns & 1);
                wait(bar_s + 16 * w + 8 * (ns & 1), (ns >> 1) & 1);
                ++ns;
                __syncwarp();
                tc_fence_after_sync();
                uint32_t v[2][32];
                tmem_ld32(t_s, v[0]);
                tmem_ld32(t_s + 32, v[1]);
                tmem_wait_ld(v[0]);
                tmem_wait_ld(v[1]);
                if (!whole) {
                    const int limit = min(pos + 1, u.len) - key0;            // columns from here on lie ahead or beyond the context
                    const int low = p.window ? pos - p.window + 1 - key0 : -0x40000000, sink = p.sinks - key0;
#pragma unroll
                    for (int col = 0; col < kChunkKeys; ++col)
                        if (!(col < limit && (col >= low || col < sink))) v[col >> 5][col & 31] = 0xff800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int col = 0; col < kChunkKeys; col += 2)
                    top[(col >> 1) & 3] = max3(top[(col >> 1) & 3], __uint_as_float(v[col >> 5][col & 31]), __uint_as_float(v[col >> 5][(col & 31) + 1]));
                const float mx = max3(top[0], top[1], fmaxf(top[2], top[3])) * p.scale_log2;
                const bool raise = mx > m + 8.f;   // the reference stays while no probability exceeds 2^8
                if (__any_sync(0xffffffffu, raise)) {
                    const float f = raise ? exp2_fast(m - mx) : 1.f;
                    if (raise) m = mx;
                    l *= f;
                    if (i > 0) {
                        // the product of the tile before may still be running (the one before that is not: S came behind it)
                        wait(bar_v + 8 * w, (ns - 2) & 1);
                        __syncwarp();
                        tc_fence_after_sync();
#pragma unroll
                        for (int q = 0; q < D / 16; ++q) {
                            uint32_t o[16];
                            tmem_ld16(t_o + 16 * q, o);
                            tmem_wait_ld16(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st16(t_o + 16 * q, o);
                        }
                    }
                }
                if (dual) named_sync(2 + w, 256);  // the other row tile's exponentials are done
                const float mm = m == -INFINITY ? 0.f : m;
                const uint64_t scale2 = pack_f32x2(p.scale_log2, p.scale_log2), minus2 = pack_f32x2(-mm, -mm);
                uint64_t sum2[2] = {0, 0};
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint64_t x = fma_f32x2(pack_u32x2(v[q][2 * e], v[q][2 * e + 1]), scale2, minus2);
                        float a, b;
                        unpack_f32x2(x, a, b);
                        a = exp2_fast(a);
                        b = exp2_fast(b);
                        sum2[e & 1] = add_f32x2(sum2[e & 1], pack_f32x2(a, b));
                        pk[e] = to_bf16x2(a, b);
                    }
                    tmem_st16(t_s + 16 * q, pk);   // columns whose scores are in registers
                }
                if (dual && (w == 0 || i + 1 < rounds)) named_arrive(3 - w, 256);
                tmem_wait_st();
                tc_fence_before_sync();
                mbar_arrive(done);
                float s0, s1;
                unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
                l += s0 + s1;
            }

            // ---- output: this thread's row
            const bool alone = u.part < 0;
            if (rounds > 0) {
                wait(bar_o + 8 * w, outputs[w] & 1);
                __syncwarp();
                tc_fence_after_sync();
            }
            float *const parts = reinterpret_cast<float *>(p.workspace + kChunkPartOffset);
            constexpr size_t kPart = kChunkRows * (D + 2);
            float *const my_part = parts + (2 * blockIdx.x + (u.part < 0 ? 0 : u.part)) * kPart;   // not used by a unit of this block alone
            float f0 = 1.f, f1 = 0.f;              // one-tile units: factors of the two accumulators
            if (!dual) {
                if (w == 1) {
                    s_stat[0][row] = m;
                    s_stat[1][row] = l;
                }
                named_sync(1, 256);
                if (w == 0) {
                    const float m1 = s_stat[0][row], l1 = s_stat[1][row];
                    const float M = fmaxf(m, m1);
                    f0 = m == -INFINITY ? (M == -INFINITY ? 1.f : 0.f) : exp2_fast(m - M);
                    f1 = m1 == -INFINITY ? 0.f : exp2_fast(m1 - M);
                    l = l * f0 + l1 * f1;
                    m = M;
                    if (nt > 1) {                  // the second accumulator's products are complete, too
                        wait(bar_o + 8, outputs[1] & 1);
                        __syncwarp();
                        tc_fence_after_sync();
                    }
                }
            }
            const bool holds = dual || w == 0;
            const bool live = holds && my_i < tile1;
            const int hq = u.h * p.group + gq;
            const int64_t token = static_cast<int64_t>(u.token0) + u.i0 + my_i;
            if (holds) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                for (int q = 0; q < D / 32; ++q) {
                    uint32_t o[32];
                    __syncwarp();
                    tmem_ld32(t_o + 32 * q, o);
                    tmem_wait_ld(o);
                    if (!dual) {
                        uint32_t o1[32];
                        tmem_ld32(t_o + 128 + 32 * q, o1);
                        tmem_wait_ld(o1);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            o[e] = __float_as_uint(__uint_as_float(o[e]) * f0 + (nt > 1 ? __uint_as_float(o1[e]) * f1 : 0.f));
                    }
                    if (live && alone) {
                        uint8_t *dst = p.out + 2 * (token * p.out_stride + static_cast<int64_t>(hq) * D + 32 * q);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v8[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                v8[e] = to_bf16x2(__uint_as_float(o[16 * h + 2 * e]) * inv, __uint_as_float(o[16 * h + 2 * e + 1]) * inv);
                            store_32(dst + 32 * h, v8, whole_sectors);
                        }
                    } else if (live) {
                        uint4 *dst = reinterpret_cast<uint4 *>(my_part) + 8 * q * kChunkRows + my_row;       // four columns by rows: consecutive lanes are adjacent
#pragma unroll
                        for (int e = 0; e < 8; ++e) dst[e * kChunkRows] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                }
                if (live) {
                    if (alone) {
                        if (p.lse) p.lse[token * p.heads_q + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
                    } else {
                        my_part[kChunkRows * D + my_row] = m;
                        my_part[kChunkRows * D + kChunkRows + my_row] = l;
                    }
                }
                tc_fence_before_sync();
            }
            if (!dual) named_sync(1, 256);         // the second accumulator and s_stat may be written again
            if (!alone) {
                // blocks that hold a part of the unit: first .. last; the counter is the first one's
                uint32_t *const counters = reinterpret_cast<uint32_t *>(p.workspace + kAttnCounterBytes);
                const int first = u.first, blocks = u.blocks;
                fence_gpu();
                named_sync(1, 256);
                if (tid == 0) {
                    const uint32_t seen = atomicAdd(counters + first, 1u);
                    s_last = seen == static_cast<uint32_t>(blocks - 1);
                    if (s_last) counters[first] = 0;                             // ready for the next call
                }
                named_sync(1, 256);
                if (s_last) {
                    fence_gpu();
                    const int first_slot = u.first_part, last = first + blocks - 1;
                    const int r = tid, ti = (tid >> 7) * p.tile_tokens + (tid & 127) / p.group;
                    if (ti < min(((tid >> 7) + 1) * p.tile_tokens, u.tokens)) {    // one row per thread
                        auto part_of = [&](int k) { return parts + (2 * k + (k == first ? first_slot : 0)) * kPart; };
                        float M = -INFINITY, Lsum = 0.f;
#pragma unroll 4
                        for (int k = first; k <= last; ++k) {
                            const float mk = __ldcg(part_of(k) + kChunkRows * D + r), lk = __ldcg(part_of(k) + kChunkRows * D + kChunkRows + r);
                            const float top = fmaxf(M, mk), base = top == -INFINITY ? 0.f : top;
                            Lsum = Lsum * exp2_fast(M - base) + lk * exp2_fast(mk - base);
                            M = top;
                        }
                        const float inv = Lsum == 0.f ? 0.f : 1.f / Lsum;
                        const int hr = u.h * p.group + (tid & 127) % p.group;
                        const int64_t tok = static_cast<int64_t>(u.token0) + u.i0 + ti;
                        if (p.lse) p.lse[tok * p.heads_q + hr] = Lsum == 0.f ? -INFINITY : (M + log2f(Lsum)) * kLn2;
                        for (int q = 0; q < D / 64; ++q) {
                            float4 a[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) a[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                            for (int k = first; k <= last; ++k) {
                                const float mk = __ldcg(part_of(k) + kChunkRows * D + r);
                                const float4 *src = reinterpret_cast<const float4 *>(part_of(k)) + 16 * q * kChunkRows + r;
                                float4 y[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __ldcg(src + e * kChunkRows);
                                const float f = (mk == -INFINITY ? 0.f : exp2_fast(mk - M)) * inv;
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    a[e].x += f * y[e].x; a[e].y += f * y[e].y; a[e].z += f * y[e].z; a[e].w += f * y[e].w;
                                }
                            }
                            uint8_t *dst = p.out + 2 * (tok * p.out_stride + static_cast<int64_t>(hr) * D + 64 * q);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t v[8] = {to_bf16x2(a[4 * e].x, a[4 * e].y), to_bf16x2(a[4 * e].z, a[4 * e].w),
                                                       to_bf16x2(a[4 * e + 1].x, a[4 * e + 1].y), to_bf16x2(a[4 * e + 1].z, a[4 * e + 1].w),
                                                       to_bf16x2(a[4 * e + 2].x, a[4 * e + 2].y), to_bf16x2(a[4 * e + 2].z, a[4 * e + 2].w),
                                                       to_bf16x2(a[4 * e + 3].x, a[4 * e + 3].y), to_bf16x2(a[4 * e + 3].z, a[4 * e + 3].w)};
                                store_32(dst + 32 * e, v, whole_sectors);
                            }
                        }
                    }
                }
                named_sync(1, 256);                // s_last may be written again
            }
            t = ring_count(t + nt);
            outputs[0] += 1;                       // the first accumulator has a tile in every unit
            outputs[1] += dual || nt > 1;
            const int last = u.last;
            unit_done(n);
            if (last) break;
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (s_gave_up) {                               // nobody sets it any more
        constexpr int R = FMT == kFmtBf16 ? S : L::kRaw;
        if (warp == kChunkUnitWarp && s_units) wait_own(bar_q_full, (s_units - 1) & 1);
        if (warp == kChunkLoadWarp)
            for (int x = max(0, s_tiles - R); x < s_tiles; ++x) wait_own((FMT == kFmtBf16 ? bar_full : bar_raw_full) + 8 * (x % R), (x / R) & 1);
        if (warp == kChunkMmaWarp || warp == kChunkMmaWarp + 2) {
            const uint32_t bar = bar_last + 4 * (warp - kChunkMmaWarp);
            if (elect_one()) umma_commit(bar);
            __syncwarp();
            wait_own(bar, 0);
        }
        __syncthreads();
    }
    if (warp == kChunkMmaWarp) tmem_dealloc(tmem, 512);
    griddep_wait();                                // started alongside the few-rows kernel: it ends before this one does
}

}  // namespace ead
