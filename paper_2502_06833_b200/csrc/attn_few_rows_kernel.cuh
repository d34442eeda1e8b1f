// Attention for units of at most 16 packed rows (new tokens x query heads of a cache head): single-token
// decoding and very short chunks.
//
// Every key and value is read from HBM once and used for 8 or 16 rows only, so HBM bounds it; the
// kernel is built to keep many bytes in flight and little else.  The block's kWarps warps (8; 12 for an 8-bit cache
// and at most 8 rows) work independently: each has its own ring of 8 KiB stages (4 KiB of keys, 4 KiB of values) filled by
// TMA boxes of one page each and takes every kWarps-th tile of the block's stretch, so no barrier stands between the loads
// of consecutive tiles or units.  Products are mma.sync with the keys (values) as the 16-row
// operand and the packed query rows as the 8-column operand: a tensor-memory accumulator has 128 rows, of which
// 8 would carry anything.  S^T = K Q^T has the layout that, transposed 8 x 8, is the second
// operand of O^T = V^T P^T.
//
// 8-bit keys and values are widened in registers on their way from shared memory to the MMA, and instructions, not
// bytes, are what an 8-bit cache is short of, so the scales are applied where there is least to apply them to.
// Keys: codes are exact in f16; the products of one scale block are summed apart and the four sums of a key are
// scaled in 32 bits.  The query rows are f16 then, too: each row is first divided by a power of two that
// brings its largest element to 1..2.  Elements down to 2^-17 of that are exact, smaller ones lose at most 2^-25 (the
// chunk kernel takes them as the bf16 they are).
// Values: an e4m3 byte placed 4 bits down in a bf16 is 2^-120 of its value, subnormals included; the factor 2^(120 + k)
// goes to the probabilities (an exact change of exponent), once per key and scale block instead of once per value.
//
// Measured (head_dim 128, 8 cache heads), in graph replay: bf16, 64 contexts of 1024-8192, 4 query heads each: 191-197 us, 6.2 TB/s,
// 0.95 of the device's copy rate.  e4m3, 24 contexts of 4001-32001, 5 query heads each: 188-190 us, 5.0 TB/s, 0.77; scales applied to
// every value instead took 234 us with 8 warps, and 12 warps instead of 8 are worth 15 %.  As calls: 198 and 199 us.  With 3-4 new
// tokens per sequence (two groups of 8 rows), 32 contexts of 1000-8000, 4 query heads each: bf16 114-116 us, e4m3 117-119.
#pragma once
#include <type_traits>

#include "attn_common.cuh"

namespace ead {

constexpr int kFewHalf = 4096;                    // bytes of keys (of values) per stage
constexpr int kFewScaleBytes = 256;               // scale bytes of keys and values per stage
constexpr float kLazyLog2 = 8.f;                  // the reference maximum moves when a logit exceeds it by 2^8

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    // volatile: stays before the refill of the stage its operands came from
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with an accumulator of zeros.
__device__ __forceinline__ void mma16816_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Codes in bits 0-15 (16-31) as a pair of f16.
__device__ __forceinline__ uint32_t codes_to_f16x2_lo(uint32_t codes)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(codes));
    return r;
}
__device__ __forceinline__ uint32_t codes_to_f16x2_hi(uint32_t codes)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(codes));
    return r;
}
// Codes 0 and 2 (1 and 3) as a pair of bf16 times 2^-120.
__device__ __forceinline__ uint32_t codes_to_bf16x2_even(uint32_t codes)
{
    return ((codes << 8) & 0x80008000u) | ((codes << 4) & 0x07F007F0u);
}
__device__ __forceinline__ uint32_t codes_to_bf16x2_odd(uint32_t codes)
{
    return (codes & 0x80008000u) | ((codes >> 4) & 0x07F007F0u);
}
// 2^(byte - 127) for byte `g` of a key's scale bytes (0 for byte 0, which the library never writes).
__device__ __forceinline__ float key_scale(uint32_t bytes, int g)
{
    return __uint_as_float(__byte_perm(bytes, 0, 0x0444u | g << 12) >> 1);
}
constexpr uint32_t kValueScaleTop = 125;          // largest byte whose factor 2^(120 + k), times a probability of up to 2^8, is a bf16

// The NG scale bytes of one key, as the low bytes of a register.
template <int NG>
__device__ __forceinline__ uint32_t lds_scales(uint32_t addr)
{
    uint32_t v;
    if (NG == 4) {
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    } else {
        asm volatile("{\n\t.reg .b16 t;\n\tld.shared.b16 t, [%1];\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(v) : "r"(addr) : "memory");
    }
    return v;
}

// A warp's place in the string of tiles: unit, its keys, and where the unit lies.
struct FewCursor {
    int b, h;                                     // sequence, cache head
    int begin;                                    // the unit's first tile, counted from the first of the block's stretch
    SeqInfo s;
    KeyRange r;
};

__device__ __forceinline__ int few_tiles(const AttnParams &p, const SeqInfo &s, int shift, KeyRange *r)
{
    if (s.n < 1 || s.n * static_cast<int64_t>(p.group) > p.few_rows) return 0;
    *r = key_range(s.p0, s.p0 + s.n - 1, s.len, p.window, p.sinks, shift);
    return r->tiles;
}
// Moves on to the unit that holds tile g of the string (g is in this unit or a later one; the search ends with the batch,
// whatever its arrays hold: the last sequence then counts as one without an end).
__device__ __forceinline__ void few_seek(const AttnParams &p, int shift, int g, FewCursor *c)
{
    while (g >= c->begin + c->r.tiles) {
        c->begin += c->r.tiles;
        if (c->r.tiles > 0 && c->h + 1 < p.cache.heads) {
            ++c->h;
        } else {
            c->h = 0;
            do {
                if (c->b + 1 >= p.batch.B) {
                    c->r.tiles = 0x7fffffff - max(c->begin, 0);
                    return;
                }
                ++c->b;
                c->s = seq_info(p.batch, c->b);
                c->r.tiles = few_tiles(p, c->s, shift, &c->r);
            } while (c->r.tiles == 0);
        }
    }
}

// Units of at most so many tiles are not divided among blocks: joining parts costs more than the imbalance where contexts are
// short.  Measured, 48 against 0 (always divided), us: 4 contexts of 300 keys, 2 heads of 128, bf16 8.2 / 12.8; 64 of 300, 8 heads
// of 128, bf16 20.9 / 25.2, e4m3 23.9 / 30.0; 16 of 1500, 8 heads of 64, e4m3 14.0 / 19.5; one of 777, 8 heads of 64, bf16 9.9 / 13.9;
// one of 1500, 2 heads of 128, bf16 16.7 / 15.6 (the largest loss).  Longer units, divided either way, differ by up to 6 %.
constexpr int kFewWholeTiles = 48;

// NB: packed rows in groups of 8 (1 or 2).
template <int FMT, int D, int NB>
struct FewLayout {
    static constexpr int kRowBytes = FMT == kFmtBf16 ? 2 * D : D;           // bytes of one key
    static constexpr int kTile = kFewHalf / kRowBytes;                      // keys per tile: 16, 32 or 64
    static constexpr int kShift = kTile == 16 ? 4 : kTile == 32 ? 5 : 6;
    static constexpr int kLine = kRowBytes < 128 ? kRowBytes : 128;         // bytes of a key in one box
    static constexpr int kBoxes = kRowBytes / kLine;                        // boxes per key row (2 for 256-byte keys)
    static constexpr int kRows = 8 * NB;
    // An 8-bit cache is bound by instructions, not bytes: three warps per scheduler, a tile's steps one after the other.
    // Otherwise two warps per scheduler and a tile's steps side by side.
    static constexpr bool kManyWarps = FMT == kFmtE4m3 && NB == 1;
    static constexpr int kWarps = kManyWarps ? 12 : 8;
    static constexpr int kSide = kManyWarps ? 1 : kTile / 16;               // steps of 16 keys worked on at once
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kMergeRow = D + 4;                                 // floats; the padding spreads the rows over the banks
    static constexpr int kByRows = kRows * kMergeRow + 2 * kRows, kByLanes = kRows * D + NB * 128;   // output, maxima and sums
    static constexpr int kMergeWarp = kByRows > kByLanes ? kByRows : kByLanes;
    static constexpr int kMergeBytes = kWarps / 2 * kMergeWarp * 4;
    static constexpr int kStages = NB == 1 && !kManyWarps ? 3 : 2;
    static constexpr int kRing = kWarps * kStages * 2 * kFewHalf;
    static constexpr int kScales = FMT == kFmtE4m3 ? kWarps * kStages * kFewScaleBytes : 0;
    static_assert(kMergeWarp % 4 == 0, "rows are read 16 bytes at a time");
    static constexpr int kSmem = 1024 + kRing + kScales + kMergeBytes + kWarps * kStages * 8;
};

template <int FMT, int D, int NB>
__global__ void __launch_bounds__(FewLayout<FMT, D, NB>::kThreads, 1)
    ead_attn_few_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, AttnParams p,
                             int box_shift, int min_tiles)
{
    using L = FewLayout<FMT, D, NB>;
    constexpr int S = L::kStages, TT = L::kTile, R = L::kRows, kFewWarps = L::kWarps, kFewThreads = L::kThreads;
    constexpr int NS = L::kSide, PER = 8 / (TT / 16);   // steps of 16 keys at once, fragment loads per step
    const int box_keys = 1 << box_shift;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int64_t s_scan[kFewWarps];
    __shared__ int s_b[2];
    __shared__ int64_t s_before[2];
    __shared__ int s_last;
    const uint32_t raw = smem_u32(smem_raw), ring0 = (raw + 1023u) & ~1023u;
    uint8_t *const ring_ptr = smem_raw + (ring0 - raw);
    uint8_t *const scales_ptr = ring_ptr + L::kRing;
    float *const merge = reinterpret_cast<float *>(scales_ptr + L::kScales);
    const uint32_t bars = smem_u32(reinterpret_cast<uint8_t *>(merge) + L::kMergeBytes);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvCacheView &c = p.cache;

    griddep_launch_dependents();                   // the chunk kernel of the same step needs nothing of this one but its SMs
    if (tid == 0) {
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
    }
    if (tid < kFewWarps * S) mbar_init(bars + 8 * tid, 1);
    fence_mbar_init();

    // ---- the string of tiles: its length, and the sequence in which this block's stretch begins
    const int per = (p.batch.B + kFewThreads - 1) / kFewThreads;
    const int b_lo = min(tid * per, p.batch.B), b_hi = min(b_lo + per, p.batch.B);
    int64_t mine = 0;
    KeyRange kr;
    for (int b = b_lo; b < b_hi; ++b) {
        bool bad;
        const SeqInfo s = seq_info(p.batch, b, &bad);
        mine += few_tiles(p, s, L::kShift, &kr);
        if (blockIdx.x == 0 && bad) flag_status(p.status, kStatusBadCount);
        if (blockIdx.x == 0 && s.n > 0 && s.p0 + s.n > p.batch.max_len) flag_status(p.status, kStatusBadPage);
    }
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) s_scan[warp] = upto;
    __syncthreads();
    int64_t total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    upto += before;                                // tiles of one head up to and including this thread's sequences
    const int64_t W = total * c.heads;
    const int64_t ctas = min(static_cast<int64_t>(gridDim.x), max(static_cast<int64_t>(1), (W + min_tiles - 1) / min_tiles));
    if (W == 0 || blockIdx.x >= ctas) return;
    const Stretches even(W, static_cast<int>(ctas));
    // The sequences in which the two ends of the block's stretch lie.  (The code up to the first loads runs once and
    // from a cold instruction cache: loops stay loops.)
#pragma unroll 1
    for (int64_t b = b_lo, at = upto - mine; b < b_hi; ++b) {
        const int t = per == 1 ? static_cast<int>(mine) : few_tiles(p, seq_info(p.batch, b), L::kShift, &kr);
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            const int64_t g = even.begin(blockIdx.x + e);
            if (g >= at * c.heads && g < (at + t) * c.heads) {
                s_b[e] = b;
                s_before[e] = at * c.heads;
            }
        }
        at += t;
    }
    __syncthreads();
    FewCursor cur;
    int64_t cur_begin = 0, g0 = 0, g1 = W;
    bool next_unit = false;
#pragma unroll 1
    for (int e = 1; e >= 0; --e) {                 // a short unit is not divided: an end within it moves to its nearer end
        int64_t g = even.begin(blockIdx.x + e);
        if (g < W) {
            cur.b = s_b[e];
            cur.s = seq_info(p.batch, cur.b);
            cur.r.tiles = few_tiles(p, cur.s, L::kShift, &cur.r);
            const int64_t off = g - s_before[e];
            cur.h = off < 0x7fffffff ? static_cast<int>(off) / cur.r.tiles : static_cast<int>(off / cur.r.tiles);
            cur_begin = s_before[e] + static_cast<int64_t>(cur.h) * cur.r.tiles;
            next_unit = false;
            if (cur.r.tiles <= kFewWholeTiles && g > cur_begin) {
                next_unit = 2 * (g - cur_begin) >= cur.r.tiles;
                g = next_unit ? cur_begin + cur.r.tiles : cur_begin;
            }
        }
        (e ? g1 : g0) = g;
    }
    if (g0 >= g1) return;
    cur.begin = static_cast<int>(cur_begin - g0);
    const int n_tiles = static_cast<int>(g1 - g0);  // from here on tiles are counted from g0
    if (next_unit) few_seek(p, L::kShift, 0, &cur);

    // ---- loads: this warp's tiles are warp, warp + kFewWarps, ...
    const uint32_t my_ring = ring0 + warp * S * 2 * kFewHalf;
    const uint32_t my_scales = smem_u32(scales_ptr) + warp * S * kFewScaleBytes;
    const uint32_t my_bars = bars + warp * S * 8;
    FewCursor ahead = cur;
    int g_ahead = warp;
    const int boxes = TT >> box_shift;              // at most 8
    // This lane's box of a tile that is to be loaded.
    struct Box {
        int entry;                                 // page as the table has it, or -2 if no query sees any of it
        int key0, h;
        bool tile;                                 // is there such a tile?
    };
    // One tile early, so that the entry is there when the tile is issued (nothing here waits for it).
    auto look_up = [&]() {
        Box x{-2, 0, 0, g_ahead < n_tiles};
        if (x.tile) {
            few_seek(p, L::kShift, g_ahead, &ahead);
            x.key0 = ahead.r.base(g_ahead - ahead.begin, L::kShift) + lane * box_keys;
            x.h = ahead.h;
            if (lane < boxes && x.key0 < ahead.r.hi && (x.key0 + box_keys > ahead.r.lo || x.key0 < p.sinks))
                x.entry = max(__ldg(p.batch.page_table + static_cast<int64_t>(ahead.b) * p.batch.table_stride + (x.key0 >> c.page_shift)), -1);
            g_ahead += kFewWarps;
        }
        return x;
    };
    auto issue = [&](int stage, const Box &x) {
        if (!x.tile) return;
        int page = x.entry;
        if (page != -2 && (page < 0 || page >= c.n_pages)) {
            flag_status(p.status, kStatusBadPage);
            page = c.n_pages;                      // outside the pool: the copy delivers zeros
        }
        const int key0 = x.key0;
        const unsigned live = __ballot_sync(0xffffffffu, lane < boxes && page >= 0);
        const uint32_t bar = my_bars + 8 * stage, dst = my_ring + stage * 2 * kFewHalf;
        const uint32_t box_bytes = box_keys * L::kRowBytes;
        const uint32_t sc_bytes = box_keys * (D / kFmtBlock);
        if (FMT == kFmtE4m3) {
            const unsigned scaled = __ballot_sync(0xffffffffu, lane < boxes && page >= 0 && page < c.n_pages);
            if (lane == 0) mbar_arrive_expect_tx(bar, 2 * __popc(live) * box_bytes + 2 * __popc(scaled) * sc_bytes);
        } else if (lane == 0) {
            mbar_arrive_expect_tx(bar, 2 * __popc(live) * box_bytes);
        }
        __syncwarp();
        if (lane < boxes && page >= 0) {
            const int slot = key0 & (c.page_size - 1);
            tma_load_5d(dst + lane * box_bytes, &tmK, 0, slot, 0, x.h, page, bar);
            tma_load_5d(dst + kFewHalf + lane * box_bytes, &tmV, 0, slot, 0, x.h, page, bar);
            if (FMT == kFmtE4m3) {
                const uint32_t sc = my_scales + stage * kFewScaleBytes + lane * sc_bytes;
                if (page < c.n_pages) {
                    const int64_t at = scale_offset(c, page, x.h, slot);
                    bulk_load(sc, c.k_scale + at, sc_bytes, bar);
                    bulk_load(sc + kFewScaleBytes / 2, c.v_scale + at, sc_bytes, bar);
                } else {
                    for (uint32_t y = 0; y < sc_bytes; y += 4) {
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(sc + y), "r"(0) : "memory");
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(sc + kFewScaleBytes / 2 + y), "r"(0) : "memory");
                    }
                }
            }
        }
        __syncwarp();
    };
    Box next_box = look_up();
#pragma unroll 1
    for (int i = 0; i < S; ++i) {
        issue(i, next_box);
        next_box = look_up();
    }

    // ---- tiles, unit by unit
    const int qc = (lane & 3) * 2;                 // this lane's packed rows: qc, qc + 1 (and 8 more)
    // Where this lane's row of an 8 x 16-byte matrix lies within a tile, for the first four fragment loads of a step;
    // later ones are a line (256-byte keys), later steps 16 keys further on.
    const int mi = lane >> 3, mr = lane & 7;       // matrix and row this lane addresses
    const uint32_t line_step = L::kBoxes == 2 ? box_keys * 128u : 0u;
    auto chunk_at = [&](int key, int ch) -> uint32_t {
        if (L::kLine == 64) return key * 64u + ((ch ^ ((key >> 1) & 3)) << 4);
        const uint32_t row = L::kBoxes == 2 ? (key >> box_shift) * 2u * box_keys + (key & (box_keys - 1)) : key;
        return row * 128u + ((ch ^ (key & 7)) << 4);
    };
    uint32_t off_k[4], off_v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        off_k[j] = chunk_at(mr + (mi & 1) * 8, 2 * j + (mi >> 1));
        off_v[j] = FMT == kFmtBf16 ? chunk_at(mr + (mi >> 1) * 8, 2 * j + (mi & 1)) : off_k[j];
    }
    // Query rows as the 8-column operand: a lane holds rows lane / 4 (+ 8), elements by the layout of the keys.  With one
    // group of rows those of the next unit are fetched while this one's parts are joined.
    uint32_t q_next[D / 16][NB][2];
    auto query_rows = [&](const FewCursor &u) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int row = nb * 8 + (lane >> 2);
            const int i = row / p.group, gq = row - i * p.group;
            const uint8_t *src = p.q + 2 * ((static_cast<int64_t>(u.s.token0) + i) * p.q_stride + (static_cast<int64_t>(u.h) * p.group + gq) * D);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                q_next[ks][nb][0] = q_next[ks][nb][1] = 0;
                if (row < u.s.n * p.group) {
                    if (FMT == kFmtBf16) {
                        q_next[ks][nb][0] = __ldg(reinterpret_cast<const uint32_t *>(src + 2 * (16 * ks + (lane & 3) * 2)));
                        q_next[ks][nb][1] = __ldg(reinterpret_cast<const uint32_t *>(src + 2 * (16 * ks + (lane & 3) * 2 + 8)));
                    } else {                       // four consecutive codes per lane: elements 4c .. 4c + 3 of the step
                        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(src + 2 * (16 * ks + (lane & 3) * 4)));
                        q_next[ks][nb][0] = v.x;
                        q_next[ks][nb][1] = v.y;
                    }
                }
            }
        }
    };
    int stage = 0;
    uint32_t phase = 0;
    int g = warp, unit_lo = 0;
    while (unit_lo < n_tiles) {
        const int unit_end = cur.begin + cur.r.tiles, unit_hi = min(unit_end, n_tiles);
        const int rows = cur.s.n * p.group;
        const int64_t token0 = cur.s.token0;
        if (NB == 2 || unit_lo == 0) query_rows(cur);
        uint32_t qf[D / 16][NB][2];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                qf[ks][nb][0] = q_next[ks][nb][0];
                qf[ks][nb][1] = q_next[ks][nb][1];
            }
        float row_scale[NB][2];                    // of this lane's rows' logits
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            row_scale[nb][0] = row_scale[nb][1] = p.scale_log2;
            if (FMT == kFmtE4m3) {                 // the four lanes of a row bring it to f16
                uint32_t top = 0;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        top = max(top, max(abs_bits(bf16_lo(qf[ks][nb][e])), abs_bits(bf16_hi(qf[ks][nb][e]))));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // exponent of the largest element; a row of zeros or one that is not finite stays as it is
                const int ex = top < 0x00800000u || top >= 0x7f800000u ? 127 : min(static_cast<int>(top >> 23), 253);
                const float down = __uint_as_float(static_cast<uint32_t>(254 - ex) << 23);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const __half2 h = __floats2half2_rn(bf16_lo(qf[ks][nb][e]) * down, bf16_hi(qf[ks][nb][e]) * down);
                        qf[ks][nb][e] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                const float up = __uint_as_float(static_cast<uint32_t>(ex) << 23);
#pragma unroll
                for (int e = 0; e < 2; ++e) row_scale[nb][e] = p.scale_log2 * __shfl_sync(0xffffffffu, up, (qc + e) * 4);
            }
        }
        int pos[NB][2];                            // positions of this lane's rows
        float m[NB][2], l[NB][2];
        float o[D / 16][NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                pos[nb][e] = cur.s.p0 + (nb * 8 + qc + e) / p.group;
                m[nb][e] = -INFINITY;
                l[nb][e] = 0.f;
            }
#pragma unroll
        for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][nb][e] = 0.f;
        const int pb = cur.s.p0 + cur.s.n - 1;

        for (; g < unit_hi; g += kFewWarps) {
            const int base = cur.r.base(g - cur.begin, L::kShift);
            const bool whole = base + TT - 1 <= cur.s.p0 && base + TT <= cur.s.len &&
                               (p.window == 0 || base > pb - p.window || base + TT <= p.sinks);
            uint32_t kb = my_ring + stage * 2 * kFewHalf, vb = kb + kFewHalf;
            if (!wait_phase(my_bars + 8 * stage, phase, p, nullptr)) {
                // the status says that the result is not valid; this warp's loads come in, then it leaves (barriers do not wait for it)
                for (int x = (g - warp) / kFewWarps, end = min(x + S, (n_tiles - warp + kFewWarps - 1) / kFewWarps); x < end; ++x)
                    wait_own(my_bars + 8 * (x % S), (x / S) & 1);
                return;
            }
            __syncwarp();
            // Steps of 16 keys, NS of them side by side: the fragment loads for the keys, all score products, the loads
            // for the values (their latency runs under the softmax), then the products with them.
#pragma unroll 1
            for (int t0 = 0; t0 < TT; t0 += 16 * NS, kb += 16 * NS * L::kRowBytes, vb += 16 * NS * L::kRowBytes) {
            uint32_t frag[NS * PER][4];
#pragma unroll
            for (int x = 0; x < NS * PER; ++x)
                ldsm4(frag[x], kb + off_k[x % PER & 3] + (x / PER) * 16 * L::kRowBytes + (x % PER >> 2) * line_step);
            bool far = false;                                    // some value scale is too large for the probabilities to take it in
            uint32_t ksc[NS][2], vsc[NS][4];
            if (FMT == kFmtE4m3) {
                constexpr int NG = D / kFmtBlock;               // scale bytes per key
                const uint32_t sb = my_scales + stage * kFewScaleBytes + t0 * NG;
                uint32_t over = 0;
#pragma unroll
                for (int st = 0; st < NS; ++st) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) ksc[st][i] = lds_scales<NG>(sb + (st * 16 + (lane >> 2) + 8 * i) * NG);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        vsc[st][i] = lds_scales<NG>(sb + 128 + (st * 16 + qc + (i & 1) + 8 * (i >> 1)) * NG);
                        over |= vsc[st][i] | (vsc[st][i] + (127u - kValueScaleTop) * 0x01010101u);   // bit 7 of a byte above 125
                    }
                }
                far = __any_sync(0xffffffffu, (over & 0x80808080u) != 0);
            }
            float s[NS][NB][4];
#pragma unroll
            for (int st = 0; st < NS; ++st)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[st][nb][0] = s[st][nb][1] = s[st][nb][2] = s[st][nb][3] = 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    const uint32_t(&a)[4] = frag[st * PER + j];
                    if (FMT == kFmtBf16) {
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma16816(s[st][nb], a[0], a[1], a[2], a[3], qf[j][nb][0], qf[j][nb][1]);
                    } else {                                    // one scale block: two steps of 16 dimensions
                        float sb[NB][4];
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {       // matrices 0, 2 (keys 0-7) and 1, 3 (keys 8-15)
                            mma16816_f16_first(sb[nb], codes_to_f16x2_lo(a[0]), codes_to_f16x2_lo(a[1]), codes_to_f16x2_hi(a[0]),
                                               codes_to_f16x2_hi(a[1]), qf[2 * j][nb][0], qf[2 * j][nb][1]);
                            mma16816_f16(sb[nb], codes_to_f16x2_lo(a[2]), codes_to_f16x2_lo(a[3]), codes_to_f16x2_hi(a[2]),
                                         codes_to_f16x2_hi(a[3]), qf[2 * j + 1][nb][0], qf[2 * j + 1][nb][1]);
                        }
                        const float f0 = key_scale(ksc[st][0], j), f1 = key_scale(ksc[st][1], j);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            s[st][nb][0] = fmaf(sb[nb][0], f0, s[st][nb][0]);
                            s[st][nb][1] = fmaf(sb[nb][1], f0, s[st][nb][1]);
                            s[st][nb][2] = fmaf(sb[nb][2], f1, s[st][nb][2]);
                            s[st][nb][3] = fmaf(sb[nb][3], f1, s[st][nb][3]);
                        }
                    }
                }
#pragma unroll
            for (int x = 0; x < NS * PER; ++x) {
                ldsm4_t(frag[x], vb + off_v[x % PER & 3] + (x / PER) * 16 * L::kRowBytes + (x % PER >> 2) * line_step);
            }
            // logits in units of log 2; what is not seen is -inf
            bool above = false;                                 // some logit exceeds its row's reference by too much
#pragma unroll
            for (int st = 0; st < NS; ++st)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float &z = s[st][nb][e];
                        z *= row_scale[nb][e & 1];
                        if (!whole) {
                            const int j = base + t0 + st * 16 + (lane >> 2) + 8 * (e >> 1);
                            if (!(j < cur.s.len && seen_by(pos[nb][e & 1], p.window, p.sinks, j))) z = -INFINITY;
                        }
                        above |= z > m[nb][e & 1] + kLazyLog2;
                    }
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = m[nb][e];
#pragma unroll
                        for (int st = 0; st < NS; ++st) x = fmaxf(x, fmaxf(s[st][nb][e], s[st][nb][e + 2]));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        const float f = x == -INFINITY ? 1.f : exp2_fast(m[nb][e] - x);
                        m[nb][e] = x;
                        l[nb][e] *= f;
#pragma unroll
                        for (int mt = 0; mt < D / 16; ++mt) {
                            o[mt][nb][e] *= f;
                            o[mt][nb][e + 2] *= f;
                        }
                    }
            }
            uint32_t pf[NS][NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float mm[2] = {m[nb][0] == -INFINITY ? 0.f : m[nb][0], m[nb][1] == -INFINITY ? 0.f : m[nb][1]};
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = exp2_fast(s[st][nb][e] - mm[e & 1]);
                        l[nb][e & 1] += x[e];
                    }
                    pf[st][nb][0] = transpose8x8(to_bf16x2(x[0], x[1]));
                    pf[st][nb][1] = transpose8x8(to_bf16x2(x[2], x[3]));
                }
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                // values no query sees may be anything, and were not even loaded: zeros, so that 0 * NaN cannot arise
                uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int j = base + t0 + st * 16 + qc + 8 * i;
                        keep[i] = (seen_by_any(cur.r, p.sinks, j) ? 0xffffu : 0u) | (seen_by_any(cur.r, p.sinks, j + 1) ? 0xffff0000u : 0u);
                    }
                }
                if (FMT == kFmtBf16) {
#pragma unroll
                    for (int mt = 0; mt < D / 16; ++mt) {
                        uint32_t(&a)[4] = frag[st * PER + mt];
                        if (!whole) {
                            a[0] &= keep[0]; a[1] &= keep[0];
                            a[2] &= keep[1]; a[3] &= keep[1];
                        }
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma16816(o[mt][nb], a[0], a[1], a[2], a[3], pf[st][nb][0], pf[st][nb][1]);
                    }
                } else {
                    // scale bytes of keys 2c, 2c + 1, then of keys 2c + 8, 2c + 9, one per half, block by block
                    uint32_t pair[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t e0 = vsc[st][2 * i] & 0x00ff00ffu, e1 = vsc[st][2 * i + 1] & 0x00ff00ffu;
                        const uint32_t o0 = (vsc[st][2 * i] >> 8) & 0x00ff00ffu, o1 = (vsc[st][2 * i + 1] >> 8) & 0x00ff00ffu;
                        pair[i][0] = __byte_perm(e0, e1, 0x5410);
                        pair[i][1] = __byte_perm(o0, o1, 0x5410);
                        pair[i][2] = __byte_perm(e0, e1, 0x7632);
                        pair[i][3] = __byte_perm(o0, o1, 0x7632);
                    }
                    if (!whole) {                  // any code is finite: with a finite factor what no query sees counts 0
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) pair[i][j] &= keep[i];
                    }
                    auto values = [&](auto is_far) {
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) {
                            const uint32_t(&a)[4] = frag[st * PER + j];
                            uint32_t w[NB][2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                // the factors: 2^(120 + k), or 2^k where the values themselves are brought to size
                                uint32_t f = pair[i][j] * 128u + (decltype(is_far)::value ? 0u : 0x3C003C00u);
                                if (decltype(is_far)::value) {                   // byte 255 marks NaNs
                                    if ((f & 0xffffu) == 0x7f80u) f |= 0x40u;
                                    if ((f >> 16) == 0x7f80u) f |= 0x400000u;
                                }
#pragma unroll
                                for (int nb = 0; nb < NB; ++nb) w[nb][i] = mul_bf16x2(pf[st][nb][i], f);
                            }
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                uint32_t v[4];
                                v[0] = codes_to_bf16x2_even(a[2 * u]);
                                v[1] = codes_to_bf16x2_odd(a[2 * u]);
                                v[2] = codes_to_bf16x2_even(a[2 * u + 1]);
                                v[3] = codes_to_bf16x2_odd(a[2 * u + 1]);
                                if (decltype(is_far)::value) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) v[i] = mul_bf16x2(v[i], 0x7B807B80u);   // 2^120
                                }
#pragma unroll
                                for (int nb = 0; nb < NB; ++nb) mma16816(o[2 * j + u][nb], v[0], v[1], v[2], v[3], w[nb][0], w[nb][1]);
                            }
                        }
                    };
                    if (far)
                        values(std::true_type{});
                    else
                        values(std::false_type{});
                }
            }
            }
            __syncwarp();                          // every lane has read the stage before it is filled again
            issue(stage, next_box);
            next_box = look_up();
            if (++stage == S) {
                stage = 0;
                phase ^= 1;
            }
        }

        FewCursor after = cur;
        if (unit_hi < n_tiles) {
            few_seek(p, L::kShift, unit_hi, &after);
            if (NB == 1) query_rows(after);
        }
        // ---- the warps' parts of the unit come together: the upper half of the warps hand theirs to the lower half lane by lane,
        // those lay them out by rows
        constexpr int kHalf = kFewWarps / 2;
        if (warp >= kHalf) {
            float *mw = merge + (warp - kHalf) * L::kMergeWarp + lane;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mw[((mt * NB + nb) * 4 + e) * 32] = o[mt][nb][e];
            }
            float *ml = mw + R * D;                // behind the fragments
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    ml[(nb * 4 + e) * 32] = m[nb][e];
                    ml[(nb * 4 + 2 + e) * 32] = l[nb][e];
                }
        }
        __syncthreads();
        if (warp < kHalf) {
            const float *src = merge + warp * L::kMergeWarp + lane, *ml = src + R * D;
            float f[NB][2], f2[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float m2 = ml[(nb * 4 + e) * 32], l2 = ml[(nb * 4 + 2 + e) * 32], M = fmaxf(m[nb][e], m2);
                    f[nb][e] = m[nb][e] == -INFINITY ? 0.f : exp2_fast(m[nb][e] - M);
                    f2[nb][e] = m2 == -INFINITY ? 0.f : exp2_fast(m2 - M);
                    l[nb][e] = l[nb][e] * f[nb][e] + l2 * f2[nb][e];
                    m[nb][e] = M;
                }
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[mt][nb][e] = o[mt][nb][e] * f[nb][e & 1] + src[((mt * NB + nb) * 4 + e) * 32] * f2[nb][e & 1];
            __syncwarp();
            float *mw = merge + warp * L::kMergeWarp;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[nb][e] += __shfl_xor_sync(0xffffffffu, l[nb][e], x);
                    const int row = nb * 8 + qc + e;
#pragma unroll
                    for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int d = 16 * mt + (FMT == kFmtBf16 ? (lane >> 2) + 8 * u : 2 * (lane >> 2) + u);
                            mw[row * L::kMergeRow + d] = o[mt][nb][e + 2 * u];
                        }
                    if (lane < 4) {
                        mw[R * L::kMergeRow + row] = m[nb][e];
                        mw[R * L::kMergeRow + R + row] = l[nb][e];
                    }
                }
        }
        __syncthreads();
        const bool begins = unit_lo == cur.begin, ends = unit_hi == unit_end;
        float *const parts = reinterpret_cast<float *>(p.workspace + kDecodePartOffset);
        uint32_t *const counters = reinterpret_cast<uint32_t *>(p.workspace);
        float *const my_part = parts + (2 * blockIdx.x + (begins ? 1 : 0)) * kDecodePartFloats;   // a block has one part of each kind at most
        constexpr int kQuads = D / 4;
        auto store = [&](int row, int dq, float M, float Lsum, float4 v) {
            const int i = row / p.group, gq = row - i * p.group;
            const float inv = Lsum == 0.f ? 0.f : 1.f / Lsum;
            const int hq = cur.h * p.group + gq;
            *reinterpret_cast<uint2 *>(p.out + 2 * ((token0 + i) * p.out_stride + static_cast<int64_t>(hq) * D + 4 * dq)) =
                make_uint2(to_bf16x2(v.x * inv, v.y * inv), to_bf16x2(v.z * inv, v.w * inv));
            if (p.lse && dq == 0) p.lse[(token0 + i) * p.heads_q + hq] = Lsum == 0.f ? -INFINITY : (M + log2f(Lsum)) * kLn2;
        };
        for (int x = tid; x < rows * kQuads; x += kFewThreads) {
            const int row = x / kQuads, dq = x - row * kQuads;
            float M = -INFINITY, Lsum = 0.f;
#pragma unroll
            for (int w = 0; w < kHalf; ++w) M = fmaxf(M, merge[w * L::kMergeWarp + R * L::kMergeRow + row]);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kHalf; ++w) {
                const float *src = merge + w * L::kMergeWarp;
                const float mm = src[R * L::kMergeRow + row];
                const float f = mm == -INFINITY ? 0.f : exp2_fast(mm - M);
                const float4 y = *reinterpret_cast<const float4 *>(src + row * L::kMergeRow + 4 * dq);
                Lsum += f * src[R * L::kMergeRow + R + row];
                v.x += f * y.x; v.y += f * y.y; v.z += f * y.z; v.w += f * y.w;
            }
            if (begins && ends) {
                store(row, dq, M, Lsum, v);
            } else {
                *reinterpret_cast<float4 *>(my_part + row * D + 4 * dq) = v;
                if (dq == 0) {
                    my_part[kDecodeRows * 128 + row] = M;
                    my_part[kDecodeRows * 128 + kDecodeRows + row] = Lsum;
                }
            }
        }
        if (!(begins && ends)) {
            // blocks that hold a part of the unit: first .. last; the counter is the first one's
            const int first = even.block_of(g0 + cur.begin), last = even.block_of(g0 + unit_end - 1);
            fence_gpu();
            __syncthreads();
            if (tid == 0) {
                const uint32_t seen = atomicAdd(counters + first, 1u);
                s_last = seen == static_cast<uint32_t>(last - first);
                if (s_last) counters[first] = 0;   // ready for the next call
            }
            __syncthreads();
            if (s_last) {
                fence_gpu();
                for (int x = tid; x < rows * kQuads; x += kFewThreads) {
                    const int row = x / kQuads, dq = x - row * kQuads;
                    float M = -INFINITY, Lsum = 0.f;
                    for (int k = first; k <= last; ++k)
                        M = fmaxf(M, __ldcg(parts + (2 * k + (k == first ? 1 : 0)) * kDecodePartFloats + kDecodeRows * 128 + row));
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int k = first; k <= last; ++k) {
                        const float *src = parts + (2 * k + (k == first ? 1 : 0)) * kDecodePartFloats;
                        const float mm = __ldcg(src + kDecodeRows * 128 + row);
                        const float f = mm == -INFINITY ? 0.f : exp2_fast(mm - M);
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(src + row * D + 4 * dq));
                        Lsum += f * __ldcg(src + kDecodeRows * 128 + kDecodeRows + row);
                        v.x += f * y.x; v.y += f * y.y; v.z += f * y.z; v.w += f * y.w;
                    }
                    store(row, dq, M, Lsum, v);
                }
            }
        }
        __syncthreads();                           // the merge buffer is free again
        unit_lo = unit_hi;
        cur = after;
    }
}

}  // namespace ead
