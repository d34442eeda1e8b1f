// What the attention kernels share: parameters, which keys a run of queries sees as a list of tiles,
// how work is dealt out to blocks, and how parts of one result are joined.
//
// A UNIT is a run of query rows that share their keys: (sequence, cache head, run of new tokens), all
// query heads of the group together.  Its keys are cut into tiles, all units' tiles are strung up one
// after the other, and every block takes an equal stretch of that string.  A block whose stretch ends inside a
// unit leaves its part (running maximum, sum, unnormalised output) in the workspace; the last block of a unit to arrive
// joins the parts in the order of the blocks, so the result does not depend on who comes last.
#pragma once
#include "kv_format.cuh"
#include "ptx_sm100.cuh"

namespace ead {

struct AttnParams {
    KvCacheView cache;
    KvBatchView batch;
    const uint8_t *q;
    uint8_t *out;
    float *lse;
    int64_t q_stride, out_stride;                 // elements between tokens
    int32_t heads_q, group, window, sinks;
    int32_t few_rows;                             // units of at most this many packed rows go to the few-rows kernel
    int32_t tile_tokens;                          // chunk kernel: whole tokens in a tile of 128 rows
    float scale_log2;                             // scale * log2(e): logits are kept in units of log 2
    uint32_t *status;
    uint8_t *workspace;
    uint32_t wait_ns, wait_hint;                  // when a wait has run out, and how long one look at a barrier may last
};

constexpr float kLn2 = 0.6931471805599453f;

// Workspace: arrival counters, one of 32 bits per block (zero between calls), of the few-rows kernel, then of the chunk kernel,
// then the partial results of each.
constexpr size_t kAttnCounterBytes = 4096;        // per kernel
constexpr int kAttnMaxCtas = 160;
static_assert(kAttnMaxCtas * sizeof(uint32_t) <= kAttnCounterBytes, "a counter per block");
constexpr int kDecodeRows = 16;                   // most packed rows of a unit of the few-rows kernel
constexpr size_t kDecodePartFloats = kDecodeRows * (128 + 2);
constexpr size_t kDecodePartOffset = 2 * kAttnCounterBytes;

// The new tokens and the readable context of a sequence.
struct SeqInfo {
    int n, p0, len;                               // new tokens, position of the first one, keys in the cache
    int token0;                                   // first new token's row of the step
};
// A sequence whose new tokens contradict the host's bounds counts as one without any (`bad`).
__device__ __forceinline__ SeqInfo seq_info(const KvBatchView &bt, int b, bool *bad = nullptr)
{
    SeqInfo s;
    const int kv = max(__ldg(bt.kv_len + b), 0), end = __ldg(bt.new_start + b + 1);
    s.token0 = __ldg(bt.new_start + b);
    s.n = end - s.token0;
    s.p0 = kv - s.n;
    s.len = min(kv, bt.max_len);
    const bool wrong = s.n < 0 || s.n > bt.max_new || s.token0 < 0 || end > bt.n_tokens;
    if (wrong) s.n = 0;
    if (bad) *bad = wrong;
    return s;
}

// Tiles of 2^shift keys that queries at positions pa .. pb see: those of the sinks, then those of
// the window.  At least one tile, so that rows that see nothing are still written.
struct KeyRange {
    int lo, hi;                                   // window part [lo, hi); sinks are [0, min(sinks, lo))
    int sink_tiles, first_tile, tiles;
    __host__ __device__ __forceinline__ int base(int t, int shift) const
    {
        return (t < sink_tiles ? t : t - sink_tiles + first_tile) << shift;
    }
};
// (A negative pb + 1 leaves nothing.  Positions are at least -2^30 and the window at most 2^30: nothing overflows.)
__host__ __device__ __forceinline__ KeyRange key_range(int pa, int pb, int len, int window, int sinks, int shift)
{
    KeyRange r;
    r.hi = min(max(pb + 1, 0), len);
    r.lo = window ? min(max(pa - window + 1, 0), r.hi) : 0;
    r.first_tile = r.lo >> shift;
    r.sink_tiles = min((min(sinks, r.lo) + (1 << shift) - 1) >> shift, r.first_tile);
    r.tiles = max(1, r.sink_tiles + ((r.hi + (1 << shift) - 1) >> shift) - r.first_tile);
    return r;
}
// Whether any of the unit's queries sees key j, and whether one at position pos does.
__device__ __forceinline__ bool seen_by_any(const KeyRange &r, int sinks, int j) { return j < r.hi && (j >= r.lo || j < sinks); }
__device__ __forceinline__ bool seen_by(int pos, int window, int sinks, int j)
{
    return j <= pos && (window == 0 || j > pos - window || j < sinks);
}

// W items dealt out to `blocks` stretches of nearly equal length, the longer ones first.
struct Stretches {
    int64_t len;
    int longer;                                   // stretches of len + 1
    __device__ __forceinline__ Stretches(int64_t W, int blocks)
    {
        len = W < 0x7fffffff ? static_cast<int>(W) / blocks : W / blocks;
        longer = static_cast<int>(W - len * blocks);
    }
    __device__ __forceinline__ int64_t begin(int i) const { return i * len + min(i, longer); }
    __device__ __forceinline__ int block_of(int64_t item) const
    {
        const int64_t head = longer * (len + 1);
        return item < head ? div(item, len + 1) : longer + div(item - head, len);
    }
    static __device__ __forceinline__ int div(int64_t a, int64_t b)
    {
        return a < 0x7fffffff && b < 0x7fffffff ? static_cast<int>(a) / static_cast<int>(b) : static_cast<int>(a / b);
    }
};

// 2^x with 2^-inf = 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Waits for a phase of an mbarrier.  False if the wait has run out (recorded in the status) or another one of the block has
// (recorded in `gave_up`, shared memory, for warps that wait for one another; NULL for one that waits for its own loads alone).
// BRIEF: the first look takes no time (a plain try_wait may be held up for as long as the hardware likes), and with a limit of 0 there is
// no other.
template <bool BRIEF = false, typename Params>
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, const Params &p, uint32_t *gave_up)
{
    if (BRIEF ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    while ((BRIEF && p.wait_ns == 0) || !mbar_try_wait_hint(bar, parity, p.wait_hint)) {
        if (gave_up && *reinterpret_cast<volatile uint32_t *>(gave_up)) return false;
        if (globaltimer_ns() - t0 >= p.wait_ns) {
            if (gave_up) *reinterpret_cast<volatile uint32_t *>(gave_up) = 1u;
            flag_status(p.status, kStatusWaitExpired);
            return false;
        }
    }
    return true;
}
// After that: waits for a copy or product of one's own that is under way, so that none outlives the block.
__device__ __forceinline__ void wait_own(uint32_t bar, uint32_t parity)
{
    const uint64_t t0 = globaltimer_ns();
    while (!mbar_try_wait_hint(bar, parity, 20000u) && globaltimer_ns() - t0 < kWaitLimitNs) { }
}

// Orders the block's partial results in the workspace before an arrival, and the other blocks' before a read.
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }

}  // namespace ead
