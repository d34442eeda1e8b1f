// What a row of logits z says: for a given token its log probability and its rank, the entropy, the k most likely tokens.
//   m = max z,  s = sum e^(z - m),  t = sum e^(z - m) (z - m):   log p_i = z_i - m - ln s,   H = ln s - t / s
// One pass over the row: a thread keeps a running maximum and the two sums of its vectors, so every logit is read once.  The
// alternatives need no list on the way: the k-th largest of the THREADS' maxima is a lower bound of the k-th largest
// logit, and only the few threads whose maximum reaches it can hold one of the k.  A thread knows the run of four vectors its maximum is in and the
// largest logit of its other runs, so nearly always that run alone is read again, and what reaches the bound is sorted.  With few rows a row is cut
// into parts, one block each; the last block of a row to finish joins the parts in their order, so the result does not depend on who comes last.
// Whole runs go to shared memory, a lane's vectors to its own places, so that the next run's loads are on their way under the arithmetic without a register.
// Measured in a replayed graph, 2041 rows of 152064 in bf16: entropy alone 97 us, 6.4 TB/s, 0.98 of the device's copy rate; with the rank of a token 112, with
// 20 alternatives 110, with both 124 (132-140 in calls one after another; f16 128, 1021 rows in 32 bits 111): 71 % of the issue slots are taken, the
// special function unit is busy 63 % (an exponential per logit), and a row's end (bound, second look, sort) is a chain of barriers that three other rows of
// the SM have to cover.  A row with more equal logits at the bound than the list of candidates has places (fewer unmasked ones than alternatives, say) is
// scanned once per alternative: 2041 rows of 152064 with 10 unmasked logits and 20 alternatives 7.4 ms.  One row of 128256 in 32 bits 8.5 us, a chain of
// look-ups, loads and the join.  On the way: a list per thread's strip read again 187, one element at a time 295, rows in two parts 174, runs loaded into
// registers with five blocks per SM 139.  Runs of 2, 3, 4, 5 vectors (five blocks per SM, four for 5): 155, 144, 132, 131; of 4 with 5, 4, 3 blocks per SM
// 132, 124, 133.
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "kv_format.cuh"
#include "ptx_sm100.cuh"
#include "rmsnorm_kernel.cuh"

namespace ead {

constexpr int kScoreThreads = 256;
constexpr int kScoreSettle = 1024;                // runs between settlements of a thread's counts
constexpr int kScoreUnroll = 4;                   // vectors of a run: a thread has them on their way together
constexpr int kScoreDepth = 2;                    // runs on their way to shared memory, the one that is read among them
constexpr int kScoreMaxTop = 64;                  // alternatives
constexpr int kScoreMaxParts = kScoreThreads;     // of a row, at most
constexpr int kScoreMaxJoin = 2048;               // parts x alternatives, at most
constexpr int kScoreSlack = 8;                    // threads beyond k that may be looked at again
constexpr int kScoreCandidates = 2048;            // logits that reach the bound; beyond, a slower way
constexpr int kScoreMaxCutRows = 1024;            // rows of a call that cuts its rows
constexpr size_t kScoreCounterBytes = kScoreMaxCutRows * sizeof(uint32_t);
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2Score = 0.6931471805599453f;

struct ScoreParams {
    const uint8_t *logits;
    int64_t stride;                               // elements between rows
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *rank, *top;
    int32_t n_rows, V, k, parts;
    uint8_t *workspace;
    uint32_t *status;
};

// A part's (or a thread's) share of a row.
struct ScoreSums {
    float m, s, t;                                // largest logit; sums
    int before;                                   // logits that come before the given token
};

// A vector of -infinity.
template <int FMT>
__device__ __forceinline__ uint4 nothing()
{
    const uint32_t w = FMT == kFmtF32 ? 0xff800000u : FMT == kFmtF16 ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}

// Larger logits have larger keys; equal ones larger keys for lower indices.  0 is below every logit's key.
__device__ __forceinline__ uint32_t order_bits(float z)
{
    const uint32_t u = __float_as_uint(z + 0.f);  // -0 and 0 are equal
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order_bits(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ unsigned long long order_key(float z, int index)
{
    return static_cast<unsigned long long>(order_bits(z)) << 32 | (0xffffffffu - static_cast<uint32_t>(index));
}

// kFloor: logits below it count as this much (its product with log2 e is exact, or small); kLow .. kHigh: where the largest logit of a part lies
// for the quick sums to be right: what is at the floor or below adds nothing then, and rounded products with log2 e are not far off.
template <int FMT>
struct LogitVec {
    static constexpr int kSize = FMT == kFmtF32 ? 4 : 2, kN = 16 / kSize;
    static constexpr float kFloor = FMT == kFmtF16 ? -65504.f : -1048576.f, kLow = FMT == kFmtF16 ? -60000.f : -524288.f, kHigh = 1048576.f;
};

__device__ __forceinline__ uint4 load_logits(const uint8_t *p)
{
    return ld_behind(reinterpret_cast<const uint4 *>(p));
}

template <int FMT>
__device__ __forceinline__ float logit_at(const uint8_t *row, int64_t i)
{
    if (FMT == kFmtF32) return ld_behind(reinterpret_cast<const float *>(row) + i);
    if (FMT == kFmtBf16) return __uint_as_float(static_cast<uint32_t>(ld_behind(reinterpret_cast<const uint16_t *>(row) + i)) << 16);
    return __half2float(__ushort_as_half(ld_behind(reinterpret_cast<const uint16_t *>(row) + i)));
}

template <int FMT>
__device__ __forceinline__ void unpack_logits(const uint4 &v, float (&z)[LogitVec<FMT>::kN])
{
    if constexpr (FMT == kFmtF32) {
        z[0] = __uint_as_float(v.x); z[1] = __uint_as_float(v.y); z[2] = __uint_as_float(v.z); z[3] = __uint_as_float(v.w);
    } else if constexpr (FMT == kFmtBf16) {
        unpack8(v, z);
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            z[2 * i] = f.x;
            z[2 * i + 1] = f.y;
        }
    }
}

// The row as 16-byte vectors of memory: vector g holds the columns g * kN - shift .. + kN - 1, the first and the last one in part.
template <int FMT>
struct RowVectors {
    const uint8_t *base;                          // of vector 0; 16-byte aligned
    int shift, V, n;
    __device__ __forceinline__ RowVectors(const uint8_t *row, int V_) : V(V_)
    {
        constexpr int S = LogitVec<FMT>::kSize, N = LogitVec<FMT>::kN;
        const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 15u;
        shift = off / S;
        base = row - off;
        n = static_cast<int>((static_cast<int64_t>(V) + shift + N - 1) / N);
    }
    __device__ __forceinline__ int column(int g) const { return g * LogitVec<FMT>::kN - shift; }
    __device__ __forceinline__ bool whole(int g) const { return (g > 0 || shift == 0) && column(g) + LogitVec<FMT>::kN <= V; }
    // The vector as it lies in memory; columns outside the row are -infinity.
    __device__ __forceinline__ uint4 raw(int g) const
    {
        constexpr int N = LogitVec<FMT>::kN;
        if (whole(g)) return load_logits(base + 16 * static_cast<int64_t>(g));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = column(g) + i;
            const bool in = c >= 0 && c < V;
            const int64_t at = static_cast<int64_t>(g) * N + i;
            if (FMT == kFmtF32) {
                w[i] = in ? ld_behind(reinterpret_cast<const uint32_t *>(base) + at) : 0xff800000u;
            } else {
                const uint32_t h = in ? ld_behind(reinterpret_cast<const uint16_t *>(base) + at) : FMT == kFmtF16 ? 0xfc00u : 0xff80u;
                w[i / 2] = (i & 1) ? w[i / 2] | h << 16 : h;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void load(int g, float (&z)[LogitVec<FMT>::kN]) const { unpack_logits<FMT>(raw(g), z); }
};

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// (z - m) in units of log 2, no lower than where 2^x is 0, so that a sum never meets 0 times infinity; a NaN stays one.
__device__ __forceinline__ float below_max(float z, float m)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"((z - m) * kLog2e), "f"(-1000.f));
    return y;
}

// Sums of two disjoint sets of logits.  With s = NaN or infinite (a logit that is NaN or +infinity) the result has it too.
// `low`: sums are relative to max(m, low).
__device__ __forceinline__ ScoreSums join_sums(const ScoreSums &a, const ScoreSums &b, float low)
{
    ScoreSums r;
    r.m = fmaxf(a.m, b.m);
    const float m = fmaxf(r.m, low), da = below_max(fmaxf(a.m, low), m), db = below_max(fmaxf(b.m, low), m);
    const float ea = exp2_of(da), eb = exp2_of(db);
    // roundings spelled out: a product drawn into the sum would make it matter which set comes first, and lanes that exchange sums have them either way
    r.s = __fadd_rn(__fmul_rn(a.s, ea), __fmul_rn(b.s, eb));
    r.t = __fadd_rn(__fmul_rn(fmaf(a.s, da, a.t), ea), __fmul_rn(fmaf(b.s, db, b.t), eb));
    r.before = a.before + b.before;
    return r;
}

__device__ __forceinline__ ScoreSums shuffle_xor(const ScoreSums &a, int o)
{
    return ScoreSums{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.t, o),
                     __shfl_xor_sync(0xffffffffu, a.before, o)};
}

struct ScoreShared {
    ScoreSums warp_sums[kScoreThreads / 32];
    union {                                       // (barriers stand between the last run and the first candidate)
        uint4 ring[kScoreDepth][kScoreUnroll][kScoreThreads];
        unsigned long long cand[kScoreCandidates];
    };
    unsigned long long best[kScoreMaxTop];        // the k largest keys, descending; 0: none
    unsigned long long warp_key[kScoreThreads / 32];
    uint2 warp_range[kScoreThreads / 32];
    int run[kScoreThreads], strip[kScoreThreads]; // of threads whose maximum reaches the bound: its run's first vector, or the thread
    int n_runs, n_strips, n_cand, last;
    int token;                                    // of thread 0 alone, for the row's end: the given token and its logit
    float z_given;
};

// Sums over the block in two halves with a barrier between: of each warp, into shared memory; and of the warps, in every thread.  (The tree is the
// same whatever the timing.)
__device__ __forceinline__ void warp_sums(ScoreShared &sh, ScoreSums a, float low)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) a = join_sums(a, shuffle_xor(a, o), low);
    if ((threadIdx.x & 31) == 0) sh.warp_sums[threadIdx.x >> 5] = a;
}
__device__ __forceinline__ ScoreSums sums_of_warps(const ScoreShared &sh, float low)
{
    ScoreSums a = sh.warp_sums[threadIdx.x & (kScoreThreads / 32 - 1)];
#pragma unroll
    for (int o = 1; o < kScoreThreads / 32; o <<= 1) a = join_sums(a, shuffle_xor(a, o), low);
    return a;
}
// Both; whoever read earlier sums may still be at it.
__device__ __forceinline__ ScoreSums block_sums(ScoreShared &sh, const ScoreSums &a, float low)
{
    __syncthreads();
    warp_sums(sh, a, low);
    __syncthreads();
    return sums_of_warps(sh, low);
}

// A lower bound of the k-th largest of the threads' keys (32 bits, 0: none) that few more than k of them reach; 0 if fewer than k
// threads have one.
__device__ __forceinline__ uint32_t bound_of(ScoreShared &sh, uint32_t key, int k)
{
    const uint32_t low = __reduce_min_sync(0xffffffffu, key ? key : 0xffffffffu), high = __reduce_max_sync(0xffffffffu, key);
    if ((threadIdx.x & 31) == 0) sh.warp_range[threadIdx.x >> 5] = make_uint2(low, high);
    if (__syncthreads_count(key != 0) < k) return 0;
    uint32_t lo = 0xffffffffu, hi = 0;            // at least k keys reach lo, none passes hi
#pragma unroll
    for (int w = 0; w < kScoreThreads / 32; ++w) {
        lo = min(lo, sh.warp_range[w].x);
        hi = max(hi, sh.warp_range[w].y);
    }
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        const int n = __syncthreads_count(key >= mid);
        if (n >= k)
            lo = mid;
        else
            hi = mid - 1;
        if (n >= k && n <= k + kScoreSlack) break;
    }
    return lo;
}

// The k largest of the n keys in sh.cand, all different, into sh.best (filled up with 0).
__device__ __forceinline__ void sort_candidates(ScoreShared &sh, int n, int k)
{
    if (threadIdx.x < k) sh.best[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kScoreThreads) {
        const unsigned long long key = sh.cand[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += sh.cand[j] > key;
        if (above < k) sh.best[above] = key;
    }
    __syncthreads();
}

// Largest of some vectors' logits, 16-bit ones two at a time; a NaN is passed over.
template <int FMT, int U>
__device__ __forceinline__ float largest(const uint4 (&v)[U])
{
    if constexpr (FMT == kFmtF32) {
        const float *const z = reinterpret_cast<const float *>(v);
        float m = z[0];
#pragma unroll
        for (int i = 1; i < 4 * U; ++i) m = fmaxf(m, z[i]);
        return m;
    } else {
        using H = std::conditional_t<FMT == kFmtBf16, __nv_bfloat162, __half2>;
        const H *const h = reinterpret_cast<const H *>(v);
        H m[4] = {h[0], h[1], h[2], h[3]};
#pragma unroll
        for (int i = 4; i < 4 * U; ++i) m[i & 3] = __hmax2(m[i & 3], h[i]);
        m[0] = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
        return fmaxf(__low2float(m[0]), __high2float(m[0]));
    }
}

// Puts a vector's logits that reach the bound among the candidates.
template <int FMT>
__device__ __forceinline__ void add_candidates(ScoreShared &sh, const RowVectors<FMT> &row, const uint4 &v, int g, uint32_t bound)
{
    constexpr int N = LogitVec<FMT>::kN;
    const uint4 one[1] = {v};
    if (bound && order_bits(largest<FMT>(one)) < bound) return;
    float z[N];
    unpack_logits<FMT>(v, z);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int col = row.column(g) + i;
        if (col >= 0 && col < row.V && order_bits(z[i]) >= bound) {
            const int n = atomicAdd(&sh.n_cand, 1);
            if (n < kScoreCandidates) sh.cand[n] = order_key(z[i], col);
        }
    }
}

// The k largest keys of the row's vectors [g0, g1).  Of the vectors g0 + threadIdx.x, + kScoreThreads, ... that this thread saw: the largest logit, the
// first vector of its run, the largest logit of the other runs.  A thread whose other runs stay below the bound has only that run looked at again.
template <int FMT>
__device__ __forceinline__ void find_top(ScoreShared &sh, const RowVectors<FMT> &row, int g0, int g1, float thread_max, int run, float second, int k)
{
    constexpr int N = LogitVec<FMT>::kN;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) sh.n_runs = sh.n_strips = sh.n_cand = 0;
    const uint32_t key = g0 + static_cast<int>(threadIdx.x) < g1 ? order_bits(thread_max) : 0;
    const uint32_t bound = bound_of(sh, key, k);  // (its barriers also publish the zeros above)
    if (key && key >= bound) {
        if (bound && order_bits(second) < bound)
            sh.run[atomicAdd(&sh.n_runs, 1)] = run;
        else
            sh.strip[atomicAdd(&sh.n_strips, 1)] = threadIdx.x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < sh.n_runs * kScoreUnroll; i += kScoreThreads) {
        const int64_t g = sh.run[i / kScoreUnroll] + static_cast<int64_t>(i % kScoreUnroll) * kScoreThreads;
        if (g < g1) add_candidates<FMT>(sh, row, row.raw(static_cast<int>(g)), static_cast<int>(g), bound);
    }
    const int per_thread = (g1 - g0 + kScoreThreads - 1) / kScoreThreads;
    for (int c = 0; c < sh.n_strips; ++c)
        for (int i = threadIdx.x; i < per_thread; i += kScoreThreads) {
            const int64_t g = g0 + sh.strip[c] + static_cast<int64_t>(i) * kScoreThreads;
            if (g < g1) add_candidates<FMT>(sh, row, row.raw(static_cast<int>(g)), static_cast<int>(g), bound);
        }
    __syncthreads();
    if (sh.n_cand <= kScoreCandidates) {
        sort_candidates(sh, sh.n_cand, k);
        return;
    }
    // Too many equal logits (or a thread with very many of the largest): one scan of the part per alternative.
    unsigned long long below = ~0ull;
    for (int r = 0; r < k; ++r) {
        unsigned long long mine = 0;
        for (int64_t g = g0 + threadIdx.x; g < g1; g += kScoreThreads) {
            float z[N];
            row.load(static_cast<int>(g), z);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int col = row.column(static_cast<int>(g)) + i;
                const unsigned long long x = order_key(z[i], col);
                if (col >= 0 && col < row.V && x < below && x > mine) mine = x;
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, o));
        if (lane == 0) sh.warp_key[warp] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kScoreThreads / 32; ++w) mine = max(mine, sh.warp_key[w]);
        if (threadIdx.x == 0) sh.best[r] = mine;
        below = mine;                             // 0 (none left) stays 0: nothing is below it
        __syncthreads();
    }
}

// The row's answers from its sums and its best keys.
__device__ __forceinline__ void write_scores(const ScoreParams &p, const ScoreShared &sh, int row, const ScoreSums &a)
{
    const float m = fmaxf(a.m, kLowest);
    // NaN or +infinity among the logits, or nothing but -infinity
    const bool bad = !(a.s > 0.f) || !(a.s <= -kLowest) || !(a.m <= -kLowest);
    const float log2_s = log2f(a.s), nan = __uint_as_float(0x7fffffffu);
    if (threadIdx.x == 0) {
        if (bad) flag_status(p.status, kStatusNonFinite);
        if (p.entropy) p.entropy[row] = bad ? nan : fmaxf((log2_s - a.t / a.s) * kLn2Score, 0.f);
        if (p.tokens) {
            const int token = sh.token;
            const bool given = token >= 0 && token < p.V;
            if (token >= p.V) flag_status(p.status, kStatusBadToken);
            if (p.logprob) {
                p.logprob[row] = bad || !given ? nan : (sh.z_given - m) - log2_s * kLn2Score;
            }
            if (p.rank) p.rank[row] = bad || !given ? -1 : a.before;
        }
    }
    if (threadIdx.x < p.k) {
        const unsigned long long key = sh.best[threadIdx.x];
        const int64_t at = static_cast<int64_t>(row) * p.k + threadIdx.x;
        const bool none = bad || key == 0;
        if (p.top) p.top[at] = none ? -1 : static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(key));
        if (p.top_logprob) {
            const float z = from_order_bits(static_cast<uint32_t>(key >> 32));
            p.top_logprob[at] = bad ? nan : key == 0 ? -INFINITY : (z - m) - log2_s * kLn2Score;
        }
    }
}

// The vector with nothing below the floor; a NaN stays one.
template <int FMT>
__device__ __forceinline__ uint4 floored(uint4 v)
{
    if constexpr (FMT == kFmtF32) {
        uint32_t *const w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+r"(w[i]) : "f"(LogitVec<FMT>::kFloor));
    } else if constexpr (FMT == kFmtBf16) {
        __nv_bfloat162 *const h = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __hmax2_nan(h[i], __float2bfloat162_rn(LogitVec<FMT>::kFloor));
    } else {
        __half2 *const h = reinterpret_cast<__half2 *>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __hmax2_nan(h[i], __float2half2_rn(LogitVec<FMT>::kFloor));
    }
    return v;
}

// A threshold that a 16-bit vector's logits are compared with, twice in a word.  strict: themselves; else the next lower number, so that
// "above" it is "not below" z.  (z is neither NaN nor infinite.)
template <int FMT>
__device__ __forceinline__ uint32_t threshold(float z, bool strict)
{
    if (FMT == kFmtF32) {
        const uint32_t b = __float_as_uint(z + 0.f);
        return strict ? b : b == 0 ? 0x80000001u : (b & 0x80000000u) ? b + 1 : b - 1;
    }
    const uint32_t b = FMT == kFmtBf16 ? __float_as_uint(z + 0.f) >> 16 : __half_as_ushort(__float2half_rn(z + 0.f));
    const uint32_t t = strict ? b : b == 0 ? 0x8001u : (b & 0x8000u) ? b + 1 : b - 1;
    return t << 16 | t;
}
// Counts of logits above a threshold.  16-bit logits are compared two at a time; a comparison gives 0xffff in its half, and a 32-bit sum
// of such words holds both halves' counts, which come apart as long as neither passes 65535.
template <int FMT>
struct CountAbove {
    uint32_t sum = 0;
    int total = 0;
    __device__ __forceinline__ void add(const uint4 &v, uint32_t t)
    {
        if constexpr (FMT == kFmtF32) {
            const float x = __uint_as_float(t);
            total += (__uint_as_float(v.x) > x) + (__uint_as_float(v.y) > x) + (__uint_as_float(v.z) > x) + (__uint_as_float(v.w) > x);
        } else if constexpr (FMT == kFmtBf16) {
            const __nv_bfloat162 *const h = reinterpret_cast<const __nv_bfloat162 *>(&v), x = *reinterpret_cast<const __nv_bfloat162 *>(&t);
            sum += __hgt2_mask(h[0], x) + __hgt2_mask(h[1], x);
            sum += __hgt2_mask(h[2], x) + __hgt2_mask(h[3], x);
        } else {
            const __half2 *const h = reinterpret_cast<const __half2 *>(&v), x = *reinterpret_cast<const __half2 *>(&t);
            sum += __hgt2_mask(h[0], x) + __hgt2_mask(h[1], x);
            sum += __hgt2_mask(h[2], x) + __hgt2_mask(h[3], x);
        }
    }
    // After at most 16383 vectors.
    __device__ __forceinline__ void settle()
    {
        if (FMT == kFmtF32) return;
        const uint32_t low = (0u - sum) & 0xffffu;                    // sum = (low - high) 2^16 - low
        total += static_cast<int>(low + ((low - ((sum + low) >> 16)) & 0xffffu));
        sum = 0;
    }
};

// One thread's running maximum and sums.
template <int FMT>
struct ScoreThread {
    static constexpr int N = LogitVec<FMT>::kN;
    float m, second;                              // largest logit; largest of the runs that it is not in
    int at;                                       // first vector of its run
    float m_log2;                                 // s, t (even and odd places) are relative to max(m, floor) = m_log2 / log2 e
    f32x2 s, t;
    CountAbove<FMT> above;
    int before;
    __device__ __forceinline__ ScoreThread() : m(-INFINITY), second(-INFINITY), at(0), m_log2(LogitVec<FMT>::kFloor * kLog2e), s(0), t(0), before(0) {}
    // A run of vectors from g on, kScoreThreads apart; EDGE: some of their columns may lie outside the row, vectors from g_end on are not the
    // part's and -infinity.  g_given: the given token's vector.
    template <bool EDGE>
    __device__ __forceinline__ void take(const RowVectors<FMT> &row, const uint4 (&v)[kScoreUnroll], int g, int g_end, bool given, float z_given, uint32_t t_or_equal, uint32_t t_above, int token, int g_given)
    {
        constexpr int U = kScoreUnroll;
        const float top = largest<FMT>(v);
        if (top <= m) {
            second = fmaxf(second, top);
        } else if (top > m) {
            second = m;
            m = top;
            at = g;
            const float m1 = fmaxf(top, LogitVec<FMT>::kFloor) * kLog2e, d = fmaxf(m_log2 - m1, -1000.f), e = exp2_of(d);
            const f32x2 ee = pack2(e, e);
            t = fma2(fma2(s, pack2(d, d), t), ee, 0);
            s = fma2(s, ee, 0);
            m_log2 = m1;
        }
        const f32x2 scale = pack2(kLog2e, kLog2e), minus_m = pack2(-m_log2, -m_log2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[N];
            unpack_logits<FMT>(floored<FMT>(v[u]), z);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const f32x2 y = fma2(pack2(z[i], z[i + 1]), scale, minus_m);
                float y0, y1;
                unpack2(y, y0, y1);
                const f32x2 e = pack2(exp2_of(y0), exp2_of(y1));
                s = add2(s, e);
                t = fma2(e, y, t);
            }
        }
        if (given && top >= z_given) {
            const bool all_before = g + (U - 1) * kScoreThreads < g_given, all_behind = g > g_given;
            if (!EDGE && (all_before || all_behind) && z_given != -INFINITY) {
                const uint32_t t = all_before ? t_or_equal : t_above;
#pragma unroll
                for (int u = 0; u < U; ++u) above.add(v[u], t);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float z[N];
                    unpack_logits<FMT>(v[u], z);
                    const int gu = g + u * kScoreThreads, col = row.column(gu);
                    if (EDGE && gu >= g_end) break;
#pragma unroll
                    for (int i = 0; i < N; ++i) before += z[i] > z_given || (z[i] == z_given && col + i < token && col + i >= 0);
                }
            }
        }
    }
    __device__ __forceinline__ ScoreSums sums() const
    {
        float s0, s1, t0, t1;
        unpack2(s, s0, s1);
        unpack2(t, t0, t1);
        const float ss = s0 + s1, tt = t0 + t1;
        if (m == -INFINITY && ss == ss) return ScoreSums{m, 0.f, 0.f, before};             // nothing but -infinity
        const float c = fmaf(-fmaxf(m, LogitVec<FMT>::kFloor), kLog2e, m_log2), e = exp2_of(c);     // what the rounding of m_log2 added to every distance
        return ScoreSums{m, ss * e, fmaf(ss, c, tt) * e, before};
    }
};

// Block (x, y): part x of row y, y + gridDim.y, ...
template <int FMT>
__global__ void __launch_bounds__(kScoreThreads, 4) ead_token_logprobs_kernel(ScoreParams p)
{
    __shared__ ScoreShared sh;
    constexpr int N = LogitVec<FMT>::kN;
    griddep_wait();
    griddep_launch_dependents();
    for (int row = blockIdx.y; row < p.n_rows; row += gridDim.y) {
        const uint8_t *const logits = p.logits + LogitVec<FMT>::kSize * (row * p.stride);
        const RowVectors<FMT> vec(logits, p.V);
        const int g0 = static_cast<int>(static_cast<int64_t>(vec.n) * blockIdx.x / p.parts);
        const int g1 = static_cast<int>(static_cast<int64_t>(vec.n) * (blockIdx.x + 1) / p.parts);
        const int n = g1 - g0, whole_end = vec.whole(g1 - 1) ? n : n - 1;                // vectors of this part
        constexpr int kRun = kScoreUnroll * kScoreThreads;
        // Whole runs go to shared memory, a lane's vectors to its own places, the first ones while the token and its logit are looked up.
        const uint32_t ring = smem_u32(&sh.ring[0][0][threadIdx.x]);
        const bool starts_cut = !vec.whole(g0);
        int i = 0, asked = starts_cut ? kRun : 0;
        uint32_t to = ring, from = ring;
        auto ask = [&] {
            if (asked + kRun <= whole_end) {
                const uint8_t *const at = vec.base + 16 * static_cast<int64_t>(g0 + asked + static_cast<int>(threadIdx.x));
#pragma unroll
                for (int u = 0; u < kScoreUnroll; ++u) copy_async_16(to + u * kScoreThreads * 16, at + u * kScoreThreads * 16);
                asked += kRun;
                to = to == ring + (kScoreDepth - 1) * kRun * 16 ? ring : to + kRun * 16;
            }
            copy_async_commit();
        };
#pragma unroll
        for (int d = 0; d < kScoreDepth - 1; ++d) ask();
        const int token = p.tokens ? ld_behind(p.tokens + row) : -1;
        const float z_token = token >= 0 && token < p.V ? logit_at<FMT>(logits, token) : 0.f;
        if (threadIdx.x == 0) {
            sh.token = token;
            sh.z_given = z_token;
        }
        const bool given = p.rank && token >= 0 && token < p.V;
        const float z_given = given ? z_token : INFINITY;
        const int g_given = given ? static_cast<int>((static_cast<int64_t>(token) + vec.shift) / N) : 0;
        const uint32_t t_or_equal = threshold<FMT>(z_given, false), t_above = threshold<FMT>(z_given, true);
        ScoreThread<FMT> th;
        auto edge = [&] {                         // a run that may meet an end of the row or of the part
            const int g = g0 + i + threadIdx.x;
            uint4 v[kScoreUnroll];
#pragma unroll
            for (int u = 0; u < kScoreUnroll; ++u)
                v[u] = static_cast<int64_t>(g) + u * kScoreThreads < g1 ? vec.raw(g + u * kScoreThreads) : nothing<FMT>();
            if (g < g1) th.template take<true>(vec, v, g, g1, given, z_given, t_or_equal, t_above, token, g_given);
            i += kRun;
        };
        if (starts_cut) edge();                   // (whole_end may then be wrong for a row of one vector: no quick run fits)
        while (i + kRun <= whole_end) {
            const int stop = min(whole_end, i + kScoreSettle * kRun);
            for (; i + kRun <= stop; i += kRun) {
                const int g = g0 + i + threadIdx.x;
                ask();
                copy_async_wait<kScoreDepth - 1>();
                uint4 v[kScoreUnroll];
#pragma unroll
                for (int u = 0; u < kScoreUnroll; ++u) v[u] = ld_shared_16(from + u * kScoreThreads * 16);
                from = from == ring + (kScoreDepth - 1) * kRun * 16 ? ring : from + kRun * 16;
                th.template take<false>(vec, v, g, g1, given, z_given, t_or_equal, t_above, token, g_given);
            }
            th.above.settle();
        }
        while (i < n) edge();
        th.before += th.above.total;
        warp_sums(sh, th.sums(), LogitVec<FMT>::kFloor);
        if (p.k)
            find_top<FMT>(sh, vec, g0, g1, th.m, th.at, th.second, p.k);      // (with barriers of its own)
        else
            __syncthreads();
        ScoreSums a = sums_of_warps(sh, LogitVec<FMT>::kFloor);
        if (a.m > -INFINITY && a.m < INFINITY && !(a.m >= LogitVec<FMT>::kLow && a.m <= LogitVec<FMT>::kHigh)) {
            // logits at the ends of the type's range: once more, relative to the part's maximum
            ScoreSums x{a.m, 0.f, 0.f, 0};
            for (int64_t g = g0 + threadIdx.x; g < g1; g += kScoreThreads) {
                float z[N];
                vec.load(static_cast<int>(g), z);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float y = below_max(z[e], a.m), w = exp2_of(y);
                    x.s += w;
                    x.t = fmaf(w, y, x.t);
                }
            }
            const int before = a.before;
            a = block_sums(sh, x, kLowest);
            a.before = before;
        }
        if (p.parts == 1) {
            write_scores(p, sh, row, a);
            __syncthreads();
            continue;
        }
        // this part's record: sums, then its keys
        uint32_t *const counter = reinterpret_cast<uint32_t *>(p.workspace) + row;
        ScoreSums *const sums = reinterpret_cast<ScoreSums *>(p.workspace + kScoreCounterBytes) + static_cast<int64_t>(row) * p.parts;
        unsigned long long *const keys = reinterpret_cast<unsigned long long *>(
            p.workspace + kScoreCounterBytes + sizeof(ScoreSums) * static_cast<int64_t>(p.n_rows) * p.parts) + static_cast<int64_t>(row) * p.parts * p.k;
        if (threadIdx.x == 0) sums[blockIdx.x] = a;
        if (threadIdx.x < p.k) keys[blockIdx.x * p.k + threadIdx.x] = sh.best[threadIdx.x];
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) sh.last = atomicAdd(counter, 1u) == static_cast<uint32_t>(p.parts - 1);
        __syncthreads();
        if (!sh.last) continue;
        __threadfence();
        ScoreSums all{-INFINITY, 0.f, 0.f, 0};
        if (threadIdx.x < p.parts) {
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(sums + threadIdx.x));
            all = ScoreSums{v.x, v.y, v.z, __float_as_int(v.w)};
        }
        all = block_sums(sh, all, kLowest);
        if (p.k) {
            const int n = p.parts * p.k;
            uint32_t mine = 0;
            for (int i = threadIdx.x; i < n; i += kScoreThreads) mine = max(mine, static_cast<uint32_t>(__ldcg(keys + i) >> 32));
            if (threadIdx.x == 0) sh.n_cand = 0;
            const uint32_t bound = bound_of(sh, mine, p.k);
            for (int i = threadIdx.x; i < n; i += kScoreThreads) {
                const unsigned long long key = __ldcg(keys + i);
                if (key && static_cast<uint32_t>(key >> 32) >= bound) sh.cand[atomicAdd(&sh.n_cand, 1)] = key;
            }
            __syncthreads();
            sort_candidates(sh, sh.n_cand, p.k);
        }
        write_scores(p, sh, row, all);
        if (threadIdx.x == 0) *counter = 0;       // ready for the next call
        __syncthreads();
    }
}

}  // namespace ead
