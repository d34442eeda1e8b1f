// What a row of logits z says: for a given token its log probability and its rank, the entropy, the k most likely tokens.
//   m = max z,  s = sum e^(z - m),  t = sum e^(z - m) (z - m):   log p_i = z_i - m - ln s,   H = ln s - t / s
// One pass over the row: a thread keeps a running maximum and the two sums of its vectors, so every logit is read once.  The
// alternatives need no list on the way: the k-th largest of the THREADS' maxima is a lower bound of the k-th largest
// logit, and only the few threads whose maximum reaches it can hold one of the k; their vectors are read again (from L2) and what
// reaches the bound is sorted.  With few rows a row is cut into parts, one block each; the last block of a row to finish joins
// the parts in their order, so the result does not depend on who comes last.  HBM bounds it at size.
#pragma once
#include <cuda_fp16.h>

#include "kv_format.cuh"
#include "rmsnorm_kernel.cuh"

namespace ead {

constexpr int kScoreThreads = 512;
constexpr int kScoreMaxTop = 64;                  // alternatives
constexpr int kScoreMaxParts = 512;               // parts of a row, at most this many
constexpr int kScoreMaxJoin = 2048;               // parts x alternatives, at most
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
    float m, s, t;                                // largest logit; sums relative to max(m, lowest finite value)
    int before;                                   // logits that come before the given token
};

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

template <int FMT>
struct LogitVec {
    static constexpr int kSize = FMT == kFmtF32 ? 4 : 2, kN = 16 / kSize;
};

__device__ __forceinline__ uint4 load_logits(const uint8_t *p)
{
    return __ldg(reinterpret_cast<const uint4 *>(p));
}

template <int FMT>
__device__ __forceinline__ float logit_at(const uint8_t *row, int64_t i)
{
    if (FMT == kFmtF32) return __ldg(reinterpret_cast<const float *>(row) + i);
    if (FMT == kFmtBf16) return __uint_as_float(static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t *>(row) + i)) << 16);
    return __half2float(__ushort_as_half(__ldg(reinterpret_cast<const uint16_t *>(row) + i)));
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
    // Columns outside the row read as -infinity.
    __device__ __forceinline__ void load(int g, float (&z)[LogitVec<FMT>::kN]) const
    {
        constexpr int N = LogitVec<FMT>::kN;
        if (whole(g)) {
            unpack_logits<FMT>(load_logits(base + 16 * static_cast<int64_t>(g)), z);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column(g) + i;
                z[i] = c >= 0 && c < V ? logit_at<FMT>(base, static_cast<int64_t>(g) * N + i) : -INFINITY;
            }
        }
    }
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
__device__ __forceinline__ ScoreSums join_sums(const ScoreSums &a, const ScoreSums &b)
{
    ScoreSums r;
    r.m = fmaxf(a.m, b.m);
    const float m = fmaxf(r.m, kLowest), da = below_max(fmaxf(a.m, kLowest), m), db = below_max(fmaxf(b.m, kLowest), m);
    const float ea = exp2_of(da), eb = exp2_of(db);
    r.s = a.s * ea + b.s * eb;
    r.t = fmaf(a.s, da, a.t) * ea + fmaf(b.s, db, b.t) * eb;
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
    unsigned long long cand[kScoreCandidates];
    unsigned long long best[kScoreMaxTop];        // the k largest keys, descending; 0: none
    unsigned long long warp_key[kScoreThreads / 32];
    int chosen[kScoreThreads];                    // threads whose maximum reaches the bound
    int n_chosen, n_cand, last;
};

// Sums over the block, in every thread.  (The tree is the same whatever the timing.)
__device__ __forceinline__ ScoreSums block_sums(ScoreShared &sh, ScoreSums a)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) a = join_sums(a, shuffle_xor(a, o));
    if ((threadIdx.x & 31) == 0) sh.warp_sums[threadIdx.x >> 5] = a;
    __syncthreads();
    a = sh.warp_sums[threadIdx.x & (kScoreThreads / 32 - 1)];
#pragma unroll
    for (int o = 1; o < kScoreThreads / 32; o <<= 1) a = join_sums(a, shuffle_xor(a, o));
    return a;
}

// A lower bound of the k-th largest of the threads' keys (32 bits, 0: none), as large as possible; 0 if fewer than k threads have one.
__device__ __forceinline__ uint32_t bound_of(uint32_t key, int k)
{
    uint32_t bound = 0;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
        const int n = __syncthreads_count(key >= (bound | bit));
        if (n >= k) bound |= bit;
        if (n == k) break;
    }
    return bound;
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

// The k largest keys of the row's vectors [g0, g1).  `thread_max`: of the vectors g0 + threadIdx.x, + kScoreThreads, ...
template <int FMT>
__device__ __forceinline__ void find_top(ScoreShared &sh, const RowVectors<FMT> &row, int g0, int g1, float thread_max, int k)
{
    constexpr int N = LogitVec<FMT>::kN;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) sh.n_chosen = sh.n_cand = 0;
    const uint32_t key = g0 + static_cast<int>(threadIdx.x) < g1 ? order_bits(thread_max) : 0;
    const uint32_t bound = bound_of(key, k);      // (its barriers also publish the zeros above)
    if (key && key >= bound) sh.chosen[atomicAdd(&sh.n_chosen, 1)] = threadIdx.x;
    __syncthreads();
    for (int c = warp; c < sh.n_chosen; c += kScoreThreads / 32)
        for (int64_t g = g0 + sh.chosen[c] + static_cast<int64_t>(lane) * kScoreThreads; g < g1; g += 32 * kScoreThreads) {
            float z[N];
            row.load(static_cast<int>(g), z);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int col = row.column(static_cast<int>(g)) + i;
                if (col >= 0 && col < row.V && order_bits(z[i]) >= bound) {
                    const int at = atomicAdd(&sh.n_cand, 1);
                    if (at < kScoreCandidates) sh.cand[at] = order_key(z[i], col);
                }
            }
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
template <int FMT>
__device__ __forceinline__ void write_scores(const ScoreParams &p, const ScoreShared &sh, int row, const uint8_t *logits, const ScoreSums &a)
{
    const float m = fmaxf(a.m, kLowest);
    // NaN or +infinity among the logits, or nothing but -infinity
    const bool bad = !(a.s > 0.f) || !(a.s <= -kLowest) || !(a.m <= -kLowest);
    const float log2_s = log2f(a.s), nan = __uint_as_float(0x7fffffffu);
    if (threadIdx.x == 0) {
        if (bad) flag_status(p.status, kStatusNonFinite);
        if (p.entropy) p.entropy[row] = bad ? nan : fmaxf((log2_s - a.t / a.s) * kLn2Score, 0.f);
        if (p.tokens) {
            const int token = __ldg(p.tokens + row);
            const bool given = token >= 0 && token < p.V;
            if (token >= p.V) flag_status(p.status, kStatusBadToken);
            if (p.logprob) {
                const float z = given ? logit_at<FMT>(logits, token) : 0.f;
                p.logprob[row] = bad || !given ? nan : (z - m) - log2_s * kLn2Score;
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

// Block (x, y): part x of row y, y + gridDim.y, ...
template <int FMT>
__global__ void __launch_bounds__(kScoreThreads) ead_token_logprobs_kernel(ScoreParams p)
{
    __shared__ ScoreShared sh;
    constexpr int N = LogitVec<FMT>::kN;
    for (int row = blockIdx.y; row < p.n_rows; row += gridDim.y) {
        const uint8_t *const logits = p.logits + LogitVec<FMT>::kSize * (row * p.stride);
        const RowVectors<FMT> vec(logits, p.V);
        const int g0 = static_cast<int>(static_cast<int64_t>(vec.n) * blockIdx.x / p.parts);
        const int g1 = static_cast<int>(static_cast<int64_t>(vec.n) * (blockIdx.x + 1) / p.parts);
        const int token = p.tokens ? __ldg(p.tokens + row) : -1;
        const bool given = p.rank && token >= 0 && token < p.V;
        const float z_given = given ? logit_at<FMT>(logits, token) : INFINITY;
        ScoreSums a{-INFINITY, 0.f, 0.f, 0};
        float m = kLowest;                        // max(a.m, kLowest)
        for (int64_t g64 = g0 + threadIdx.x; g64 < g1; g64 += kScoreThreads) {
            const int g = static_cast<int>(g64);
            float z[N];
            vec.load(g, z);
            float top = z[0];
#pragma unroll
            for (int i = 1; i < N; ++i) top = fmaxf(top, z[i]);
            if (top > a.m) {
                a.m = top;
                const float m1 = fmaxf(top, kLowest), d = below_max(m, m1), e = exp2_of(d);
                a.t = fmaf(a.s, d, a.t) * e;
                a.s *= e;
                m = m1;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float y = below_max(z[i], m), e = exp2_of(y);
                a.s += e;
                a.t = fmaf(e, y, a.t);
            }
            if (given && top >= z_given) {
                const int col = vec.column(g);
#pragma unroll
                for (int i = 0; i < N; ++i) a.before += z[i] > z_given || (z[i] == z_given && col + i < token && col + i >= 0);
            }
        }
        const float thread_max = a.m;
        if (p.k) find_top<FMT>(sh, vec, g0, g1, thread_max, p.k);
        a = block_sums(sh, a);
        if (p.parts == 1) {
            write_scores<FMT>(p, sh, row, logits, a);
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
        __syncthreads();                          // warp_sums is used again
        all = block_sums(sh, all);
        if (p.k) {
            const int n = p.parts * p.k;
            uint32_t mine = 0;
            for (int i = threadIdx.x; i < n; i += kScoreThreads) mine = max(mine, static_cast<uint32_t>(__ldcg(keys + i) >> 32));
            if (threadIdx.x == 0) sh.n_cand = 0;
            const uint32_t bound = bound_of(mine, p.k);
            for (int i = threadIdx.x; i < n; i += kScoreThreads) {
                const unsigned long long key = __ldcg(keys + i);
                if (key && static_cast<uint32_t>(key >> 32) >= bound) sh.cand[atomicAdd(&sh.n_cand, 1)] = key;
            }
            __syncthreads();
            sort_candidates(sh, sh.n_cand, p.k);
        }
        write_scores<FMT>(p, sh, row, logits, all);
        if (threadIdx.x == 0) *counter = 0;       // ready for the next call
        __syncthreads();
    }
}

}  // namespace ead
