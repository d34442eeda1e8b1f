// Root-mean-square norm of every query and key head, and the position rotation, in one pass over a step's projections; the
// results go into tensors (dense) or, with the values, straight into the paged cache in its format:
//   y = x / sqrt(mean(x^2) + eps) * weight,   (a, b) -> (a cos - b sin, b cos + a sin),   angle = position * inv_freq[j]
// A warp takes one token (with few tokens: some of its heads).  Its rows are on their way to shared memory, several runs deep, while it looks up the
// token's place and computes the angles once, the product in 64 bits and brought within half a turn before it is rounded to 32; then it
// streams the heads.  Weight, cos and sin come together in two factors per element that a lane keeps for all heads,
//   y_e = (x_e f_e + x_partner g_e) / sqrt(mean(x^2) + eps),   f = weight cos,   g = -+ weight of the partner sin
// Two forms: heads rotated as a whole in halves (a lane holds 8 elements of either half), and all others (a lane holds 8 consecutive elements, partners
// exchange the bf16 words as they were loaded).  Every element is read once and written once: HBM bounds it at size, launch and the
// chain of look-ups at one step.
// Measured: 18125 tokens of 32 + 8 + 8 heads of 128 into an 8-bit cache 79 us in a replayed graph, 5.2 TB/s, 0.79 of the device's copy rate, 81-85 us in
// calls one after another; into a bf16 cache 77 us, 5.8 TB/s.  (On the way: the other form, with rows two runs ahead in registers, 93; a block per token with angles
// shared 174.)  The other form, half of each head or neighbouring pairs: 92-94 us into 8 bits, 84 into bf16, with 82 % of the issue slots taken (64
// registers; into a cache 8 and 24 bytes of them spill).  64 tokens of 40 + 8 + 8 heads 3.7-4.0 us; 4001 tokens of 32 + 8 heads of 64, 32
// elements of each rotated, 9.8-9.9 us, 4.1-4.2 TB/s.  More runs ahead do not help (whole heads: 3 runs 80.6, 4 78.7, 5 79.0), more warps per SM cost registers
// (whole heads: 16 warps 78.7, 24 81.5, 32 107; the other form: 32 warps 9.8, 24 11.5).
#pragma once
#include "quantise_kernel.cuh"

namespace ead {

constexpr int kRopeThreads = 256;
constexpr int kRopeDepth = 4;                     // runs on their way to shared memory, the one that is read among them
constexpr int kRopePartDepth = 6;                 // the same for heads that are rotated in part
constexpr int kRopeRun = 256;                     // elements that a warp takes at a time

struct RopeParams {
    KvCacheView cache;                            // !DENSE
    KvBatchView batch;                            // !DENSE
    const int32_t *positions;
    const uint8_t *q, *k, *v;
    uint8_t *q_out, *k_out;                       // k_out: DENSE
    int64_t q_stride, kv_stride, q_out_stride, k_out_stride;   // elements between tokens
    const float *inv_freq;
    const uint8_t *q_weight, *k_weight;           // bf16 [dim] or NULL
    int32_t n_tokens, heads_q, heads_kv, dim, rot, interleaved;
    int32_t split;                                // warps that share a token
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

__device__ __forceinline__ void unpack8(const uint4 &v, f32x2 (&f)[4])
{
    f[0] = pack2(bf16_lo(v.x), bf16_hi(v.x));
    f[1] = pack2(bf16_lo(v.y), bf16_hi(v.y));
    f[2] = pack2(bf16_lo(v.z), bf16_hi(v.z));
    f[3] = pack2(bf16_lo(v.w), bf16_hi(v.w));
}

__device__ __forceinline__ uint4 to_bf16x8(const f32x2 (&y)[4])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(y[i], f[2 * i], f[2 * i + 1]);
    return pack8(f);
}

// What a lane needs to turn its 8 elements of a head.
struct RopeLane {
    f32x2 f[4], g[4];                             // factors of the elements and of their partners
    int partner;                                  // lane that has the partners; -1: this one, pairs are neighbours
    bool turned, norm;
};

// The factors of queries or keys from their weight and the token's cos and sin (1 and 0 behind the rotated part).
__device__ __forceinline__ void set_factors(const RopeParams &p, RopeLane &l, const uint8_t *weight, const float2 *turn, int lane)
{
    const int e0 = (lane & ((p.dim >> 3) - 1)) * 8, half = p.rot >> 1;
    l.norm = weight != nullptr;
    uint4 w = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), o = w;                 // ones
    if (weight) {
        const int in_head = lane & ((p.dim >> 3) - 1);
        w = o = ld_behind(reinterpret_cast<const uint4 *>(weight) + in_head);
        if (l.partner >= 0) o = ld_behind(reinterpret_cast<const uint4 *>(weight) + (l.partner & ((p.dim >> 3) - 1)));
    }
    if (l.partner < 0) o = make_uint4(__byte_perm(w.x, 0, 0x1032), __byte_perm(w.y, 0, 0x1032), __byte_perm(w.z, 0, 0x1032), __byte_perm(w.w, 0, 0x1032));
    f32x2 a[4], b[4];
    unpack8(w, a);
    unpack8(o, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = e0 + 2 * i, j0 = p.interleaved ? e >> 1 : e < half ? e : e - half, j1 = p.interleaved ? j0 : j0 + 1;
        const float2 u = l.turned ? turn[j0] : make_float2(1.f, 0.f), v = l.turned ? turn[j1] : make_float2(1.f, 0.f);
        l.f[i] = mul2(a[i], pack2(u.x, v.x));
        l.g[i] = mul2(b[i], p.interleaved ? pack2(-u.y, v.y) : e < half ? pack2(-u.y, -v.y) : pack2(u.y, v.y));
    }
}

// 8 elements per lane of a run of heads, normalised and rotated.
__device__ __forceinline__ void norm_and_rotate(const RopeParams &p, const RopeLane &l, const uint4 &x, f32x2 (&y)[4])
{
    f32x2 a[4], b[4];
    unpack8(x, a);
    uint4 o;
    if (l.partner >= 0)
        o = make_uint4(__shfl_sync(0xffffffffu, x.x, l.partner), __shfl_sync(0xffffffffu, x.y, l.partner), __shfl_sync(0xffffffffu, x.z, l.partner),
                       __shfl_sync(0xffffffffu, x.w, l.partner));
    else
        o = make_uint4(__byte_perm(x.x, 0, 0x1032), __byte_perm(x.y, 0, 0x1032), __byte_perm(x.z, 0, 0x1032), __byte_perm(x.w, 0, 0x1032));
    if (!l.turned) o = make_uint4(0, 0, 0, 0);    // (an infinity must not meet the 0 of the sine)
    unpack8(o, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fma2(a[i], l.f[i], mul2(b[i], l.g[i]));
    if (l.norm) {
        f32x2 squares = mul2(a[0], a[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) squares = fma2(a[i], a[i], squares);
        float sum, odd;
        unpack2(squares, sum, odd);
        sum += odd;
#pragma unroll
        for (int i = 1; i < 8; i <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
        if (p.dim == 128) sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        const float r = rsqrtf(sum * (p.dim == 128 ? 1.f / 128 : 1.f / 64) + p.eps);
        const f32x2 rr = pack2(r, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], rr);
    }
}

// The warp's token and share of its heads, and the token's place.
struct RopeToken {
    int t, share, position, page, slot;
};
// False: no token.
__device__ __forceinline__ bool token_of(const RopeParams &p, int warp, RopeToken &k)
{
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kRopeThreads / 32) + warp;
    k.t = p.split == 1 ? static_cast<int>(unit) : static_cast<int>(unit / p.split);
    k.share = static_cast<int>(unit - static_cast<int64_t>(k.t) * p.split);
    k.page = k.slot = 0;
    return k.t < p.n_tokens;
}
// False: the token has no place, nothing of it is written.
template <bool DENSE>
__device__ __forceinline__ bool find_place(const RopeParams &p, int lane, RopeToken &k)
{
    if (DENSE) {
        k.position = ld_behind(p.positions + k.t);
        return true;
    }
    const int b = find_sequence<true>(p.batch.new_start, p.batch.B, k.t, lane);
    const int first = ld_behind(p.batch.new_start + b), last = ld_behind(p.batch.new_start + b + 1);
    const bool bad = first < 0 || k.t < first || k.t >= last || last > p.batch.n_tokens || last - first > p.batch.max_new;
    const int cached = ld_behind(p.batch.kv_len + b) - (last - k.t);
    k.page = bad ? -1 : find_page<true>(p.cache, p.batch, b, cached);
    k.position = p.positions ? ld_behind(p.positions + k.t) : cached;
    k.slot = cached & (p.cache.page_size - 1);
    if (k.page < 0 && lane == 0 && k.share == 0) flag_status(p.status, bad ? kStatusBadCount : kStatusBadPage);
    return k.page >= 0;
}

// Where a token's values go in a pool of the cache, from element e0 of a head on: its first head's, and the scale's (e4m3).
struct RopePlace {
    uint8_t *pool, *scale;
};
template <int FMT>
__device__ __forceinline__ RopePlace place_of(const KvCacheView &c, const RopeToken &k, uint8_t *values, uint8_t *scales, int e0)
{
    RopePlace r;
    r.pool = values + (FMT == kFmtBf16 ? 2 : 1) * (pool_offset(c, k.page, 0, k.slot) + e0);
    r.scale = FMT == kFmtE4m3 ? scales + scale_offset(c, k.page, 0, k.slot) + (e0 >> 5) : nullptr;
    return r;
}
// 8 elements of a head; 4 lanes hold a block of 32.
template <int FMT>
__device__ __forceinline__ void put8(const RopePlace &at, int64_t offset, int scale_offset, bool live, const f32x2 (&y)[4], int lane)
{
    if (FMT == kFmtBf16) {
        if (live) *reinterpret_cast<uint4 *>(at.pool + 2 * offset) = to_bf16x8(y);
        return;
    }
    float f[8];
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        unpack2(y[j], f[2 * j], f[2 * j + 1]);
        amax = __vimax3_u32(amax, abs_bits(f[2 * j]), abs_bits(f[2 * j + 1]));
    }
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const int byte = scale_byte(amax);
    if (live) {
        *reinterpret_cast<uint2 *>(at.pool + offset) = to_e4m3x8(f, inverse_scale(byte));
        if ((lane & 3) == 0) at.scale[scale_offset] = static_cast<uint8_t>(byte);
    }
}

// The form for heads that are rotated in part or in neighbouring pairs.
// Warp (token, share of its heads); queries first, then keys, then (for the cache) values, each in runs of kRopeRun elements.
template <int FMT, bool DENSE>
__global__ void __launch_bounds__(kRopeThreads, 4) ead_rotate_kernel(RopeParams p)
{
    __shared__ alignas(16) float2 s_turn[kRopeThreads / 32][64];
    __shared__ alignas(16) uint8_t s_ring[kRopeThreads / 32][kRopePartDepth][512];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    griddep_wait();
    griddep_launch_dependents();
    RopeToken k;
    if (!token_of(p, warp, k)) return;
    const int t = k.t, nq = p.heads_q * p.dim, nk = p.heads_kv * p.dim;
    const int runs_q = (nq + kRopeRun - 1) / kRopeRun, runs_k = (nk + kRopeRun - 1) / kRopeRun, runs = runs_q + (DENSE ? 1 : 2) * runs_k;
    const int begin = runs * k.share / p.split, end = runs * (k.share + 1) / p.split;
    const uint32_t ring = smem_u32(s_ring[warp]) + lane * 16;
    const uint8_t *const row_q = p.q + 2 * t * p.q_stride, *const row_k = p.k + 2 * t * p.kv_stride, *const row_v = DENSE ? nullptr : p.v + 2 * t * p.kv_stride;
    int asked = begin, to_place = 0, from_place = 0;      // next run to ask for, its place, and the place of the next one to read
    auto ask = [&] {
        if (asked < end) {
            const int r = asked < runs_q ? asked : asked < runs_q + runs_k ? asked - runs_q : asked - runs_q - runs_k, e = r * kRopeRun + lane * 8;
            const uint8_t *const row = asked < runs_q ? row_q : asked < runs_q + runs_k ? row_k : row_v;
            if (e < (asked < runs_q ? nq : nk)) copy_async_16(ring + to_place * 512, row + 2 * e);
            ++asked;
            to_place = to_place + 1 == kRopePartDepth ? 0 : to_place + 1;
        }
        copy_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kRopePartDepth - 1; ++i) ask();
    if (!find_place<DENSE>(p, lane, k)) {
        copy_async_wait<0>();
        return;
    }
    float2 *const turn = s_turn[warp];
    const int in_head = lane & ((p.dim >> 3) - 1), e0 = in_head * 8, half = p.rot >> 1, shift = p.dim == 128 ? 7 : 6;
    RopeLane l;
    l.turned = e0 < p.rot;
    l.partner = p.interleaved ? -1 : !l.turned ? lane : e0 < half ? lane + (half >> 3) : lane - (half >> 3);
    if (begin < runs_q + runs_k) {                // (the angles are not for values)
        for (int i = lane; i < half; i += 32) turn[i] = rotation(k.position, ld_behind(p.inv_freq + i));
        __syncwarp();
    }
    // Runs r0 .. r1 - 1 of one kind with n elements; `done` takes a run's elements.
    auto stream = [&](int r0, int r1, int n, auto done) {
        for (int r = r0; r < r1; ++r) {
            ask();
            copy_async_wait<kRopePartDepth - 1>();
            const int e = r * kRopeRun + lane * 8;
            const uint4 x = e < n ? ld_shared_16(ring + from_place * 512) : make_uint4(0, 0, 0, 0);
            from_place = from_place + 1 == kRopePartDepth ? 0 : from_place + 1;
            done(e, e < n, x);
        }
    };
    const int q1 = min(end, runs_q), k0 = max(begin, runs_q) - runs_q, k1 = min(end, runs_q + runs_k) - runs_q;
    if (begin < q1) {
        set_factors(p, l, p.q_weight, turn, lane);
        uint8_t *const to = p.q_out + 2 * t * p.q_out_stride;
        stream(begin, q1, nq, [&](int e, bool live, const uint4 &x) {
            f32x2 y[4];
            norm_and_rotate(p, l, x, y);
            if (live) *reinterpret_cast<uint4 *>(to + 2 * e) = to_bf16x8(y);
        });
    }
    const int64_t head_stride = DENSE ? 0 : p.cache.head_stride;
    const int scale_stride = DENSE ? 0 : p.cache.page_size * (p.cache.head_dim / kFmtBlock);
    if (k0 < k1) {
        set_factors(p, l, p.k_weight, turn, lane);
        uint8_t *const to = DENSE ? p.k_out + 2 * t * p.k_out_stride : nullptr;
        const RopePlace at = DENSE ? RopePlace{} : place_of<FMT>(p.cache, k, p.cache.k, p.cache.k_scale, e0);
        stream(k0, k1, nk, [&](int e, bool live, const uint4 &x) {
            f32x2 y[4];
            norm_and_rotate(p, l, x, y);
            if (!DENSE)
                put8<FMT>(at, (e >> shift) * head_stride, (e >> shift) * scale_stride, live, y, lane);
            else if (live)
                *reinterpret_cast<uint4 *>(to + 2 * e) = to_bf16x8(y);
        });
    }
    if (DENSE) return;
    const int v0 = max(begin, runs_q + runs_k) - runs_q - runs_k, v1 = end - runs_q - runs_k;
    if (v0 < v1) {
        const RopePlace at = place_of<FMT>(p.cache, k, p.cache.v, p.cache.v_scale, e0);
        stream(v0, v1, nk, [&](int e, bool live, const uint4 &x) {
            f32x2 y[4];
            unpack8(x, y);
            put8<FMT>(at, (e >> shift) * head_stride, (e >> shift) * scale_stride, live, y, lane);
        });
    }
}

// The form for heads that are rotated as a whole, pairs in their two halves: a lane holds 8 elements of either half, so partners meet in a register
// and half as many lanes share a sum.  What the warp reads depends on the token alone: it is on its way to shared memory, kRopeDepth runs deep, while
// the token's place and angles are found.  (A lane copies and reads its own pieces: no barrier.)
template <int FMT, bool DENSE>
__global__ void __launch_bounds__(kRopeThreads, 2) ead_rotate_halves_kernel(RopeParams p)
{
    __shared__ alignas(16) float2 s_turn[kRopeThreads / 32][64];
    __shared__ alignas(16) uint8_t s_ring[kRopeThreads / 32][kRopeDepth][2][512];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    griddep_wait();
    griddep_launch_dependents();
    const int half = p.dim >> 1, per_head = half >> 3, in_head = lane & (per_head - 1), e0 = in_head * 8, heads_run = 32 / per_head, head0 = lane / per_head;
    const int runs_q = (p.heads_q + heads_run - 1) / heads_run, runs_k = (p.heads_kv + heads_run - 1) / heads_run, runs = runs_q + (DENSE ? 1 : 2) * runs_k;
    RopeToken k;
    if (!token_of(p, warp, k)) return;
    const int begin = runs * k.share / p.split, end = runs * (k.share + 1) / p.split;
    const uint32_t ring = smem_u32(s_ring[warp]) + lane * 16;
    const uint8_t *const row_q = p.q + 2 * (k.t * p.q_stride + e0), *const row_k = p.k + 2 * (k.t * p.kv_stride + e0);
    const uint8_t *const row_v = DENSE ? nullptr : p.v + 2 * (k.t * p.kv_stride + e0);
    int asked = begin, to = 0, from = 0;          // next run to ask for, its place, and the place of the next one to read
    auto ask = [&] {
        if (asked < end) {
            const int r = asked < runs_q ? asked : asked < runs_q + runs_k ? asked - runs_q : asked - runs_q - runs_k;
            const uint8_t *const row = asked < runs_q ? row_q : asked < runs_q + runs_k ? row_k : row_v;
            const int head = r * heads_run + head0;
            if (head < (asked < runs_q ? p.heads_q : p.heads_kv)) {
                copy_async_16(ring + to * 1024, row + 2 * head * p.dim);
                copy_async_16(ring + to * 1024 + 512, row + 2 * (head * p.dim + half));
            }
            ++asked;
            to = to + 1 == kRopeDepth ? 0 : to + 1;
        }
        copy_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kRopeDepth - 1; ++i) ask();
    if (!find_place<DENSE>(p, lane, k)) {
        copy_async_wait<0>();
        return;
    }
    float2 *const turn = s_turn[warp];
    if (begin < runs_q + runs_k) {                // (the angles are not for values)
        for (int i = lane; i < half; i += 32) turn[i] = rotation(k.position, ld_behind(p.inv_freq + i));
        __syncwarp();
    }
    // Runs r0 .. r1 - 1 of n heads; `done` takes a run's head and the two pieces.
    auto stream = [&](int r0, int r1, int n, auto done) {
        for (int r = r0; r < r1; ++r) {
            ask();
            copy_async_wait<kRopeDepth - 1>();
            const int head = r * heads_run + head0;
            const bool live = head < n;
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (live) {
                x = ld_shared_16(ring + from * 1024);
                y = ld_shared_16(ring + from * 1024 + 512);
            }
            from = from + 1 == kRopeDepth ? 0 : from + 1;
            done(head, live, x, y);
        }
    };
    const int64_t head_stride = DENSE ? 0 : p.cache.head_stride;
    const int scale_stride = DENSE ? 0 : p.cache.page_size * (p.cache.head_dim / kFmtBlock);
    auto put = [&](const RopePlace &at, int head, bool live, const f32x2 (&y)[4], const f32x2 (&z)[4]) {
        const RopePlace high{at.pool + (FMT == kFmtBf16 ? 2 : 1) * half, FMT == kFmtE4m3 ? at.scale + (half >> 5) : nullptr};
        put8<FMT>(at, head * head_stride, head * scale_stride, live, y, lane);
        put8<FMT>(high, head * head_stride, head * scale_stride, live, z, lane);
    };
    // Queries or keys: `weight` and the angles in four factors per pair of elements.
    auto turn_heads = [&](int r0, int r1, int n, const uint8_t *weight, auto done) {
        f32x2 fy[4], gy[4], fz[4], gz[4];
        {
            uint4 w = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), u = w;             // ones
            if (weight) {
                w = ld_behind(reinterpret_cast<const uint4 *>(weight + 2 * e0));
                u = ld_behind(reinterpret_cast<const uint4 *>(weight + 2 * (e0 + half)));
            }
            f32x2 wy[4], wz[4];
            unpack8(w, wy);
            unpack8(u, wz);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 cs = *reinterpret_cast<const float4 *>(turn + e0 + 2 * i);
                const f32x2 c = pack2(cs.x, cs.z), sn = pack2(cs.y, cs.w);
                fy[i] = mul2(wy[i], c);
                gy[i] = mul2(wz[i], pack2(-cs.y, -cs.w));
                fz[i] = mul2(wz[i], c);
                gz[i] = mul2(wy[i], sn);
            }
        }
        stream(r0, r1, n, [&](int head, bool live, const uint4 &x, const uint4 &v) {
            f32x2 a[4], b[4], y[4], z[4];
            unpack8(x, a);
            unpack8(v, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = fma2(a[i], fy[i], mul2(b[i], gy[i]));
                z[i] = fma2(b[i], fz[i], mul2(a[i], gz[i]));
            }
            if (weight) {
                f32x2 squares = mul2(a[0], a[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) squares = fma2(a[i], a[i], squares);
#pragma unroll
                for (int i = 0; i < 4; ++i) squares = fma2(b[i], b[i], squares);
                float sum, odd;
                unpack2(squares, sum, odd);
                sum += odd;
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if (per_head == 8) sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                const float r = rsqrtf(sum * (per_head == 8 ? 1.f / 128 : 1.f / 64) + p.eps);
                const f32x2 rr = pack2(r, r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[i] = mul2(y[i], rr);
                    z[i] = mul2(z[i], rr);
                }
            }
            done(head, live, y, z);
        });
    };
    auto to_rows = [&](uint8_t *row) {
        return [=](int head, bool live, const f32x2 (&y)[4], const f32x2 (&z)[4]) {
            uint8_t *const to = row + 2 * (head * p.dim + e0);
            if (!live) return;
            *reinterpret_cast<uint4 *>(to) = to_bf16x8(y);
            *reinterpret_cast<uint4 *>(to + 2 * half) = to_bf16x8(z);
        };
    };
    const int q1 = min(end, runs_q), k0 = max(begin, runs_q) - runs_q, k1 = min(end, runs_q + runs_k) - runs_q;
    if (begin < q1) turn_heads(begin, q1, p.heads_q, p.q_weight, to_rows(p.q_out + 2 * k.t * p.q_out_stride));
    if (k0 < k1) {
        if constexpr (DENSE) {
            turn_heads(k0, k1, p.heads_kv, p.k_weight, to_rows(p.k_out + 2 * k.t * p.k_out_stride));
        } else {
            const RopePlace at = place_of<FMT>(p.cache, k, p.cache.k, p.cache.k_scale, e0);
            turn_heads(k0, k1, p.heads_kv, p.k_weight, [&](int head, bool live, const f32x2 (&y)[4], const f32x2 (&z)[4]) { put(at, head, live, y, z); });
        }
    }
    if (DENSE) return;
    const int v0 = max(begin, runs_q + runs_k) - runs_q - runs_k, v1 = end - runs_q - runs_k;
    if (v0 < v1) {
        const RopePlace at = place_of<FMT>(p.cache, k, p.cache.v, p.cache.v_scale, e0);
        stream(v0, v1, p.heads_kv, [&](int head, bool live, const uint4 &x, const uint4 &v) {
            f32x2 y[4], z[4];
            unpack8(x, y);
            unpack8(v, z);
            put(at, head, live, y, z);
        });
    }
}

}  // namespace ead
