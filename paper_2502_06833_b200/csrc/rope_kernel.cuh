// Root-mean-square norm of every query and key head, and the position rotation, in one pass over a step's projections; the
// results go into tensors (dense) or, with the values, straight into the paged cache in its format:
//   y = x / sqrt(mean(x^2) + eps) * weight,   (a, b) -> (a cos - b sin, b cos + a sin),   angle = position * inv_freq[j]
// A warp takes one token (with few tokens: some of its heads): it looks up the token's place, computes the angles once, the product in 64 bits and
// brought within half a turn before it is rounded to 32, and then streams the heads.  A lane holds 8 consecutive elements of a head, a head is 8
// or 16 neighbouring lanes.  Weight, cos and sin come together in two factors per element that a lane keeps for all heads,
//   y_e = (x_e f_e + x_partner g_e) / sqrt(mean(x^2) + eps),   f = weight cos,   g = -+ weight of the partner sin
// so partners exchange the bf16 words as they were loaded.  Every element is read once and written once: HBM bounds it at size, launch and the
// chain of look-ups at one step.
#pragma once
#include "quantise_kernel.cuh"

namespace ead {

constexpr int kRopeThreads = 256;
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
        w = o = __ldg(reinterpret_cast<const uint4 *>(weight) + in_head);
        if (l.partner >= 0) o = __ldg(reinterpret_cast<const uint4 *>(weight) + (l.partner & ((p.dim >> 3) - 1)));
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

// Warp (token, share of its heads); queries first, then keys, then (for the cache) values, each in runs of kRopeRun elements.
template <int FMT, bool DENSE>
__global__ void __launch_bounds__(kRopeThreads, 4) ead_rotate_kernel(RopeParams p)
{
    __shared__ alignas(16) float2 s_turn[kRopeThreads / 32][64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    griddep_wait();
    griddep_launch_dependents();
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kRopeThreads / 32) + warp;
    const int t = p.split == 1 ? static_cast<int>(unit) : static_cast<int>(unit / p.split), share = static_cast<int>(unit - static_cast<int64_t>(t) * p.split);
    if (t >= p.n_tokens) return;
    const int nq = p.heads_q * p.dim, nk = p.heads_kv * p.dim;
    const int runs_q = (nq + kRopeRun - 1) / kRopeRun, runs_k = (nk + kRopeRun - 1) / kRopeRun, runs = runs_q + (DENSE ? 1 : 2) * runs_k;
    const int begin = runs * share / p.split, end = runs * (share + 1) / p.split;
    int position, page = 0, slot = 0;
    if (DENSE) {
        position = __ldg(p.positions + t);
    } else {
        const int b = find_sequence(p.batch.new_start, p.batch.B, t, lane);
        const int first = __ldg(p.batch.new_start + b), last = __ldg(p.batch.new_start + b + 1);
        const bool bad = first < 0 || t < first || t >= last || last > p.batch.n_tokens || last - first > p.batch.max_new;
        const int cached = __ldg(p.batch.kv_len + b) - (last - t);
        page = bad ? -1 : find_page(p.cache, p.batch, b, cached);
        position = p.positions ? __ldg(p.positions + t) : cached;
        slot = cached & (p.cache.page_size - 1);
        if (page < 0) {                           // no place: nothing of the token is written
            if (lane == 0 && share == 0) flag_status(p.status, bad ? kStatusBadCount : kStatusBadPage);
            return;
        }
    }
    float2 *const turn = s_turn[warp];
    const int in_head = lane & ((p.dim >> 3) - 1), e0 = in_head * 8, half = p.rot >> 1, shift = p.dim == 128 ? 7 : 6;
    RopeLane l;
    l.turned = e0 < p.rot;
    l.partner = p.interleaved ? -1 : !l.turned ? lane : e0 < half ? lane + (half >> 3) : lane - (half >> 3);
    if (begin < runs_q + runs_k) {                // (the angles are not for values)
        for (int i = lane; i < half; i += 32) turn[i] = rotation(position, __ldg(p.inv_freq + i));
        __syncwarp();
    }
    // Runs r0 .. r1 - 1 of one kind; `done` takes a run's elements.
    auto stream = [&](int r0, int r1, const uint8_t *row, int n, auto done) {
        const uint8_t *from = row + 2 * (r0 * kRopeRun + lane * 8);
        int e = r0 * kRopeRun + lane * 8;         // of a run's first element
        auto load = [&](int ahead) { return e + ahead * kRopeRun < n ? *reinterpret_cast<const uint4 *>(from + 2 * ahead * kRopeRun) : make_uint4(0, 0, 0, 0); };
        uint4 x0 = load(0), x1 = r0 + 1 < r1 ? load(1) : x0;
        for (int r = r0; r < r1; r += 2, e += 2 * kRopeRun, from += 4 * kRopeRun) {
            const uint4 y0 = x0;
            if (r + 2 < r1) x0 = load(2);
            done(e, e < n, y0);
            if (r + 1 >= r1) break;
            const uint4 y1 = x1;
            if (r + 3 < r1) x1 = load(3);
            done(e + kRopeRun, e + kRopeRun < n, y1);
        }
    };
    const int q1 = min(end, runs_q), k0 = max(begin, runs_q) - runs_q, k1 = min(end, runs_q + runs_k) - runs_q;
    if (begin < q1) {
        set_factors(p, l, p.q_weight, turn, lane);
        uint8_t *const to = p.q_out + 2 * t * p.q_out_stride;
        stream(begin, q1, p.q + 2 * t * p.q_stride, nq, [&](int e, bool live, const uint4 &x) {
            f32x2 y[4];
            norm_and_rotate(p, l, x, y);
            if (live) *reinterpret_cast<uint4 *>(to + 2 * e) = to_bf16x8(y);
        });
    }
    // a key or value of the cache
    uint8_t *pool = nullptr, *scale = nullptr;
    const int64_t head_stride = DENSE ? 0 : p.cache.head_stride;
    const int scale_stride = DENSE ? 0 : p.cache.page_size * (p.cache.head_dim / kFmtBlock);
    auto put = [&](int e, bool live, const f32x2 (&y)[4]) {
        const int head = e >> shift;
        const int64_t to = head * head_stride;
        if (FMT == kFmtBf16) {
            if (live) *reinterpret_cast<uint4 *>(pool + 2 * to) = to_bf16x8(y);
            return;
        }
        float f[8];
        uint32_t amax = 0;                        // 4 lanes hold a block of 32
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unpack2(y[j], f[2 * j], f[2 * j + 1]);
            amax = __vimax3_u32(amax, abs_bits(f[2 * j]), abs_bits(f[2 * j + 1]));
        }
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const int byte = scale_byte(amax);
        if (live) {
            *reinterpret_cast<uint2 *>(pool + to) = to_e4m3x8(f, inverse_scale(byte));
            if ((lane & 3) == 0) scale[head * scale_stride] = static_cast<uint8_t>(byte);
        }
    };
    auto set_pool = [&](uint8_t *values, uint8_t *scales) {
        pool = values + (FMT == kFmtBf16 ? 2 : 1) * (pool_offset(p.cache, page, 0, slot) + e0);
        if (FMT == kFmtE4m3) scale = scales + scale_offset(p.cache, page, 0, slot) + (e0 >> 5);
    };
    if (k0 < k1) {
        set_factors(p, l, p.k_weight, turn, lane);
        uint8_t *const to = DENSE ? p.k_out + 2 * t * p.k_out_stride : nullptr;
        if (!DENSE) set_pool(p.cache.k, p.cache.k_scale);
        stream(k0, k1, p.k + 2 * t * p.kv_stride, nk, [&](int e, bool live, const uint4 &x) {
            f32x2 y[4];
            norm_and_rotate(p, l, x, y);
            if (!DENSE)
                put(e, live, y);
            else if (live)
                *reinterpret_cast<uint4 *>(to + 2 * e) = to_bf16x8(y);
        });
    }
    if (DENSE) return;
    const int v0 = max(begin, runs_q + runs_k) - runs_q - runs_k, v1 = end - runs_q - runs_k;
    if (v0 < v1) {
        set_pool(p.cache.v, p.cache.v_scale);
        stream(v0, v1, p.v + 2 * t * p.kv_stride, nk, [&](int e, bool live, const uint4 &x) {
            if (FMT == kFmtBf16) {
                if (live) *reinterpret_cast<uint4 *>(pool + 2 * (e >> shift) * head_stride) = x;
                return;
            }
            f32x2 y[4];
            unpack8(x, y);
            put(e, live, y);
        });
    }
}

}  // namespace ead
