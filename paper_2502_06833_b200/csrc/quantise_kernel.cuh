// bf16 values into 8-bit blocks: rows with a scale per 32 or 128 consecutive values (activations; of a gated MLP
// y = silu(gate) * x is taken on the way), and matrices with a scale per 128 x 128 (weights).
// Every value is read once and every code written once, so HBM bounds both at size and the launch at one step.
// Measured: 8191 rows of 13824 with a gate 95-102 us in a replayed graph, 5.6-5.9 TB/s, 0.85-0.91 of the device's copy rate, with 80 % of the issue slots
// taken (one exponential and one reciprocal per value), 104-111 us in calls one after another; 64 rows of 8960 2.1-3.0 us.  With one pass of 512 values per
// warp 145 us, 4 passes 103, 8 98, 14 and all 27 of a row 96.5.  Weights in 128 x 128 blocks: 152064 x 1536 132 us, 5.3 TB/s, 7168 x 5120 24 us, 4.7 TB/s
// (each block of threads has its tile's loads out at once and waits for all of them; a weight is brought into the format once).
#pragma once
#include "kv_format.cuh"
#include "ptx_sm100.cuh"
#include "rmsnorm_kernel.cuh"

namespace ead {

constexpr int kQuantThreads = 256;
constexpr int kQuantPass = 512;                    // values of a row that a warp takes at a time

struct QuantParams {
    const uint8_t *x, *gate;
    uint8_t *out, *out_scale;
    int64_t x_stride, gate_stride, out_stride;     // elements
    int32_t rows, cols, scale_cols;
    int32_t passes;                                // ceil(cols / kQuantPass)
    int32_t split;                                 // warps that share a row
};

__device__ __forceinline__ uint2 to_e4m3x8(const float (&y)[8], float inv)
{
    return make_uint2(to_e4m3x2(y[0] * inv, y[1] * inv) | to_e4m3x2(y[2] * inv, y[3] * inv) << 16,
                      to_e4m3x2(y[4] * inv, y[5] * inv) | to_e4m3x2(y[6] * inv, y[7] * inv) << 16);
}

// g / (1 + e^-g): the exponential and the quotient by the special function unit, 2^-22 each; the exponential's argument is rounded to 32 bits, which
// adds 1.25 x 2^-24 |g|: the result is within 2^-20 + 1.25 x 2^-24 |g| of itself (2^-17 at -87), where a code's rounding takes 2^-4.  The argument
// in an exact and a small part would bring 2^-20 at every gate for 103 us instead of 95 (8191 rows of 13824).  0 for gates below -87.3, where the divisor
// passes 2^126 (the product is below 2^-118 of x there).
__device__ __forceinline__ float silu(float g) { return __fdividef(g, 1.f + __expf(-g)); }

// A warp takes a stretch of a row, kQuantPass values at a time, a lane 8 consecutive ones of each half of them: BLOCK / 8 neighbouring lanes share a
// scale.  The next values' loads are on their way under the arithmetic.
template <int BLOCK, bool GATED>
__global__ void __launch_bounds__(kQuantThreads) ead_quantise_rows_kernel(QuantParams p)
{
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5);      // (the host sees to it that these fit)
    const int row = static_cast<int>(unit / static_cast<uint32_t>(p.split)), share = static_cast<int>(unit - static_cast<uint32_t>(row) * p.split);
    if (row >= p.rows) return;
    const int pass0 = static_cast<int>(static_cast<int64_t>(p.passes) * share / p.split), pass1 = static_cast<int>(static_cast<int64_t>(p.passes) * (share + 1) / p.split);
    const uint8_t *const x_row = p.x + 2 * row * p.x_stride, *const g_row = GATED ? p.gate + 2 * row * p.gate_stride : nullptr;
    uint8_t *const out_row = p.out + row * p.out_stride, *const scale_row = p.out_scale + static_cast<int64_t>(row) * p.scale_cols;
    uint4 x[2], g[2];
    auto load = [&](int pass) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = pass * kQuantPass + h * (kQuantPass / 2) + lane * 8;
            x[h] = g[h] = make_uint4(0, 0, 0, 0);
            if (col < p.cols) {
                x[h] = ld_behind(reinterpret_cast<const uint4 *>(x_row + 2 * static_cast<int64_t>(col)));
                if (GATED) g[h] = ld_behind(reinterpret_cast<const uint4 *>(g_row + 2 * static_cast<int64_t>(col)));
            }
        }
    };
    load(pass0);
    for (int pass = pass0; pass < pass1; ++pass) {
        uint4 xn[2], gn[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            xn[h] = x[h];
            gn[h] = g[h];
        }
        if (pass + 1 < pass1) load(pass + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = pass * kQuantPass + h * (kQuantPass / 2) + lane * 8;
            float y[8];
            unpack8(xn[h], y);
            if (GATED) {
                float a[8];
                unpack8(gn[h], a);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] *= silu(a[k]);
            }
            uint32_t amax = 0;
#pragma unroll
            for (int k = 0; k < 8; k += 2) amax = __vimax3_u32(amax, abs_bits(y[k]), abs_bits(y[k + 1]));
            if (GATED && amax >= 0x7f800000u) {    // a product of finite values that passes 32 bits saturates like any other large value
                float u[8], a[8];
                unpack8(xn[h], u);
                unpack8(gn[h], a);
                amax = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (abs_bits(y[k]) == 0x7f800000u && isfinite(u[k]) && isfinite(a[k])) y[k] = copysignf(3.402823466e38f, y[k]);
                    amax = max(amax, abs_bits(y[k]));
                }
            }
#pragma unroll
            for (int o = 1; o < BLOCK / 8; o <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const int byte = scale_byte(amax);
            if (col < p.cols) {
                *reinterpret_cast<uint2 *>(out_row + col) = to_e4m3x8(y, inverse_scale(byte));
                if ((lane & (BLOCK / 8 - 1)) == 0) scale_row[col / BLOCK] = static_cast<uint8_t>(byte);
            }
        }
    }
}

// A block takes 128 x 128 values: thread t columns 8 (t mod 16) .. + 7 of rows t / 16 + 16 i.
__global__ void __launch_bounds__(kQuantThreads) ead_quantise_tiles_kernel(QuantParams p)
{
    __shared__ uint32_t part[kQuantThreads / 32];
    griddep_wait();
    griddep_launch_dependents();
    const int64_t row0 = static_cast<int64_t>(blockIdx.x / p.scale_cols) * 128 + threadIdx.x / 16;
    const int col = static_cast<int>(blockIdx.x % p.scale_cols) * 128 + (threadIdx.x & 15) * 8;
    uint4 x[8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        if (col < p.cols && row0 + 16 * i < p.rows) x[i] = ld_behind(reinterpret_cast<const uint4 *>(p.x + 2 * ((row0 + 16 * i) * p.x_stride + col)));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float y[8];
        unpack8(x[i], y);
#pragma unroll
        for (int k = 0; k < 8; ++k) amax = max(amax, abs_bits(y[k]));
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 32; ++i) amax = max(amax, part[i]);
    const int byte = scale_byte(amax);
    const float inv = inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float y[8];
        unpack8(x[i], y);
        if (col < p.cols && row0 + 16 * i < p.rows) *reinterpret_cast<uint2 *>(p.out + (row0 + 16 * i) * p.out_stride + col) = to_e4m3x8(y, inv);
    }
    if (threadIdx.x == 0) p.out_scale[blockIdx.x] = static_cast<uint8_t>(byte);
}

}  // namespace ead
