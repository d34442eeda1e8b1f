// The paged cache as the kernels see it, the lookup of a new token's place in it, and the 8-bit
// block format (e4m3 codes with one power-of-two scale byte per 32 values).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ead_internal.cuh"
#include "ptx_sm100.cuh"

namespace ead {

constexpr int kFmtBf16 = 0;
constexpr int kFmtE4m3 = 1;
constexpr int kFmtF32 = 2;
constexpr int kFmtF16 = 3;
constexpr int kFmtBlock = 32;
constexpr int kMaxBatch = 4096;                    // sequences of a step
constexpr uint32_t kStatusBadPage = 0x10u;
constexpr uint32_t kStatusBadToken = 0x20u;

struct KvCacheView {
    uint8_t *k, *v;                               // pools
    uint8_t *k_scale, *v_scale;                   // [n_pages, heads, page_size, head_dim / 32], e4m3 only
    int64_t page_stride, head_stride, slot_stride;   // elements
    int32_t heads, head_dim, page_size, page_shift, n_pages;
};

struct KvBatchView {
    const int32_t *new_start, *kv_len, *page_table;
    int32_t B, n_tokens, max_new, max_len, table_stride;
};

__device__ __forceinline__ void flag_status(uint32_t *status, uint32_t bits)
{
    if (status) atomicOr(status, bits);
}

// Largest b with start[b] <= t, found by the whole warp: every lane probes one of 32 equally spaced
// entries, so 1024 sequences take two dependent loads instead of a binary search's ten.
// start[0] = 0 and start[B] > t.  BEHIND: see ld_behind.
template <bool BEHIND = false>
__device__ __forceinline__ int find_sequence(const int32_t *start, int B, int t, int lane)
{
    int lo = 0, n = B;                            // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) >> 5;
        const int at = lo + lane * step;
        const bool le = lane * step < n && (BEHIND ? ld_behind(start + at) : __ldg(start + at)) <= t;
        const unsigned hits = __ballot_sync(0xffffffffu, le);
        const int last = 31 - __clz(hits | 1u);
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

// Page that holds position `pos` of sequence b, or -1 (nothing there, or an index outside the pool).
template <bool BEHIND = false>
__device__ __forceinline__ int find_page(const KvCacheView &c, const KvBatchView &bt, int b, int pos)
{
    if (pos < 0 || pos >= bt.max_len) return -1;
    const int32_t *const entry = bt.page_table + static_cast<int64_t>(b) * bt.table_stride + (pos >> c.page_shift);
    const int page = BEHIND ? ld_behind(entry) : __ldg(entry);
    return page >= 0 && page < c.n_pages ? page : -1;
}

__device__ __forceinline__ int64_t pool_offset(const KvCacheView &c, int page, int head, int slot)
{
    return page * c.page_stride + head * c.head_stride + slot * c.slot_stride;
}
__device__ __forceinline__ int64_t scale_offset(const KvCacheView &c, int page, int head, int slot)
{
    return ((static_cast<int64_t>(page) * c.heads + head) * c.page_size + slot) * (c.head_dim / kFmtBlock);
}

// Bits of |x|: they order like the magnitudes, with infinities and NaNs on top.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale byte of a block whose largest magnitude has these bits: 448 = 1.75 * 2^8, so its exponent
// less 8, one more when its mantissa exceeds 1.75 (the addition below carries exactly then);
// 255 for a block that is not finite.
__device__ __forceinline__ int scale_byte(uint32_t amax_bits)
{
    if (amax_bits >= 0x7f800000u) return 255;
    const int e = static_cast<int>((amax_bits + 0x1FFFFFu) >> 23) - 8;
    return min(max(e, 7), 246);                   // 2^-120 .. 2^119
}
// 2^(127 - byte), the factor that takes a value to its code's magnitude; NaN for byte 255, which
// turns every code of the block into 0x7F.
__device__ __forceinline__ float inverse_scale(int byte)
{
    return __uint_as_float(byte == 255 ? 0x7fffffffu : static_cast<uint32_t>(254 - byte) << 23);
}
// 2^(byte - 127); NaN for byte 255; byte 0, which the library never writes, is a subnormal.
__device__ __forceinline__ float scale_value(int byte)
{
    return __uint_as_float(byte == 255 ? 0x7fffffffu : byte == 0 ? 0x00400000u : static_cast<uint32_t>(byte) << 23);
}
// Two values to e4m3 codes (first value in the low byte): nearest even, saturating, NaN -> 0x7F.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes), __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Two 32-bit values in one register pair, for the instructions that take two at a time.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

}  // namespace ead
