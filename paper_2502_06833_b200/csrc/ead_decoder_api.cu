// Host side of the decoder-side operators declared in include/ead.h: paged key/value cache, chunk
// attention over it, residual norm.  Stateless: arguments are checked, kernels are enqueued.
#include "../../include/ead.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <mutex>

#include "attn_chunk_kernel.cuh"
#include "attn_few_rows_kernel.cuh"
#include "kv_cache_kernels.cuh"
#include "rmsnorm_kernel.cuh"
#include "tma_host.h"

using namespace ead;

namespace {

#define EAD_CUDA(x)                          \
    do {                                     \
        if ((x) != cudaSuccess) {            \
            cudaGetLastError();              \
            return EAD_ECUDA;                \
        }                                    \
    } while (0)

constexpr int kMaxDevices = 64;
constexpr int kNormThreadsPerSm = 2048;   // what an SM holds; further rows are taken by the same blocks in turn
// Tokens per warp of an 8-bit cache's write and read, where a call moves at least kKvLongRunValues values; otherwise, and for
// bf16, one.  Measured, one against four tokens per warp: e4m3, write of 24 k tokens with 8 heads of 128 35.0 against 31.1 us,
// read of 107 k 143 against 114, write of 2^24 values 12.5 against 11.7, of 2^23 7.3 against 7.7, of 2^20 3.1 against 3.7.  bf16
// never gains (2^24 values 12.5 against 13.7, 2^26 47.6 against 48.6): twice the stores keep the memory busy by themselves.
constexpr int kKvRun = 4;
constexpr int64_t kKvLongRunValues = 1 << 24;
// Least work per block of the chunk kernel (a tile of 128 rows x 64 keys: 1), so that a short call does not cut every unit into
// parts.  16, 24 and 48 did not differ beyond noise.
constexpr int kChunkMinCost = 24;
static_assert(kChunkMinCost >= kChunkUnitCost + 2, "every block's stretch has to hold the beginning of a tile");
// Tiles of 8 KiB per block before another block is worth its part in the join; it decides calls with less than that per SM.
// Measured, 8 / 16 / 32 tiles, us: one context of 777 keys, 8 heads of 64, bf16 9.7 / 9.9 / 15.2; 4 of 777, 2 heads of 128, bf16
// 16.0 / 13.2 / 14.4; 4 of 300, 8 heads of 64, bf16 7.6 / 10.5 / 17.3, e4m3 13.4 / 23.0 / 37.1; 16 of 777, 8 heads of 128, e4m3
// 14.1 / 14.2 / 23.6.
constexpr int kFewMinTiles = 16;

struct DeviceInfo {
    bool ready = false;
    int sms = 0;
};

std::mutex g_mu;
std::atomic<uint32_t> g_wait_ns{static_cast<uint32_t>(kWaitLimitNs)};   // of the attention kernels' bounded waits
static_assert(kWaitLimitNs <= 0x7fffffffu, "held in 32 bits");
DeviceInfo g_dev[kMaxDevices];

int launched() { return cudaGetLastError() == cudaSuccess ? EAD_OK : EAD_ECUDA; }

// A pool as {128-byte (or 64-byte) line of a key, slot, line, head, page}; a box is `keys` consecutive slots of one
// head of one page, `lines` of its lines one after the other, with the swizzle that makes eight keys' chunks conflict-free.
bool encode_pool(CUtensorMap *tm, const KvCacheView &c, int format, void *base, int keys, int lines)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const bool bf16 = format == EAD_FMT_BF16;
    const int size = bf16 ? 2 : 1, row = c.head_dim * size, line = std::min(row, 128);
    const cuuint64_t dims[5] = {static_cast<cuuint64_t>(line / size), static_cast<cuuint64_t>(c.page_size),
                                static_cast<cuuint64_t>(row / line), static_cast<cuuint64_t>(c.heads),
                                static_cast<cuuint64_t>(c.n_pages)};
    const cuuint64_t strides[4] = {static_cast<cuuint64_t>(c.slot_stride * size), static_cast<cuuint64_t>(line),
                                   static_cast<cuuint64_t>(c.head_stride * size),
                                   static_cast<cuuint64_t>(c.page_stride * size)};
    const cuuint32_t box[5] = {static_cast<cuuint32_t>(line / size), static_cast<cuuint32_t>(keys),
                               static_cast<cuuint32_t>(lines), 1, 1};
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    return fn(tm, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, base, dims, strides, box, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, line == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The query rows as {dimension, head, token}; a box is 64 dimensions of a cache head's query heads for the tokens of a row tile.
bool encode_queries(CUtensorMap *tm, const AttnParams &p)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(p.cache.head_dim), static_cast<cuuint64_t>(p.heads_q),
                                static_cast<cuuint64_t>(p.batch.n_tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(2 * p.cache.head_dim), static_cast<cuuint64_t>(2 * p.q_stride)};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(p.group), static_cast<cuuint32_t>(p.tile_tokens)}, ones[3] = {1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint8_t *>(p.q), dims, strides, box, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FMT, int D, int NB>
int launch_few_rows(const AttnParams &p, int sms, cudaStream_t s)
{
    using L = FewLayout<FMT, D, NB>;
    const int keys = std::min(p.cache.page_size, L::kTile);
    CUtensorMap tk, tv;
    if (!encode_pool(&tk, p.cache, FMT, p.cache.k, keys, L::kBoxes) || !encode_pool(&tv, p.cache, FMT, p.cache.v, keys, L::kBoxes))
        return EAD_ECUDA;
    ead_attn_few_rows_kernel<FMT, D, NB><<<std::min(sms, kAttnMaxCtas), L::kThreads, L::kSmem, s>>>(tk, tv, p, __builtin_ctz(keys), kFewMinTiles);
    return launched();
}

template <int FMT, int D>
int launch_few_rows(const AttnParams &p, int sms, cudaStream_t s)
{
    return p.few_rows <= 8 ? launch_few_rows<FMT, D, 1>(p, sms, s) : launch_few_rows<FMT, D, 2>(p, sms, s);
}

template <int FMT, int D>
int launch_chunk(const AttnParams &p, int sms, cudaStream_t s)
{
    using L = ChunkLayout<FMT, D>;
    const int keys = std::min(p.cache.page_size, kChunkKeys);
    CUtensorMap tk, tv;
    if (!encode_pool(&tk, p.cache, FMT, p.cache.k, keys, 1) || !encode_pool(&tv, p.cache, FMT, p.cache.v, keys, FMT == kFmtBf16 ? D / 64 : 1))
        return EAD_ECUDA;
    CUtensorMap tq;
    if (!encode_queries(&tq, p)) return EAD_ECUDA;
    // Behind the few-rows kernel of the same call it may start as that one's blocks leave their SMs.
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(std::min(sms, kAttnMaxCtas));
    cfg.blockDim = dim3(L::kThreads);
    cfg.dynamicSmemBytes = L::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.few_rows ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, ead_attn_chunk_kernel<FMT, D>, tk, tv, tq, p, static_cast<int>(__builtin_ctz(keys)), kChunkMinCost) != cudaSuccess) {
        cudaGetLastError();
        return EAD_ECUDA;
    }
    return EAD_OK;
}

template <int FMT, int D, int NB>
bool allow_smem()
{
    return cudaFuncSetAttribute(ead_attn_few_rows_kernel<FMT, D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                FewLayout<FMT, D, NB>::kSmem) == cudaSuccess;
}
template <int FMT, int D>
bool allow_smem()
{
    return allow_smem<FMT, D, 1>() && allow_smem<FMT, D, 2>() &&
           cudaFuncSetAttribute(ead_attn_chunk_kernel<FMT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                ChunkLayout<FMT, D>::kSmem) == cudaSuccess;
}

// Makes `device` current; on its first use checks the architecture and sets kernel attributes.
int use_device(int device, DeviceInfo **out)
{
    if (device < 0 || device >= kMaxDevices) return EAD_EINVALID_ARG;
    std::lock_guard<std::mutex> lock(g_mu);
    DeviceInfo &d = g_dev[device];
    if (!d.ready) {
        int n = 0, major = 0;
        EAD_CUDA(cudaGetDeviceCount(&n));
        if (device >= n) return EAD_EINVALID_ARG;
        EAD_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device));
        if (major != 10) return EAD_EUNSUPPORTED_ARCH;
        EAD_CUDA(cudaSetDevice(device));
        EAD_CUDA(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, device));
        if (!allow_smem<kFmtBf16, 64>() || !allow_smem<kFmtBf16, 128>() || !allow_smem<kFmtE4m3, 64>() ||
            !allow_smem<kFmtE4m3, 128>()) {
            cudaGetLastError();
            return EAD_ECUDA;
        }
        d.ready = true;
    }
    EAD_CUDA(cudaSetDevice(device));
    *out = &d;
    return EAD_OK;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_cache(const ead_kv_cache *c, KvCacheView *v)
{
    if (!c || (c->format != EAD_FMT_BF16 && c->format != EAD_FMT_E4M3) || c->reserved) return EAD_EINVALID_ARG;
    if (c->heads_kv < 1 || c->heads_kv > 128 || (c->head_dim != 64 && c->head_dim != 128)) return EAD_EINVALID_ARG;
    if (c->page_size < 8 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) || c->n_pages < 1)
        return EAD_EINVALID_ARG;
    if (!c->k || !c->v || c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < c->head_dim) return EAD_EINVALID_ARG;
    const bool e4m3 = c->format == EAD_FMT_E4M3;
    if (e4m3 != (c->k_scale != nullptr) || e4m3 != (c->v_scale != nullptr)) return EAD_EINVALID_ARG;
    const int per16 = e4m3 ? 16 : 8;                  // elements in 16 bytes
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->page_stride % per16 || c->head_stride % per16 ||
        c->slot_stride % per16)
        return EAD_EALIGNMENT;
    if (e4m3 && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))) return EAD_EALIGNMENT;
    v->k = static_cast<uint8_t *>(c->k);
    v->v = static_cast<uint8_t *>(c->v);
    v->k_scale = c->k_scale;
    v->v_scale = c->v_scale;
    v->page_stride = c->page_stride;
    v->head_stride = c->head_stride;
    v->slot_stride = c->slot_stride;
    v->heads = c->heads_kv;
    v->head_dim = c->head_dim;
    v->page_size = c->page_size;
    v->page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
    v->n_pages = c->n_pages;
    return EAD_OK;
}

int check_batch(const ead_kv_batch *b, const KvCacheView &c, bool needs_len, KvBatchView *v)
{
    if (!b || b->reserved || b->B < 1 || b->B > kMaxBatch || b->n_tokens < 0 || b->max_new < 0 || b->max_len < 0)
        return EAD_EINVALID_ARG;
    if (!b->new_start || (needs_len && !b->kv_len) || !b->page_table || b->table_stride < 1) return EAD_EINVALID_ARG;
    if (b->n_tokens > static_cast<int64_t>(b->B) * b->max_new) return EAD_EINVALID_ARG;
    if (b->max_len > static_cast<int64_t>(b->table_stride) * c.page_size) return EAD_EINVALID_ARG;
    if (b->max_len > (1 << 30) || b->n_tokens > (1 << 30)) return EAD_EINVALID_ARG;   // positions stay within 32 bits
    if (!aligned(b->new_start, 4) || !aligned(b->kv_len, 4) || !aligned(b->page_table, 4)) return EAD_EALIGNMENT;
    v->new_start = b->new_start;
    v->kv_len = b->kv_len;
    v->page_table = b->page_table;
    v->B = b->B;
    v->n_tokens = b->n_tokens;
    v->max_new = b->max_new;
    v->max_len = b->max_len;
    v->table_stride = b->table_stride;
    return EAD_OK;
}

// Caller's bf16 rows of `elements` values, `stride` apart.
int check_rows(const void *p, int64_t stride, int64_t elements)
{
    if (!p || stride < elements) return EAD_EINVALID_ARG;
    if (!aligned(p, 16) || stride % 8) return EAD_EALIGNMENT;
    return EAD_OK;
}

int move_setup(const ead_kv_cache *cache, const ead_kv_batch *batch, const void *k, const void *v, int64_t stride,
               uint32_t *status, bool needs_len, int32_t device, KvMoveParams *p, DeviceInfo **d)
{
    int rc = check_cache(cache, &p->cache);
    if (rc == EAD_OK) rc = check_batch(batch, p->cache, needs_len, &p->batch);
    const int64_t row = static_cast<int64_t>(p->cache.heads) * p->cache.head_dim;
    if (rc != EAD_OK || p->batch.n_tokens == 0) return rc;      // nothing to do: the rows may have no address
    rc = check_rows(k, stride, row);
    if (rc == EAD_OK) rc = check_rows(v, stride, row);
    if (rc == EAD_OK && !aligned(status, 4)) rc = EAD_EALIGNMENT;
    if (rc == EAD_OK) rc = use_device(device, d);
    if (rc != EAD_OK) return rc;
    p->rows_k = static_cast<uint8_t *>(const_cast<void *>(k));
    p->rows_v = static_cast<uint8_t *>(const_cast<void *>(v));
    p->row_stride = stride;
    p->status = status;
    return EAD_OK;
}

// Units of up to 16 packed rows have a kernel of their own.  Where longer chunks are there as well, only up to 8:
// a second group of 8 rows costs every unit, and the other kernel runs anyway.  `most`: packed rows of the largest unit.
int few_rows_limit(int group, int64_t most)
{
    return group > kDecodeRows ? 0 : most <= 8 || (most > kDecodeRows && group <= 8) ? 8 : kDecodeRows;
}

// One warp per run of tokens and stretch of a token's values.
bool long_runs(const KvMoveParams &p)
{
    return int64_t{2} * p.batch.n_tokens * p.cache.heads * p.cache.head_dim >= kKvLongRunValues;
}

dim3 move_grid(const KvMoveParams &p, int run)
{
    const int warps = (p.batch.n_tokens + run - 1) / run, per_block = kKvThreads / 32;
    return dim3((warps + per_block - 1) / per_block, (2 * p.cache.heads * p.cache.head_dim + kKvPass - 1) / kKvPass);
}

}  // namespace

extern "C" int ead_kv_write(const ead_kv_cache *cache, const ead_kv_batch *batch, const void *k_new, const void *v_new,
                            int64_t new_stride, uint32_t *status, int32_t device, void *stream)
{
    KvMoveParams p{};
    DeviceInfo *d = nullptr;
    const int rc = move_setup(cache, batch, k_new, v_new, new_stride, status, true, device, &p, &d);
    if (rc != EAD_OK || p.batch.n_tokens == 0) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cache->format == EAD_FMT_BF16)
        ead_kv_write_kernel<kFmtBf16, 1><<<move_grid(p, 1), kKvThreads, 0, s>>>(p);
    else if (!long_runs(p))
        ead_kv_write_kernel<kFmtE4m3, 1><<<move_grid(p, 1), kKvThreads, 0, s>>>(p);
    else
        ead_kv_write_kernel<kFmtE4m3, kKvRun><<<move_grid(p, kKvRun), kKvThreads, 0, s>>>(p);
    return launched();
}

extern "C" int ead_kv_read(const ead_kv_cache *cache, const ead_kv_batch *batch, const int32_t *first, void *k_out,
                           void *v_out, int64_t out_stride, uint32_t *status, int32_t device, void *stream)
{
    KvMoveParams p{};
    DeviceInfo *d = nullptr;
    if (!aligned(first, 4)) return EAD_EALIGNMENT;
    const int rc = move_setup(cache, batch, k_out, v_out, out_stride, status, false, device, &p, &d);
    if (rc != EAD_OK || p.batch.n_tokens == 0) return rc;
    p.first = first;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cache->format == EAD_FMT_BF16)
        ead_kv_read_kernel<kFmtBf16, 1><<<move_grid(p, 1), kKvThreads, 0, s>>>(p);
    else if (!long_runs(p))
        ead_kv_read_kernel<kFmtE4m3, 1><<<move_grid(p, 1), kKvThreads, 0, s>>>(p);
    else
        ead_kv_read_kernel<kFmtE4m3, kKvRun><<<move_grid(p, kKvRun), kKvThreads, 0, s>>>(p);
    return launched();
}

extern "C" int ead_kv_attention(const ead_kv_cache *cache, const ead_kv_batch *batch, const void *q, int64_t q_stride,
                                int32_t heads_q, float scale, int32_t window, int32_t sinks, void *out,
                                int64_t out_stride, float *lse, void *workspace, uint32_t *status, int32_t device,
                                void *stream)
{
    AttnParams p{};
    DeviceInfo *d = nullptr;
    int rc = check_cache(cache, &p.cache);
    if (rc == EAD_OK) rc = check_batch(batch, p.cache, true, &p.batch);
    if (rc != EAD_OK) return rc;
    if (heads_q < p.cache.heads || heads_q % p.cache.heads || heads_q / p.cache.heads > 128) return EAD_EINVALID_ARG;
    if (!std::isfinite(scale) || !(scale > 0.f) || window < 0 || sinks < 0 || !workspace) return EAD_EINVALID_ARG;
    if (p.batch.n_tokens == 0) return EAD_OK;
    const int64_t row = static_cast<int64_t>(heads_q) * p.cache.head_dim;
    rc = check_rows(q, q_stride, row);
    if (rc == EAD_OK) rc = check_rows(out, out_stride, row);
    if (rc == EAD_OK && (!aligned(lse, 4) || !aligned(workspace, 256) || !aligned(status, 4))) rc = EAD_EALIGNMENT;
    if (rc == EAD_OK) rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    p.q = static_cast<const uint8_t *>(q);
    p.out = static_cast<uint8_t *>(out);
    p.lse = lse;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.heads_q = heads_q;
    p.group = heads_q / p.cache.heads;
    p.window = std::min(window, 1 << 30);     // positions lie below
    p.sinks = window ? sinks : 0;
    p.scale_log2 = scale * kLog2e;
    p.workspace = static_cast<uint8_t *>(workspace);
    p.status = status;
    p.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    p.wait_hint = std::min(p.wait_ns, 20000u);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t most = static_cast<int64_t>(p.batch.max_new) * p.group;
    p.tile_tokens = 128 / p.group;
    p.few_rows = few_rows_limit(p.group, most);
    if (most > 0x7fffffff) return EAD_EINVALID_ARG;
    // the few-rows kernel counts a block's tiles, of at least 16 keys, in 32 bits (a block takes minutes for so many)
    if (p.few_rows && static_cast<int64_t>(p.batch.B) * p.cache.heads * (p.batch.max_len / 16 + 2) / std::min(d->sms, kAttnMaxCtas) > (1 << 30))
        return EAD_ELIMIT;
    const bool bf16 = cache->format == EAD_FMT_BF16, wide = p.cache.head_dim == 128;
    if (p.few_rows) {
        rc = bf16 ? (wide ? launch_few_rows<kFmtBf16, 128>(p, d->sms, s) : launch_few_rows<kFmtBf16, 64>(p, d->sms, s))
                  : (wide ? launch_few_rows<kFmtE4m3, 128>(p, d->sms, s) : launch_few_rows<kFmtE4m3, 64>(p, d->sms, s));
        if (rc != EAD_OK) return rc;
    }
    if (most > p.few_rows)
        rc = bf16 ? (wide ? launch_chunk<kFmtBf16, 128>(p, d->sms, s) : launch_chunk<kFmtBf16, 64>(p, d->sms, s))
                  : (wide ? launch_chunk<kFmtE4m3, 128>(p, d->sms, s) : launch_chunk<kFmtE4m3, 64>(p, d->sms, s));
    return rc;
}

extern "C" int ead_kv_wait_limit(int32_t ns)
{
    g_wait_ns.store(ns < 0 ? static_cast<uint32_t>(kWaitLimitNs) : static_cast<uint32_t>(ns), std::memory_order_relaxed);
    return EAD_OK;
}

extern "C" int ead_plan_chunk(int32_t n_new, int32_t kv_len, int32_t max_new, int32_t heads_per_kv, int32_t window, int32_t sinks,
                              int64_t *out)
{
    if (!out || n_new < 0 || n_new > max_new || max_new > (1 << 30) || kv_len < 0 || kv_len > (1 << 30) || heads_per_kv < 1 ||
        heads_per_kv > 128 || window < 0 || sinks < 0 || static_cast<int64_t>(max_new) * heads_per_kv > 0x7fffffff)
        return EAD_EINVALID_ARG;
    AttnParams p{};
    p.group = heads_per_kv;
    p.window = std::min(window, 1 << 30);
    p.sinks = window ? sinks : 0;
    p.tile_tokens = 128 / p.group;
    p.few_rows = few_rows_limit(p.group, static_cast<int64_t>(max_new) * p.group);
    const SeqInfo s{n_new, kv_len - n_new, kv_len, 0};
    out[0] = chunk_blocks(p, s);
    out[1] = chunk_cost(p, s, 0, 1);
    return EAD_OK;
}

extern "C" int ead_add_rmsnorm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                               void *residual_out, int64_t residual_out_stride, const void *weight, float eps,
                               int32_t n_rows, int32_t H, int32_t format, void *out, int64_t out_stride,
                               uint8_t *out_scale, int32_t device, void *stream)
{
    const bool e4m3 = format == EAD_FMT_E4M3;
    if ((format != EAD_FMT_BF16 && !e4m3) || n_rows < 0 || H < 8 || !weight || e4m3 != (out_scale != nullptr))
        return EAD_EINVALID_ARG;
    if (!std::isfinite(eps) || eps < 0.f) return EAD_EINVALID_ARG;
    if (H > EAD_NORM_MAX_H) return EAD_ELIMIT;
    if (H % (e4m3 ? kFmtBlock : 8) || !aligned(weight, 16)) return EAD_EALIGNMENT;
    if (n_rows == 0) return EAD_OK;
    int rc = check_rows(x, x_stride, H);
    if (rc == EAD_OK) rc = check_rows(out, out_stride, H);
    if (rc == EAD_OK && residual) rc = check_rows(residual, residual_stride, H);
    if (rc == EAD_OK && residual_out) rc = check_rows(residual_out, residual_out_stride, H);
    DeviceInfo *d = nullptr;
    if (rc == EAD_OK) rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    NormParams p{};
    p.x = static_cast<const uint8_t *>(x);
    p.residual = static_cast<const uint8_t *>(residual);
    p.weight = static_cast<const uint8_t *>(weight);
    p.residual_out = static_cast<uint8_t *>(residual_out);
    p.out = static_cast<uint8_t *>(out);
    p.out_scale = out_scale;
    p.x_stride = x_stride;
    p.residual_stride = residual_stride;
    p.residual_out_stride = residual_out_stride;
    p.out_stride = out_stride;
    p.H = H;
    p.eps = eps;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int groups = H / 8;
    const int nv = groups <= 512 ? 1 : groups <= 1024 ? 2 : 4;
    const int threads = ((groups + nv - 1) / nv + 31) / 32 * 32;
    const int blocks = std::min(n_rows, kNormThreadsPerSm / threads * d->sms);
#define EAD_LAUNCH_NORM(NV)                                                                    \
    (e4m3 ? ead_add_rmsnorm_kernel<kFmtE4m3, NV><<<blocks, threads, 0, s>>>(p, n_rows)         \
          : ead_add_rmsnorm_kernel<kFmtBf16, NV><<<blocks, threads, 0, s>>>(p, n_rows))
    if (nv == 1)
        EAD_LAUNCH_NORM(1);
    else if (nv == 2)
        EAD_LAUNCH_NORM(2);
    else
        EAD_LAUNCH_NORM(4);
#undef EAD_LAUNCH_NORM
    return launched();
}
