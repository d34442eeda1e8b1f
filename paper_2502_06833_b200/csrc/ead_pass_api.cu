// Host side of the operators of a decoder's 8-bit pass declared in include/ead.h: product with block scales, quantisation,
// norm and rotation of query and key heads, log probabilities of given tokens.  Stateless: arguments are checked, kernels are enqueued.
#include "../../include/ead.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "decoder_host.h"
#include "linear_kernel.cuh"
#include "logprob_kernel.cuh"
#include "quantise_kernel.cuh"
#include "rope_kernel.cuh"
#include "tma_host.h"

using namespace ead;

namespace {

// Most tokens of a product that single blocks serve.  Measured, 7168 x 5120, us, single blocks against pairs: 128 tokens 12.8 / 13.4, 160 tokens 14.2 / 14.0,
// 200 tokens 17.2 / 14.2; 2048 x 5120: 160 tokens 10.5 / 11.5, 200 tokens 12.0 / 11.5; 14336 x 5120: 18.0 / 19.4, 21.7 / 20.3.
constexpr int kLinFewTokens = 160;
// What a pair's tile costs beside its tokens, in tokens.  Measured, us per round of tiles, 4099 x 7168 x 5120: 8.1 for 64 tokens, 9.5 for 96, 10.6 for 128, 11.8
// for 160, 13.1 for 192, 14.3 for 208, 15.7 for 240; 1024 x 7168 x 5120: 7.2, 8.4, 9.1, 11.5, 12.0, 15.3, 16.5.
constexpr int kLinPairFixed = 100;
// What the join of a tile's parts costs, in stages of 128 values along K.
constexpr double kLinJoinStages = 4;
// Blocks of a call that scores few rows, per SM, and the least 16-byte vectors of a part: a run of a block (one row of 128256 in 32 bits: parts of 256
// vectors 9.3 us, of 512 10.0, of 1024 8.8, of 2048 9.5).
constexpr int kScoreBlocksPerSm = 2;
constexpr int kScoreMinVectors = kScoreUnroll * kScoreThreads;

// Passes of 512 values of a warp that quantises (quantise_kernel.cuh has the figures), and the warps per SM below which it has fewer.
constexpr int kQuantMinPasses = 14;
constexpr int kQuantWarpsPerSm = 64;
// Warps per SM that a call with few tokens is divided into, for the rotation.  (16, 32 and 64 differ by less than 0.2 us for 64 tokens; 4001 tokens of 2560
// elements, at that time: 12.1, 12.5, 13.8.)
constexpr int kRopeWarpsPerSm = 32;

DeviceTable g_devices;
int g_clusters[kMaxDevices][kLinMaxSplit + 1];    // clusters of ead_linear's blocks that a device holds at a time, by their size

template <int BLOCK, bool F32, bool PAIR>
bool prepare_linear()
{
    return cudaFuncSetAttribute(ead_linear_kernel<BLOCK, F32, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinSmem) == cudaSuccess;
}

cudaLaunchConfig_t linear_config(int blocks, int threads, int cluster, int smem, cudaStream_t s, cudaLaunchAttribute *attr)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cfg;
}

int use_device(int device, DeviceInfo **out)
{
    return g_devices.use(device, out, [device] {
        if (!prepare_linear<32, false, false>() || !prepare_linear<32, true, false>() || !prepare_linear<128, false, false>() ||
            !prepare_linear<128, true, false>() || !prepare_linear<32, false, true>() || !prepare_linear<32, true, true>() ||
            !prepare_linear<128, false, true>() || !prepare_linear<128, true, true>())
            return false;
        for (int c = 1; c <= kLinMaxSplit; ++c) {
            cudaLaunchAttribute attr[2];
            const cudaLaunchConfig_t cfg = linear_config(c, LinLayout<128, false>::kThreads, c, kLinSmem, nullptr, attr);
            if (cudaOccupancyMaxActiveClusters(&g_clusters[device][c], ead_linear_kernel<128, false, false>, &cfg) != cudaSuccess) return false;
        }
        return true;
    });
}

// How a product is divided (what the comments of linear_kernel.cuh describe).
struct LinearPlan {
    bool pair;
    int tile_tokens, token_tiles, split, whole, rest, blocks;
};

LinearPlan plan_linear(int T, int N, int kblocks, int block, const int *clusters)
{
    const int most = block == 128 ? LinLayout<128, true>::kMaxTokens : LinLayout<32, true>::kMaxTokens;
    const int64_t features = (N + int64_t{kLinM} - 1) / kLinM;
    LinearPlan best{};
    if (T <= kLinFewTokens) {
        best.tile_tokens = (T + 15) / 16 * 16;
        best.token_tiles = 1;
        double cost = 1e300;
        for (int c = 1; c <= std::min(kLinMaxSplit, kblocks); ++c) {
            const int64_t held = clusters[c], blocks = held * c;
            if (held < 1) continue;
            int64_t whole = features / blocks * blocks, rest = features - whole;
            if (c == 1 || rest > held) {
                whole = features;
                rest = 0;
            }
            const double t = static_cast<double>((whole + blocks - 1) / blocks) * kblocks + (rest ? (kblocks + c - 1) / c + kLinJoinStages : 0);
            if (t < cost) {
                cost = t;
                best.split = c;
                best.whole = static_cast<int>(whole);
                best.rest = static_cast<int>(rest);
                best.blocks = static_cast<int>(whole ? std::min(blocks, (whole + c - 1) / c * c) : rest * c);
            }
        }
        return best;
    }
    if (clusters[2] < 1) return best;             // no pair fits (a device of which only a part is there): refused
    const int64_t pairs = clusters[2], feature_pairs = (features + 1) / 2, least = (T + int64_t{most} - 1) / most;
    int64_t cost = INT64_MAX;
    for (int64_t n = least; n <= least + pairs; ++n) {
        const int tile = static_cast<int>((T + n - 1) / n + 15) / 16 * 16;
        const int64_t tiles = feature_pairs * ((T + int64_t{tile} - 1) / tile), rounds = (tiles + pairs - 1) / pairs;
        const int64_t t = rounds * (tile + kLinPairFixed);
        if (t < cost) {
            cost = t;
            best = LinearPlan{true, tile, static_cast<int>((T + int64_t{tile} - 1) / tile), 2, static_cast<int>(tiles), 0, static_cast<int>(2 * std::min(pairs, tiles))};
        }
        if (tile == 16) break;
    }
    return best;
}

// 8-bit rows as boxes of 128 bytes x `rows`, with the 128-byte swizzle.
bool encode_codes(CUtensorMap *tm, const ead_e4m3_matrix &m, int rows)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(m.cols), static_cast<cuuint64_t>(m.rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(m.row_stride)};
    const cuuint32_t box[2] = {kLinK, static_cast<cuuint32_t>(rows)}, ones[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.codes, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int check_matrix(const ead_e4m3_matrix *m, int block_rows)
{
    if (!m || m->reserved || m->rows < 0 || m->cols < kFmtBlock || m->cols > (1 << 30) || m->rows > (1 << 30)) return EAD_EINVALID_ARG;
    if (m->block_rows != block_rows) return EAD_EINVALID_ARG;
    if (m->block_cols != 128 && (m->block_cols != kFmtBlock || block_rows != 1)) return EAD_EINVALID_ARG;
    if (m->rows == 0) return EAD_OK;              // nothing there: it may have no address
    if (!m->codes || !m->scale || m->row_stride < m->cols || m->row_stride > (int64_t{1} << 39)) return EAD_EINVALID_ARG;
    if (m->cols % kFmtBlock || !aligned(m->codes, 16) || m->row_stride % 16) return EAD_EALIGNMENT;
    if (m->block_cols == kFmtBlock && !aligned(m->scale, 4)) return EAD_EALIGNMENT;
    return EAD_OK;
}

int check_rope(const ead_rope *r, RopeParams *p)
{
    if (!r || r->reserved || (r->head_dim != 64 && r->head_dim != 128) || r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 16)
        return EAD_EINVALID_ARG;
    if ((r->interleaved != 0 && r->interleaved != 1) || !std::isfinite(r->eps) || r->eps < 0.f) return EAD_EINVALID_ARG;
    if (r->rot_dim && !r->inv_freq) return EAD_EINVALID_ARG;
    if (!aligned(r->inv_freq, 4) || !aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return EAD_EALIGNMENT;
    p->inv_freq = r->inv_freq;
    p->q_weight = static_cast<const uint8_t *>(r->q_weight);
    p->k_weight = static_cast<const uint8_t *>(r->k_weight);
    p->dim = r->head_dim;
    p->rot = r->rot_dim;
    p->interleaved = r->interleaved;
    p->eps = r->eps;
    return EAD_OK;
}

// A kernel whose setup runs under the end of the one before it in the stream.
template <typename Params>
int launch_early(void (*kernel)(Params), dim3 grid, int threads, const Params &p, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
        cudaGetLastError();
        return EAD_ECUDA;
    }
    return EAD_OK;
}

template <int FMT, bool DENSE>
int launch_rotate(RopeParams &p, int n_tokens, int sms, cudaStream_t s)
{
    const bool halves = p.rot == p.dim && !p.interleaved;
    const int run = halves ? 2 * kRopeRun : kRopeRun;
    const int64_t values = (static_cast<int64_t>(p.heads_q) + (DENSE ? 1 : 2) * p.heads_kv) * p.dim;
    const int runs = static_cast<int>((values + run - 1) / run);
    p.n_tokens = n_tokens;
    p.split = static_cast<int>(std::min<int64_t>(runs, std::max<int64_t>(1, int64_t{kRopeWarpsPerSm} * sms / n_tokens)));
    const int64_t blocks = (static_cast<int64_t>(n_tokens) * p.split + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    return halves ? launch_early(ead_rotate_halves_kernel<FMT, DENSE>, static_cast<unsigned>(blocks), kRopeThreads, p, s)
                  : launch_early(ead_rotate_kernel<FMT, DENSE>, static_cast<unsigned>(blocks), kRopeThreads, p, s);
}

template <int BLOCK, bool F32, bool PAIR>
int launch_linear(const CUtensorMap &tw, const CUtensorMap &tx, LinearParams p, int blocks, cudaStream_t s)
{
    using L = LinLayout<BLOCK, PAIR>;
    const int stage = L::stage_bytes(p.tile_tokens);
    p.stages = std::min(kLinMaxStages, (kLinSmem - L::fixed_bytes()) / stage);
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = linear_config(blocks, L::kThreads, p.split, L::fixed_bytes() + p.stages * stage, s, attr);
    if (cudaLaunchKernelEx(&cfg, ead_linear_kernel<BLOCK, F32, PAIR>, tw, tx, p) != cudaSuccess) {
        cudaGetLastError();
        return EAD_ECUDA;
    }
    return EAD_OK;
}

template <int BLOCK, bool F32>
int launch_linear(const CUtensorMap &tw, const CUtensorMap &tx, const LinearParams &p, const LinearPlan &plan, cudaStream_t s)
{
    return plan.pair ? launch_linear<BLOCK, F32, true>(tw, tx, p, plan.blocks, s) : launch_linear<BLOCK, F32, false>(tw, tx, p, plan.blocks, s);
}

}  // namespace

extern "C" int ead_linear(const ead_e4m3_matrix *x, const ead_e4m3_matrix *w, const void *bias, int32_t format, void *out, int64_t out_stride,
                          uint32_t *status, int32_t device, void *stream)
{
    int rc = check_matrix(x, 1);
    if (rc == EAD_OK) rc = check_matrix(w, 128);
    if (rc != EAD_OK) return rc;
    const bool f32 = format == EAD_FMT_F32;
    if ((format != EAD_FMT_BF16 && !f32) || x->cols != w->cols) return EAD_EINVALID_ARG;
    if (x->rows == 0 || w->rows == 0) return EAD_OK;
    if (!out || out_stride < w->rows) return EAD_EINVALID_ARG;
    if (!aligned(out, f32 ? 4 : 2) || !aligned(bias, 2) || !aligned(status, 4)) return EAD_EALIGNMENT;
    LinearParams p{};
    p.x_scale = x->scale;
    p.w_scale = w->scale;
    p.bias = static_cast<const uint8_t *>(bias);
    p.out = static_cast<uint8_t *>(out);
    p.out_stride = out_stride;
    p.T = x->rows;
    p.N = w->rows;
    p.kblocks = (x->cols + kLinK - 1) / kLinK;
    p.x_scale_cols = (x->cols + x->block_cols - 1) / x->block_cols;
    p.w_scale_cols = p.kblocks;
    // every tile has an index of 32 bits, whatever the plan
    if ((p.N / kLinM + int64_t{1}) * (p.T / 16 + int64_t{1}) > (1 << 30)) return EAD_ELIMIT;
    DeviceInfo *d = nullptr;
    rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    const LinearPlan plan = plan_linear(p.T, p.N, p.kblocks, x->block_cols, g_clusters[device]);
    if (!plan.blocks) return EAD_ECUDA;
    p.tile_tokens = plan.tile_tokens;
    p.token_tiles = plan.token_tiles;
    p.whole = plan.whole;
    p.rest = plan.rest;
    p.split = plan.split;
    p.wide = aligned(out, 16) && out_stride % (f32 ? 4 : 8) == 0;
    p.status = status;
    p.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    p.wait_hint = std::min(p.wait_ns, 20000u);
    CUtensorMap tw, tx;
    if (!encode_codes(&tw, *w, kLinM) || !encode_codes(&tx, *x, plan.pair ? p.tile_tokens / 2 : p.tile_tokens)) return EAD_ECUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return x->block_cols == 128 ? (f32 ? launch_linear<128, true>(tw, tx, p, plan, s) : launch_linear<128, false>(tw, tx, p, plan, s))
                                : (f32 ? launch_linear<32, true>(tw, tx, p, plan, s) : launch_linear<32, false>(tw, tx, p, plan, s));
}

extern "C" int ead_quantise(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, const ead_e4m3_matrix *out, int32_t device,
                            void *stream)
{
    if (!out) return EAD_EINVALID_ARG;
    const bool tiles = out->block_rows == 128;
    int rc = check_matrix(out, tiles ? 128 : 1);
    if (rc != EAD_OK) return rc;
    if (tiles && gate) return EAD_EINVALID_ARG;
    if (out->rows == 0) return EAD_OK;
    rc = check_rows(x, x_stride, out->cols);
    if (rc == EAD_OK && gate) rc = check_rows(gate, gate_stride, out->cols);
    DeviceInfo *d = nullptr;
    if (rc == EAD_OK) rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    QuantParams p{};
    p.x = static_cast<const uint8_t *>(x);
    p.gate = static_cast<const uint8_t *>(gate);
    p.out = static_cast<uint8_t *>(out->codes);
    p.out_scale = out->scale;
    p.x_stride = x_stride;
    p.gate_stride = gate_stride;
    p.out_stride = out->row_stride;
    p.rows = out->rows;
    p.cols = out->cols;
    p.scale_cols = (p.cols + out->block_cols - 1) / out->block_cols;
    p.passes = (p.cols + kQuantPass - 1) / kQuantPass;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t most = static_cast<int64_t>(kQuantWarpsPerSm) * d->sms;          // with few rows a warp has one pass, with many kQuantMinPasses
    const int passes = static_cast<int>(std::min<int64_t>(kQuantMinPasses, std::max<int64_t>(1, static_cast<int64_t>(p.rows) * p.passes / most)));
    p.split = (p.passes + passes - 1) / passes;
    const int64_t blocks = tiles ? static_cast<int64_t>((p.rows + int64_t{127}) / 128) * p.scale_cols
                                 : (static_cast<int64_t>(p.rows) * p.split + kQuantThreads / 32 - 1) / (kQuantThreads / 32);
    if (blocks > 0x1fffffff) return EAD_ELIMIT;   // warps are counted in 32 bits
    const unsigned grid = static_cast<unsigned>(blocks);
    if (tiles) return launch_early(ead_quantise_tiles_kernel, grid, kQuantThreads, p, s);
    if (out->block_cols == 128)
        return gate ? launch_early(ead_quantise_rows_kernel<128, true>, grid, kQuantThreads, p, s) : launch_early(ead_quantise_rows_kernel<128, false>, grid, kQuantThreads, p, s);
    return gate ? launch_early(ead_quantise_rows_kernel<32, true>, grid, kQuantThreads, p, s) : launch_early(ead_quantise_rows_kernel<32, false>, grid, kQuantThreads, p, s);
}

extern "C" int ead_qk_norm_rope(const ead_rope *rope, const int32_t *positions, int32_t n_tokens, const void *q, int64_t q_stride, int32_t heads_q,
                                const void *k, int64_t k_stride, int32_t heads_kv, void *q_out, int64_t q_out_stride, void *k_out,
                                int64_t k_out_stride, int32_t device, void *stream)
{
    RopeParams p{};
    int rc = check_rope(rope, &p);
    if (rc != EAD_OK) return rc;
    if (n_tokens < 0 || n_tokens > (1 << 30) || heads_q < 0 || heads_q > 16384 || heads_kv < 0 || heads_kv > 128) return EAD_EINVALID_ARG;
    if (n_tokens == 0 || heads_q + heads_kv == 0) return EAD_OK;
    if (!positions) return EAD_EINVALID_ARG;
    if (heads_q) rc = check_rows(q, q_stride, static_cast<int64_t>(heads_q) * p.dim);
    if (rc == EAD_OK && heads_q) rc = check_rows(q_out, q_out_stride, static_cast<int64_t>(heads_q) * p.dim);
    if (rc == EAD_OK && heads_kv) rc = check_rows(k, k_stride, static_cast<int64_t>(heads_kv) * p.dim);
    if (rc == EAD_OK && heads_kv) rc = check_rows(k_out, k_out_stride, static_cast<int64_t>(heads_kv) * p.dim);
    if (rc == EAD_OK && !aligned(positions, 4)) rc = EAD_EALIGNMENT;
    DeviceInfo *d = nullptr;
    if (rc == EAD_OK) rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    p.positions = positions;
    p.q = static_cast<const uint8_t *>(q);
    p.k = static_cast<const uint8_t *>(k);
    p.q_out = static_cast<uint8_t *>(q_out);
    p.k_out = static_cast<uint8_t *>(k_out);
    p.q_stride = q_stride;
    p.kv_stride = k_stride;
    p.q_out_stride = q_out_stride;
    p.k_out_stride = k_out_stride;
    p.heads_q = heads_q;
    p.heads_kv = heads_kv;
    return launch_rotate<kFmtBf16, true>(p, n_tokens, d->sms, static_cast<cudaStream_t>(stream));
}

extern "C" int ead_kv_rotate_write(const ead_rope *rope, const ead_kv_cache *cache, const ead_kv_batch *batch, const int32_t *positions,
                                   const void *q, int64_t q_stride, int32_t heads_q, const void *k, const void *v, int64_t kv_stride, void *q_out,
                                   int64_t q_out_stride, uint32_t *status, int32_t device, void *stream)
{
    RopeParams p{};
    int rc = check_rope(rope, &p);
    if (rc == EAD_OK) rc = check_cache(cache, &p.cache);
    if (rc == EAD_OK) rc = check_batch(batch, p.cache, true, &p.batch);
    if (rc != EAD_OK) return rc;
    if (rope->head_dim != cache->head_dim || heads_q < 0 || heads_q > 16384) return EAD_EINVALID_ARG;
    if (p.batch.n_tokens == 0) return EAD_OK;
    const int64_t q_row = static_cast<int64_t>(heads_q) * p.dim, kv_row = static_cast<int64_t>(p.cache.heads) * p.dim;
    if (heads_q) rc = check_rows(q, q_stride, q_row);
    if (rc == EAD_OK && heads_q) rc = check_rows(q_out, q_out_stride, q_row);
    if (rc == EAD_OK) rc = check_rows(k, kv_stride, kv_row);
    if (rc == EAD_OK) rc = check_rows(v, kv_stride, kv_row);
    if (rc == EAD_OK && (!aligned(positions, 4) || !aligned(status, 4))) rc = EAD_EALIGNMENT;
    DeviceInfo *d = nullptr;
    if (rc == EAD_OK) rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    p.positions = positions;
    p.q = static_cast<const uint8_t *>(q);
    p.k = static_cast<const uint8_t *>(k);
    p.v = static_cast<const uint8_t *>(v);
    p.q_out = static_cast<uint8_t *>(q_out);
    p.q_stride = q_stride;
    p.kv_stride = kv_stride;
    p.q_out_stride = q_out_stride;
    p.heads_q = heads_q;
    p.heads_kv = p.cache.heads;
    p.status = status;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cache->format == EAD_FMT_BF16 ? launch_rotate<kFmtBf16, false>(p, p.batch.n_tokens, d->sms, s)
                                         : launch_rotate<kFmtE4m3, false>(p, p.batch.n_tokens, d->sms, s);
}

extern "C" int ead_token_logprobs(const void *logits, int32_t format, int64_t stride, int32_t n_rows, int32_t V, const int32_t *tokens,
                                  float *logprob, float *entropy, int32_t *rank, int32_t k, int32_t *top, float *top_logprob, void *workspace,
                                  uint32_t *status, int32_t device, void *stream)
{
    if ((format != EAD_FMT_BF16 && format != EAD_FMT_F16 && format != EAD_FMT_F32) || n_rows < 0 || V < 1 || V > (1 << 30) || k < 0 || !workspace)
        return EAD_EINVALID_ARG;
    if (k > kScoreMaxTop) return EAD_ELIMIT;
    if (!tokens && (logprob || rank)) return EAD_EINVALID_ARG;
    if (n_rows == 0) return EAD_OK;
    if (!logits || stride < V) return EAD_EINVALID_ARG;
    if (!aligned(logits, format == EAD_FMT_F32 ? 4 : 2) || !aligned(workspace, 256) || !aligned(tokens, 4) || !aligned(logprob, 4) ||
        !aligned(entropy, 4) || !aligned(rank, 4) || !aligned(top, 4) || !aligned(top_logprob, 4) || !aligned(status, 4))
        return EAD_EALIGNMENT;
    DeviceInfo *d = nullptr;
    const int rc = use_device(device, &d);
    if (rc != EAD_OK) return rc;
    ScoreParams p{};
    p.logits = static_cast<const uint8_t *>(logits);
    p.stride = stride;
    p.tokens = tokens;
    p.logprob = logprob;
    p.entropy = entropy;
    p.rank = rank;
    p.k = top || top_logprob ? k : 0;
    p.top = top;
    p.top_logprob = top_logprob;
    p.n_rows = n_rows;
    p.V = V;
    p.workspace = static_cast<uint8_t *>(workspace);
    p.status = status;
    const int per = format == EAD_FMT_F32 ? 4 : 8, blocks = kScoreBlocksPerSm * d->sms;
    const int64_t vectors = (static_cast<int64_t>(V) + per - 1) / per;
    int64_t parts = std::min<int64_t>(blocks / n_rows, (vectors + kScoreMinVectors - 1) / kScoreMinVectors);
    parts = std::min<int64_t>(parts, kScoreMaxParts);
    if (p.k) parts = std::min<int64_t>(parts, kScoreMaxJoin / p.k);
    p.parts = static_cast<int>(std::max<int64_t>(parts, 1));
    const dim3 grid(p.parts, std::min(n_rows, 65535));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return format == EAD_FMT_BF16 ? launch_early(ead_token_logprobs_kernel<kFmtBf16>, grid, kScoreThreads, p, s)
           : format == EAD_FMT_F16 ? launch_early(ead_token_logprobs_kernel<kFmtF16>, grid, kScoreThreads, p, s)
                                   : launch_early(ead_token_logprobs_kernel<kFmtF32>, grid, kScoreThreads, p, s);
}
