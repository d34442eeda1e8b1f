// What the host sides of the decoder-side operators share: device table, checks of descriptions and rows.
#pragma once
#include "../../include/ead.h"

#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <mutex>

#include "kv_format.cuh"

namespace ead {

#define EAD_CUDA(x)                          \
    do {                                     \
        if ((x) != cudaSuccess) {            \
            cudaGetLastError();              \
            return EAD_ECUDA;                \
        }                                    \
    } while (0)

constexpr int kMaxDevices = 64;

inline std::atomic<uint32_t> g_wait_ns{static_cast<uint32_t>(kWaitLimitNs)};   // of the kernels' bounded waits
static_assert(kWaitLimitNs <= 0x7fffffffu, "held in 32 bits");

struct DeviceInfo {
    bool ready = false;
    int sms = 0;
};

// Devices that were used so far, one table per source file: on a device's first use its architecture is checked and
// the file's kernels get their attributes (`prepare`).
class DeviceTable {
public:
    // Makes `device` current.
    template <typename F>
    int use(int device, DeviceInfo **out, F prepare)
    {
        if (device < 0 || device >= kMaxDevices) return EAD_EINVALID_ARG;
        std::lock_guard<std::mutex> lock(mu_);
        DeviceInfo &d = dev_[device];
        if (!d.ready) {
            int n = 0, major = 0;
            EAD_CUDA(cudaGetDeviceCount(&n));
            if (device >= n) return EAD_EINVALID_ARG;
            EAD_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device));
            if (major != 10) return EAD_EUNSUPPORTED_ARCH;
            EAD_CUDA(cudaSetDevice(device));
            EAD_CUDA(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, device));
            if (!prepare()) {
                cudaGetLastError();
                return EAD_ECUDA;
            }
            d.ready = true;
        }
        EAD_CUDA(cudaSetDevice(device));
        *out = &d;
        return EAD_OK;
    }

private:
    std::mutex mu_;
    DeviceInfo dev_[kMaxDevices];
};

inline int launched() { return cudaGetLastError() == cudaSuccess ? EAD_OK : EAD_ECUDA; }

inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline int check_cache(const ead_kv_cache *c, KvCacheView *v)
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

inline int check_batch(const ead_kv_batch *b, const KvCacheView &c, bool needs_len, KvBatchView *v)
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
inline int check_rows(const void *p, int64_t stride, int64_t elements)
{
    if (!p || stride < elements) return EAD_EINVALID_ARG;
    if (!aligned(p, 16) || stride % 8) return EAD_EALIGNMENT;
    return EAD_OK;
}

}  // namespace ead
