// What the host sides of the serving operators share: set-up once per device, checks of pointers and strides, launches.
#pragma once
#include <atomic>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>
#include <mutex>

#include "../../include/mmv.h"
#include "host_state.h"

namespace mmv {

constexpr int kMaxDevices = 64;
constexpr int kMaxHeads = 1024;
constexpr int kPagedMaxSms = 160;

struct ServeDevice {
    std::mutex lock;
    std::atomic<bool> ok{false};
    int sm_count = 0;
};

// The current device, after `setup` has succeeded on it once (only success is remembered); null if it fails.
template <typename F>
ServeDevice* device_once(ServeDevice (&all)[kMaxDevices], F setup) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    ServeDevice* d = &all[dev];
    if (d->ok.load(std::memory_order_acquire)) return d;
    std::lock_guard<std::mutex> guard(d->lock);
    if (d->ok.load(std::memory_order_relaxed)) return d;
    int sm = 0;
    if (cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return nullptr;
    d->sm_count = sm;
    if (!setup()) {
        cudaGetLastError();
        return nullptr;
    }
    d->ok.store(true, std::memory_order_release);
    return d;
}

template <typename K>
bool allow_smem(K kernel, int bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// a stride of an axis that holds more than one entry keeps its rows on 16-byte words (`per` values each)
inline bool word_stride(int64_t stride, int64_t extent, int per = 8) { return extent <= 1 || stride % per == 0; }
inline bool overlap(const void* a, size_t abytes, const void* b, size_t bbytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return abytes && bbytes && x < y + bbytes && y < x + abytes;
}
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// `after`: the kernel may start while the one in front of it in the stream still runs (it waits before it reads).
template <typename... KP, typename... A>
mmv_status launch(void (*kernel)(KP...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool after, const A&... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 1 : 0;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, args...);
    ++g_launches;
    if (err == cudaSuccess) return MMV_OK;
    cudaGetLastError();
    return MMV_ERR_CUDA;
}

// [token][head][column] as boxes of 64 columns of one head of 64 tokens, 128-byte swizzle; what lies outside reads as zero.
inline bool token_map(CUtensorMap* map, const void* x, int dim, int heads, int64_t ntok, int64_t stride_head, int64_t stride_token) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    if (ntok == 0) {                                                  // never read
        *map = CUtensorMap{};
        return true;
    }
    const cuuint64_t row = static_cast<cuuint64_t>(dim) * 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(ntok)};
    const cuuint64_t strides[2] = {heads > 1 ? static_cast<cuuint64_t>(stride_head) * 2 : row,
                                   ntok > 1 ? static_cast<cuuint64_t>(stride_token) * 2 : row * static_cast<cuuint64_t>(heads)};
    const cuuint32_t box[3] = {64, 1, 64}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline bool value_type(int dt) { return dt == MMV_F16_TO_F32 || dt == MMV_BF16_TO_F32; }

// Query heads of one key head in parts of up to `most`, of nearly equal size.
struct PagedHeads {
    int group, parts, rows;
};
inline PagedHeads paged_heads(int heads, int kv_heads, int most) {
    PagedHeads h;
    h.group = heads / kv_heads;
    h.parts = (h.group + most - 1) / most;
    h.rows = (h.group + h.parts - 1) / h.parts;
    return h;
}
inline int paged_padded(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

}  // namespace mmv
