// Host-side helpers of the library's source files: sizes, launch attributes, the driver's encoder of tensor maps.  Each file
// that includes this has them (and what they remember) for itself.
#pragma once

#include <atomic>
#include <cstddef>
#include <cstdint>
#include <map>
#include <mutex>
#include <utility>

#include <cuda.h>
#include <cuda_runtime.h>

#include "perq.h"

// The device error word of the product kernels (perq_matmul.cu), which perq_device_error reads with the others' own.
__attribute__((visibility("hidden"))) cudaError_t perq_mm_read_error(unsigned int *flags);
__attribute__((visibility("hidden"))) cudaError_t perq_mm_clear_error();

namespace {

constexpr size_t kMaxSmem = 227 * 1024;

inline bool is_pow2(long long v) { return v > 0 && (v & (v - 1)) == 0; }
inline int ilog2(int v) { int l = 0; while ((1 << l) < v) ++l; return l; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int sm_count()
{
    static std::atomic<int> cached[64];          // per device ordinal; 0 = not asked yet
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    const bool slot = dev >= 0 && dev < 64;
    if (slot && cached[dev].load() > 0) return cached[dev].load();
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (slot) cached[dev].store(n);
    return n;
}

// Opt-in to more than 48 KB of dynamic shared memory.  The attribute belongs to (kernel, device): it is set
// the first time and whenever a launch needs more than was set before (the call costs a microsecond or two,
// which matters for the small launches).
std::mutex g_smem_attr_mutex;
std::map<std::pair<const void *, int>, size_t> g_smem_attr_set;

template <typename K>
int allow_smem(K kernel, size_t bytes)
{
    if (bytes <= 48 * 1024) return PERQ_OK;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PERQ_ERR_CUDA;
    const void *func = reinterpret_cast<const void *>(kernel);
    std::lock_guard<std::mutex> lock(g_smem_attr_mutex);
    size_t &have = g_smem_attr_set[std::make_pair(func, dev)];
    if (have >= bytes) return PERQ_OK;
    if (cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return PERQ_ERR_CUDA;
    }
    have = bytes;
    return PERQ_OK;
}

// The driver's encoder of tensor maps, asked for once (the library does not link against libcuda).
typedef CUresult (*TensorMapEncode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                    const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncode tensor_map_encode()
{
    static std::atomic<void *> cached{nullptr};
    void *fn = cached.load();
    if (fn == nullptr) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return nullptr;
        }
        cached.store(fn);
    }
    return reinterpret_cast<TensorMapEncode>(fn);
}

}  // namespace
