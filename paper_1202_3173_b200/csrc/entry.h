// What the host entry points of the language-model operators share: status and message, ranges of memory, the device.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <string>

#include "kernels.h"
#include "strassen_b200.h"

namespace strassen {
namespace entry {

inline int fail(int status, const std::string &msg)
{
    set_last_error(msg.c_str());
    return status;
}

inline int cuda_fail(cudaError_t e, const char *what) { return fail(STRASSEN_CUDA_ERROR, std::string(what) + ": " + cudaGetErrorString(e)); }

constexpr int64_t kMaxExtent = int64_t(1) << 30;          // of one dimension; products of two fit 64-bit byte offsets
constexpr int64_t kMaxLd = int64_t(1) << 40;

inline int type_size(int type)
{
    switch (type) {
    case STRASSEN_BF16:
    case STRASSEN_F16: return 2;
    case STRASSEN_F32: return 4;
    case STRASSEN_E4M3: return 1;
    }
    return 0;
}

// Rows of a strided matrix as a byte range.
struct Range {
    uintptr_t lo, hi;
};
inline Range rows_of(const void *p, int64_t m, int64_t k, int64_t ld, int size)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return {lo, lo + (m > 0 && p ? uintptr_t((m - 1) * ld + k) * uintptr_t(size) : 0)};
}
inline bool overlap(const Range &a, const Range &b) { return a.lo < b.hi && b.lo < a.hi; }
inline bool misaligned(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(size) != 0; }
inline bool same_rows(const void *p, int64_t ldp, const void *q, int64_t ldq, int64_t m) { return p == q && (m <= 1 || ldp == ldq); }

constexpr int kMaxDevices = 64;
inline std::atomic<int> g_sms[kMaxDevices];       // SM count of a device that was found to be an sm_100 part; 0: not looked at yet

inline int current_device(int *sms)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail(STRASSEN_INVALID_ARG, "device ordinal out of range");
    *sms = g_sms[dev].load(std::memory_order_acquire);
    if (*sms > 0) return STRASSEN_OK;
    int major = 0;
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
    if (major != 10)
        return fail(STRASSEN_CUDA_ERROR, "this library holds sm_100a code only; the current device is not a B200-class GPU");
    g_sms[dev].store(*sms, std::memory_order_release);
    return STRASSEN_OK;
}

}  // namespace entry
}  // namespace strassen
