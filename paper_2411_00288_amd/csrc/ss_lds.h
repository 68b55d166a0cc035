// Launches of kernels with more than 64 KB of shared memory.
#ifndef SS_LDS_H_
#define SS_LDS_H_
#include "ss_internal.h"
#include <atomic>

namespace ss {

// A kernel's shared memory may pass 64 KB once its limit is raised, which is done at its first such launch on a device.
template <auto KERNEL>
int allow_lds(size_t bytes)
{
    if (bytes <= 65536) return SS_OK;
    static std::atomic<unsigned long long> done{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return SS_ERR_HIP;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev >= 64 || !(done.load(std::memory_order_acquire) & bit)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return SS_ERR_HIP;
        if (dev < 64) done.fetch_or(bit, std::memory_order_release);
    }
    return SS_OK;
}

}  // namespace ss

#endif
