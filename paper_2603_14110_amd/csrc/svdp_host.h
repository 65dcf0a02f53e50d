// Host-side helpers of the C-ABI entry points: sizes, launches, and the record of granted LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>
#include <mutex>
#include <utility>

#include "../../include/svdp.h"
#include "svdp_device.h"

namespace {

constexpr size_t ALIGN = 256;
constexpr size_t LDS_DEFAULT = 64 * 1024;     // dynamic LDS a kernel may use without asking
constexpr int MAX_DEVICES = 64;

inline size_t align_up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Enqueues a kernel.  Straight to hipLaunchKernel: the <<<>>> form goes through a push and a pop of the launch
// configuration besides (2.4 -> 2.25 us a launch of twenty arguments), and launches are what bounds small calls: a list of two
// rows 9.7 -> 8.5 us, the step of d = 256, D = 1024 12.7 -> 11.6 (10.5 to 12.5 by the host it runs on).  A refused launch is the
// last error, which hip_status() reports.
template <typename... P, typename... A>
inline void launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, A &&...args)
{
    [&](P... p) {
        void *at[] = {const_cast<void *>(static_cast<const void *>(&p))...};
        (void)hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, at, lds, st);
    }(std::forward<A>(args)...);
}

inline svdp_status hip_status(hipError_t e)
{
    if (e == hipSuccess) e = hipGetLastError();
    else (void)hipGetLastError();
    return e == hipSuccess ? SVDP_OK : SVDP_ERR_HIP;
}

// Dynamic LDS above the default limit has to be enabled per kernel and device once.  What was
// enabled is remembered per kernel (the template parameter is the kernel itself) and device;
// the driver call is made under a lock, so that the remembered size never runs ahead of it.
std::mutex g_grant_mutex;
template <auto Kernel>
bool grant_lds(size_t bytes)
{
    static std::atomic<int> granted[MAX_DEVICES];
    if (bytes <= LDS_DEFAULT) return true;
    if (bytes > svdp::LDS_MAX) return false;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) {
        (void)hipGetLastError();
        return false;
    }
    if ((int)bytes <= granted[dev].load(std::memory_order_acquire)) return true;
    std::lock_guard<std::mutex> lock(g_grant_mutex);
    if ((int)bytes <= granted[dev].load(std::memory_order_relaxed)) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                            (int)bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    granted[dev].store((int)bytes, std::memory_order_release);
    return true;
}

}  // namespace
