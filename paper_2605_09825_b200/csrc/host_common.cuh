// Host-side helpers every translation unit of the library shares: device properties, one-time
// set-up per device, argument checks.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"

namespace mxfp4 {

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int kMaxDevices = 64;      // size of the per-device tables below

struct DeviceInfo {
    int sm_count = 0;
    int cc_major = 0;
    bool ok = false;
};

// Per-device set-up that runs once however many host threads reach it at the same time: the
// first caller on a device runs `f` (which returns a status code), the others wait for it, and
// everybody gets that status.  One instance per table (device properties, a kernel's
// shared-memory attribute, the copy streams of the host-buffer call, ...).
struct PerDeviceOnce {
    std::once_flag flag[kMaxDevices];
    int status[kMaxDevices] = {};
    template <class F>
    int run(int dev, F&& f)
    {
        std::call_once(flag[dev], [&] { status[dev] = f(); });
        return status[dev];
    }
};

// Ordinal of the current device, or -1 if it cannot be had or lies beyond the tables.
static inline int current_device()
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return -1;
    return dev;
}

// Whether this translation unit has been called on a device.  Every entry point asks for device_info() before it
// launches anything, which sets it; until then the unit's status word cannot be set either.
static inline std::atomic<bool>& unit_used(int dev)
{
    static std::atomic<bool> used[kMaxDevices];
    return used[dev];
}

static inline const DeviceInfo& device_info()
{
    static DeviceInfo info[kMaxDevices];
    static PerDeviceOnce once;
    static const DeviceInfo none;
    const int dev = current_device();
    if (dev < 0) return none;
    once.run(dev, [&] {
        unit_used(dev) = true;
        cudaDeviceProp prop;
        if (cudaGetDeviceProperties(&prop, dev) == cudaSuccess) {
            info[dev].sm_count = prop.multiProcessorCount;
            info[dev].cc_major = prop.major;
            info[dev].ok = true;
        }
        return 0;
    });
    return info[dev];
}

// Raises a kernel's dynamic shared-memory limit on the current device, once per device.
template <class Kernel>
static int ensure_smem_attribute(PerDeviceOnce& once, Kernel kernel, size_t smem)
{
    const int dev = current_device();
    if (dev < 0) return MXFP4_ERR_CUDA;
    return once.run(dev, [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) ==
                       cudaSuccess
                   ? MXFP4_OK : MXFP4_ERR_CUDA;
    });
}

static inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Current device usable by the library's kernels?  MXFP4_OK, MXFP4_ERR_CUDA or MXFP4_ERR_DEVICE.
static inline int device_status_code(const DeviceInfo& dev)
{
    if (!dev.ok) return MXFP4_ERR_CUDA;
    return dev.cc_major == 10 ? MXFP4_OK : MXFP4_ERR_DEVICE;
}

// The status of this translation unit's kernels, cleared if it was set; 0 without a look at the device where the
// unit has not been called (a look costs a copy of its own, 11 us).
static inline int take_unit_status(int* status)
{
    const int dev = current_device();
    *status = 0;
    return dev >= 0 && !unit_used(dev) ? 0 : take_device_status(status);
}

// The same of the other translation units (each has its own status word).
int block128_take_status(int* status);
int residual_norm_take_status(int* status);
int logprobs_take_status(int* status);

}  // namespace mxfp4
