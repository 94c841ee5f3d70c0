// What launches of several kernels share.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

namespace ngpu {

// More LDS than the 64 KB of a launch by default, asked for once a device (bits of `devices`), as HIP's documentation has it.
// (The runtime of ROCm 7 launches without being asked: step, decode and top-k rely on that with 65 KB.)
template <class K>
hipError_t allow_lds(K *kernel, int bytes, std::atomic<uint64_t> &devices) {
    int device;
    if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
    const uint64_t bit = uint64_t(1) << device % 64;
    if (device < 64 && (devices.load(std::memory_order_relaxed) & bit)) return hipSuccess;
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && device < 64) devices.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

}  // namespace ngpu
