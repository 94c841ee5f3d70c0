// Reductions of floats over a wavefront and over a few wavefronts' results, and a lane's rank in a mask.
#pragma once

#include <type_traits>

#include "group.h"

namespace ngpu {

// Bits of a wavefront's mask that belong to the lanes before this one.
__device__ __forceinline__ int lanes_below(unsigned long long mask) {
    return int(__builtin_amdgcn_mbcnt_hi(unsigned(mask >> 32), __builtin_amdgcn_mbcnt_lo(unsigned(mask), 0u)));
}

// The inverse of float_key.
__device__ __forceinline__ float key_float(unsigned k) {
    return __int_as_float(int(k ^ (~unsigned(int(k) >> 31) | 0x80000000u)));
}

// Sum over W values that repeat every W lanes: pairs, then pairs of pairs, so
// every lane adds the same numbers in the same order.
template <int W>
__device__ __forceinline__ float sum_over_waves(float x) {
    auto moved = [](float v, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if (W >= 2) x += moved(x, std::integral_constant<int, 0xB1>{});    // lane ^ 1
    if (W >= 4) x += moved(x, std::integral_constant<int, 0x4E>{});    // lane ^ 2
    if (W >= 8) x += moved(x, std::integral_constant<int, 0x141>{});   // other half of 8
    if (W >= 16) x += moved(x, std::integral_constant<int, 0x140>{});  // other half of 16
    return x;
}

// Sum over the wavefront, in a fixed order, uniform in every lane.
__device__ __forceinline__ float wave_sum(float x) {
    x = sum_over_waves<16>(x);   // of each row of 16 lanes
    float r = 0.0f;
#pragma unroll
    for (int i = 0; i < kWave; i += 16) r += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i));
    return r;
}

// Maximum over the wavefront, uniform; no lane may hold NaN.
__device__ __forceinline__ float wave_max(float x) { return key_float(wave_max_u32(float_key(x))); }

}  // namespace ngpu
