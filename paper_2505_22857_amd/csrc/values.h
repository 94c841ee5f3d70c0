// Values of the serving kernels: half-width types and order keys.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

namespace ngpu {

// The bits of a bfloat16 or half value, so that loads and stores of both are
// plain 16-bit ones.
struct Bf16 {
    uint16_t bits;
};
struct F16 {
    uint16_t bits;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float(unsigned(x.bits) << 16); }
__device__ __forceinline__ float to_float(F16 x) {
    return float(__builtin_bit_cast(_Float16, x.bits));
}
template <class T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ Bf16 from_float<Bf16>(float x) {   // to nearest, ties to even; NaN stays NaN
    return {__builtin_bit_cast(uint16_t, __bf16(x))};
}
template <>
__device__ __forceinline__ F16 from_float<F16>(float x) {
    return {__builtin_bit_cast(uint16_t, _Float16(x))};
}

}  // namespace ngpu
