// Values in 8 bits: e4m3 (largest 448, NaN 0x7f, no infinities) and their scales.
#pragma once

#include "values.h"

namespace ngpu {

struct E4m3 {
    uint8_t bits;
};

constexpr float kMost8 = 448.0f;          // the largest value
constexpr int kLeastScale = -100;         // exponent of the least scale that is chosen

// The four values in a word's bytes, and two of them, lower or upper.
template <bool UPPER>
__device__ __forceinline__ float2 to_floats8(int word) {
    const auto x = __builtin_amdgcn_cvt_pk_f32_fp8(word, UPPER);
    return make_float2(x[0], x[1]);
}
__device__ __forceinline__ float to_float(E4m3 x) { return to_floats8<false>(int(x.bits)).x; }

// Rounded to nearest, ties to even; |x| < 464, NaN stays NaN.  Four values to a word's bytes.
__device__ __forceinline__ int pack8(float a, float b, float c, float d) {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// The least power of two s >= 2^-100 with 448 s >= m, for finite m >= 0: with m = f 2^e, 1 <= f < 2, and 448 = 1.75
// * 2^8 it is 2^(e - 8), or twice that where f > 1.75.
__device__ __forceinline__ float least_scale(float m) {
    const unsigned u = __float_as_uint(m);
    const int e = int(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float(unsigned(max(e, kLeastScale) + 127) << 23);
}

}  // namespace ngpu
