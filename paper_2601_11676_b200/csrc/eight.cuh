// 8-bit rows of a paged cache: a code is an e4m3 number (a sign, four bits of exponent biased by 7, three behind the point),
// a row of one K/V head at one position has the power of two 2^e that its codes are multiplied with, stored as e + 127.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace halo {

// Every value of a row is then a normal bf16 number or 0: code * 2^e lies in [2^-126, 1.75 * 2^127].
constexpr int kEightMin = -117, kEightMax = 119;
constexpr int kEightNan = 255;   // a row that held a NaN or an infinity: all of it reads back as NaN

// The smallest e with amax <= 448 * 2^e, 448 = 1.75 * 2^8 the largest e4m3 number; amax finite.
__device__ __forceinline__ int eight_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, kEightMin), kEightMax);
}
__device__ __forceinline__ float eight_power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// 2^e of a scale byte; NaN for kEightNan
__device__ __forceinline__ float eight_unit(uint32_t byte) { return __uint_as_float(byte == kEightNan ? 0x7fc00000u : byte << 23); }
// Two codes, the first in the low byte: nearest, ties to even.
__device__ __forceinline__ uint32_t eight_pair(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// The four codes of a word as numbers: exponent and significand fall into the fields of an fp32 number, which is the value
// times 2^-120 (subnormal codes included), and 2^120 puts that right without rounding.
__device__ __forceinline__ void eight_widen(uint32_t w, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = w >> (8 * i);
        f[i] = __uint_as_float(((c & 0x80u) << 24) | ((c & 0x7fu) << 20)) * 0x1p120f;
    }
}

}  // namespace halo
