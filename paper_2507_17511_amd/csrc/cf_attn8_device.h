// Device-side building blocks of the kernels over the cache in 8 bits: e4m3 codes, the powers of two that they are scaled by.
#pragma once

#include "cf_attn_device.h"
#include "cf_attn8.h"

namespace cf {
namespace attn {

constexpr int kLeastExponent = -100, kMostExponent = 119;       // of scales: elements are finite in fp32 and bf16, and none of them subnormal

template <int DT> struct Code;
template <> struct Code<BF16> {
    static constexpr float kMost = 2.9774707105582116e38f;      // 448 x 2^119
    template <bool HIGH> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH)); }
};
template <> struct Code<F16> {
    static constexpr float kMost = 61440.0f;                    // 240 x 2^8: the next code times 2^8 is past fp16
    template <bool HIGH> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HIGH)); }
};

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // -126 <= e <= 127

// The exponent of the least scale that brings `most` to 448 = 1.75 x 2^8 at most.
__device__ __forceinline__ int exponent_for(float most)
{
    const uint32_t w = __float_as_uint(most);
    const int e = (int)(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, kLeastExponent), kMostExponent);
}
__device__ __forceinline__ int exponent_of(float scale) { return min(max((int)(__float_as_uint(scale) >> 23 & 255u) - 127, kLeastExponent), kMostExponent); }

// Four codes of four elements that lie within +-448 (or are NaN).
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

}  // namespace attn
}  // namespace cf
