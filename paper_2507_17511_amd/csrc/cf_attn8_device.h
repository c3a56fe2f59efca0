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

// Moves between lanes.  CONTROL: 0x110 + n from n lanes below, of sixteen; 0x142 (0x143) from the last lane of the sixteen (half) below; 0xb1, 0x4e the other lane of a pair, pair of a
// four; 0x141 (0x140) eight (sixteen) lanes turned round.  Lanes that nothing comes to have 0.
template <int CONTROL, int ROWS = 0xf> __device__ __forceinline__ uint32_t moved(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CONTROL, ROWS, 0xf, false); }
template <int CONTROL> __device__ __forceinline__ float moved(float x) { return __uint_as_float(moved<CONTROL>(__float_as_uint(x))); }
template <int CONTROL> __device__ __forceinline__ double moved(double x)
{
    const u32x2 w = __builtin_bit_cast(u32x2, x);
    return __builtin_bit_cast(double, (u32x2){moved<CONTROL>(w[0]), moved<CONTROL>(w[1])});
}
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }     // stays at the largest number

// Sums over sixteen lanes up to each, and over the wave's.
__device__ __forceinline__ uint32_t sums_of_sixteen(uint32_t x)
{
    x = add(x, moved<0x111>(x));
    x = add(x, moved<0x112>(x));
    x = add(x, moved<0x114>(x));
    return add(x, moved<0x118>(x));
}
__device__ __forceinline__ uint32_t sums(uint32_t x)
{
    x = sums_of_sixteen(x);
    x = add(x, moved<0x142, 0xa>(x));
    return add(x, moved<0x143, 0xc>(x));
}

}  // namespace attn
}  // namespace cf
