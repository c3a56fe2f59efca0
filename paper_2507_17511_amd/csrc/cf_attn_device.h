// Device-side building blocks shared by the attention kernels: 16-bit element formats, the matrix
// instructions on them, and the exchange of a value between the halves of a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cf_attn.h"

namespace cf {
namespace attn {

#define CF_GLOBAL __attribute__((address_space(1)))
#define CF_LDS __attribute__((address_space(3)))
#define CF_CONST __attribute__((address_space(4)))     // memory that nothing writes during the launch

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int BF16 = 1, F16 = 2;    // cf_dtype
constexpr float kLn2 = 0.693147180559945309f;
// Where a row's reference, which its scores (times log2 e) are taken relative to, begins: the lowest finite number, and not -infinity, so that
// score - reference is -infinity, and the weight 0, for a masked score of a row that has seen no other.
constexpr float kNoMax = -3.402823466e38f;
// A row's accumulators are scaled down when a score passes the reference in use by more than Elem::kMostOver powers of two.  bf16: the reference is a maximum, weights
// reach 2^8 at most, their rounding is relative, and sums of 2^31 of them stay finite in fp32.  fp16 holds numbers from 2^-14 on in full and none below 2^-25, and keys that weigh
// less than that next to the largest may weigh much together, behind a first token that all rows attend to, say.  So there
// - a score that passes the reference by more than kJump, as the first keys' do, sets it kLift below itself: what shares a tile with it keeps more of its bits;
// - the reference falls, too, and the accumulators are scaled up, where all of a row's keys at hand (64 at most) are less than kLeastOver over it, or their weights sum up to
//   less than kLeastSum.  Other sums are off by the rounding of 64 weights to 2^-24 at most: 2^-8 of the least if all were rounded one way, and they average out.
// The sum of all weights stays below 2^kMostTotal; past kFullTotal nothing falls: what is at hand is below 2^-60 of the row.
constexpr float kJump = 15.0f, kLift = 6.0f;
constexpr float kLeastOver = -11.0f;
constexpr float kLeastSum = 0.00048828125f;                 // 2^-11
constexpr float kMostTotal = 60.0f;
constexpr float kFullTotal = 288230376151711744.0f;        // 2^58
// Where the maximum is not looked for (see k_attn_prompt): the most that the weights of a lane's keys of one tile may sum up to.  No weight is
// larger than that, so that all of them are finite in fp16.
constexpr float kMostSum = 32768.0f;
// ... and the largest maximum of which half a unit in the last place is 1/4 at most.
constexpr float kMostExact = 4194304.0f;

template <typename T> __device__ __forceinline__ const CF_GLOBAL T *gconst(const void *p) { return (const CF_GLOBAL T *)p; }
template <typename T> __device__ __forceinline__ CF_GLOBAL T *gmut(void *p) { return (CF_GLOBAL T *)p; }

template <int DT> struct Elem;
// Whether one of two 16-bit numbers is infinite or NaN: a carry out of the exponent, to the sign's place, tells.  Carries may be OR-ed over many.
template <uint32_t EXPONENT> struct OddPair {
    static __device__ __forceinline__ uint32_t carry(uint32_t w) { return (w & EXPONENT * 0x10001u) + (0x8000u - EXPONENT) * 0x10001u; }
    static __device__ __forceinline__ bool any(uint32_t carries) { return (carries & 0x80008000u) != 0; }
};
template <> struct Elem<BF16> {
    using Odd = OddPair<0x7f80u>;
    static constexpr bool kFollow = false;                          // whether the reference follows the scores down
    static constexpr float kMostOver = 8.0f;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2)); }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0); }
};
template <> struct Elem<F16> {
    using Odd = OddPair<0x7c00u>;
    static constexpr bool kFollow = true;
    static constexpr float kMostOver = 15.0f;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2)); }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0); }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger of a lane's value and that of the lane 32 (16) away; NaN yields to a number.
__device__ __forceinline__ float max_halves(float x)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_quarters(float x)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_quarters(float x)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The reference after keys whose largest score is `top`; whether it may fall, and the largest part of the row's sum that a lane has.
template <int DT> __device__ __forceinline__ float reference(float m, float top, bool fall, float total)
{
    if constexpr (!Elem<DT>::kFollow) return fmaxf(m, top);
    const float raised = top > m + kJump ? top - kLift : fmaxf(m, top);
    return fall && top < m + kLeastOver && top > -__builtin_inff() ? fmaxf(top, m - fmaxf(kMostTotal - __log2f(total), 0.0f)) : raised;
}

// Enqueues a kernel of 256 (so many) threads a workgroup.  -> what came of it, and not of some call before it: the runtime remembers an error until it is asked.
template <int THREADS, typename Args> hipError_t enqueue_of(void (*kernel)(Args), int64_t workgroups, hipStream_t s, Args a)
{
    void *args[] = {&a};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)workgroups), dim3(THREADS), args, 0, s);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
}
template <typename Args> hipError_t enqueue(void (*kernel)(Args), int64_t workgroups, hipStream_t s, Args a) { return enqueue_of<256>(kernel, workgroups, s, a); }

__device__ __forceinline__ float lse_of(float m, float l) { return l > 0.0f || l != l ? (m + __log2f(l)) * kLn2 : -__builtin_inff(); }
__device__ __forceinline__ float inverse_of(float l) { return l > 0.0f || l != l ? 1.0f / l : 0.0f; }

}  // namespace attn
}  // namespace cf
