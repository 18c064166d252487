// Numbers in 8 and 16 bits, as the caches hold them (HIP translation units only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wg {

typedef __bf16 Half2 __attribute__((ext_vector_type(2)));
typedef __bf16 Half8 __attribute__((ext_vector_type(8)));
typedef float Float2 __attribute__((ext_vector_type(2)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef uint32_t Word2 __attribute__((ext_vector_type(2)));
typedef uint32_t Word4 __attribute__((ext_vector_type(4)));

constexpr float kMost8 = 448.f;                      // the largest number of the format (e4m3: 4 exponent bits, 3 of mantissa)
constexpr int kLeastExp = -64, kMostExp = 120;       // exponents that a scale may have

// Two numbers to bfloat16: nearest, ties to even.
__device__ __forceinline__ uint32_t pk_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(Float2{a, b}, Half2)); }
// Numbers to 8 bits: nearest, ties to even; what is too large is the largest (NaN stays NaN).
__device__ __forceinline__ float within(float x) { return __builtin_fabsf(x) > kMost8 ? __builtin_copysignf(kMost8, x) : x; }
__device__ __forceinline__ uint32_t to_bytes(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(within(a), within(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(within(c), within(d), r, true);
}
__device__ __forceinline__ float low(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float high(uint32_t two) { return __uint_as_float(two & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t rescaled(uint32_t bytes, float ratio)
{
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)bytes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)bytes, true);
    return to_bytes(a[0] * ratio, a[1] * ratio, b[0] * ratio, b[1] * ratio);
}
// The larger of a and the magnitude of a number (bfloat16, in the upper half of a word), unless that is none or infinite.
__device__ __forceinline__ float top_of(float a, float x) { const float y = __builtin_fabsf(x); return __builtin_fmaxf(a, y < __builtin_inff() ? y : 0.f); }

// The least power of two times which 448 reaches `top`: 448 = 1.75 * 2^8.  A power of two costs no precision, the format keeps 3 bits of mantissa at any
// scale, and where a page's scale grows its earlier tokens are rounded again only at the format's low end.
__device__ __forceinline__ float scale_for(float top)
{
    const uint32_t bits = __float_as_uint(top);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
    e = e < kLeastExp ? kLeastExp : e > kMostExp ? kMostExp : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

}  // namespace wg
