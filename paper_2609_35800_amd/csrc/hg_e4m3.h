// The codes of the 8-bit cache: e4m3 (4 exponent bits, bias 7, 3 mantissa bits;
// largest 448, smallest 2^-9, 0x7F NaN) times a power of two.
#pragma once

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

// Biased exponent of 2^e, the smallest with amax <= 448 * 2^e, e in [-100, 119]:
// 448 = 1.75 * 2^8, so e is amax's exponent - 8, or - 7 for mantissas past 1.75.  In
// this range every code * 2^e is a normal BF16 number or 0.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, 127 - 100), 127 + 119);
}
__device__ __forceinline__ float exponent_scale(int biased) { return __uint_as_float((uint32_t)biased << 23); }
__device__ __forceinline__ float exponent_inverse(int biased) { return __uint_as_float((uint32_t)(254 - biased) << 23); }

// Biased exponent of a stored scale, within the range above (whatever is stored,
// the arithmetic on it stays in range); `other` for one that is not finite.
__device__ __forceinline__ int stored_exponent(float scale, int other) {
  const int e = (int)(__float_as_uint(scale) >> 23) & 0xFF;
  return e == 0xFF ? other : min(max(e, 127 - 100), 127 + 119);
}

// Infinities (and what a scale at the end of its range leaves above) to the largest code.
__device__ __forceinline__ float saturate(float x) {
  return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f);
}

// Four values to codes, nearest, ties to even; Small: none is past 448 or NaN.
template <bool Small>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  if constexpr (!Small) {
    a = saturate(a);
    b = saturate(b);
    c = saturate(c);
    d = saturate(d);
  }
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// Eight BF16 values, times inv, to codes.
template <bool Small>
__device__ __forceinline__ u32x2 to_codes8(u32x4 x, float inv) {
  return u32x2{to_codes<Small>(bf16_lo(x[0]) * inv, bf16_hi(x[0]) * inv, bf16_lo(x[1]) * inv, bf16_hi(x[1]) * inv),
               to_codes<Small>(bf16_lo(x[2]) * inv, bf16_hi(x[2]) * inv, bf16_lo(x[3]) * inv, bf16_hi(x[3]) * inv)};
}

// 2^d for d <= 0; 0 where that is below the normal numbers, and a code times it
// below every code.
__device__ __forceinline__ float exponent_ratio(int d) { return exponent_scale(max(127 + d, 0)); }

// Four codes times a ratio to codes.
__device__ __forceinline__ uint32_t rescale_codes(uint32_t x, float ratio) {
  return to_codes<false>(__builtin_amdgcn_cvt_f32_fp8((int)x, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)x, 1) * ratio,
                  __builtin_amdgcn_cvt_f32_fp8((int)x, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)x, 3) * ratio);
}

// Two codes (the lower or the upper of a word) times a power of two to BF16, exact.
template <bool Upper>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t x, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, Upper));
}

}  // namespace
}  // namespace hg
