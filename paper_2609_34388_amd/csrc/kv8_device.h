// The 8-bit block: 16 tokens of one KV head (include/recguide.h has the
// format), where its bytes lie, and its conversions.
#pragma once

#include "attention_device.h"

namespace rg {
namespace {

template <int D>
struct Kv8 {
  static constexpr int V = 16 * D, BLOCK = 32 * D;  // V's first byte
  static __device__ __forceinline__ int k_code(int slot, int d) { return (d >> 5) * 512 + slot * 32 + (d & 31); }
  static __device__ __forceinline__ int v_code(int slot, int d) { return V + ((slot >> 3) * D + d) * 8 + (slot & 7); }
};

// Exponent (biased by 127) of the scale for a largest magnitude's fp32 bits:
// the magnitude over the scale lies in [224, 448) unless clamped.  The upper
// end keeps 448 times the scale below 2^128, the lower one every product a
// normal bf16.
__device__ __forceinline__ int kv8_exponent(uint32_t bits) { return min(max((int)((bits + 0x200000u) >> 23) - 8, 10), 246); }

// Bytes 2 SEL and 2 SEL + 1 of a word of codes, times the scale, as two bf16
// (exact: four significant bits times a power of two).
template <int SEL>
__device__ __forceinline__ uint32_t decode2_8(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, SEL != 0));
}
// Eight codes as bf16.
__device__ __forceinline__ u32x4 decode8_8(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{decode2_8<0>(lo, scale), decode2_8<1>(lo, scale), decode2_8<0>(hi, scale), decode2_8<1>(hi, scale)};
}

// Four values as codes at a scale given by its reciprocal: nearest, ties to
// even, magnitudes past 448 as 448; what is not finite as NaN.
__device__ __forceinline__ uint32_t encode4_8(float a, float b, float c, float d, float inv) {
  auto held = [&](float x) {
    const float y = fminf(fmaxf(x * inv, -448.f), 448.f);
    return fabsf(x) < __builtin_huge_valf() ? y : __builtin_nanf("");
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(held(a), held(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(held(c), held(d), w, true);
}

}  // namespace
}  // namespace rg
