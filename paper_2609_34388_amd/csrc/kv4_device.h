// The 4-bit block: 16 tokens of one KV head (include/recguide.h has the
// format), where its parts lie, and its conversions.
#pragma once

#include "attention_device.h"

namespace rg {
namespace {

template <int D>
struct Kv4 {
  static constexpr int DT = D / 32;  // scale groups of a token, and dims of a V unit
  static constexpr int KS = 8 * D, VC = KS + D / 2, VS = VC + 8 * D, BLOCK = 17 * D;
  static constexpr int VB = D / 64;  // bytes of a V unit of one token
  // Byte of element d (even) of K, of the scale of its group g.
  static __device__ __forceinline__ int k_code(int slot, int d) { return (d >> 6) * 512 + slot * 32 + ((d & 63) >> 1); }
  static __device__ __forceinline__ int k_scale(int slot, int g) { return KS + slot * DT + g; }
  // Byte of V unit u (dims DT u .. DT u + DT - 1), of the scale of group g.
  static __device__ __forceinline__ int v_unit(int slot, int u) {
    return VC + (((slot >> 3) * 32 + u) * 8 + (slot & 7)) * VB;
  }
  static __device__ __forceinline__ int v_scale(int slot, int g) { return VS + ((slot >> 3) * DT + g) * 8 + (slot & 7); }
};

// Scale byte (1 .. 252) as its power of two.  Of kNanScale, and of any float with
// its exponent, the conversions make NaN whatever the code (all codes of both kinds
// measured), zero included.
constexpr uint32_t kNanScale = 255;
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Elements 2 SEL and 2 SEL + 1 of eight 4-bit codes, as bf16 (exact: two
// significant bits times a power of two).
template <int SEL>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ __forceinline__ u32x4 decode8(uint32_t codes, float scale) {
  return u32x4{decode2<0>(codes, scale), decode2<1>(codes, scale), decode2<2>(codes, scale), decode2<3>(codes, scale)};
}

// Eight bf16 as 4-bit codes: nearest, ties to even, saturating at 6.
__device__ __forceinline__ uint32_t encode8(u32x4 x, float scale) {
  // (a bit cast of a vector's element itself would take element 0)
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), scale, 3);
  return c;
}

}  // namespace
}  // namespace rg
