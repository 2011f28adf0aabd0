// The 4-bit KV cache format and its conversions (device side, shared by the kernel sources).
//
// A group is 32 consecutive dimensions of one token of one head: 32 E2M1 codes (sign, then the
// magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one E8M0 byte b, the scale 2^(b - 127) (the MXFP4
// format of the OCP Microscaling specification).  The scale is the smallest power of two for
// which the group's largest magnitude is at most 7 times it (up to 7 rounds to 6): over normal,
// heavy-tailed and uniform groups that leaves a root-mean-square error of 11.2, 12.9 and 9.9 % of
// the values', against 11.5, 13.9 and 9.9 % for "at most 6" and 11.5, 13.1 and 14.1 % for the
// specification's floor rule.  b stays in [2, 252], so that every value a code stands for
// is a normal bf16 number or zero: a stored value is exact in bf16, and attention over the cache
// rounds nothing more than attention over bf16 rows does.  A group with an infinity or a NaN has
// b = 255 and reads back as NaN.
//
// One block (16 tokens) of one head is 17 D bytes, K and V together (17 lines of 128 bytes at
// D = 128), so that what a work-group reads is one piece of memory:
//   K codes   [16 tokens][D / 2]            byte i of a row: dimensions 2 i (low half) and 2 i + 1
//   V codes   [2 halves][D / 2 pairs][8]    byte j of pair i: dimensions 2 i, 2 i + 1 of token 8 half + j
//   K scales  [16 tokens][D / 32]
//   V scales  [D / 32][16 tokens]
// A lane of Q.K^T reads 32 (D = 64: 16) dimensions of one token; a lane of P.V reads 8 tokens of
// 4 dimensions: each is 16 (8) bytes in one place.
#pragma once

#include <hip/hip_runtime.h>

namespace mx4 {

template <int D>
struct Layout {
  static constexpr int kGroups = D / 32;
  static constexpr int kRow = D / 2;               // bytes of a K row
  static constexpr int kHalf = 4 * D;              // bytes of 8 tokens of V
  static constexpr int kV = 8 * D;                 // where V's codes, K's and V's scales start
  static constexpr int kKScale = 16 * D;
  static constexpr int kVScale = 16 * D + 16 * kGroups;
  static constexpr int kBytes = 17 * D;            // one block of one head
};

constexpr uint32_t kNanScale = 255;

// the scale byte of a group whose largest magnitude has these bf16 bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  // exponent field - 2, one more where the mantissa is over 1.75 (0x60): top <= 7 * 2^(b - 127)
  const int b = static_cast<int>((top + 0x1f) >> 7) - 2;
  return top >= 0x7f80 ? kNanScale : static_cast<uint32_t>(min(max(b, 2), 252));
}
// its value as the conversions take it (255: infinity, which reads back as NaN)
__device__ __forceinline__ float scale_value(uint32_t b) { return __builtin_bit_cast(float, b << 23); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// byte B of `codes` as two bf16 values
template <int B>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
// eight bf16 values as eight codes (round to nearest even, saturating at 6)
__device__ __forceinline__ uint32_t encode8(const uint32_t (&x)[4], float scale) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x[2]), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x[3]), scale, 3);
  return c;
}
// the largest magnitude's bits of the 32 values that four neighbouring lanes hold
__device__ __forceinline__ uint32_t group_top(const uint32_t (&x)[4]) {
  u16x2 m = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
  uint32_t t = max(static_cast<uint32_t>(m[0]), static_cast<uint32_t>(m[1]));
  t = max(t, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(t), 0xB1, 0xf, 0xf, true)));   // lane ^ 1
  return max(t, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(t), 0x4E, 0xf, 0xf, true)));  // lane ^ 2
}

}  // namespace mx4
