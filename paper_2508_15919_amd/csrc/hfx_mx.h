// The 4-bit page pool: where things lie in a page, and the conversions to and from it (device code).
//
// A block is the 16 tokens of one page and one kv-head, 17 D bytes in a row:
//   key codes    [16 tokens][D / 32][16 bytes]      byte b of a group: dimensions 2b (low four bits) and 2b + 1 of 32
//   value codes  [2][D / 64][16][2][8 tokens]       [half of the page][64 dimensions][i][32 of them][token]: dimensions i (low) and i + 16 of 32
//   key scales   [16 tokens][D / 32]
//   value scales [2][D / 64][8 tokens][2]
// The order in which the matrix cores take their operands: a lane of the scaled 4-bit product takes 32 dimensions of one key with one
// scale, 16 bytes in a row; of the values a lane needs 8 tokens of one dimension in bf16, and a byte of value codes gives one token's
// dimensions of two neighbouring product tiles.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hfx_desc.h"

namespace hfx {

template <int D>
struct Mx {
  static constexpr int kGroups = D / 32;             // scales of a token and head
  static constexpr int kKeys = 0, kValues = 8 * D, kKeyScales = 16 * D, kValueScales = 16 * D + D / 2, kBlock = 17 * D;
  static constexpr int kHalf = 4 * D;                // value codes of 8 tokens
  static constexpr int kHalfScales = D / 4;
};

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// Two codes (byte `Byte` of `codes`) times two to the power of a scale byte in bits 23 to 30 of `scale`, as bf16, the low four bits' one low.  The
// instruction looks at the exponent of its scale operand alone, so that a scale byte anywhere in a register takes one shift; a scale byte of 255 makes NaN.
template <int Byte>
__device__ __forceinline__ unsigned from_fp4(unsigned codes, unsigned scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __builtin_bit_cast(float, scale), Byte));
}
// Byte `Byte` of a register of scale bytes in the place where from_fp4 looks.
template <int Byte>
__device__ __forceinline__ unsigned scale_at(unsigned scales) {
  return Byte == 3 ? scales >> 1 : scales << (23 - 8 * Byte);
}

// Scale byte of 32 values whose largest magnitude has the bits `top`: the smallest power of two under which that value is nearest to a
// magnitude of at most 6, that is, less than 7.  At least 2 and at most 252, so that every value of a block is a normal bf16 number or zero;
// 255 where the block holds something that is not finite.
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
  const int e = (int)((top + 0x200000u) >> 23) - 2;
  return top >= 0x7f800000u ? 255u : (unsigned)min(max(e, 2), 252);
}

// Codes of eight values under the scale 2^(e - 127), nearest, ties to the even code; the first value in the lowest four bits.
__device__ __forceinline__ unsigned to_fp4(const float* x, unsigned e) {
  const float scale = __builtin_bit_cast(float, e << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
  return c;
}

}  // namespace hfx
