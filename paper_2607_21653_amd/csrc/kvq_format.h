// The 4-bit KV cache format, shared by the kernels that write, read and attend over it: OCP
// microscaling MXFP4. A token's head vector of D dims is D / 32 groups of 32 e2m1 codes (sign, 2
// exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), each group with an e8m0 scale byte s
// that stands for 2^(s - 127), 255 for NaN. Every value is exact in bf16: 2 significant bits and, with
// the scale bytes that are written (2 .. 252), exponents -126 .. 127.
//
// A block of 16 tokens of one kv head is a record of 17 D / 2 bytes per cache, codes first:
//   K  codes [16 tokens][D / 2]       scales [16 tokens][D / 32]
//   V  codes [4][D / 8][4 tokens][4]  scales [4][D / 32][4 tokens]   (token 4 a + c; dims 8 i .. +7)
// Dim 2 i is the low nibble of byte i. The V order is the MFMA operand order of V^T: the 16 bytes of
// lane 16 a + r are 4 tokens of one octet of dims, so a wavefront reads a block's codes as one
// contiguous load, as it does with K's rows.
#pragma once
#include "device_common.h"

namespace molt {

constexpr uint32_t kKvqScaleNan = 255u;

template <int D>
struct KvqRecord {
  static constexpr int kCodes = 8 * D;        // bytes of codes
  static constexpr int kBytes = 17 * D / 2;
  // byte offset of the 4 code bytes of dims 8 oct .. +7 of a token, and of its group's scale
  MOLT_DEV static int k_code(int token, int oct) { return token * (D / 2) + oct * 4; }
  MOLT_DEV static int k_scale(int token, int group) { return kCodes + token * (D / 32) + group; }
  MOLT_DEV static int v_code(int token, int oct) { return ((token >> 2) * (D / 8) + oct) * 16 + (token & 3) * 4; }
  MOLT_DEV static int v_scale(int token, int group) { return kCodes + ((token >> 2) * (D / 32) + group) * 4 + (token & 3); }
};

// Scale byte of a group from the bits of its largest magnitude a (f32): the exponent e with
// a / 2^e in [3.5, 7), so that no element is more than one unit 2^e off (6 is the largest code; above
// 5 and up to 7 it is the nearest or as near as 4 and 6 are to 5): the exponent field of a, one more
// from mantissa 1.75 on, less 2. Kept in 2 .. 252, where every nonzero code is a normal finite bf16.
MOLT_DEV uint32_t kvq_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kKvqScaleNan;
  const int s = int((amax_bits + 0x00200000u) >> 23) - 2;
  return uint32_t(s < 2 ? 2 : s > 252 ? 252 : s);
}

// 8 values as e2m1 codes of x / 2^(s - 127) in 4 bytes, x[0] in the low nibble: round to nearest, ties
// to the even code, saturating. The hardware conversion (v_cvt_scalef32_pk_fp4_f32) does this and takes
// the scale's exponent field only: compared on gfx950 with a bit-level rounding over every bf16 value of
// 51 scales and over ties and their neighbours, no code differs. A NaN group's codes are 0.
MOLT_DEV uint32_t kvq_encode8(const float (&x)[8], uint32_t s) {
  if (s == kKvqScaleNan) return 0u;
  const float sc = __uint_as_float(s << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], sc, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], sc, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], sc, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], sc, 3);
  return r;
}

// The two values of byte I of w (dims 2 I and 2 I + 1 of an octet) as packed bf16. Only the exponent
// field of `scale` counts (its sign and mantissa are ignored, 255 gives NaN: compared on gfx950 for every
// code and scale byte), so a scale byte may be shifted into place with its neighbours still around it.
template <int I>
MOLT_DEV uint32_t kvq_decode2(uint32_t w, uint32_t scale_bits) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale_bits), I));
}

// The same as packed f16, exact for the scale bytes of 2^-21 .. 2^10 (codes up to 6 and down to 0.5, which is
// subnormal below 2^-13): compared on gfx950 for every code and the scale bytes 104 .. 140.
template <int I>
MOLT_DEV uint32_t kvq_decode2_f16(uint32_t w, uint32_t scale_bits) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, __uint_as_float(scale_bits), I));
}
constexpr uint32_t kKvqF16First = 106u;      // 106 .. 137: 2^-21 .. 2^10
// nonzero if one of 8 scale bytes is outside 106 .. 137 (a borrow from a byte's difference comes from one that is)
MOLT_DEV uint32_t kvq_outside_f16(uint32_t a, uint32_t b) {
  return ((a - kKvqF16First * 0x01010101u) | (b - kKvqF16First * 0x01010101u)) & 0xe0e0e0e0u;
}

// byte i of four scale bytes, at the exponent field
MOLT_DEV uint32_t kvq_scale_bits(uint32_t bytes, int i) {
  return i == 0 ? bytes << 23 : i == 1 ? bytes << 15 : i == 2 ? bytes << 7 : bytes >> 1;
}

}  // namespace molt
