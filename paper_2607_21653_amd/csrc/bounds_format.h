// Bounds of the keys of a block and kv head (molt_key_bounds_update of molt.h): the record, its codes and scale.
#pragma once
#include "device_common.h"

template <int D>
struct BoundsRecord {
  static constexpr int kExponent = 2 * D;        // codes of the largest keys, of the smallest, the exponent, 15 bytes unused
  static constexpr int kBytes = 2 * D + 16;
};
constexpr int kBoundsMinExponent = -100;
constexpr int kBoundsMaxExponent = 122;          // of finite values past 127 * 2^121, the largest of f32 and bf16 among them
constexpr int kBoundsNotFinite = 127;            // exponent of a block that holds an infinity or NaN

// The smallest e >= -100 with a <= 127 * 2^e, for the bits of a finite a >= 0: a = 2^(E - 127) (1 + m / 2^23), and
// 127 = 2^6 (1 + 0x7e0000 / 2^23). Subnormals are under 127 * 2^-100.
MOLT_DEV int bounds_exponent(uint32_t a) {
  const int e = int(a >> 23) - 133 + ((a & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return max(e, kBoundsMinExponent);
}
// 2^e for e in -126 .. 127
MOLT_DEV float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

// four codes (-127 .. 127) as bytes, the first lowest
MOLT_DEV uint32_t pack_codes(int a, int b, int c, int d) {
  return (uint32_t(a) & 0xffu) | (uint32_t(b) & 0xffu) << 8 | (uint32_t(c) & 0xffu) << 16 | uint32_t(d) << 24;
}
