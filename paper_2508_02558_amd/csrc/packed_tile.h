// The cache of 4 bits a value: its layout, and the conversions between its codes and numbers.
//
// A value is a 4-bit number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and negatives, sign in bit 3) times 2^e with one e for 32 of them, 4.25 bits in
// all: the form for which gfx950 converts two codes to two scaled bf16 numbers, exactly, in one instruction.  e belongs to 32 channels of
// a key and to one channel of 32 value rows: each time to numbers that are contracted with each other, so that a lane of a
// matrix instruction, which holds eight of them, needs one scale.
//
// A (batch, KV head) is a run of tiles of 32 rows, 34 d bytes each, one after the other, so that a wavefront fetches a tile with whole
// 1 KB requests that need no reordering in registers or LDS: lane (m = lane % 32, half = lane / 32) gets its own 16 bytes.
//   key codes    [d/32 groups of channels][32 keys][16 bytes]; request i: group 2 i + half of key m
//   value codes  [d/64: i][half][32: m][16 bytes]: channels (d/32) m + 2 i + j, j = 0, 1, eight bytes each; nibble 4 a + p of them is
//                row 8 a + 4 half + p, the order in which the logits of a 32x32 product lie in the registers of a lane
//   key scales   [32 keys][d/32 groups], value scales [d channels]: bytes e + 127 of 2^e, 255 for NaN
#pragma once

#include "mfma_tile.h"

namespace sdllm {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

template <int HD>
struct PackedLayout {
  static constexpr int kLoads = HD / 64;                 // 16-byte loads per lane of a tile's keys, and of its values
  static constexpr int kGroups = HD / 32;                // scales of a key; channels of a value row per lane
  static constexpr int kKeys = 0, kValues = 16 * HD, kKeyScales = 32 * HD, kValueScales = 33 * HD, kTile = 34 * HD;
};
static_assert(PackedLayout<128>::kTile == packed_tile_bytes(128) && PackedLayout<64>::kTile == packed_tile_bytes(64), "as the host sizes it");

// The float 2^e of a scale byte; 255 makes what is converted with it NaN.
__device__ __forceinline__ float scale_of_byte(uint32_t word, int byte) { return __builtin_bit_cast(float, ((word >> (8 * byte)) & 0xff) << 23); }

// Eight numbers of a word of codes, lowest nibble first.
__device__ __forceinline__ bf16x8 unpack8(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Scale byte of a group from the largest of its magnitudes' bits (as float; NaN above infinity above all numbers): the smallest e in
// [-125, 125] with magnitudes below 7 2^e.  Up to there rounding to 6 2^e is no further than half of that number's step of 2 2^e; the limits keep
// every number that the codes stand for normal and finite.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int byte = (int)((top + 0x200000u) >> 23) - 2;   // a mantissa of 1.75 and more carries
  return byte < 2 ? 2 : byte > 252 ? 252 : byte;
}

}  // namespace sdllm
