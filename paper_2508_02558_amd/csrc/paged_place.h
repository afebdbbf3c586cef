// What the kernels of the paged cache's attention share about values and places: masks, the softmax reference, values that are no numbers, and where a tile's rows are.
#pragma once

#include "attn_tile_math.h"
#include "paged_tile.h"

namespace sdllm {

// Logits of keys that a row does not see become -inf; `seen` is the row's bits of the tile (seen_bits).
__device__ __forceinline__ void mask_logits(f32x16& s, uint32_t seen, int half) {
  seen >>= 4 * half;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = or_minus_infinity(s[i], bit_mask(seen, 8 * (i >> 2) + (i & 3)));
}

// The softmax reference of a row moves when a maximum exceeds it by more than kRescaleSlack (attn_tile_math.h).  Numerators against it are rounded to bf16, the
// type of what they multiply: half a step, 2^-8, of each, as much as the rounding of the result.
template <int NE>
__device__ __forceinline__ void move_reference_to(float m_loc, float& m_ref, float& l_run, f32x16 (&acc)[NE]) {
  if (__ballot(m_loc > m_ref + kRescaleSlack) != 0) {
    const float m_new = fmaxf(m_ref, fmaxf(m_loc, __shfl_xor(m_loc, 32)));
    const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    l_run *= alpha;
#pragma unroll
    for (int e = 0; e < NE; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[e][i] *= alpha;
  }
}

// Takes values that are no numbers out of a masked tile's operands (paged_tile.h); true for all lanes if there are any.  bf16: two values a word.
template <int N>
__device__ __forceinline__ bool take_specials(f32x4 (&f)[N]) {
  auto special = [](float v) { return ((__builtin_bit_cast(uint32_t, v) & 0x7f800000u) + 0x00800000u) & 0x80000000u; };   // bit 31: the exponent is all ones
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= special(f[i][j]);
  if (__ballot(any != 0) == 0) return false;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) f[i][j] = special(f[i][j]) ? 0.f : f[i][j];
  return true;
}
template <int N>
__device__ __forceinline__ bool take_specials(i16x8 (&f)[N]) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  // bits 15 and 31: the exponents that are all ones
  auto special = [](uint32_t v) { return ((v & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
  u16x2 most = {0, 0};   // of the magnitudes
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u32x4 v = __builtin_bit_cast(u32x4, f[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[j] & 0x7fff7fffu));
  }
  if (__ballot(special(__builtin_bit_cast(uint32_t, most)) != 0) == 0) return false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 v = __builtin_bit_cast(u32x4, f[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] &= ~((special(v[j]) >> 15) * 0xffffu);
    f[i] = __builtin_bit_cast(i16x8, v);
  }
  return true;
}

// add_specials' share of four channels of a row of V
template <typename E>
__device__ __forceinline__ f32x4 special_values(const char* v, int channel, bool sees) {
  const E* u = reinterpret_cast<const E*>(v) + channel;
  f32x4 z;
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = sees && !(fabsf((float)u[k]) < INFINITY) ? (float)u[k] : 0.f;
  return z;
}

// Where the rows of an item are, in bytes (ES an element): its pages' and its own (kSeeTree) rows of the KV head
struct ItemBase {
  const char *k, *v, *k_own, *v_own;
  int64_t page;
  uint32_t stride, stride_own, row_mask;
};
template <int ES, int SEES>
__device__ __forceinline__ ItemBase item_base(const PagedAttnParams& p, const PagedItem& w) {
  ItemBase r{};
  const PagedCache& c = p.cache;
  const int64_t at = ES * (w.g * c.sh);
  r.k = (const char*)p.k_pages + at;
  r.v = (const char*)p.v_pages + at;
  r.page = ES * c.sp;
  r.stride = (uint32_t)(c.sr * ES);
  r.row_mask = (1u << c.page_shift) - 1;
  if (SEES == kSeeTree) {
    const int64_t own = ES * (w.b * p.blk_sb + w.g * p.blk_sh);
    r.k_own = (const char*)p.k_blk + own;
    r.v_own = (const char*)p.v_blk + own;
    r.stride_own = (uint32_t)(p.blk_sr * ES);
  }
  return r;
}

// Where the rows of a tile are, worked out for 64 tiles at once, one per lane, and handed out by readlane.  Rows 0-15 and 16-31 lie in one page each, or in the
// same; a half that nobody sees any of is the other's rows.
struct TilePlace {
  int64_t at0, at1; // bytes from ItemBase's pointers to row 0 and to row 16
  uint32_t bits;    // of [lo, hi): lo, hi << 6; kOwn, kWhole
};
constexpr uint32_t kOwn = 1 << 12, kWhole = 1 << 13;   // kWhole: 32 rows of the cache, one stride apart

template <int SEES>
__device__ __forceinline__ TilePlace place_of(const PagedAttnParams& p, const PagedItem& w, const ItemBase& i, const PagedTile& x) {
  TilePlace r;
  const bool own = SEES == kSeeTree && x.own;
  auto half_at = [&](int h) {
    const int seen = x.at + min(max(16 * h, x.lo), x.hi - 1), first = seen & ~15;
    return own ? (int64_t)first * i.stride_own : page_of(p.cache, w.b, seen) * i.page + (int64_t)(first & (int)i.row_mask) * i.stride;
  };
  r.at0 = half_at(0);
  r.at1 = half_at(1);
  const bool whole = !own && x.lo == 0 && x.hi == kTileKeys && r.at1 - r.at0 == 16 * (int64_t)i.stride;
  r.bits = (uint32_t)(x.lo | x.hi << 6) | (own ? kOwn : 0u) | (whole ? kWhole : 0u);
  return r;
}
__device__ __forceinline__ int64_t readlane64(int64_t v, int lane) {
  const uint64_t u = (uint64_t)v;
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)u, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32);
}
__device__ __forceinline__ TilePlace place_from(const TilePlace& r, int lane) {
  return {readlane64(r.at0, lane), readlane64(r.at1, lane), (uint32_t)__builtin_amdgcn_readlane((int)r.bits, lane)};
}
// Row r of a tile, or the nearest that somebody sees, in bytes from ItemBase's pointers
__device__ __forceinline__ int64_t row_at(const TilePlace& t, const ItemBase& i, int r) {
  r = min(max(r, (int)(t.bits & 63)), (int)(t.bits >> 6 & 63) - 1);
  return t.at0 + ((r & 16) != 0 ? t.at1 - t.at0 : 0) + (uint32_t)(r & 15) * (t.bits & kOwn ? i.stride_own : i.stride);
}

}  // namespace sdllm
