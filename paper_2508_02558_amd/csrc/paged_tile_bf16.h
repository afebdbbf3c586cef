// bf16 tiles of the paged cache in LDS, and what the matrix cores take of them: 32 keys by 32 query columns, fragments as in attn_tile_math.h (K rows as
// the A operand of the logits, V columns through the transposing LDS read, P^T as the B operand), for head_dim 64 and 128.
//
// A tile of one tensor comes as HD / 16 fetches of 1 KB of consecutive LDS, each of whole rows in order; which 16-byte piece of its row a lane brings is free, so
// the pieces of a row are permuted to keep the operand reads off each other's banks.
#pragma once

#include "attn_tile_math.h"
#include "paged_tile.h"

namespace sdllm {

template <int HD>
struct BfTile {
  static constexpr int kRow = HD * 2, kBytes = kTileKeys * kRow;
  static constexpr int kPieces = kRow / 16;             // of a row
  static constexpr int kRowsPerFetch = kWave / kPieces;
  static constexpr int kFetches = kTileKeys / kRowsPerFetch;
  static constexpr int NP = HD / 16;                    // operands of the logits
  static constexpr int NE = HD / 32;                    // accumulators
  // row r holds piece c of K in place c ^ k_turn(r), of V in place c ^ v_turn(r)
  static __device__ __forceinline__ int k_turn(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int v_turn(int r) { return HD == 128 ? (r & 3) << 2 : (r & 2) << 1; }

  static __device__ __forceinline__ void read_k(const uint8_t* tile, int half, int col, bf16x8 (&a)[NP]) {
    const uint32_t at = (uint32_t)(col * kRow + ((half ^ k_turn(col)) << 4));
#pragma unroll
    for (int i = 0; i < NP; ++i) a[i] = *reinterpret_cast<const bf16x8*>(tile + (at ^ (uint32_t)(i * 32)));
  }
  static __device__ __forceinline__ void read_v(const uint8_t* tile, int lane, i16x8 (&f)[2 * NE]) {
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const int half = lane >> 5, grp = (lane >> 4) & 1, s16 = lane & 15, r = half * 4 + (s16 >> 2);
    const uint32_t at = (uint32_t)(r * kRow + ((v_turn(r) << 4) ^ (grp * 32 + (s16 & 3) * 8)));
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const uint8_t* from = tile + (at ^ (uint32_t)(e * 64)) + st * 16 * kRow;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)from);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from + 8 * kRow));
        f[st * NE + e] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
  }
  static __device__ __forceinline__ void logits(const bf16x8 (&a)[NP], const bf16x8 (&qf)[NP], f32x16& s) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], qf[i], s, 0, 0, 0);
  }
  static __device__ __forceinline__ void pv(const i16x8 (&f)[2 * NE], const bf16x8 (&pb)[2], f32x16 (&acc)[NE]) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int e = 0; e < NE; ++e)
        acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[st * NE + e]), pb[st], acc[e], 0, 0, 0);
  }
};

// Logits of keys that a row does not see become -inf; `seen` is the row's bits of the tile (seen_bits).
__device__ __forceinline__ void mask_logits(f32x16& s, uint32_t seen, int half) {
  seen >>= 4 * half;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = or_minus_infinity(s[i], bit_mask(seen, 8 * (i >> 2) + (i & 3)));
}

// Softmax numerators of a tile's raw logits as the B operands of the second product, against a reference that moves when a maximum exceeds it by
// more than kRescaleSlack (attn_tile_math.h).  Rounded to bf16, the type of what they multiply: half a step, 2^-8, of each numerator,
// as much as the rounding of the result.
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

template <int NE>
__device__ __forceinline__ void numerators(const f32x16& s, float scale_log2, float& m_ref, float& l_run, f32x16 (&acc)[NE], bf16x8 (&pb)[2]) {
  float m_loc = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m_loc = fmaxf(m_loc, s[i]);
  move_reference_to<NE>(m_loc * scale_log2, m_ref, l_run, acc);
  float l_loc = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -m_ref));
    l_loc += x;
    pb[i >> 3][i & 7] = (__bf16)x;
  }
  l_run += l_loc;
}

// Takes values that are no numbers out of a masked tile's operands (paged_tile.h), two values a word; true for all lanes if there are any.
template <int N>
__device__ __forceinline__ bool take_specials(i16x8 (&f)[N]) {
  // bits 15 and 31: the exponents that are all ones
  auto special = [](uint32_t v) { return ((v & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u32x4 v = __builtin_bit_cast(u32x4, f[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= special(v[j]);
  }
  if (__ballot(any != 0) == 0) return false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 v = __builtin_bit_cast(u32x4, f[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] &= ~((special(v[j]) >> 15) * 0xffffu);
    f[i] = __builtin_bit_cast(i16x8, v);
  }
  return true;
}

// add_specials' share of one row of V
template <int NE>
__device__ __forceinline__ void add_special_row(const char* v, bool sees, int half, f32x16 (&acc)[NE]) {
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const bf16x4 u = *reinterpret_cast<const bf16x4*>(v + 2 * out_col0(e, i4, half));
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[e][i4 * 4 + k] += sees && !(fabsf((float)u[k]) < INFINITY) ? (float)u[k] : 0.f;
    }
}

// Where the rows of an item are (bf16), in bytes: its pages' and its own (kSeeTree) rows of the KV head
struct ItemBase {
  const char *k, *v, *k_own, *v_own;
  int64_t page;
  uint32_t stride, stride_own, row_mask;
};
template <int SEES>
__device__ __forceinline__ ItemBase item_base(const PagedAttnParams& p, const PagedItem& w) {
  ItemBase r{};
  const PagedCache& c = p.cache;
  const int64_t at = 2 * (w.g * c.sh);
  r.k = (const char*)p.k_pages + at;
  r.v = (const char*)p.v_pages + at;
  r.page = 2 * c.sp;
  r.stride = (uint32_t)(c.sr * 2);
  r.row_mask = (1u << c.page_shift) - 1;
  if (SEES == kSeeTree) {
    const int64_t own = 2 * (w.b * p.blk_sb + w.g * p.blk_sh);
    r.k_own = (const char*)p.k_blk + own;
    r.v_own = (const char*)p.v_blk + own;
    r.stride_own = (uint32_t)(p.blk_sr * 2);
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
