// Tiles of the paged cache in LDS and what the matrix cores make of them.
#pragma once

#include "paged_place.h"

namespace sdllm {

// 32 keys by C query columns of tensors of type E on the matrix cores: K rows as the A operand of the logits, V columns through the transposing LDS read as that of the second
// product, P^T as its B operand.  A tile of one tensor comes as fetches of 1 KB of consecutive LDS, each of whole rows in order; which 16-byte
// piece of its row a lane brings is free: row r holds piece c of K in place c ^ k_turn(r), of V in place c ^ v_turn(r), which keeps the operand
// reads off each other's banks.
template <typename E, int HD>
struct Tile {
  static constexpr int kRow = HD * (int)sizeof(E), kBytes = kTileKeys * kRow;
  static constexpr int kPieces = kRow / 16;             // of a row
  static constexpr int kRowsPerFetch = kWave / kPieces, kFetches = kTileKeys / kRowsPerFetch;
};

typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
__device__ __forceinline__ i16x8 transposed(const uint8_t* lo, const uint8_t* hi) {
  return __builtin_shufflevector(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)lo), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)hi), 0, 1, 2, 3, 4, 5,
                                 6, 7);
}

template <typename E, int HD, int C>
struct Math;

// Fragments as in attn_tile_math.h: lane (col, half) holds keys 8 (i / 4) + 4 half + i % 4 of its column.
template <int HD>
struct Math<__bf16, HD, 32> : Tile<__bf16, HD> {
  using T = Tile<__bf16, HD>;
  using Q = bf16x8;
  using K = bf16x8;
  using V = i16x8;
  using P = bf16x8;
  using Acc = f32x16;
  static constexpr int NQ = HD / 16, NK = HD / 16, NV = HD / 16, NS = 16, NA = HD / 32, NB = 2, kSlots = NA * 4;
  static __device__ __forceinline__ int k_turn(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int v_turn(int r) { return HD == 128 ? (r & 3) << 2 : (r & 2) << 1; }
  static __device__ __forceinline__ int key_base(int lane) { return 4 * (lane >> 5); }
  static __device__ __forceinline__ int key(int i) { return 8 * (i >> 2) + (i & 3); }
  static __device__ __forceinline__ int q_piece(int i, int lane) { return 2 * i + (lane >> 5); }
  static __device__ __forceinline__ float over_row(float v, bool sum) {
    const float o = __shfl_xor(v, 32);
    return sum ? v + o : fmaxf(v, o);
  }
  static __device__ __forceinline__ void read_k(const uint8_t* tile, int lane, bf16x8 (&a)[NK]) {
    const int half = lane >> 5, col = lane & 31;
    const uint32_t at = (uint32_t)(col * T::kRow + ((half ^ k_turn(col)) << 4));
#pragma unroll
    for (int i = 0; i < NK; ++i) a[i] = *reinterpret_cast<const bf16x8*>(tile + (at ^ (uint32_t)(i * 32)));
  }
  static __device__ __forceinline__ void read_v(const uint8_t* tile, int lane, i16x8 (&f)[NV]) {
    const int half = lane >> 5, grp = (lane >> 4) & 1, s16 = lane & 15, r = half * 4 + (s16 >> 2);
    const uint32_t at = (uint32_t)(r * T::kRow + ((v_turn(r) << 4) ^ (grp * 32 + (s16 & 3) * 8)));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint8_t* from = tile + (at ^ (uint32_t)(i % NA * 64)) + i / NA * 16 * T::kRow;
      f[i] = transposed(from, from + 8 * T::kRow);
    }
  }
  static __device__ __forceinline__ void logits(const bf16x8 (&a)[NK], const bf16x8 (&q)[NQ], float (&s)[NS]) {
    f32x16 c;
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], q[i], c, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = c[i];
  }
  static __device__ __forceinline__ void product(const i16x8 (&f)[NV], const bf16x8 (&pb)[NB], Acc (&acc)[NA]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      acc[i % NA] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[i]), pb[i / NA], acc[i % NA], 0, 0, 0);
  }
  // slot i: four results of consecutive channels, the first of them channel()
  static __device__ __forceinline__ f32x4 slot(const Acc (&acc)[NA], int i) {
    return {acc[i >> 2][(i & 3) * 4], acc[i >> 2][(i & 3) * 4 + 1], acc[i >> 2][(i & 3) * 4 + 2], acc[i >> 2][(i & 3) * 4 + 3]};
  }
  static __device__ __forceinline__ void add(Acc (&acc)[NA], int i, const f32x4& z) {
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[i >> 2][(i & 3) * 4 + k] += z[k];
  }
  static __device__ __forceinline__ int channel(int i, int lane) { return out_col0(i >> 2, i & 3, lane >> 5); }
  static constexpr int kCols = 32;                      // lane l holds results of column l % kCols
};

// 16 columns: half the work of a tile.  Row 4 q + r of half h of the logits is key 8 q + 4 h + r, so that lane (col, q) holds keys 8 q .. 8 q + 7 of its
// column, as the second product takes them.
template <int HD>
struct Math<__bf16, HD, 16> : Tile<__bf16, HD> {
  using T = Tile<__bf16, HD>;
  using Q = bf16x8;
  using K = bf16x8;
  using V = i16x8;
  using P = bf16x8;
  using Acc = f32x4;
  static constexpr int NQ = HD / 32, NK = HD / 16, NV = HD / 16, NS = 8, NA = HD / 16, NB = 1, kSlots = NA;
  static __device__ __forceinline__ int k_turn(int r) { return HD == 128 ? (r & 3) | (r >> 3) << 2 : ((r >> 1) & 1) | (r >> 3) << 1; }
  static __device__ __forceinline__ int v_turn(int r) { return HD == 128 ? (r & 3) << 1 | (r & 8) : (r & 2) | (r & 8) >> 1; }
  static __device__ __forceinline__ int key_base(int lane) { return 8 * (lane >> 4); }
  static __device__ __forceinline__ int key(int i) { return i; }
  static __device__ __forceinline__ int q_piece(int i, int lane) { return 4 * i + (lane >> 4); }
  static __device__ __forceinline__ float over_row(float v, bool sum) {
#pragma unroll
    for (int o = 16; o < kWave; o <<= 1) {
      const float x = __shfl_xor(v, o);
      v = sum ? v + x : fmaxf(v, x);
    }
    return v;
  }
  static __device__ __forceinline__ void read_k(const uint8_t* tile, int lane, bf16x8 (&a)[NK]) {
    const int q = lane >> 4, m = lane & 15, r = 8 * (m >> 2) + (m & 3);   // and r + 4, whose pieces turn alike
    const uint32_t at = (uint32_t)(r * T::kRow + ((q ^ k_turn(r)) << 4));
#pragma unroll
    for (int i = 0; i < NK; ++i) a[i] = *reinterpret_cast<const bf16x8*>(tile + (at ^ (uint32_t)(i / 2 * 64)) + i % 2 * 4 * T::kRow);
  }
  static __device__ __forceinline__ void read_v(const uint8_t* tile, int lane, i16x8 (&f)[NV]) {
    const int q = lane >> 4, s16 = lane & 15, r = 8 * q + (s16 >> 2);     // and r + 4
    const uint32_t at = (uint32_t)(r * T::kRow + ((v_turn(r) << 4) ^ ((s16 & 3) * 8)));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint8_t* from = tile + (at ^ (uint32_t)(i * 32));
      f[i] = transposed(from, from + 4 * T::kRow);
    }
  }
  static __device__ __forceinline__ void logits(const bf16x8 (&a)[NK], const bf16x8 (&q)[NQ], float (&s)[NS]) {
    f32x4 c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < NK; ++i) c[i % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], q[i / 2], c[i % 2], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = c[i >> 2][i & 3];
  }
  static __device__ __forceinline__ void product(const i16x8 (&f)[NV], const bf16x8 (&pb)[NB], Acc (&acc)[NA]) {
#pragma unroll
    for (int i = 0; i < NA; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[i]), pb[0], acc[i], 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 slot(const Acc (&acc)[NA], int i) { return acc[i]; }
  static __device__ __forceinline__ void add(Acc (&acc)[NA], int i, const f32x4& z) { acc[i] += z; }
  static __device__ __forceinline__ int channel(int i, int lane) { return 16 * i + 4 * (lane >> 4); }
  static constexpr int kCols = 16;
};

// fp32: lane (col, part) holds keys 16 (i / 4) + 4 part + i % 4 of its column.  The order in which channels are contracted is free: a 16-byte piece of a row is
// four operands, of the logits four channels of a key, of the second product four columns of V, so that results are columns 64 c + 4 m + e for row m of product 4 c + e.
template <int HD>
struct Math<float, HD, 16> : Tile<float, HD> {
  using T = Tile<float, HD>;
  using Q = f32x4;
  using K = f32x4;
  using V = f32x4;
  using P = f32x4;
  using Acc = f32x4;
  static constexpr int NQ = HD / 16, NK = HD / 8, NV = HD / 8, NS = 8, NA = HD / 16, NB = 2, kSlots = NA;
  static __device__ __forceinline__ int k_turn(int r) { return r & 15; }
  static __device__ __forceinline__ int v_turn(int) { return 0; }
  static __device__ __forceinline__ int key_base(int lane) { return 4 * (lane >> 4); }
  static __device__ __forceinline__ int key(int i) { return 16 * (i >> 2) + (i & 3); }
  static __device__ __forceinline__ int q_piece(int i, int lane) { return 4 * i + (lane >> 4); }
  static __device__ __forceinline__ float over_row(float v, bool sum) { return Math<__bf16, HD, 16>::over_row(v, sum); }
  static __device__ __forceinline__ void read_k(const uint8_t* tile, int lane, f32x4 (&a)[NK]) {
    const int part = lane >> 4, col = lane & 15;
    const uint32_t at = (uint32_t)(col * T::kRow + ((part ^ k_turn(col)) << 4));
#pragma unroll
    for (int i = 0; i < NK; ++i) a[i] = *reinterpret_cast<const f32x4*>(tile + (at ^ (uint32_t)(i / 2 * 64)) + i % 2 * 16 * T::kRow);   // keys col and 16 + col
  }
  static __device__ __forceinline__ void read_v(const uint8_t* tile, int lane, f32x4 (&f)[NV]) {
    const uint8_t* from = tile + 4 * (lane >> 4) * T::kRow + (lane & 15) * 16;
#pragma unroll
    for (int i = 0; i < NV; ++i) f[i] = *reinterpret_cast<const f32x4*>(from + key(i & 7) * T::kRow + (i >> 3) * 256);
  }
  static __device__ __forceinline__ void logits(const f32x4 (&a)[NK], const f32x4 (&q)[NQ], float (&s)[NS]) {
    f32x4 c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) c[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[2 * t + h][k], q[t][k], c[h], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = c[i >> 2][i & 3];
  }
  static __device__ __forceinline__ void product(const f32x4 (&f)[NV], const f32x4 (&pb)[NB], Acc (&acc)[NA]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < NA; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[(e >> 2) * 8 + i][e & 3], pb[i >> 2][i & 3], acc[e], 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 slot(const Acc (&acc)[NA], int i) {
    const int e = i & ~3, r = i & 3;
    return {acc[e][r], acc[e + 1][r], acc[e + 2][r], acc[e + 3][r]};
  }
  static __device__ __forceinline__ void add(Acc (&acc)[NA], int i, const f32x4& z) {
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[(i & ~3) + k][i & 3] += z[k];
  }
  static __device__ __forceinline__ int channel(int i, int lane) { return 64 * (i >> 2) + 16 * (lane >> 4) + 4 * (i & 3); }
  static constexpr int kCols = 16;
};

// Results of a share, as the lanes of a wave hold them: [share][kCols columns of its block][slot][lane], so that a wave writes 1 KB at a time
template <class M>
__device__ __forceinline__ f32x4* partial_slot(const PagedAttnParams& p, int64_t share, int cols, int i, int lane) {
  return reinterpret_cast<f32x4*>(p.part_o) + ((share * (p.block_cols / M::kCols) + cols) * M::kSlots + i) * kWave + lane;
}

}  // namespace sdllm
