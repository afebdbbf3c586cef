// The cache of 4 bits a value (packed_tile.h): gathering the retained rows into it (Alg. 1 steps 12-14, with each value rounded to the
// numbers of the cache), and reading it back as rows.  Bound by memory: 3.76 bytes of bf16 rows come or go for each byte of cache.
#include "packed_tile.h"

namespace sdllm {

namespace {

constexpr int kPackThreads = 64;   // a wavefront to a workgroup, which is gone as soon as it is done: 8 x 32 heads x 2160 rows and back 129 us, with four 132

// bits of a number as float, sign off
template <typename T> __device__ __forceinline__ uint32_t magnitude(T x) { return __builtin_bit_cast(uint32_t, (float)x) & 0x7fffffffu; }

template <typename T> struct Pieces;   // 16 bytes of a row, and two numbers
template <> struct Pieces<__bf16> { using Vec = bf16x8; using Pair = bf16x2; static constexpr int N = 8; };
template <> struct Pieces<float> { using Vec = f32x4; using Pair = f32x2; static constexpr int N = 4; };

__device__ __forceinline__ float power_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

template <int DPP>
__device__ __forceinline__ uint32_t lane_move(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP, 0xf, 0xf, false); }

// One wavefront packs the keys or the values of one tile: whole rows come with 16 bytes a lane (keys) or two numbers a lane (values, so that a
// lane has all rows of its channels), all requested together; the codes meet in LDS as they lie in the cache and leave with 16
// bytes a lane.  The rows are read past the caches: they are many times what is written.
template <typename T, int HD>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const PackParams p) {
  using L = PackedLayout<HD>;
  using P = Pieces<T>;
  __shared__ __attribute__((aligned(16))) uint8_t codes_lds[L::kValues], scales_lds[HD];
  const int lane = threadIdx.x;
  const bool values = blockIdx.x & 1;
  const int unit = blockIdx.x >> 1;
  const int row = p.by_tiles.quotient(unit), tile = unit - row * p.tiles;      // (batch, KV head), tile of it
  const int b = p.by_hkv.quotient(row), g = row - b * p.hkv;
  const int first = tile * kTileKeys, n = min(kTileKeys, p.n - first);
  const int named = p.idx[(size_t)row * p.n + first + min(lane & 31, n - 1)];
  const int picked = min(max(named, 0), p.seq_len - 1);   // never leave the source tensor, whatever idx holds
  const size_t base = b * p.s_sb + g * p.s_sh;

  if (!values) {
    // the lanes of a group of 32 channels are neighbours
    constexpr int kPerRow = HD / P::N, kRows = kWave / kPerRow, kLoads = kTileKeys / kRows;   // lanes of a key, keys of a request
    typename P::Vec k[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int key = j * kRows + lane / kPerRow;
      k[j] = __builtin_nontemporal_load(reinterpret_cast<const typename P::Vec*>((const T*)p.k + base + (size_t)__shfl(picked, key) * p.s_sr) + lane % kPerRow);
    }
    constexpr int kGroupLanes = 32 / P::N;
    const int group = lane % kPerRow / kGroupLanes, at = lane % kGroupLanes;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int key = j * kRows + lane / kPerRow;
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < P::N; ++c) top = max(top, magnitude(k[j][c]));
      top = max(top, lane_move<0xb1>(top));                // of lanes 1, 0, 3, 2
      top = max(top, lane_move<0x4e>(top));                // 2, 3, 0, 1
      if constexpr (kGroupLanes == 8) top = max(top, lane_move<0x141>(top));   // 7 .. 0
      const bool there = key < n;
      const uint32_t byte = there ? scale_byte(top) : 2;
      const float scale = power_of(byte);
      uint32_t word = 0;
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)k[j][0], (float)k[j][1], scale, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)k[j][2], (float)k[j][3], scale, 1);
      uint8_t* to = codes_lds + (group * 32 + key) * 16;
      if constexpr (P::N == 8) {
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)k[j][4], (float)k[j][5], scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)k[j][6], (float)k[j][7], scale, 3);
        reinterpret_cast<uint32_t*>(to)[at] = there ? word : 0;
      } else {
        reinterpret_cast<uint16_t*>(to)[at] = (uint16_t)(there ? word : 0);
      }
      if (at == 0) scales_lds[key * L::kGroups + group] = (uint8_t)byte;
    }
  } else {
    constexpr int kHalves = HD / 64;                         // of the rows, that a lane takes; with 64 channels those of its half
    const int pair = lane % (HD / 2), half = lane >> 5;
    typename P::Pair v[kHalves][16];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r >> 2) + 4 * (kHalves == 2 ? h : half) + (r & 3);
        const int from = kHalves == 2 ? __builtin_amdgcn_readlane(picked, key) : __shfl(picked, key);
        v[h][r] = __builtin_nontemporal_load(reinterpret_cast<const typename P::Pair*>((const T*)p.v + base + (size_t)from * p.s_sr) + pair);
      }
    uint32_t top[2] = {0, 0}, byte[2];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (n < kTileKeys && 8 * (r >> 2) + (r & 3) >= n - 4 * (kHalves == 2 ? h : half)) v[h][r] = typename P::Pair{0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) top[j] = max(top[j], magnitude(v[h][r][j]));
      }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (kHalves == 1) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
      byte[j] = scale_byte(top[j]);
    }
    // channels 2 pair and 2 pair + 1 are j = 0, 1 of lane m and request i
    const int m = pair / L::kLoads, i = pair % L::kLoads;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      u32x4 codes;
#pragma unroll
      for (int w = 0; w < 4; ++w) {                        // word 2 j + st: rows 8 st .. 8 st + 7 of v
        const int j = w >> 1, r0 = 8 * (w & 1);
        const float scale = power_of(byte[j]);
        uint32_t word = 0;
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)v[h][r0][j], (float)v[h][r0 + 1][j], scale, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)v[h][r0 + 2][j], (float)v[h][r0 + 3][j], scale, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)v[h][r0 + 4][j], (float)v[h][r0 + 5][j], scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)v[h][r0 + 6][j], (float)v[h][r0 + 7][j], scale, 3);
        codes[w] = word;
      }
      *reinterpret_cast<u32x4*>(codes_lds + ((i * 2 + (kHalves == 2 ? h : half)) * 32 + m) * 16) = codes;
    }
    if (kHalves == 2 || half == 0) *reinterpret_cast<uint16_t*>(scales_lds + 2 * pair) = (uint16_t)(byte[0] | byte[1] << 8);
  }

  wave_lds_sync();
  uint8_t* to = p.cache + (size_t)row * p.head_bytes + (size_t)tile * L::kTile;
  uint8_t* codes_to = to + (values ? L::kValues : L::kKeys);
#pragma unroll
  for (int at = 0; at < L::kValues; at += 1024) *reinterpret_cast<u32x4*>(codes_to + at + lane * 16) = *reinterpret_cast<const u32x4*>(codes_lds + at + lane * 16);
  if (lane < HD / 16) *reinterpret_cast<u32x4*>(to + (values ? L::kValueScales : L::kKeyScales) + lane * 16) = *reinterpret_cast<const u32x4*>(scales_lds + lane * 16);
}

// One wavefront unpacks the keys or the values of one tile.
template <typename T, int HD>
__global__ __launch_bounds__(kPackThreads) void unpack_kernel(const PackParams p) {
  using L = PackedLayout<HD>;
  using P = Pieces<T>;
  const int lane = threadIdx.x;
  const int unit = blockIdx.x >> 1;
  const int row = p.by_tiles.quotient(unit), tile = unit - row * p.tiles;
  const int b = p.by_hkv.quotient(row), g = row - b * p.hkv;
  const int first = tile * kTileKeys, n = min(kTileKeys, p.n - first);
  const uint8_t* in = p.cache + (size_t)row * p.head_bytes + (size_t)tile * L::kTile;
  const size_t base = b * p.s_sb + g * p.s_sh + (size_t)first * p.s_sr;

  if (!(blockIdx.x & 1)) {
    // a lane takes eight channels, the lanes of a row are neighbours
    constexpr int kPerRow = HD / 8;
#pragma unroll
    for (int r0 = 0; r0 < kTileKeys; r0 += kWave / kPerRow) {
      const int key = r0 + lane / kPerRow, chunk = lane % kPerRow;
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(in + L::kKeys + ((chunk >> 2) * 32 + key) * 16 + (chunk & 3) * 4);
      const float scale = scale_of_byte(in[L::kKeyScales + key * L::kGroups + (chunk >> 2)], 0);
      const bf16x8 x = unpack8(codes, scale);
      if (key < n) {
        T* dst = (T*)p.k_out + base + (size_t)key * p.s_sr + chunk * 8;
#pragma unroll
        for (int c = 0; c < 8 / P::N; ++c) {
          typename P::Vec y;
#pragma unroll
          for (int u = 0; u < P::N; ++u) y[u] = (T)(float)x[c * P::N + u];
          __builtin_nontemporal_store(y, reinterpret_cast<typename P::Vec*>(dst) + c);
        }
      }
    }
    return;
  }
  // a lane takes HD / 32 neighbouring channels of the sixteen rows of its half
  const int m = lane & 31, half = lane >> 5;
  bf16x8 x[L::kGroups][2];
#pragma unroll
  for (int i = 0; i < L::kLoads; ++i) {
    const u32x4 codes = *reinterpret_cast<const u32x4*>(in + L::kValues + ((i * 2 + half) * 32 + m) * 16);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float scale = scale_of_byte(in[L::kValueScales + m * L::kGroups + 2 * i + j], 0);
#pragma unroll
      for (int st = 0; st < 2; ++st) x[2 * i + j][st] = unpack8(codes[2 * j + st], scale);
    }
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int key = 8 * (r >> 2) + 4 * half + (r & 3);
    if (key < n) {
      typedef __attribute__((ext_vector_type(HD / 32))) T Out;
      Out y;
#pragma unroll
      for (int e = 0; e < L::kGroups; ++e) y[e] = (T)(float)x[e][r >> 3][r & 7];
      __builtin_nontemporal_store(y, reinterpret_cast<Out*>((T*)p.v_out + base + (size_t)key * p.s_sr + m * L::kGroups));
    }
  }
}

template <typename T, int HD>
hipError_t launch_tiles(const PackParams& p, bool pack, hipStream_t s) {
  const dim3 grid((uint32_t)p.rows * p.tiles * 2);
  return launch(pack ? pack_kernel<T, HD> : unpack_kernel<T, HD>, grid, dim3(kPackThreads), 0, s, p);
}

hipError_t launch_any(const PackParams& p, int dtype, int d, bool pack, hipStream_t s) {
  if (dtype == 0) return d == 128 ? launch_tiles<__bf16, 128>(p, pack, s) : launch_tiles<__bf16, 64>(p, pack, s);
  return d == 128 ? launch_tiles<float, 128>(p, pack, s) : launch_tiles<float, 64>(p, pack, s);
}

}  // namespace

hipError_t launch_pack(const PackParams& p, int dtype, int d, hipStream_t s) { return launch_any(p, dtype, d, true, s); }
hipError_t launch_unpack(const PackParams& p, int dtype, int d, hipStream_t s) { return launch_any(p, dtype, d, false, s); }

}  // namespace sdllm
