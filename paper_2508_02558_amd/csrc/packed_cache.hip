// The cache of 4 bits a value (packed_tile.h): gathering the retained rows into it (Alg. 1 steps 12-14, with each value rounded to the
// numbers of the cache), and reading it back as rows.  Bound by memory: 3.76 bytes of bf16 rows come or go for each byte of cache.
#include "packed_tile.h"

namespace sdllm {

namespace {

constexpr int kPackThreads = 256;

// bits of a number as float, sign off
template <typename T> __device__ __forceinline__ uint32_t magnitude(T x) { return __builtin_bit_cast(uint32_t, (float)x) & 0x7fffffffu; }

template <typename T> struct Pieces;   // 16 bytes of a row
template <> struct Pieces<__bf16> { using Vec = bf16x8; using Pair = bf16x2; static constexpr int N = 8; };
template <> struct Pieces<float> { using Vec = f32x4; using Pair = f32x2; static constexpr int N = 4; };

// One wavefront packs one tile.
template <typename T, int HD>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const PackParams p) {
  using L = PackedLayout<HD>;
  using P = Pieces<T>;
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * (kPackThreads / kWave) + (threadIdx.x >> 6);
  if (unit >= p.rows * p.tiles) return;
  const int row = unit / p.tiles, tile = unit - row * p.tiles;      // (batch, KV head), tile of it
  const int b = row / p.hkv, g = row - b * p.hkv;
  const int first = tile * kTileKeys, n = min(kTileKeys, p.n - first);
  const int32_t* idx = p.idx + (size_t)row * p.n + first;
  uint8_t* out = p.cache + (size_t)row * p.head_bytes + (size_t)tile * L::kTile;
  const size_t base = b * p.s_sb + g * p.s_sh;
  const int m = lane & 31, half = lane >> 5;

  {  // keys: a lane takes 32 channels of one key
    const bool there = m < n;
    const char* src = (const char*)p.k + (base + (size_t)idx[there ? m : 0] * p.s_sr) * sizeof(T);
    uint8_t scale_bytes[L::kLoads];
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const int group = 2 * i + half;
      typename P::Vec x[32 / P::N];
#pragma unroll
      for (int c = 0; c < 32 / P::N; ++c) x[c] = reinterpret_cast<const typename P::Vec*>(src + group * 32 * sizeof(T))[c];
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < 32; ++c) top = max(top, magnitude(x[c / P::N][c % P::N]));
      const uint32_t byte = there ? scale_byte(top) : 2;
      const float scale = __builtin_bit_cast(float, byte << 23);
      u32x4 codes;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t word = 0;
        auto at = [&](int c) { return (float)x[(8 * w + c) / P::N][(8 * w + c) % P::N]; };
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, at(0), at(1), scale, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, at(2), at(3), scale, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, at(4), at(5), scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, at(6), at(7), scale, 3);
        codes[w] = there ? word : 0;
      }
      *reinterpret_cast<u32x4*>(out + L::kKeys + (group * 32 + m) * 16) = codes;
      scale_bytes[i] = (uint8_t)byte;
    }
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) out[L::kKeyScales + m * L::kGroups + 2 * i + half] = scale_bytes[i];
  }

  {  // values: a lane takes two neighbouring channels; with 64 of them, of the rows of its half
    constexpr int kHalves = HD / 64;                       // of the rows, that a lane takes
    const int pair = lane % (HD / 2);
    typename P::Pair x[kHalves][16];
    uint32_t top[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r >> 2) + 4 * (kHalves == 2 ? h : half) + (r & 3);
        const bool there = key < n;
        const T* src = (const T*)p.v + base + (size_t)idx[there ? key : 0] * p.s_sr + 2 * pair;
        x[h][r] = *reinterpret_cast<const typename P::Pair*>(src);
        if (!there) x[h][r] = typename P::Pair{0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) top[j] = max(top[j], magnitude(x[h][r][j]));
      }
    uint32_t byte[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (kHalves == 1) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
      byte[j] = scale_byte(top[j]);
    }
    // channels 2 pair and 2 pair + 1 are j = 0, 1 of lane m and request i
    const int lane_m = pair / L::kLoads, i = pair % L::kLoads;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      u32x4 codes;
#pragma unroll
      for (int w = 0; w < 4; ++w) {                        // word 2 j + st: rows 8 st .. 8 st + 7 of x
        const int j = w >> 1, r0 = 8 * (w & 1);
        const float scale = __builtin_bit_cast(float, byte[j] << 23);
        uint32_t word = 0;
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)x[h][r0][j], (float)x[h][r0 + 1][j], scale, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)x[h][r0 + 2][j], (float)x[h][r0 + 3][j], scale, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)x[h][r0 + 4][j], (float)x[h][r0 + 5][j], scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, (float)x[h][r0 + 6][j], (float)x[h][r0 + 7][j], scale, 3);
        codes[w] = word;
      }
      *reinterpret_cast<u32x4*>(out + L::kValues + ((i * 2 + (kHalves == 2 ? h : half)) * 32 + lane_m) * 16) = codes;
    }
    if (kHalves == 2 || half == 0) *reinterpret_cast<uint16_t*>(out + L::kValueScales + 2 * pair) = (uint16_t)(byte[0] | byte[1] << 8);
  }
}

// One wavefront unpacks one tile.
template <typename T, int HD>
__global__ __launch_bounds__(kPackThreads) void unpack_kernel(const PackParams p) {
  using L = PackedLayout<HD>;
  using P = Pieces<T>;
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * (kPackThreads / kWave) + (threadIdx.x >> 6);
  if (unit >= p.rows * p.tiles) return;
  const int row = unit / p.tiles, tile = unit - row * p.tiles;
  const int b = row / p.hkv, g = row - b * p.hkv;
  const int first = tile * kTileKeys, n = min(kTileKeys, p.n - first);
  const uint8_t* in = p.cache + (size_t)row * p.head_bytes + (size_t)tile * L::kTile;
  const size_t base = b * p.s_sb + g * p.s_sh + (size_t)first * p.s_sr;

  // keys: a lane takes eight channels, the lanes of a row are neighbours
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
        reinterpret_cast<typename P::Vec*>(dst)[c] = y;
      }
    }
  }

  // values: a lane takes HD / 32 neighbouring channels of the sixteen rows of its half
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
      *reinterpret_cast<Out*>((T*)p.v_out + base + (size_t)key * p.s_sr + m * L::kGroups) = y;
    }
  }
}

template <typename T, int HD>
hipError_t launch_tiles(const PackParams& p, bool pack, hipStream_t s) {
  const int per_block = kPackThreads / kWave;
  const dim3 grid((uint32_t)(((int64_t)p.rows * p.tiles + per_block - 1) / per_block));
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
