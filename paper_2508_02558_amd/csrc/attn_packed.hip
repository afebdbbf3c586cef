// Block-query attention over a cache of 4 bits a value (packed_tile.h) and the block's own keys and values (Alg. 3, cache_state == 2).
//
// The query rows of the heads of a KV head are one list of columns (head, row); 32 of them are a 32x32 matrix block, whatever the block length, so
// that single tokens of grouped heads share one.  A wavefront owns 32 columns and takes tiles of 32 keys: its lanes' own bytes of the
// tile come straight from memory (no LDS), eight codes turn into one operand of v_mfma_f32_32x32x16_bf16 by four conversions, and
//   logits^T = K_tile Q^T   (K rows as A operand: a lane holds sixteen logits of one column),
//   O^T += V_tile^T P^T     (V codes lie in the order of those sixteen logits),
// with the running maximum and sum of a softmax.  The numbers of the cache are bf16 numbers, so for fp32 tensors the queries and the
// probabilities enter as the sum of three bf16 parts, all 24 bits of them: three times the products, and exact ones.
// Keys are split over the wavefronts of a workgroup, merged through LDS, and over workgroups, whose partials a second launch folds.
#include "attn_merge.h"
#include "attn_tile_math.h"
#include "packed_tile.h"

namespace sdllm {

namespace {

constexpr int kCols = 32;

// Upper halves of the bits of eight floats
__device__ __forceinline__ bf16x8 upper_halves(const uint32_t (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = x[2 * i] >> 16 | (x[2 * i + 1] & 0xffff0000u);
  return __builtin_bit_cast(bf16x8, w);
}

// bf16 numbers whose sum the numbers are: one, for those that are bf16 or may be rounded to it, or three, which hold the 24 bits of any float
// (eight each, cut off and not rounded, so that the largest float stays one).  An infinity is its first part.
template <int PARTS>
__device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8 (&part)[PARTS]) {
  if constexpr (PARTS == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) part[0][i] = (__bf16)x[i];
  } else {
    float rest[8];
    uint32_t bits[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int n = 0; n < PARTS; ++n) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bits[i] = __builtin_bit_cast(uint32_t, rest[i]);
        const float cut = __builtin_bit_cast(float, bits[i] & 0xffff0000u);
        rest[i] = n == 0 && __builtin_isinf(x[i]) ? 0.f : rest[i] - cut;
      }
      part[n] = upper_halves(bits);
    }
  }
}

// The same with zeros for infinities, for products with further parts: infinity times a part that is 0 would be NaN where infinity
// times the number is not.
__device__ __forceinline__ bf16x8 without_infinities(const bf16x8& x) {
  u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7fffu) == 0x7f80u) w[i] &= 0xffff0000u;
    if ((w[i] & 0x7fff0000u) == 0x7f800000u) w[i] &= 0xffffu;
  }
  return __builtin_bit_cast(bf16x8, w);
}

template <typename T> struct Parts;
template <> struct Parts<__bf16> { static constexpr int N = 1, kWaves = kPackedWavesBf16; };
template <> struct Parts<float> { static constexpr int N = 3, kWaves = kPackedWavesF32; };

// Eight consecutive numbers of a row
__device__ __forceinline__ void load8(const __bf16* at, bf16x8 (&part)[1]) { part[0] = *reinterpret_cast<const bf16x8*>(at); }
__device__ __forceinline__ void load8(const float* at, bf16x8 (&part)[3]) {
  const f32x4 lo = reinterpret_cast<const f32x4*>(at)[0], hi = reinterpret_cast<const f32x4*>(at)[1];
  const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  split_parts(x, part);
}

__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Products of parts down to 2^-24 of the first one, the small ones first
template <int PARTS>
__device__ __forceinline__ f32x16 mfma_parts(const bf16x8 (&a)[PARTS], const bf16x8 (&b)[PARTS], f32x16 c) {
  if constexpr (PARTS == 3) {
    const bf16x8 a0 = without_infinities(a[0]);
    c = mfma(a[2], b[0], c);
    c = mfma(a[1], b[1], c);
    c = mfma(a0, b[2], c);
    c = mfma(a[1], b[0], c);
    c = mfma(a0, b[1], c);
  }
  return mfma(a[0], b[0], c);
}

// A tile as its lanes fetch it
template <int HD>
struct RawTile {
  u32x4 k[PackedLayout<HD>::kLoads], v[PackedLayout<HD>::kLoads];
  uint32_t ks, vs;                                       // scale bytes: groups of the lane's key, channels of its value rows

  __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
    using L = PackedLayout<HD>;
    const int m = lane & 31;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) k[i] = *reinterpret_cast<const u32x4*>(tile + L::kKeys + (i * 64 + lane) * 16);
    if constexpr (HD == 128) {
      ks = *reinterpret_cast<const uint32_t*>(tile + L::kKeyScales + m * 4);
      vs = *reinterpret_cast<const uint32_t*>(tile + L::kValueScales + m * 4);
    } else {
      ks = *reinterpret_cast<const uint16_t*>(tile + L::kKeyScales + m * 2);
      vs = *reinterpret_cast<const uint16_t*>(tile + L::kValueScales + m * 2);
    }
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) v[i] = *reinterpret_cast<const u32x4*>(tile + L::kValues + (i * 64 + lane) * 16);
  }
};

// Softmax of a tile's raw logits against the running reference: s becomes the numerators.
template <int NE>
__device__ __forceinline__ void softmax_step(f32x16& s, int rows, float scale_log2, int half, float& m_ref, float& l_run, f32x16 (&acc)[NE]) {
  const float m_loc = tile_mask_max(s, rows, scale_log2, half);
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
  float l_loc = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -m_ref));
    l_loc += s[i];
  }
  l_run += l_loc;
}

template <int PARTS>
__device__ __forceinline__ void prob_parts(const f32x16& s, bf16x8 (&pb)[2][PARTS]) {
#pragma unroll
  for (int st = 0; st < 2; ++st) {
    const float x[8] = {s[8 * st], s[8 * st + 1], s[8 * st + 2], s[8 * st + 3], s[8 * st + 4], s[8 * st + 5], s[8 * st + 6], s[8 * st + 7]};
    split_parts(x, pb[st]);
  }
}

template <int HD> constexpr int park_row() { return 16 * (HD / 32) * 4 + 16; }
template <int HD> constexpr int wave_lds() { return 64 * park_row<HD>() + 64 * 4; }

template <typename T, int HD>
__global__ __launch_bounds__(Parts<T>::kWaves * kWave) void attn_packed_kernel(const PackedAttnParams p) {
  using L = PackedLayout<HD>;
  constexpr int PARTS = Parts<T>::N, NE = L::kGroups, NF = HD / 16;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int half = lane >> 5, m = lane & 31;

  // columns of a KV head and split side by side on an XCD: they read the same tiles
  const int wg = xcd_contiguous_id(blockIdx.x, gridDim.x);
  const int pair = wg / p.col_tiles, ct = wg - pair * p.col_tiles;
  const int bg = pair / p.n_split, split = pair - bg * p.n_split;
  const int b = bg / p.hkv, g = bg - b * p.hkv;
  const int t_end = min(p.blk_tiles + p.tiles, (split + 1) * p.tiles_per_split);

  const int col = min(ct * kCols + m, p.cols - 1);       // past the end: the last column again, not stored
  const int h = g * p.group + col / p.nq, row = col - col / p.nq * p.nq;

  const uint8_t* cache = p.cache + (size_t)bg * p.head_bytes;
  // tiles: those of the block, then those of the cache
  int t = split * p.tiles_per_split + wave;
  RawTile<HD> next;
  int t_cached = t;                                      // first tile of the cache that the wave takes
  while (t_cached < p.blk_tiles) t_cached += nw;
  if (t_cached < t_end) next.load(cache + (size_t)(t_cached - p.blk_tiles) * L::kTile, lane);

  // Q^T operands: fragment 4 i + st holds channels 32 (2 i + half) + 8 st ..
  bf16x8 qf[NF][PARTS];
  const T* q = (const T*)p.q + b * p.q_sb + h * p.q_sh + row * p.q_sr;
#pragma unroll
  for (int f = 0; f < NF; ++f) load8(q + 32 * (2 * (f >> 2) + half) + 8 * (f & 3), qf[f]);

  f32x16 acc[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  float m_ref = kNoMax, l_run = 0.f;

  for (; t < t_end && t < p.blk_tiles; t += nw) {        // the block's own rows, from memory as they lie there
    const int first = t * kTileKeys, n = min(kTileKeys, p.nq - first);
    const size_t base = b * p.blk_sb + g * p.blk_sh + (size_t)first * p.blk_sr;
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    const T* k = (const T*)p.k_blk + base + (size_t)min(m, n - 1) * p.blk_sr;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      bf16x8 kf[PARTS];
      load8(k + 32 * (2 * (f >> 2) + half) + 8 * (f & 3), kf);
      s = mfma_parts(kf, qf[f], s);
    }
    softmax_step<NE>(s, n, p.scale_log2, half, m_ref, l_run, acc);
    bf16x8 pb[2][PARTS];
    prob_parts<PARTS>(s, pb);
    // a lane takes HD / 32 neighbouring channels of each of its sixteen keys
    typedef __attribute__((ext_vector_type(HD / 32))) T Few;
    Few v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = 8 * (r >> 2) + 4 * half + (r & 3);
      v[r] = *reinterpret_cast<const Few*>((const T*)p.v_blk + base + (size_t)min(key, n - 1) * p.blk_sr + m * NE);
      if (key >= n) v[r] = Few(0);
    }
#pragma unroll
    for (int e = 0; e < NE; ++e)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const float x[8] = {(float)v[8 * st][e],     (float)v[8 * st + 1][e], (float)v[8 * st + 2][e], (float)v[8 * st + 3][e],
                            (float)v[8 * st + 4][e], (float)v[8 * st + 5][e], (float)v[8 * st + 6][e], (float)v[8 * st + 7][e]};
        bf16x8 vf[PARTS];
        split_parts(x, vf);
        acc[e] = mfma_parts(vf, pb[st], acc[e]);
      }
  }

  for (; t < t_end; t += nw) {
    const RawTile<HD> raw = next;
    if (t + nw < t_end) next.load(cache + (size_t)(t + nw - p.blk_tiles) * L::kTile, lane);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const float scale = scale_of_byte(raw.ks >> (8 * half), 2 * i);
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const bf16x8 kf = unpack8(raw.k[i][st], scale);
#pragma unroll
        for (int n = PARTS - 1; n >= 0; --n) s = mfma(kf, qf[4 * i + st][n], s);
      }
    }
    softmax_step<NE>(s, p.n_cached - (t - p.blk_tiles) * kTileKeys, p.scale_log2, half, m_ref, l_run, acc);
    bf16x8 pb[2][PARTS];
    prob_parts<PARTS>(s, pb);
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const float scale = scale_of_byte(raw.vs, e);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const bf16x8 vf = unpack8(raw.v[e >> 1][2 * (e & 1) + st], scale);
#pragma unroll
        for (int n = PARTS - 1; n >= 0; --n) acc[e] = mfma(vf, pb[st][n], acc[e]);
      }
    }
  }
  const float l_tot = l_run + __shfl_xor(l_run, 32);

  // Merge of the wavefronts: each parks its results, [lane][register i][e] (registers i of all e are neighbouring channels), and its columns'
  // (reference, sum); then wave w folds registers w, w + nw, ... of all of them.
  uint8_t* mine = smem + wave * wave_lds<HD>();
  typedef __attribute__((ext_vector_type(NE))) float Res;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    Res v;
#pragma unroll
    for (int e = 0; e < NE; ++e) v[e] = acc[e][i];
    *reinterpret_cast<Res*>(mine + lane * park_row<HD>() + i * NE * 4) = v;
  }
  float* ml = reinterpret_cast<float*>(mine + 64 * park_row<HD>());
  if (lane < 32) { ml[lane] = m_ref; ml[32 + lane] = l_tot; }
  __syncthreads();
  float m_tot = kNoMax, l_all = 0.f;
  for (int w = 0; w < nw; ++w) m_tot = fmaxf(m_tot, reinterpret_cast<const float*>(smem + w * wave_lds<HD>() + 64 * park_row<HD>())[m]);
  for (int w = 0; w < nw; ++w) {
    const float* of = reinterpret_cast<const float*>(smem + w * wave_lds<HD>() + 64 * park_row<HD>());
    l_all = __builtin_fmaf(of[32 + m], __builtin_amdgcn_exp2f(of[m] - m_tot), l_all);
  }
  const bool stored = ct * kCols + m < p.cols;
  const size_t slot = ((size_t)(bg * p.col_tiles + ct) * p.n_split + split);
  for (int i = wave; i < 16; i += nw) {
    Res o = Res(0.f);
    for (int w = 0; w < nw; ++w) {
      const uint8_t* of = smem + w * wave_lds<HD>();
      const float f = __builtin_amdgcn_exp2f(reinterpret_cast<const float*>(of + 64 * park_row<HD>())[m] - m_tot);
      o += *reinterpret_cast<const Res*>(of + lane * park_row<HD>() + i * NE * 4) * f;
    }
    const int ch = NE * (8 * (i >> 2) + 4 * half + (i & 3));
    if (p.n_split == 1) {
      typedef __attribute__((ext_vector_type(HD / 32))) T Few;
      Few y;
#pragma unroll
      for (int e = 0; e < NE; ++e) y[e] = (T)(o[e] / l_all);
      if (stored) *reinterpret_cast<Few*>((T*)p.out + b * p.o_sb + h * p.o_sh + row * p.o_sr + ch) = y;
    } else {
      *reinterpret_cast<Res*>(p.part_o + (slot * kCols + m) * HD + ch) = o;
    }
  }
  if (p.n_split > 1 && wave == 0 && lane < 32) {
    p.part_ml[slot * 64 + lane] = m_tot;
    p.part_ml[slot * 64 + 32 + lane] = l_all;
  }
}

// One thread folds the splits of four channels of a column.
template <typename T, int HD>
__global__ __launch_bounds__(256) void attn_packed_merge_kernel(const PackedAttnParams p) {
  const int unit = blockIdx.x / (kCols * HD / 4 / 256), at = (blockIdx.x % (kCols * HD / 4 / 256)) * 256 + threadIdx.x;
  const int m = at / (HD / 4), c4 = at % (HD / 4) * 4;
  const int bg = unit / p.col_tiles, ct = unit - bg * p.col_tiles;
  const int col = ct * kCols + m;
  if (col >= p.cols) return;
  const size_t slot = (size_t)unit * p.n_split;
  const RowPiece r = fold_splits<kCols>(p.part_ml + slot * 64 + m, p.part_o + (slot * kCols + m) * HD + c4, (size_t)kCols * HD, p.n_split, 0, 1);
  const int b = bg / p.hkv, g = bg - b * p.hkv, h = g * p.group + col / p.nq, row = col % p.nq;
  store_piece<T>(r, (T*)p.out + b * p.o_sb + h * p.o_sh + row * p.o_sr + c4);
}

template <typename T, int HD>
hipError_t launch_as(const PackedAttnParams& p, hipStream_t s) {
  const int units = p.batch * p.hkv * p.col_tiles;
  const size_t lds = (size_t)p.waves * wave_lds<HD>();
  static LdsOptIn opt;
  hipError_t e = opt.ensure(reinterpret_cast<const void*>(attn_packed_kernel<T, HD>), Parts<T>::kWaves * wave_lds<HD>());
  if (e != hipSuccess) return e;
  e = launch(attn_packed_kernel<T, HD>, dim3((uint32_t)units * p.n_split), dim3(p.waves * kWave), lds, s, p);
  if (e != hipSuccess || p.n_split == 1) return e;
  return launch(attn_packed_merge_kernel<T, HD>, dim3((uint32_t)units * (kCols * HD / 4 / 256)), dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_attn_packed(const PackedAttnParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == 0) return d == 128 ? launch_as<__bf16, 128>(p, s) : launch_as<__bf16, 64>(p, s);
  return d == 128 ? launch_as<float, 128>(p, s) : launch_as<float, 64>(p, s);
}

}  // namespace sdllm
