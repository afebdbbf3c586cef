// Norm of each query and key head and rotation by position in one pass: what turns a projection into the q_blk and k_in of a block
// step.  y = x / sqrt(mean(x^2) + eps) * w per head, then each pair (a, b) of frequency f becomes (a cos t - b sin t, a sin t + b cos t), t =
// position * inv_freq[f].  fp32 throughout, one rounding at the end; t in 64 bits, reduced to a part of a turn, because 32 bits leave of an angle of
// 10^5 no more than 2^-7, and what rounding that part to 32 bits leaves off goes into its sine and cosine.
//
// Bound by memory.  A lane holds the two 16-byte pieces of a head that are turned into each other, 4 to 16 lanes a head, and a wavefront
// 4 to 16 heads of one position, so that an angle is computed once by one lane and handed to the others.
#include "mfma_tile.h"

namespace sdllm {

namespace {

constexpr int kRopeThreads = 256;   // at most

template <typename T> struct Piece;
template <> struct Piece<__bf16> { using Vec = bf16x8; static constexpr int N = 8; };
template <> struct Piece<float> { using Vec = f32x4; static constexpr int N = 4; };

template <bool NT, class V> __device__ __forceinline__ V read(const V* at) { return NT ? __builtin_nontemporal_load(at) : *at; }
template <bool NT, class V> __device__ __forceinline__ void write(const V& v, V* at) {
  if constexpr (NT) __builtin_nontemporal_store(v, at);
  else *at = v;
}

template <typename T, int HD, bool NT>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(const QkParams p) {
  using Vec = typename Piece<T>::Vec;
  constexpr int N = Piece<T>::N;
  constexpr int kLanes = HD / (2 * N);         // of a head
  constexpr int kHeads = kWave / kLanes;       // of a wavefront at a time
  const int lane = threadIdx.x & 63;
  const int wave = blockIdx.x * (blockDim.x / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int token = wave / p.parts, part = wave - token * p.parts;
  if (token >= p.tokens) return;
  const int b = p.by_rows.quotient(token), row = token - b * p.rows;
  const int sub = lane % kLanes, slot = lane / kLanes;

  // one angle per lane
  const int freqs = p.rot >> 1;
  float cs = 1.f, sn = 0.f;
  if (lane < freqs) {
    const int position = p.positions ? p.positions[b * p.pos_stride + row] : p.pos_begin + row;
    double turns = (double)position * (double)p.inv_freq[lane] * 0.15915494309189533577;
    turns -= rint(turns);
    // in half turns, as a float and what that leaves off: sine and cosine of their sum, to first order
    const double half_turns = 2.0 * turns;
    const float near = (float)half_turns, rest = 3.14159265f * (float)(half_turns - (double)near);
    float s0, c0;
    sincospif(near, &s0, &c0);
    sn = __builtin_fmaf(c0, rest, s0);
    cs = __builtin_fmaf(-s0, rest, c0);
  }
  float c[N], s[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = __shfl(cs, sub * N + i);
    s[i] = __shfl(sn, sub * N + i);
  }
  // pieces: the two halves of the turned channels, then what is left in order; or neighbours
  const int half = p.rot / (2 * N);
  const bool turned = sub < half;
  const int first = (p.adjacent || !turned ? 2 * sub : sub) * N, second = (p.adjacent || !turned ? 2 * sub + 1 : sub + half) * N;

  const int heads = p.hq + p.hkv;
  for (int h0 = part * kHeads; h0 < heads; h0 += p.parts * kHeads) {
    const int h = h0 + slot;
    const bool there = h < heads, is_q = h < p.hq;
    const int hh = is_q ? h : h - p.hq;
    float x[2 * N];
    if (there) {
      const T* src = is_q ? (const T*)p.q_in + b * p.qi_sb + hh * p.qi_sh + row * p.qi_sr : (const T*)p.k_in + b * p.ki_sb + hh * p.ki_sh + row * p.ki_sr;
      const Vec u = read<NT>(reinterpret_cast<const Vec*>(src + first)), v = read<NT>(reinterpret_cast<const Vec*>(src + second));
#pragma unroll
      for (int i = 0; i < N; ++i) { x[i] = (float)u[i]; x[N + i] = (float)v[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) x[i] = 0.f;
    }
    if (p.norm) {
      // mean(x^2) + eps, with eps f^2 for rows that were multiplied by f
      auto mean_square = [&](float eps) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, o);
        return __builtin_fmaf(sum, 1.f / HD, eps);
      };
      float ms = mean_square(p.eps);
      // Rows whose squares are not numbers of fp32, or are so small that they lose bits, are brought near 1 by a power of two first: elements up to
      // 2^128 become 2^58, ones below 2^-41 up to 2^59.  All lanes go in for one row, the others with a factor of 1.  The test is 0.05 of 2.9 us for a
      // block's rows.
      if (__ballot(!(ms >= 0x1p-90f && ms <= 0x1p120f)) != 0) {
        const float f = ms >= 0x1p-90f ? ms <= 0x1p120f ? 1.f : 0x1p-70f : 0x1p100f;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) x[i] *= f;
        ms = mean_square(p.eps * f * f);
      }
      const float r = 1.f / sqrtf(ms);
      const T* w = (const T*)(is_q ? p.q_weight : p.k_weight);
      if (w) {
        const Vec u = *reinterpret_cast<const Vec*>(w + first), v = *reinterpret_cast<const Vec*>(w + second);
#pragma unroll
        for (int i = 0; i < N; ++i) { x[i] = x[i] * r * (float)u[i]; x[N + i] = x[N + i] * r * (float)v[i]; }
      } else {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) x[i] *= r;
      }
    }
    if (turned) {
      if (p.adjacent) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float a = x[2 * i], bb = x[2 * i + 1];
          x[2 * i] = a * c[i] - bb * s[i];
          x[2 * i + 1] = a * s[i] + bb * c[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float a = x[i], bb = x[N + i];
          x[i] = a * c[i] - bb * s[i];
          x[N + i] = a * s[i] + bb * c[i];
        }
      }
    }
    if (there) {
      T* dst = is_q ? (T*)p.q_out + b * p.qo_sb + hh * p.qo_sh + row * p.qo_sr : (T*)p.k_out + b * p.ko_sb + hh * p.ko_sh + row * p.ko_sr;
      Vec u, v;
#pragma unroll
      for (int i = 0; i < N; ++i) { u[i] = (T)x[i]; v[i] = (T)x[N + i]; }
      write<NT>(u, reinterpret_cast<Vec*>(dst + first));
      write<NT>(v, reinterpret_cast<Vec*>(dst + second));
    }
  }
}

template <typename T, int HD>
hipError_t launch_as(const QkParams& q, hipStream_t s) {
  QkParams p = q;
  constexpr int kHeads = kWave * 2 * Piece<T>::N / HD;
  const int passes = (p.hq + p.hkv + kHeads - 1) / kHeads;
  // wavefronts per position: until there are four for every SIMD
  p.parts = 1;
  while (p.parts < passes && (int64_t)p.tokens * p.parts < 16 * kNumCUs) p.parts *= 2;
  if (p.parts > passes) p.parts = passes;
  const int64_t waves = (int64_t)p.tokens * p.parts;
  // Few wavefronts are a workgroup each, spread over all CUs (32 x 32 heads 3.33 -> 3.03 us, 666 x 16 of 64 floats 3.50 -> 3.37); many
  // are not (8 x 4352 x 64: 205 us, 218 each for itself).
  const int threads = waves <= 16 * kNumCUs ? kWave : kRopeThreads;
  const dim3 grid((uint32_t)((waves * kWave + threads - 1) / threads)), block(threads);
  // Past the caches where what is written does not stay there anyway: 8 x 4352 x 64 heads, 1.14 GB, 222 -> 205 us; 666 x 16 heads of 64
  // floats, 5.5 MB, 3.5 -> 3.7.
  const int64_t bytes = (int64_t)p.tokens * (p.hq + p.hkv) * HD * sizeof(T) * 2;
  return bytes >= (int64_t)256 << 20 ? launch(qk_norm_rope_kernel<T, HD, true>, grid, block, 0, s, p) : launch(qk_norm_rope_kernel<T, HD, false>, grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == 0) return d == 128 ? launch_as<__bf16, 128>(p, s) : launch_as<__bf16, 64>(p, s);
  return d == 128 ? launch_as<float, 128>(p, s) : launch_as<float, 64>(p, s);
}

}  // namespace sdllm
