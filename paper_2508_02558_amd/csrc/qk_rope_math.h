// Norm of a head and its rotation by position, as a wavefront does them that holds several heads of one position (qk_norm_rope.hip,
// append_paged.hip).  A lane holds the two 16-byte pieces of a head that are turned into each other, 4 to 16 lanes a head, and a wavefront
// 4 to 16 heads of one position, so that an angle is computed once by one lane and handed to the others.
#pragma once

#include "mfma_tile.h"

namespace sdllm {

template <typename T> struct Piece;
template <> struct Piece<__bf16> { using Vec = bf16x8; static constexpr int N = 8; };
template <> struct Piece<float> { using Vec = f32x4; static constexpr int N = 4; };

template <bool NT, class V> __device__ __forceinline__ V read_piece(const V* at) { return NT ? __builtin_nontemporal_load(at) : *at; }
template <bool NT, class V> __device__ __forceinline__ void write_piece(const V& v, V* at) {
  if constexpr (NT) __builtin_nontemporal_store(v, at);
  else *at = v;
}

// Cosine and sine of the angle of this lane's frequency (lane < rot / 2; else 1 and 0).  The angle in 64 bits, reduced to a part of a turn, because 32
// bits leave of an angle of 10^5 no more than 2^-7, and what rounding that part to 32 bits leaves off goes into its sine and cosine.
__device__ __forceinline__ void lane_angle(int position, const float* inv_freq, int lane, int freqs, float& cs, float& sn) {
  cs = 1.f;
  sn = 0.f;
  if (lane < freqs) {
    double turns = (double)position * (double)inv_freq[lane] * 0.15915494309189533577;
    turns -= rint(turns);
    // in half turns, as a float and what that leaves off: sine and cosine of their sum, to first order
    const double half_turns = 2.0 * turns;
    const float near = (float)half_turns, rest = 3.14159265f * (float)(half_turns - (double)near);
    float s0, c0;
    sincospif(near, &s0, &c0);
    sn = __builtin_fmaf(c0, rest, s0);
    cs = __builtin_fmaf(-s0, rest, c0);
  }
}

// Where the two pieces of lane `sub` of a head begin: the two halves of the turned channels, then what is left in order; or neighbours
struct PieceAt { int first, second; bool turned; };
__device__ __forceinline__ PieceAt pieces_of(int sub, int rot, bool adjacent, int n) {
  const int half = rot / (2 * n);
  const bool turned = sub < half;
  return {(adjacent || !turned ? 2 * sub : sub) * n, (adjacent || !turned ? 2 * sub + 1 : sub + half) * n, turned};
}

// x = x / sqrt(mean x^2 + eps) w over a head's HD channels, 2 N of them in this lane; w may be null (all ones)
template <typename T, int HD>
__device__ __forceinline__ void norm_head(float (&x)[2 * Piece<T>::N], const T* w, int first, int second, float eps) {
  using Vec = typename Piece<T>::Vec;
  constexpr int N = Piece<T>::N, kLanes = HD / (2 * N);
  // mean(x^2) + eps, with eps f^2 for rows that were multiplied by f
  auto mean_square = [&](float e) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, o);
    return __builtin_fmaf(sum, 1.f / HD, e);
  };
  float ms = mean_square(eps);
  // Rows whose squares are not numbers of fp32, or are so small that they lose bits, are brought near 1 by a power of two first: elements up to
  // 2^128 become 2^58, ones below 2^-41 up to 2^59.  All lanes go in for one row, the others with a factor of 1.  The test is 0.05 of 2.9 us for a
  // block's rows.
  if (__ballot(!(ms >= 0x1p-90f && ms <= 0x1p120f)) != 0) {
    const float f = ms >= 0x1p-90f ? ms <= 0x1p120f ? 1.f : 0x1p-70f : 0x1p100f;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) x[i] *= f;
    ms = mean_square(eps * f * f);
  }
  const float r = 1.f / sqrtf(ms);
  if (w) {
    const Vec u = *reinterpret_cast<const Vec*>(w + first), v = *reinterpret_cast<const Vec*>(w + second);
#pragma unroll
    for (int i = 0; i < N; ++i) { x[i] = x[i] * r * (float)u[i]; x[N + i] = x[N + i] * r * (float)v[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) x[i] *= r;
  }
}

// (a, b) -> (a c - b s, a s + b c) for the pairs in this lane
template <int N>
__device__ __forceinline__ void turn_pairs(float (&x)[2 * N], const float (&c)[N], const float (&s)[N], bool adjacent) {
  if (adjacent) {
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

}  // namespace sdllm
