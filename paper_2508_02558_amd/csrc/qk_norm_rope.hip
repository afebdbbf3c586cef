// Norm of each query and key head and rotation by position in one pass: what turns a projection into the q_blk and k_in of a block
// step.  y = x / sqrt(mean(x^2) + eps) * w per head, then each pair (a, b) of frequency f becomes (a cos t - b sin t, a sin t + b cos t), t =
// position * inv_freq[f].  fp32 throughout, one rounding at the end; t in 64 bits (qk_rope_math.h, which has the arithmetic).
//
// Bound by memory.
#include "qk_rope_math.h"

namespace sdllm {

namespace {

constexpr int kRopeThreads = 256;   // at most

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

  const int position = p.rot == 0 ? 0 : p.positions ? p.positions[b * p.pos_stride + row] : p.pos_begin + row;
  float cs, sn;
  lane_angle(position, p.inv_freq, lane, p.rot >> 1, cs, sn);
  float c[N], s[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = __shfl(cs, sub * N + i);
    s[i] = __shfl(sn, sub * N + i);
  }
  const auto [first, second, turned] = pieces_of(sub, p.rot, p.adjacent, N);

  const int heads = p.hq + p.hkv;
  for (int h0 = part * kHeads; h0 < heads; h0 += p.parts * kHeads) {
    const int h = h0 + slot;
    const bool there = h < heads, is_q = h < p.hq;
    const int hh = is_q ? h : h - p.hq;
    float x[2 * N];
    if (there) {
      const T* src = is_q ? (const T*)p.q_in + b * p.qi_sb + hh * p.qi_sh + row * p.qi_sr : (const T*)p.k_in + b * p.ki_sb + hh * p.ki_sh + row * p.ki_sr;
      const Vec u = read_piece<NT>(reinterpret_cast<const Vec*>(src + first)), v = read_piece<NT>(reinterpret_cast<const Vec*>(src + second));
#pragma unroll
      for (int i = 0; i < N; ++i) { x[i] = (float)u[i]; x[N + i] = (float)v[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) x[i] = 0.f;
    }
    if (p.norm) norm_head<T, HD>(x, (const T*)(is_q ? p.q_weight : p.k_weight), first, second, p.eps);
    if (turned) turn_pairs<N>(x, c, s, p.adjacent);
    if (there) {
      T* dst = is_q ? (T*)p.q_out + b * p.qo_sb + hh * p.qo_sh + row * p.qo_sr : (T*)p.k_out + b * p.ko_sb + hh * p.ko_sh + row * p.ko_sr;
      Vec u, v;
#pragma unroll
      for (int i = 0; i < N; ++i) { u[i] = (T)x[i]; v[i] = (T)x[N + i]; }
      write_piece<NT>(u, reinterpret_cast<Vec*>(dst + first));
      write_piece<NT>(v, reinterpret_cast<Vec*>(dst + second));
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
