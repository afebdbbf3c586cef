// Appending to the paged cache: norm and rotation of the new queries and keys as in qk_norm_rope.hip, the keys, and the values as they
// are, stored in the rows that the page table names.  Bound by memory: everything is read and written once.  A wavefront takes heads of one new row; a
// row's place is found once per wavefront, while its heads are on their way.  8 sequences of 1024 to 4096 rows x 32/8 heads of 128: 503 MB in 95 us, 5.3 TB/s (a
// copy: 5.1); one token of 28/4 heads 3.3 us, two round trips to memory and the launch.
#include "qk_rope_math.h"

namespace sdllm {

namespace {

constexpr int kAppendThreads = 256;   // at most

template <typename T, int HD, bool NT>
__global__ __launch_bounds__(kAppendThreads) void append_paged_kernel(const AppendParams p) {
  using Vec = typename Piece<T>::Vec;
  constexpr int N = Piece<T>::N;
  constexpr int kLanes = HD / (2 * N), kHeads = kWave / kLanes;
  const QkParams& q = p.qk;
  const PagedCache& c = p.cache;
  const int lane = threadIdx.x & 63;
  const int wave = blockIdx.x * (blockDim.x / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int token = wave / q.parts, part = wave - token * q.parts;
  if (token >= q.tokens) return;
  const int b = q.by_rows.quotient(token), i = token - b * c.rows;
  if (i >= c.count(b)) return;
  const int sub = lane % kLanes, slot = lane / kLanes;

  const int row = p.pick ? min(max(p.pick[(int64_t)b * c.rows + i], 0), c.rows - 1) : i;   // of q_in, k_in and v_in
  const int place = c.length(b) + i;
  const int position = q.rot == 0 ? 0 : q.positions ? q.positions[b * q.pos_stride + row] : place + q.pos_begin;
  // where keys and values go, in elements; nowhere: < 0
  int64_t at = -1;
  if (place < c.capacity) {
    const int page = c.table[b * c.table_stride + (place >> c.page_shift)];
    if (page >= 0 && page < c.n_pages) at = page * c.sp + (place & ((1 << c.page_shift) - 1)) * c.sr;
  }
  float cs, sn;
  lane_angle(position, q.inv_freq, lane, q.rot >> 1, cs, sn);
  float co[N], si[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    co[j] = __shfl(cs, sub * N + j);
    si[j] = __shfl(sn, sub * N + j);
  }
  const auto [first, second, turned] = pieces_of(sub, q.rot, q.adjacent, N);

  // passes over heads that are normalised and turned, then over those that are copied
  const int heads = q.hq + q.hkv, passes = (heads + kHeads - 1) / kHeads, all = passes + (q.hkv + kHeads - 1) / kHeads;
  for (int pass = part; pass < all; pass += q.parts) {
    if (pass < passes) {
      const int h = pass * kHeads + slot;
      const bool there = h < heads, is_q = h < q.hq;
      const int hh = is_q ? h : h - q.hq;
      float x[2 * N];
      if (there) {
        const T* src = is_q ? (const T*)q.q_in + b * q.qi_sb + hh * q.qi_sh + row * q.qi_sr : (const T*)q.k_in + b * q.ki_sb + hh * q.ki_sh + row * q.ki_sr;
        const Vec u = read_piece<NT>(reinterpret_cast<const Vec*>(src + first)), v = read_piece<NT>(reinterpret_cast<const Vec*>(src + second));
#pragma unroll
        for (int j = 0; j < N; ++j) { x[j] = (float)u[j]; x[N + j] = (float)v[j]; }
      } else {
#pragma unroll
        for (int j = 0; j < 2 * N; ++j) x[j] = 0.f;
      }
      if (q.norm) norm_head<T, HD>(x, (const T*)(is_q ? q.q_weight : q.k_weight), first, second, q.eps);
      if (turned) turn_pairs<N>(x, co, si, q.adjacent);
      if (there && (is_q || at >= 0)) {
        T* dst = is_q ? (T*)q.q_out + b * q.qo_sb + hh * q.qo_sh + i * q.qo_sr : (T*)p.k_pages + at + hh * c.sh;
        Vec u, v;
#pragma unroll
        for (int j = 0; j < N; ++j) { u[j] = (T)x[j]; v[j] = (T)x[N + j]; }
        write_piece<NT>(u, reinterpret_cast<Vec*>(dst + first));
        write_piece<NT>(v, reinterpret_cast<Vec*>(dst + second));
      }
    } else {
      const int h = (pass - passes) * kHeads + slot;
      if (h < q.hkv && at >= 0) {
        const T* src = (const T*)p.v_in + b * q.ki_sb + h * q.ki_sh + row * q.ki_sr + sub * 2 * N;
        T* dst = (T*)p.v_pages + at + h * c.sh + sub * 2 * N;
        const Vec u = read_piece<NT>(reinterpret_cast<const Vec*>(src)), v = read_piece<NT>(reinterpret_cast<const Vec*>(src + N));
        write_piece<NT>(u, reinterpret_cast<Vec*>(dst));
        write_piece<NT>(v, reinterpret_cast<Vec*>(dst + N));
      }
    }
  }
}

template <typename T, int HD>
hipError_t launch_as(const AppendParams& a, hipStream_t s) {
  AppendParams p = a;
  QkParams& q = p.qk;
  constexpr int kHeads = kWave * 2 * Piece<T>::N / HD;
  const int passes = (q.hq + q.hkv + kHeads - 1) / kHeads + (q.hkv + kHeads - 1) / kHeads;
  // as in qk_norm_rope.hip: wavefronts per row until there are four for every SIMD, few of them spread over all CUs, much data past the caches
  // (bf16, 32/8 heads, MB read and written: 384 77 us, through the caches 84; 768 148, 158; 192 43, 48, but that much the next call finds in the memory-side cache)
  q.parts = 1;
  while (q.parts < passes && (int64_t)q.tokens * q.parts < 16 * kNumCUs) q.parts *= 2;
  if (q.parts > passes) q.parts = passes;
  const int64_t waves = (int64_t)q.tokens * q.parts;
  const int threads = waves <= 16 * kNumCUs ? kWave : kAppendThreads;
  const dim3 grid((uint32_t)((waves * kWave + threads - 1) / threads)), block(threads);
  const int64_t bytes = (int64_t)q.tokens * (q.hq + 2 * q.hkv) * HD * sizeof(T) * 2;
  return bytes >= (int64_t)256 << 20 ? launch(append_paged_kernel<T, HD, true>, grid, block, 0, s, p) : launch(append_paged_kernel<T, HD, false>, grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_append_paged(const AppendParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == 0) return d == 128 ? launch_as<__bf16, 128>(p, s) : launch_as<__bf16, 64>(p, s);
  return d == 128 ? launch_as<float, 128>(p, s) : launch_as<float, 64>(p, s);
}

}  // namespace sdllm
