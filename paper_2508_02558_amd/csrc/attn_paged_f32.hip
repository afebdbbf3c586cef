// Attention over the paged cache, fp32 tensors: exact fp32 products and sums on the matrix cores (general_tile.h).
//
// A workgroup takes 16 columns (query rows x heads of a KV head's group; paged_tile.h) and a share of their tiles; its waves take the tiles in
// turn, each with a wave-private LDS tile and no barrier in the loop, the next tile requested before one is computed, and merge through LDS at the end.
// Shares of one item leave partials that a second launch merges.
#include "attn_paged_merge.h"
#include "general_tile.h"
#include "paged_tile.h"

namespace sdllm {

namespace {

template <int D>
constexpr int f32_wave_lds() {
  using O = Ops<float, D>;
  const int parked = kWave * (O::NACC * 4 + 16);
  return (O::kKTile > parked ? O::kKTile : parked) + 512;
}

// Where the rows of a tile are: rows 0-15 and 16-31 lie in one page each, or in the same
struct TileRows { const char *k[2], *v[2]; int64_t stride; int lo, hi; };

template <int SEES>
__device__ __forceinline__ TileRows rows_of(const PagedAttnParams& p, const PagedItem& w, const PagedTile& x) {
  TileRows r;
  r.lo = x.lo;
  r.hi = x.hi;
  if (SEES == kSeeTree && x.own) {
    r.stride = p.blk_sr * 4;
    const int64_t at = 4 * (w.b * p.blk_sb + w.g * p.blk_sh) + x.at * r.stride;
#pragma unroll
    for (int h = 0; h < 2; ++h) { r.k[h] = (const char*)p.k_blk + at + 16 * h * r.stride; r.v[h] = (const char*)p.v_blk + at + 16 * h * r.stride; }
    return r;
  }
  const PagedCache& c = p.cache;
  r.stride = c.sr * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // a half that no row sees any of may have no page: the other's
    const int row = x.at + min(max(16 * h, x.lo), x.hi - 1), first = row & ~15;
    const int64_t at = 4 * (page_of(c, w.b, row) * c.sp + w.g * c.sh + (first & ((1 << c.page_shift) - 1)) * c.sr);
    r.k[h] = (const char*)p.k_pages + at;
    r.v[h] = (const char*)p.v_pages + at;
  }
  return r;
}

template <int D, int SEES>
__global__ __launch_bounds__(kGeneralMaxWaves * kWave) void attn_paged_f32_kernel(const PagedAttnParams p) {
  using O = Ops<float, D>;
  constexpr int R = O::kRows, NS = O::NS, kWaveBytes = f32_wave_lds<D>(), kPark = O::NACC * 4 + 16, kUnits = O::NACC / 4;
  constexpr float kSlack = 8.f;   // as in attn_tile_math.h: the softmax reference moves when a maximum exceeds it by more
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int part = lane / R, col = lane % R;

  PagedItem w;
  if (!find_item<SEES>(p, lane, w)) return;
  const int per_split = ceil_div(w.tiles, w.n_split);
  const int t_begin = min(w.tiles, w.split * per_split), t_end = min(w.tiles, t_begin + per_split);

  const int column = w.blk * R + col, in = min(column, w.cols - 1);
  const int row = p.by_group.quotient(in), head = w.g * p.group + in - row * p.group;
  const RowSight sight = sight_of<SEES>(p, w, row);
  typename O::Frag qf[O::NP];
  g_row_pieces<O>((const float*)p.q + w.b * p.q_sb + head * p.q_sh + row * p.q_sr, part, qf);

  // K rows as 16-byte pieces, whole rows per group of lanes; V rows as the second product takes them.  Rows that nobody sees are some other's in K, zero in V.
  u32x4 kreg[O::kLoads];
  typename O::V vreg;
  auto load_k = [&](const TileRows& r) {
    constexpr int kPerRow = O::kRow / 16, kRowsPerLoad = kWave / kPerRow;
    const int c = lane % kPerRow, r0 = lane / kPerRow;
#pragma unroll
    for (int j = 0; j < O::kLoads; ++j) {
      const int at = min(max(j * kRowsPerLoad + r0, r.lo), r.hi - 1);
      kreg[j] = *reinterpret_cast<const u32x4*>((at < 16 ? r.k[0] : r.k[1]) + (at & 15) * r.stride + c * 16);
    }
  };
  auto load_v = [&](const TileRows& r) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int key = O::key(i, part), at = min(max(key, r.lo), r.hi - 1);
      const char* src = (at < 16 ? r.v[0] : r.v[1]) + (at & 15) * r.stride + col * 16;
#pragma unroll
      for (int c = 0; c < O::NE / 4; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(src + c * 256);
        vreg.r[i][c] = key == at ? x : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  };

  uint8_t* lds_k = smem + wave * kWaveBytes;
  typename O::Acc acc[O::NE];
#pragma unroll
  for (int e = 0; e < O::NE; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;      // softmax reference of the row; sum over the keys this lane has seen

  bool specials = false;                  // values of masked tiles that are no numbers
  int t = t_begin + wave;
  PagedTile next;
  TileRows rows;
  if (t < t_end) {
    next = tile_of<SEES>(p, w, t);
    rows = rows_of<SEES>(p, w, next);
    load_k(rows);
    load_v(rows);
  }
  for (; t < t_end; t += nw) {
    const PagedTile x = next;
    const bool more = t + nw < t_end;
    g_store_rows<O>(lds_k, O::kKRow, lane, kreg);
    wave_lds_sync();
    if (more) {
      next = tile_of<SEES>(p, w, t + nw);
      rows = rows_of<SEES>(p, w, next);
      load_k(rows);
    }
    float s[NS];
    O::logits(lds_k, qf, col, part, s);
    if (!x.full) {
      const uint32_t seen = seen_bits<SEES>(p, x, sight) >> (4 * part);
#pragma unroll
      for (int i = 0; i < NS; ++i) s[i] = or_minus_infinity(s[i], bit_mask(seen, O::key(i, 0)));
    }
    float m_loc = s[0];
#pragma unroll
    for (int i = 1; i < NS; ++i) m_loc = fmaxf(m_loc, s[i]);
    m_loc *= p.scale_log2;
    if (__ballot(m_loc > m_run + kSlack) != 0) {
      const float m_new = fmaxf(m_run, parts_max<O>(m_loc));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int e = 0; e < O::NE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[e][i] *= alpha;
    }
    float l_loc = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2, -m_run));
      l_loc += s[i];
    }
    l_run += l_loc;
    if (!x.full) {
      // bit 31: exponent all ones
      auto special = [](float v) { return (__builtin_bit_cast(uint32_t, v) & 0x7f800000u) + 0x00800000u & 0x80000000u; };
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int c = 0; c < O::NE / 4; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) any |= special(vreg.r[i][c][k]);
      if (__ballot(any != 0)) {
        specials = true;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int c = 0; c < O::NE / 4; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) vreg.r[i][c][k] = special(vreg.r[i][c][k]) ? 0.f : vreg.r[i][c][k];
      }
    }
    g_pv<D>(lds_k, vreg, s, lane, acc);
    if (more) load_v(rows);   // flies under the next tile's logits
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  if (specials)
    add_specials<SEES>(p, w, sight, 4, 0, ceil_div(t_end - t_begin - wave, nw), [&](int n) { return t_begin + wave + n * nw; }, [&](const char* v, bool sees) {
#pragma unroll
      for (int e = 0; e < O::NE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float z = reinterpret_cast<const float*>(v)[64 * (e >> 2) + 4 * (4 * part + i) + (e & 3)];
          acc[e][i] += sees && !(fabsf(z) < INFINITY) ? z : 0.f;
        }
    });
  // merge of the waves: each parks its results ([lane][unit of four columns]) and its rows' statistics
  const float l_tot = parts_sum<O>(l_run);
  uint8_t* mine = smem + wave * kWaveBytes;
  float* my_ml = reinterpret_cast<float*>(mine + kWave * kPark);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < O::NE; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (O::flat(e, i) >> 2 == u) v[O::flat(e, i) & 3] = acc[e][i];
    *reinterpret_cast<f32x4*>(mine + lane * kPark + u * 16) = v;
  }
  if (lane < R) { my_ml[lane] = m_run; my_ml[32 + lane] = l_tot; }
  __syncthreads();
  auto stat_of = [&](int k) { return reinterpret_cast<const float*>(smem + k * kWaveBytes + kWave * kPark); };
  float f_w[kGeneralMaxWaves], m_tot = kNoMax, l_all = 0.f;
#pragma unroll
  for (int k = 0; k < kGeneralMaxWaves; ++k) {
    f_w[k] = k < nw ? stat_of(k)[col] : kNoMax;
    m_tot = fmaxf(m_tot, f_w[k]);
  }
#pragma unroll
  for (int k = 0; k < kGeneralMaxWaves; ++k)
    if (k < nw) {
      f_w[k] = __builtin_amdgcn_exp2f(f_w[k] - m_tot);   // a wave that saw no tile parked (kNoMax, 0, 0)
      l_all += f_w[k] * stat_of(k)[32 + col];
    }
  const float inv = 1.f / l_all;
  for (int u = wave; u < kUnits; u += nw) {
    f32x4 o4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGeneralMaxWaves; ++k)
      if (k < nw) o4 += *reinterpret_cast<const f32x4*>(smem + k * kWaveBytes + lane * kPark + u * 16) * f_w[k];
    const int d0 = O::unit_col(u, part);
    if (column < w.cols) {
      if (w.n_split > 1) *reinterpret_cast<f32x4*>(p.part_o + ((int64_t)w.slot * R + col) * D + d0) = o4;
      else *reinterpret_cast<f32x4*>((float*)p.out + w.b * p.o_sb + head * p.o_sh + row * p.o_sr + d0) = sight.none ? f32x4{0.f, 0.f, 0.f, 0.f} : o4 * inv;
    }
  }
  if (w.n_split > 1 && wave == 0 && lane < R) {
    p.part_ml[(int64_t)w.slot * 2 * R + lane] = sight.none ? -INFINITY : m_tot;
    p.part_ml[(int64_t)w.slot * 2 * R + R + lane] = l_all;
  }
}

template <int D, int SEES>
hipError_t launch_sees(const PagedAttnParams& p, const PagedPlan& pl, hipStream_t s) {
  static LdsOptIn lds;
  const auto kernel = attn_paged_f32_kernel<D, SEES>;
  hipError_t e = lds.ensure(reinterpret_cast<const void*>(kernel), kGeneralMaxWaves * f32_wave_lds<D>());
  if (e != hipSuccess) return e;
  e = launch(kernel, dim3((unsigned)p.workgroups), dim3(pl.waves * kWave), pl.waves * f32_wave_lds<D>(), s, p);
  return e != hipSuccess || !pl.splits ? e : launch_paged_merge<float, D>(p, s);
}

}  // namespace

hipError_t launch_attn_paged_f32(const PagedAttnParams& p, const PagedPlan& pl, int sees, int d, hipStream_t s) {
  if (d == 128) return sees == kSeeTree ? launch_sees<128, kSeeTree>(p, pl, s) : launch_sees<128, kSeeWindow>(p, pl, s);
  return sees == kSeeTree ? launch_sees<64, kSeeTree>(p, pl, s) : launch_sees<64, kSeeWindow>(p, pl, s);
}

}  // namespace sdllm
