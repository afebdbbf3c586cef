// Attention over the paged cache, for few query columns per KV head, single tokens and small trees, and for fp32 tensors.  Bound by memory with bf16
// tensors: all a call does is read the keys and values once.  With fp32 tensors, exact products and sums, by the matrix cores, which take sixteen times as long.
//
// A workgroup takes 16 or 32 columns (paged_tile.h) and a share of their tiles.  Each wavefront streams tiles of its own straight into LDS, no barrier in
// the loop: K of the next tile is requested as soon as this one's operands are in registers, V likewise, so that a wavefront has 8 to 16 KB under way at any time.
// Where its next 64 tiles are is worked out at once, a tile per lane.  The wavefronts merge through LDS; splits of an item leave partials.
// One token of 32 sequences of 1000 to 16000 keys x 28/4 heads of 128: 557 MB in 94 us, 5.9 TB/s with the merge, 64 x 2000 keys x 32/32 heads 6.8; two trees
// of 8 rows x 65000 and 131000 keys x 32/8 heads 137 to 141 us, 5.8 TB/s; fp32, 2000 rows x 16/2 heads 71 TFLOP/s of the 140 that a large product reaches.
#include <type_traits>

#include "attn_paged_merge.h"

namespace sdllm {

namespace {

template <typename E, int HD, int C>
constexpr int stream_wave_lds() { return 2 * Tile<E, HD>::kBytes + 2 * C * (int)sizeof(float); }   // K, V and row statistics; results are parked where the tiles were

template <typename E, int HD, int C, int NW, int SEES>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_paged_stream_kernel(const PagedAttnParams p) {
  using T = Math<E, HD, C>;
  constexpr int ES = sizeof(E), NS = T::NS, NA = T::NA, kSlots = T::kSlots, kRegs = sizeof(typename T::Acc) / 4, kWaveLds = stream_wave_lds<E, HD, C>();
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane % C;

  PagedItem w;
  if (!find_item<SEES>(p, lane, w)) return;
  // the same for all lanes, and known to be: the loop's branches are scalar
  const int per_split = __builtin_amdgcn_readfirstlane(ceil_div(w.tiles, w.n_split));
  const int t_begin = __builtin_amdgcn_readfirstlane(min(w.tiles, w.split * per_split)) + wave;
  const int t_end = __builtin_amdgcn_readfirstlane(min(w.tiles, (w.split + 1) * per_split));
  const int n_mine = max(0, (t_end - t_begin + NW - 1) / NW);   // tiles t_begin, t_begin + NW, ...

  const int column = w.blk * C + col, in = min(column, w.cols - 1);
  const int row = p.by_group.quotient(in), head = w.g * p.group + in - row * p.group;
  const RowSight sight = sight_of<SEES>(p, w, row);

  const ItemBase item = item_base<ES, SEES>(p, w);
  // tiles 64 i .. 64 i + 63 of this wavefront's, one per lane: where they are
  TilePlace places;
  auto look_up = [&](int j0) __attribute__((always_inline)) {
    places = place_of<SEES>(p, w, item, tile_of<SEES>(p, w, min(t_begin + (j0 + lane) * NW, w.tiles - 1)));
  };

  uint8_t* k_lds = smem + wave * kWaveLds;
  uint8_t* v_lds = k_lds + T::kBytes;
  const bool past_caches = w.past_caches;
  auto fetch = [&](TilePlace t, bool is_v, uint8_t* lds) __attribute__((always_inline)) {
    const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(lds));
    const char* base = t.bits & kOwn ? is_v ? item.v_own : item.k_own : is_v ? item.v : item.k;
    int l = lane;
    asm volatile("" : "+v"(l));   // a lane's places in the fetches are worked out here: kept, they would be too many registers
    const int r0 = l / T::kPieces, place = l % T::kPieces;
    auto piece = [&](int r) __attribute__((always_inline)) { return (uint32_t)(place ^ (is_v ? T::v_turn(r) : T::k_turn(r))) << 4; };
    if (t.bits & kWhole) {
      const uint32_t off = r0 * item.stride;
      const char* first = base + t.at0;
      const int64_t step = (int64_t)T::kRowsPerFetch * item.stride;
      if (past_caches) {
#pragma unroll
        for (int j = 0; j < T::kFetches; ++j) fetch_to_lds_once(to + (uint32_t)j * 1024, in_scalars(first + j * step), off + piece(j * T::kRowsPerFetch + r0));
      } else {
#pragma unroll
        for (int j = 0; j < T::kFetches; ++j) fetch_to_lds(to + (uint32_t)j * 1024, in_scalars(first + j * step), off + piece(j * T::kRowsPerFetch + r0));
      }
    } else {
#pragma unroll
      for (int j = 0; j < T::kFetches; ++j) {
        const int r = j * T::kRowsPerFetch + r0;
        fetch_to_lds(to + (uint32_t)j * 1024, base + row_at(t, item, r) + piece(r));
      }
    }
  };

  typename T::Acc acc[NA];
#pragma unroll
  for (int e = 0; e < NA; ++e)
#pragma unroll
    for (int i = 0; i < kRegs; ++i) acc[e][i] = 0.f;
  float m_run = kNoMax, l_run = 0.f;
  typename T::Q qf[T::NQ];
  typename T::K a[T::NK];
  typename T::V f[T::NV];
  typename T::P pb[T::NB];
  constexpr int kPerP = NS / T::NB;
  float s[NS];

  // Requests in order: K(0), V(0), K(1), and then for each tile j K(j+2), V(j+1).  The waits count them.  Loads by the compiler in between (pages)
  // make a wait longer, never shorter.
  PagedTile x, x_next;
  TilePlace next{};
  auto landed = [&](bool all) __attribute__((always_inline)) {
    if (all) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if constexpr (T::kFetches == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    else if constexpr (T::kFetches == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    wave_lds_sync();
  };
  bool full = true, specials = false;   // of the tile whose second product is next; values of masked tiles that are no numbers
  // logits of tile j, then the next K
  auto logits = [&](int j) __attribute__((always_inline)) {
    x = x_next;
    T::read_k(k_lds, lane, a);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (j + 1 < n_mine) {
      if (((j + 1) & 63) == 0) look_up(j + 1);
      next = place_from(places, (j + 1) & 63);
      x_next = tile_of<SEES>(p, w, t_begin + (j + 1) * NW);
      fetch(next, false, k_lds);
    }
    in_issue_order();
    T::logits(a, qf, s);
  };
  auto softmax = [&]() __attribute__((always_inline)) {
    full = x.full;
    if (!full) {
      const uint32_t seen = seen_bits<SEES>(p, x, sight) >> T::key_base(lane);
#pragma unroll
      for (int i = 0; i < NS; ++i) s[i] = or_minus_infinity(s[i], bit_mask(seen, T::key(i)));
    }
    float m_loc = s[0];
#pragma unroll
    for (int i = 1; i < NS; ++i) m_loc = fmaxf(m_loc, s[i]);
    m_loc *= p.scale_log2;
    if (__ballot(m_loc > m_run + kRescaleSlack) != 0) {
      const float m_new = fmaxf(m_run, T::over_row(m_loc, false));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int e = 0; e < NA; ++e)
#pragma unroll
        for (int i = 0; i < kRegs; ++i) acc[e][i] *= alpha;
    }
    float l_loc = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2, -m_run));
      l_loc += e;
      pb[i / kPerP][i % kPerP] = (E)e;   // rounded: bf16
    }
    l_run += l_loc;
  };

  if (n_mine > 0) {
    look_up(0);
    x_next = tile_of<SEES>(p, w, t_begin);
    TilePlace of_v = place_from(places, 0);
    fetch(of_v, false, k_lds);
    in_issue_order();
    fetch(of_v, true, v_lds);
    in_issue_order();
    const u32x4* q = reinterpret_cast<const u32x4*>((const char*)p.q + ES * (w.b * p.q_sb + head * p.q_sh + row * p.q_sr));
#pragma unroll
    for (int i = 0; i < T::NQ; ++i) qf[i] = __builtin_bit_cast(typename T::Q, q[T::q_piece(i, lane)]);
    // logits of tile j, second product of tile j - 1, softmax of tile j
#pragma clang loop unroll(disable)
    for (int j = 0; j <= n_mine; ++j) {
      if (j < n_mine) {
        if (j > 0) { of_v.at0 = next.at0; of_v.at1 = next.at1; of_v.bits = next.bits; }
        landed(j <= 1);                     // K(j); V(j-1) may still fly
        logits(j);
      }
      if (j > 0) {
        landed(j + 1 >= n_mine);            // V(j-1); K(j+1), if there is one, may still fly
        T::read_v(v_lds, lane, f);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (j < n_mine) fetch(of_v, true, v_lds);
        in_issue_order();
        if (!full) specials |= take_specials(f);
        T::product(f, pb, acc);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (j < n_mine) softmax();
    }
  }

  if (specials)
    add_specials<SEES>(p, w, sight, ES, n_mine,
                       [&](int j) __attribute__((always_inline)) {
                         const int t = t_begin + j * NW;
                         return tile_of<SEES>(p, w, t).full ? -1 : t;
                       },
                       [&](const char* v, bool sees) __attribute__((always_inline)) {
#pragma unroll
                         for (int i = 0; i < kSlots; ++i) T::add(acc, i, special_values<E>(v, T::channel(i, lane), sees));
                       });
  const float l_tot = T::over_row(l_run, true);
  // Merge: every wavefront parks its results (slot i of a lane in place i ^ its turn) and its columns' statistics; they then share out the slots, with
  // everything that a slot needs requested at once.
  auto parked = [&](int k, int i) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4*>(smem + k * kWaveLds + lane * kSlots * 16 + ((i ^ (kSlots == 16 ? lane & 15 : kSlots == 8 ? (lane >> 1) & 7 : (lane >> 2) & 3)) << 4));
  };
  auto stat_of = [&](int k) __attribute__((always_inline)) { return reinterpret_cast<float*>(smem + k * kWaveLds + 2 * T::kBytes); };
#pragma unroll
  for (int i = 0; i < kSlots; ++i) *parked(wave, i) = T::slot(acc, i);
  if (lane < C) { stat_of(wave)[lane] = m_run; stat_of(wave)[C + lane] = l_tot; }
  __syncthreads();
  constexpr int kMine = kSlots / NW > 0 ? kSlots / NW : 1;
  if (kSlots < NW && wave >= kSlots) return;
  float f_w[NW], l_w[NW], m_tot = kNoMax, l_all = 0.f;
  f32x4 part[kMine][NW];
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    f_w[k] = stat_of(k)[col];
    l_w[k] = stat_of(k)[C + col];
#pragma unroll
    for (int j = 0; j < kMine; ++j) part[j][k] = *parked(k, wave + j * NW);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < NW; ++k) m_tot = fmaxf(m_tot, f_w[k]);
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    f_w[k] = __builtin_amdgcn_exp2f(f_w[k] - m_tot);   // a wavefront that saw no tile parked (kNoMax, 0, 0)
    l_all += f_w[k] * l_w[k];
  }
  const float inv = 1.f / l_all;
  if (column >= w.cols) return;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    f32x4 o4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NW; ++k) o4 += part[j][k] * f_w[k];
    const int d0 = T::channel(wave + j * NW, lane);
    if (w.n_split > 1) {
      *partial_slot<T>(p, w.slot, 0, wave + j * NW, lane) = o4;
    } else {
      typedef __attribute__((ext_vector_type(4))) E E4;
      E4 ob;
#pragma unroll
      for (int r = 0; r < 4; ++r) ob[r] = (E)(sight.none ? 0.f : o4[r] * inv);
      *reinterpret_cast<E4*>((E*)p.out + w.b * p.o_sb + head * p.o_sh + row * p.o_sr + d0) = ob;
    }
  }
  if (w.n_split > 1 && wave == 0 && lane < C) {
    p.part_ml[(int64_t)w.slot * 2 * C + lane] = sight.none ? -INFINITY : m_tot;
    p.part_ml[(int64_t)w.slot * 2 * C + C + lane] = l_all;
  }
}

template <typename E, int HD, int C, int NW, int SEES>
hipError_t launch_sees(const PagedAttnParams& p, const PagedPlan& pl, hipStream_t s) {
  static LdsOptIn lds;
  const auto kernel = attn_paged_stream_kernel<E, HD, C, NW, SEES>;
  constexpr int kLds = NW * stream_wave_lds<E, HD, C>();
  hipError_t e = lds.ensure(reinterpret_cast<const void*>(kernel), kLds);
  if (e != hipSuccess) return e;
  e = launch(kernel, dim3((unsigned)p.workgroups), dim3(NW * kWave), kLds, s, p);
  return e != hipSuccess || !pl.splits ? e : launch_paged_merge<E, HD, C>(p, s);
}

template <typename E, int HD, int C, int NW>
hipError_t launch_waves(const PagedAttnParams& p, const PagedPlan& pl, int sees, hipStream_t s) {
  return sees == kSeeTree ? launch_sees<E, HD, C, NW, kSeeTree>(p, pl, s) : launch_sees<E, HD, C, NW, kSeeWindow>(p, pl, s);
}

template <int HD>
hipError_t launch_dim(const PagedAttnParams& p, const PagedPlan& pl, int sees, int dtype, hipStream_t s) {
  if (dtype != 0) return launch_waves<float, HD, 16, paged_waves_f32(HD)>(p, pl, sees, s);
  if (p.block_cols == 16) return pl.waves == 4 ? launch_waves<__bf16, HD, 16, 4>(p, pl, sees, s) : launch_waves<__bf16, HD, 16, 8>(p, pl, sees, s);
  return pl.waves == 4 ? launch_waves<__bf16, HD, 32, 4>(p, pl, sees, s) : launch_waves<__bf16, HD, 32, 8>(p, pl, sees, s);
}

}  // namespace

hipError_t launch_attn_paged_stream(const PagedAttnParams& p, const PagedPlan& pl, int sees, int dtype, int d, hipStream_t s) {
  const bool fits = dtype == 0 ? (p.block_cols == 16 || p.block_cols == 32) && (pl.waves == 4 || pl.waves == 8) : p.block_cols == 16 && pl.waves == paged_waves_f32(d);
  if (!fits) return hipErrorInvalidValue;
  return d == 128 ? launch_dim<128>(p, pl, sees, dtype, s) : launch_dim<64>(p, pl, sees, dtype, s);
}

}  // namespace sdllm
