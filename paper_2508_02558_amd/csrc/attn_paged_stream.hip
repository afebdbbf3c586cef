// Attention over the paged cache, bf16, few query columns per KV head: single tokens and small trees.  Bound by memory: all a call does is read the keys
// and values once.
//
// A workgroup takes 32 columns (paged_tile.h) and a share of their tiles.  Each wavefront streams tiles of its own straight into LDS, no barrier in
// the loop: K of the next tile is requested as soon as this one's operands are in registers, V likewise, so that a wavefront has 8 to 16 KB under way at any time.
// The pages of its next 64 tiles are looked up by one load, a tile per lane.  The wavefronts merge through LDS; splits of an item leave partials.
#include "attn_paged_merge.h"
#include "paged_tile_bf16.h"

namespace sdllm {

namespace {

constexpr int kStreamWaves = 8;   // most of a workgroup

template <int HD>
constexpr int stream_wave_lds() { return 2 * BfTile<HD>::kBytes + 256; }   // K, V and row statistics; the accumulators are parked where the tiles were

template <int HD, int SEES>
__global__ __launch_bounds__(kStreamWaves * kWave) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_paged_stream_kernel(const PagedAttnParams p) {
  using T = BfTile<HD>;
  constexpr int NE = T::NE, kSlots = NE * 4, kWaveLds = stream_wave_lds<HD>();
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int half = lane >> 5, col = lane & 31;

  PagedItem w;
  if (!find_item<SEES>(p, lane, w)) return;
  const int per_split = ceil_div(w.tiles, w.n_split);
  const int t_begin = min(w.tiles, w.split * per_split) + wave, t_end = min(w.tiles, (w.split + 1) * per_split);
  const int n_mine = max(0, (t_end - t_begin + nw - 1) / nw);   // tiles t_begin, t_begin + nw, ...

  const int column = w.blk * 32 + col, in = min(column, w.cols - 1);
  const int row = p.by_group.quotient(in), head = w.g * p.group + in - row * p.group;
  const RowSight sight = sight_of<SEES>(p, w, row);

  const ItemBase item = item_base<SEES>(p, w);
  // tiles 64 i .. 64 i + 63 of this wavefront's, one per lane: where they are
  TilePlace places;
  auto look_up = [&](int j0) __attribute__((always_inline)) {
    places = place_of<SEES>(p, w, item, tile_of<SEES>(p, w, min(t_begin + (j0 + lane) * nw, w.tiles - 1)));
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

  f32x16 acc[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  float m_run = kNoMax, l_run = 0.f;
  bf16x8 qf[T::NP], a[T::NP], pb[2];
  i16x8 f[2 * NE];
  f32x16 s;

  // Requests in order: K(0), V(0), K(1), and then for each tile j K(j+2), V(j+1).  The waits count them.  Loads by the compiler in between (pages)
  // make a wait longer, never shorter.
  PagedTile x, x_next;
  TilePlace next{};
  auto landed = [&](bool all) __attribute__((always_inline)) {
    if (all) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if constexpr (T::kFetches == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    wave_lds_sync();
  };
  bool full = true, specials = false;   // of the tile whose second product is next; values of masked tiles that are no numbers
  // logits of tile j, then the next K
  auto logits = [&](int j) __attribute__((always_inline)) {
    x = x_next;
    T::read_k(k_lds, half, col, a);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (j + 1 < n_mine) {
      if (((j + 1) & 63) == 0) look_up(j + 1);
      next = place_from(places, (j + 1) & 63);
      x_next = tile_of<SEES>(p, w, t_begin + (j + 1) * nw);
      fetch(next, false, k_lds);
    }
    in_issue_order();
    T::logits(a, qf, s);
  };
  auto softmax = [&]() __attribute__((always_inline)) {
    full = x.full;
    if (!full) mask_logits(s, seen_bits<SEES>(p, x, sight), half);
    numerators<NE>(s, p.scale_log2, m_run, l_run, acc, pb);
  };
  if (n_mine > 0) {
    look_up(0);
    x_next = tile_of<SEES>(p, w, t_begin);
    TilePlace of_v = place_from(places, 0);
    fetch(of_v, false, k_lds);
    in_issue_order();
    fetch(of_v, true, v_lds);
    in_issue_order();
    const u32x4* q = reinterpret_cast<const u32x4*>((const char*)p.q + 2 * (w.b * p.q_sb + head * p.q_sh + row * p.q_sr));
#pragma unroll
    for (int i = 0; i < T::NP; ++i) qf[i] = __builtin_bit_cast(bf16x8, q[i * 2 + half]);
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
        T::pv(f, pb, acc);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (j < n_mine) softmax();
    }
  }

  if (specials)
    add_specials<SEES>(p, w, sight, 2, 0, n_mine, [&](int j) { return t_begin + j * nw; },
                       [&](const char* v, bool sees) __attribute__((always_inline)) { add_special_row<NE>(v, sees, half, acc); });
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  // Merge: every wavefront parks its accumulators (slot i of a lane in place i ^ its turn) and its columns' statistics; they then share out the slots.
  auto turn = [](int l) { return HD == 128 ? l & 15 : (l >> 1) & 7; };
  auto stat_of = [&](int k) __attribute__((always_inline)) { return reinterpret_cast<float*>(smem + k * kWaveLds + 2 * T::kBytes); };
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 v = {acc[e][i4 * 4], acc[e][i4 * 4 + 1], acc[e][i4 * 4 + 2], acc[e][i4 * 4 + 3]};
      *reinterpret_cast<f32x4*>(k_lds + lane * kSlots * 16 + (((e * 4 + i4) ^ turn(lane)) << 4)) = v;
    }
  if (lane < 32) { stat_of(wave)[lane] = m_run; stat_of(wave)[32 + lane] = l_tot; }
  __syncthreads();
  float f_w[kStreamWaves], m_tot = kNoMax, l_all = 0.f;
#pragma unroll
  for (int k = 0; k < kStreamWaves; ++k) {
    f_w[k] = k < nw ? stat_of(k)[col] : kNoMax;
    m_tot = fmaxf(m_tot, f_w[k]);
  }
#pragma unroll
  for (int k = 0; k < kStreamWaves; ++k)
    if (k < nw) {
      f_w[k] = __builtin_amdgcn_exp2f(f_w[k] - m_tot);   // a wavefront that saw no tile parked (kNoMax, 0, 0)
      l_all += f_w[k] * stat_of(k)[32 + col];
    }
  const float inv = 1.f / l_all;
  if (column < w.cols) {
    for (int i = wave; i < kSlots; i += nw) {
      f32x4 o4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kStreamWaves; ++k)
        if (k < nw) o4 += *reinterpret_cast<const f32x4*>(smem + k * kWaveLds + lane * kSlots * 16 + ((i ^ turn(lane)) << 4)) * f_w[k];
      const int d0 = out_col0(i >> 2, i & 3, half);
      if (w.n_split > 1) {
        *reinterpret_cast<f32x4*>(p.part_o + ((int64_t)w.slot * 32 + col) * HD + d0) = o4;
      } else {
        bf16x4 ob;
#pragma unroll
        for (int r = 0; r < 4; ++r) ob[r] = (__bf16)(sight.none ? 0.f : o4[r] * inv);
        *reinterpret_cast<bf16x4*>((__bf16*)p.out + w.b * p.o_sb + head * p.o_sh + row * p.o_sr + d0) = ob;
      }
    }
    if (w.n_split > 1 && wave == 0 && lane < 32) {
      p.part_ml[(int64_t)w.slot * 64 + lane] = sight.none ? -INFINITY : m_tot;
      p.part_ml[(int64_t)w.slot * 64 + 32 + lane] = l_all;
    }
  }
}

template <int HD, int SEES>
hipError_t launch_sees(const PagedAttnParams& p, const PagedPlan& pl, hipStream_t s) {
  static LdsOptIn lds;
  const auto kernel = attn_paged_stream_kernel<HD, SEES>;
  hipError_t e = lds.ensure(reinterpret_cast<const void*>(kernel), kStreamWaves * stream_wave_lds<HD>());
  if (e != hipSuccess) return e;
  if (pl.waves < 1 || pl.waves > kStreamWaves || p.block_cols != 32) return hipErrorInvalidValue;
  e = launch(kernel, dim3((unsigned)p.workgroups), dim3(pl.waves * kWave), pl.waves * stream_wave_lds<HD>(), s, p);
  return e != hipSuccess || !pl.splits ? e : launch_paged_merge<__bf16, HD>(p, s);
}

}  // namespace

hipError_t launch_attn_paged_stream(const PagedAttnParams& p, const PagedPlan& pl, int sees, int d, hipStream_t s) {
  if (d == 128) return sees == kSeeTree ? launch_sees<128, kSeeTree>(p, pl, s) : launch_sees<128, kSeeWindow>(p, pl, s);
  return sees == kSeeTree ? launch_sees<64, kSeeTree>(p, pl, s) : launch_sees<64, kSeeWindow>(p, pl, s);
}

}  // namespace sdllm
