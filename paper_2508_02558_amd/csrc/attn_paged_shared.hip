// Attention over the paged cache, bf16, many query columns per KV head: prompts, and trees of grouped-query heads.  Bound by the matrix cores.
//
// A workgroup of 8 waves takes 256 / KS columns (paged_tile.h) and a share of their tiles, which its waves share through rings in LDS: wave w works
// on block w % (8 / KS) of 32 columns and, of KS key groups, on group w / (8 / KS).  A step of a group is 8 KB of K and of V, one tile of head_dim 128 or two of
// head_dim 64, so that both have sixteen matrix instructions a step.  The two waves of a SIMD are locked in opposite phases, with a barrier at each change, as in
// dense_full_mfma.hip, which says why: while one issues its matrix instructions (logits of step t+1 between the second product of
// step t), the other finds row maxima and does the first half of its exponentials.  The vector phase would be the longer one, so where the next tiles are, and which
// of them are masked, is worked out in the matrix phase: causal with head_dim 64 240 us became 200.
// Tiles that some row of a wave does not see all of are masked by 32 bits per row (seen_bits); whole tiles pay one scalar test.  Pages of the next 64 tiles are
// looked up by one load, a tile per lane.
// Rates, of 1245 TFLOP/s that a large product reaches (two machines): 4 x 4096 rows x 28/4 heads of 128, all keys seen, 1070 (897 us; without pages 1100), causal
// 925 to 995 (520 to 483); four prompts of 1024 to 4096 rows with a window of 1024 keys 695 to 720 (205 to 198; 7 of a workgroup's 45 us pass until its first logits,
// and the fifth round of workgroups is a third full); head_dim 64, 8192 rows x 16/2 heads, causal, 815 to 855 (210 to 200, twice the exponentials per product).
#include <type_traits>

#include "attn_paged_merge.h"

namespace sdllm {

namespace {

constexpr int kSharedWaves = 8;
constexpr int shared_ring(int ks) { return ks == 1 ? 5 : 4; }   // steps held
template <int HD, int KS>
constexpr int shared_lds() {
  const int ring = shared_ring(KS) * KS * (kRingK + kRingV), parked = KS == 1 ? 0 : kSharedWaves * (kWave * (HD * 2 + 16) + 256);
  return ring > parked ? ring : parked;
}

// A step of a group in LDS: eight groups of 1 KB of consecutive rows' pieces, as one fetch leaves them, rows r, r + 8, r + 16, ... in group r (mfma_tile.h).  With
// head_dim 64 a group holds eight half-sized rows; neighbours of them swap pairs of pieces.
template <int HD>
struct Step {
  static constexpr int KT = 128 / HD;                   // tiles of a step
  static constexpr int NP = HD / 16, NE = HD / 32;
  static constexpr int kRow = HD * 2, kPieces = kRow / 16;

  // row (of the step) and 16-byte piece that a lane of wave w's fetch brings
  static __device__ __forceinline__ int fetch_row(int wave, int lane) { return wave + 8 * (lane / kPieces); }
  static __device__ __forceinline__ uint32_t fetch_k_piece(int lane) { return (uint32_t)((lane % kPieces) ^ ((lane / kPieces) & 1)) << 4; }
  static __device__ __forceinline__ uint32_t fetch_v_piece(int lane) { return (uint32_t)(lane % kPieces) << 4; }

  static __device__ __forceinline__ const uint8_t* k_at(const uint8_t* step, int half, int col) {
    return step + (col & 7) * kKGroup + (col >> 3) * kRow + ((half ^ ((col >> 3) & 1)) << 4);
  }
  static __device__ __forceinline__ const uint8_t* v_at(const uint8_t* step, int lane) { return shared_v_at(step, lane); }
  // operand i of a step's logits and of its second product, i = 0 .. 7
  static __device__ __forceinline__ bf16x8 k_frag(const uint8_t* at, int i) {
    return *reinterpret_cast<const bf16x8*>(at + (HD == 128 ? i * 32 : (i & 1) * 512 + (i >> 1) * 32));
  }
  static __device__ __forceinline__ i16x8 v_frag(const uint8_t* at, int i) {
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    at += HD == 128 ? (i >> 2) * 512 + (i & 3) * 64 : (i >> 1) * 256 + (i & 1) * 64;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + kRow));   // eight keys on
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ int k_tile(int i) { return HD == 128 ? 0 : i & 1; }
  static __device__ __forceinline__ int k_part(int i) { return HD == 128 ? i : i >> 1; }
  static __device__ __forceinline__ int v_part(int i) { return HD == 128 ? i >> 2 : i >> 1; }   // 16 keys each
  static __device__ __forceinline__ int v_col(int i) { return i % NE; }
};

// Numerators r and r + 1 of 16 keys (eight in this lane), keys 16 part .. of the step, of exponents `at`
template <int KT, class At>
__device__ __forceinline__ void numerator_pair(const At& at, int part, int r, float& l, bf16x8 (&pb)[2 * KT]) {
#pragma unroll
  for (int i = r; i < r + 2; ++i) {
    const float x = __builtin_amdgcn_exp2f(at(part, i));
    l += x;
    pb[part][i] = (__bf16)x;
  }
}

template <int HD, int KS, int SEES>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_paged_shared_kernel(const PagedAttnParams p) {
  using S = Step<HD>;
  constexpr int KT = S::KT, NP = S::NP, NE = S::NE;
  constexpr int RB = kSharedWaves / KS, N = shared_ring(KS), kStepK = KS * kRingK, kStepV = KS * kRingV, kV0 = N * kStepK;
  constexpr int kCols = RB * 32;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int rb = wave % RB, kg = wave / RB;
  const bool late = wave >= kSharedWaves / 2;   // waves w and w + 4 share a SIMD: the second four run one phase behind

  PagedItem w;
  if (!find_item<SEES>(p, lane, w)) return;
  // the same for all lanes, and known to be: the loop's branches are scalar
  const int per_split = __builtin_amdgcn_readfirstlane(ceil_div(w.tiles, w.n_split));
  const int t0 = __builtin_amdgcn_readfirstlane(min(w.tiles, w.split * per_split)), n_tiles = __builtin_amdgcn_readfirstlane(min(w.tiles - t0, per_split));
  const int nsteps = ceil_div(n_tiles, KS * KT);   // step j, group k: tiles t0 + (j KS + k) KT ..

  // columns past the last compute on a copy of it and are not written back
  struct Column { int column, row, head; };
  auto column_of = [&](int c) __attribute__((always_inline)) {
    const int column = w.blk * kCols + rb * 32 + c, in = min(column, w.cols - 1), row = p.by_group.quotient(in);
    return Column{column, row, w.g * p.group + in - row * p.group};
  };
  const Column mine = column_of(col);
  const RowSight sight = sight_of<SEES>(p, w, mine.row);
  // keys [most_first, least_last] are in the window of all rows of this wave
  if (SEES == kSeeWindow) {
    const int c0 = min(w.blk * kCols + rb * 32, w.cols - 1), c1 = min(w.blk * kCols + rb * 32 + 31, w.cols - 1);
    w.least_last = last_seen(p, w.end, w.length + p.by_group.quotient(c0));
    w.most_first = first_seen(p, w.length + p.by_group.quotient(c1));
  }

  f32x16 acc[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  float m_run = kNoMax, l_run = 0.f;
  bool specials = false;   // values of masked tiles that are no numbers

  if (nsteps > 0) {
    bf16x8 qf[NP];
    {
      const u32x4* q = reinterpret_cast<const u32x4*>((const char*)p.q + 2 * (w.b * p.q_sb + mine.head * p.q_sh + mine.row * p.q_sr));
#pragma unroll
      for (int i = 0; i < NP; ++i) qf[i] = __builtin_bit_cast(bf16x8, q[i * 2 + half]);
    }
    // Tiles 64 i .. 64 i + 63 of the share, one per lane: where they are, and which of them and of the 64 before every row of this wave sees whole
    const ItemBase item = item_base<2, SEES>(p, w);
    TilePlace places;
    uint64_t whole_now = 0, whole_before = 0;
    int at_hand = 0;
    auto look_up = [&](int n0) __attribute__((always_inline)) {
      const PagedTile x = tile_of<SEES>(p, w, t0 + min(n0 + lane, n_tiles - 1));
      places = place_of<SEES>(p, w, item, x);
      whole_before = whole_now;
      whole_now = __ballot(x.full && n0 + lane < n_tiles);
      at_hand = n0 >> 6;
    };
    // A step's fetch: wave w brings rows w, w + 8, ... of every group's tiles.  A tile past the last is the last one again, masked later.
    const uint32_t lds0 = lds_address(smem);
    const int my_row = S::fetch_row(wave, lane);
    const uint32_t off_k = (uint32_t)(my_row & (kTileKeys - 1)) * item.stride + S::fetch_k_piece(lane);
    const uint32_t off_v = (uint32_t)(my_row & (kTileKeys - 1)) * item.stride + S::fetch_v_piece(lane);
    struct From { const char* group[KS]; };
    auto from = [&](bool is_v, int step) __attribute__((always_inline)) {
      const char *pages = is_v ? item.v : item.k, *own = is_v ? item.v_own : item.k_own;
      const uint32_t off = is_v ? off_v : off_k;
      From r;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int n = (step * KS + i) * KT, n0 = min(n, n_tiles - 1) & 63, n1 = min(n + KT - 1, n_tiles - 1) & 63;
        const uint32_t bits0 = (uint32_t)__builtin_amdgcn_readlane((int)places.bits, n0), bits1 = (uint32_t)__builtin_amdgcn_readlane((int)places.bits, n1);
        if (bits0 & bits1 & kWhole) {
          const int64_t a = readlane64(places.at0, n0);
          if constexpr (KT == 1) {
            r.group[i] = pages + a + off;
          } else {
            const int64_t b = readlane64(places.at0, n1);
            r.group[i] = pages + (my_row >= kTileKeys ? b : a) + off;
          }
        } else {
          int l = lane;
          asm volatile("" : "+v"(l));   // worked out here, not kept
          const int row = S::fetch_row(wave, l);
          const TilePlace a = place_from(places, n0);
          const char* at = (a.bits & kOwn ? own : pages) + row_at(a, item, row & (kTileKeys - 1));
          if constexpr (KT > 1) {
            const TilePlace b = place_from(places, n1);
            const char* other = (b.bits & kOwn ? own : pages) + row_at(b, item, row & (kTileKeys - 1));
            at = row >= kTileKeys ? other : at;
          }
          r.group[i] = at + (is_v ? S::fetch_v_piece(l) : S::fetch_k_piece(l));
        }
      }
      return r;
    };
    auto fetch = [&](bool is_v, const From& x, int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < KS; ++i)
        fetch_to_lds(lds0 + (uint32_t)(slot + (is_v ? kV0 + i * kRingV + wave * kVGroup : i * kRingK + wave * kKGroup)), x.group[i]);
    };
    auto fetch_k = [&](int step, int slot) __attribute__((always_inline)) { fetch(false, from(false, step), slot); };
    auto fetch_v = [&](int step, int slot) __attribute__((always_inline)) { fetch(true, from(true, step), slot); };
    // The 64 tiles at hand change before the K of a step that begins with the next; V of the step before has been asked for by then.
    auto turn_page = [&](int step) __attribute__((always_inline)) {
      const int n = step * KS * KT;
      if (n > 0 && (n & 63) == 0 && n < n_tiles) look_up(n);
    };
    static_assert(64 % (KS * KT) == 0, "a step's tiles are among the same 64");

    const uint8_t* k_at = S::k_at(smem + kg * kRingK, half, col);
    const uint8_t* v_at = S::v_at(smem + kV0 + kg * kRingV, lane);
    bf16x8 a[8], pb[2 * KT];
    i16x8 f[8];
    f32x16 sn[KT];
    float late_at[KT][8];   // exponents of the second half, so that the logits' registers are free for the next step's from its first product on

    bool full;
    auto look_ahead = [&](int step) __attribute__((always_inline)) {   // full: every row of this wave sees all of the step's tiles
      const int n0 = (step * KS + kg) * KT;
      const uint64_t whole = (n0 >> 6 == at_hand ? whole_now : whole_before) >> (n0 & 63);
      full = (~whole & ((1u << KT) - 1)) == 0;
    };
    auto mask = [&](int step) __attribute__((always_inline)) {
      if (full) return;
      const int n0 = (step * KS + kg) * KT;
#pragma unroll
      for (int q = 0; q < KT; ++q) {
        const PagedTile x = tile_of<SEES>(p, w, t0 + min(n0 + q, n_tiles - 1));
        mask_logits(sn[q], n0 + q >= n_tiles ? 0u : seen_bits<SEES>(p, x, sight), half);
      }
    };
    auto exponent = [&](int part, int i) __attribute__((always_inline)) { return __builtin_fmaf(sn[part >> 1][8 * (part & 1) + i], p.scale_log2, -m_run); };
    auto late_exponent = [&](int part, int i) __attribute__((always_inline)) { return late_at[part - KT][i]; };
    // Vector phase of a step: masks, row maxima, the reference, first half of the numerators
    auto vector_phase = [&](int step) __attribute__((always_inline)) {
      mask(step);
      float m_loc = sn[0][0];
#pragma unroll
      for (int q = 0; q < KT; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) m_loc = fmaxf(m_loc, sn[q][i]);
      move_reference_to<NE>(m_loc * p.scale_log2, m_run, l_run, acc);
      float l = 0.f;
#pragma unroll
      for (int part = 0; part < KT; ++part)
#pragma unroll
        for (int r = 0; r < 8; r += 2) numerator_pair<KT>(exponent, part, r, l, pb);
      l_run += l;
#pragma unroll
      for (int part = 0; part < KT; ++part)
#pragma unroll
        for (int r = 0; r < 8; ++r) late_at[part][r] = exponent(KT + part, r);
      if (!full) specials |= take_specials(f);
    };
    // Matrix phase: logits of the next step, second product of the current one, each operand register set reloaded for the next phase once it has been
    // used; the other half of the current step's numerators between the first instructions, `between(i)` (scalar work that the vector phase would wait for)
    // between the others.
    auto matrix_phase = [&](int k_slot, int v_slot, const auto& between) __attribute__((always_inline)) {
      float l = 0.f;
#pragma unroll
      for (int q = 0; q < KT; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[q][i] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sn[S::k_tile(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], qf[S::k_part(i)], sn[S::k_tile(i)], 0, 0, 0);
        acc[S::v_col(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[i]), pb[S::v_part(i)], acc[S::v_col(i)], 0, 0, 0);
        a[i] = S::k_frag(k_at + k_slot, i);
        f[i] = S::v_frag(v_at + v_slot, i);
        if (i < 4) {
#pragma unroll
          for (int j = 0; j < KT; ++j) {
            const int n = i * KT + j;   // pair: keys of the second half in order
            numerator_pair<KT>(late_exponent, KT + n / 4, n % 4 * 2, l, pb);
          }
        }
        between(i);
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += l;
    };

    // Requests are counted, in the order K(0), V(0), K(1), V(1), ..., V(N-1), K(N) and then V(t+N), K(t+N+1) for t = 0, 1, ...  Loads by the compiler
    // (pages) make a wait longer, never shorter; query rows, masks and the first pages are waited for before the first request.
    look_up(0);
#pragma unroll
    for (int i = 0; i < NP; ++i) asm volatile("" : "+v"(qf[i]));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      turn_page(j);
      fetch_k(j, j * kStepK);
      in_issue_order();
      fetch_v(j, j * kStepV);
      in_issue_order();
    }
    // V(1), K(2), ..., V(N-1) may still fly
    if (KS == 1) asm volatile("s_waitcnt vmcnt(7)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
    bare_barrier();
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = S::k_frag(k_at, i);
#pragma unroll
    for (int q = 0; q < KT; ++q)
#pragma unroll
      for (int i = 0; i < 16; ++i) sn[q][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sn[S::k_tile(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], qf[S::k_part(i)], sn[S::k_tile(i)], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = S::v_frag(v_at, i);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = S::k_frag(k_at + kStepK, i);
    look_ahead(0);
    vector_phase(0);
    // What the early waves read before a wait of the late ones stands between has landed: K(2), K(3), V(1), V(2).
    if (KS == 1) asm volatile("s_waitcnt lgkmcnt(0) vmcnt(3)" ::: "memory");   // V(3), K(4), V(4)
    else asm volatile("s_waitcnt lgkmcnt(0) vmcnt(2)" ::: "memory");           // V(3)
    bare_barrier();
    turn_page(N);
    fetch_k(N, 0);
    in_issue_order();
    if (late) bare_barrier();

    // Iteration t: matrix phase (logits of step t+1, second product of step t; reads K(t+2), V(t+1)), barrier, vector phase of step
    // t+1, barrier.  The late waves are one phase behind: vector phase t is the last that they end before the early ones'
    // matrix phase t+2, so what that reads, K(t+4) and V(t+3), has to have landed by then.  Requested behind those are V(t+N-1),
    // K(t+N) (KS = 1) and V(t+N), K(t+N+1): four requests either way.  A place in a ring is fetched into in vector phase t at the
    // earliest after the barrier that ends the late waves' vector phase t-1, at the end of which what they read there, in
    // matrix phase t-1, is in registers.
    static_assert(N == (KS == 1 ? 5 : 4), "the waits count on it");
    int t = 0, v_slot = kStepV, k_slot = 2 * kStepK, v_next = 0, k_next = kStepK;   // places of V(t+1), K(t+2), V(t+N), K(t+N+1)
    auto advance = [&](int& slot, int by) __attribute__((always_inline)) { slot = slot + by == N * by ? 0 : slot + by; };
    auto iteration = [&](auto fetches) __attribute__((always_inline)) {
      From v_from, k_from;
      __builtin_amdgcn_s_setprio(1);
      matrix_phase(k_slot, v_slot, [&](int i) __attribute__((always_inline)) {
        if (fetches && i == 4) v_from = from(true, t + N);
        if (fetches && i == 5) {
          turn_page(t + N + 1);
          k_from = from(false, t + N + 1);
        }
        if (i == 6) look_ahead(t + 1);
      });
      __builtin_amdgcn_s_setprio(0);
      bare_barrier();
      if (fetches) {
        fetch(true, v_from, v_next);
        fetch(false, k_from, k_next);
      }
      in_issue_order();
      vector_phase(t + 1);
      in_issue_order();
      advance(v_slot, kStepV); advance(k_slot, kStepK); advance(v_next, kStepV); advance(k_next, kStepK);
      if (fetches) asm volatile("s_waitcnt lgkmcnt(0) vmcnt(4)" ::: "memory");
      else asm volatile("s_waitcnt lgkmcnt(0) vmcnt(0)" ::: "memory");
      bare_barrier();
    };
    for (; t + N < nsteps; ++t) iteration(std::true_type{});
    for (; t + 1 < nsteps; ++t) iteration(std::false_type{});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land in LDS that is parked in, or another workgroup's
    float l = 0.f;
#pragma unroll
    for (int part = KT; part < 2 * KT; ++part)
#pragma unroll
      for (int r = 0; r < 8; r += 2) numerator_pair<KT>(late_exponent, part, r, l, pb);
    l_run += l;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      acc[S::v_col(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[i]), pb[S::v_part(i)], acc[S::v_col(i)], 0, 0, 0);
    if (!late) bare_barrier();
  }

  if (specials) {
    // KT tiles of every step are this group's, and are looked at together: a whole one as well if the other is masked, or past the last.  One past the last is
    // a copy that counts for nothing: it may be another group's, whose rows this one has seen no key of, and zero times an infinity is NaN in the merge.
    add_specials<SEES>(p, w, sight, 2, nsteps * KT,
                       [&](int n) __attribute__((always_inline)) {
                         const int n0 = (n / KT * KS + kg) * KT, t = n0 + n % KT;
                         if (t >= n_tiles) return -1;
                         bool whole = n0 + KT <= n_tiles;
#pragma unroll
                         for (int q = 0; q < KT; ++q) whole = whole && tile_of<SEES>(p, w, t0 + min(n0 + q, n_tiles - 1)).full;
                         return whole ? -1 : t0 + t;
                       },
                       [&](const char* v, bool sees) __attribute__((always_inline)) {
#pragma unroll
                         for (int i = 0; i < NE * 4; ++i) {
                           const f32x4 z = special_values<__bf16>(v, out_col0(i >> 2, i & 3, half), sees);
#pragma unroll
                           for (int k = 0; k < 4; ++k) acc[i >> 2][(i & 3) * 4 + k] += z[k];
                         }
                       });
  }
  float l_tot = l_run + __shfl_xor(l_run, 32);
  int again = col;
  asm volatile("" : "+v"(again));   // worked out again rather than kept
  const auto [column, row, head] = column_of(again);
  const bool there = column < w.cols, none = sight_of<SEES>(p, w, row).none;
  float* part_ml = p.part_ml + (int64_t)w.slot * 2 * kCols + rb * 32 + col;
  __bf16* out = (__bf16*)p.out + w.b * p.o_sb + head * p.o_sh + row * p.o_sr;
  using M = Math<__bf16, HD, 32>;   // results lie as there
  if constexpr (KS == 1) {
    const float inv = 1.f / l_tot;
    if (w.n_split > 1) {
#pragma unroll
      for (int i = 0; i < M::kSlots; ++i) *partial_slot<M>(p, w.slot, rb, i, lane) = M::slot(acc, i);
    } else {
      // Four channels of a lane and the four after them of the lane 32 on, twice: exchanged, so that each has eight in a row to write
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int i4 = 0; i4 < 4; i4 += 2) {
          bf16x4 ab[2];
#pragma unroll
          for (int k = 0; k < 8; ++k) ab[k >> 2][k & 3] = (__bf16)(none ? 0.f : acc[e][i4 * 4 + k] * inv);
          u32x2 x = __builtin_bit_cast(u32x2, ab[0]), y = __builtin_bit_cast(u32x2, ab[1]);
          u32x4 o;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const auto z = __builtin_amdgcn_permlane32_swap(x[k], y[k], false, false);
            o[k] = z[0];
            o[2 + k] = z[1];
          }
          if (there) *reinterpret_cast<u32x4*>(out + 32 * e + 8 * (i4 + half)) = o;
        }
    }
  } else {
    // merge of the key groups of each block of columns
    constexpr int kLane = HD * 2 + 16, kPark = kWave * kLane + 256;
    __syncthreads();                          // the tiles are done with
    uint8_t* own = smem + wave * kPark;
#pragma unroll
    for (int e = 0; e < NE; ++e)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 v = {acc[e][i4 * 4], acc[e][i4 * 4 + 1], acc[e][i4 * 4 + 2], acc[e][i4 * 4 + 3]};
        *reinterpret_cast<f32x4*>(own + lane * kLane + (e * 4 + i4) * 16) = v;
      }
    if (lane < 32) {
      float* ml = reinterpret_cast<float*>(own + kWave * kLane);
      ml[lane] = m_run;
      ml[32 + lane] = l_tot;
    }
    __syncthreads();
    auto parked = [&](int k) __attribute__((always_inline)) { return smem + (k * RB + rb) * kPark; };
    float f_w[KS], m_tot = kNoMax;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      f_w[k] = reinterpret_cast<const float*>(parked(k) + kWave * kLane)[col];
      m_tot = fmaxf(m_tot, f_w[k]);
    }
    l_tot = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      f_w[k] = __builtin_amdgcn_exp2f(f_w[k] - m_tot);
      l_tot += f_w[k] * reinterpret_cast<const float*>(parked(k) + kWave * kLane)[32 + col];
    }
    m_run = m_tot;
    const float inv = 1.f / l_tot;
#pragma unroll
    for (int j = 0; j < NE * 4 / KS; ++j) {
      const int i = kg * (NE * 4 / KS) + j;
      f32x4 o4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) o4 += *reinterpret_cast<const f32x4*>(parked(k) + lane * kLane + i * 16) * f_w[k];
      if (w.n_split > 1) {
        *partial_slot<M>(p, w.slot, rb, i, lane) = o4;
      } else if (there) {
        bf16x4 ob;
#pragma unroll
        for (int r = 0; r < 4; ++r) ob[r] = (__bf16)(none ? 0.f : o4[r] * inv);
        *reinterpret_cast<bf16x4*>(out + M::channel(i, lane)) = ob;
      }
    }
  }
  if (w.n_split > 1 && kg == 0 && lane < 32 && there) {
    part_ml[0] = none ? -INFINITY : m_run;
    part_ml[kCols] = l_tot;
  }
}

template <int HD, int KS, int SEES>
hipError_t launch_sees(const PagedAttnParams& p, const PagedPlan& pl, hipStream_t s) {
  static LdsOptIn lds;
  const auto kernel = attn_paged_shared_kernel<HD, KS, SEES>;
  constexpr int kLds = shared_lds<HD, KS>();
  hipError_t e = lds.ensure(reinterpret_cast<const void*>(kernel), kLds);
  if (e != hipSuccess) return e;
  if (p.block_cols != 256 / KS) return hipErrorInvalidValue;
  e = launch(kernel, dim3((unsigned)p.workgroups), dim3(512), kLds, s, p);
  return e != hipSuccess || !pl.splits ? e : launch_paged_merge<__bf16, HD, 32>(p, s);
}

template <int HD>
hipError_t launch_dim(const PagedAttnParams& p, const PagedPlan& pl, int sees, hipStream_t s) {
  if (p.block_cols == 256) return sees == kSeeTree ? launch_sees<HD, 1, kSeeTree>(p, pl, s) : launch_sees<HD, 1, kSeeWindow>(p, pl, s);
  return sees == kSeeTree ? launch_sees<HD, 2, kSeeTree>(p, pl, s) : launch_sees<HD, 2, kSeeWindow>(p, pl, s);
}

}  // namespace

hipError_t launch_attn_paged_shared(const PagedAttnParams& p, const PagedPlan& pl, int sees, int d, hipStream_t s) {
  return d == 128 ? launch_dim<128>(p, pl, sees, s) : launch_dim<64>(p, pl, sees, s);
}

}  // namespace sdllm
