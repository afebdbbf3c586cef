// Block-query attention over a cache of 4 bits a value (packed_tile.h) and the block's own keys and values (Alg. 3, cache_state == 2).
//
// The query rows of the heads of a KV head are one list of columns (head, row); 32 of them are a 32x32 matrix block, whatever the block length, so
// that single tokens of grouped heads share one.  A wavefront owns 32 columns and takes tiles of 32 keys, which come through a ring in
// LDS of its own, and makes
//   logits^T = K_tile Q^T   (K rows as A operand: a lane holds sixteen logits of one column),
//   O^T += V_tile^T P^T     (V codes lie in the order of those sixteen logits),
// with the running maximum and sum of a softmax.  Four conversions make one operand of v_mfma_f32_32x32x16_bf16 out of eight codes.  The numbers of the
// cache are bf16 numbers, so for fp32 tensors the queries and the probabilities enter as the sum of three bf16 parts, all 24 bits of them: three times the products,
// and exact ones.  Keys are split over the wavefronts of a workgroup, merged through LDS, and over workgroups, whose partials a second launch
// folds.
//
// What bounds it.  Calls on few heads: latency; a workgroup is 5 us without its tiles, 2.3 of them the launch, 1.4 until the queries are
// there, 1.5 to 2 for the merge (16 KB of LDS a wavefront, in and out).  Full grids: a tile is 750 cycles of vector and 512 of matrix instructions
// to a SIMD (measured rates: 4.5 cycles a conversion, fma or add, 8 an exponential, 32 a matrix instruction) and takes 1265 of it, their sum, although
// two wavefronts are there: 224 workgroups x 73 tiles keep the matrix unit busy for 31 % of 15.7 us.  256 x 69 from HBM take 21.4 to 22 us
// (3.9 TB/s), 18.2 to 18.9 from the memory-side cache.
// Measured, when calls of four tiles a wavefront and more were 2 to 3 % faster, and not kept: sums and maxima between the products of the values, where the
// matrix unit has room for them (within 1%); a higher priority for wavefronts that are there (224 x 73 -1.5%, 256 x 69 from HBM +4%); LDS for each
// wavefront to park its results in without waiting (+1 to +4%: the code is longer).  Four wavefronts instead of eight: 224 x 73 17.7 us in place of 15.8.
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
// (eight each, cut off and not rounded, so that the largest float stays one).  An infinity is its first part, and NaN with the others.
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
        rest[i] -= cut;
      }
      part[n] = upper_halves(bits);
    }
  }
}

template <typename T> struct Parts;
template <> struct Parts<__bf16> { static constexpr int N = 1, kWaves = kPackedWavesBf16; };
template <> struct Parts<float> { static constexpr int N = 3, kWaves = kPackedWavesF32; };

__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Keys past the rows become -inf; the largest of the lane's logits, scaled.
__device__ __forceinline__ float mask_max(f32x16& s, int rows, float scale_log2, int half) {
  if (rows < kTileKeys) {                                // the last tile only: a branch, not sixteen selections in every one
    asm volatile("");
    const int left = rows - 4 * half;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < left ? s[i] : -INFINITY;
  }
  float m = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
  return m * scale_log2;
}

// Softmax of a tile's raw logits against the running reference: s becomes the numerators.
template <int NE>
__device__ __forceinline__ void move_reference(float m_loc, float& m_ref, float& l_run, f32x16 (&acc)[NE]) {
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
}
template <int NE>
__device__ __forceinline__ void softmax_step(f32x16& s, int rows, float scale_log2, int half, float& m_ref, float& l_run, f32x16 (&acc)[NE]) {
  move_reference<NE>(mask_max(s, rows, scale_log2, half), m_ref, l_run, acc);
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

template <int N>
__device__ __forceinline__ void wait_vector_memory() {
  static_assert(N < 64, "what the counter holds");
  asm volatile("s_waitcnt vmcnt(%0)" :: "i"(N) : "memory");
}
// ---- rows in LDS: 32 rows of a tensor as they are fetched, 16-byte pieces of a row in another order in each, so that lanes that read
// the same piece of neighbouring rows meet different banks
template <typename T, int HD>
struct Rows {
  static constexpr int kPieces = HD * (int)sizeof(T) / 16, kRow = HD * (int)sizeof(T), kBytes = 32 * kRow;
  static constexpr int kFetches = kBytes / 1024, kPerFetch = 64 / kPieces;        // fetch instructions, rows of one
  static __device__ __forceinline__ int turn(int row) { return kPieces >= 16 ? row & (kPieces - 1) : row >> 1 & (kPieces - 1); }
  // byte `at` of a row
  static __device__ __forceinline__ const uint8_t* place(const uint8_t* rows, int row, int at) {
    return rows + row * kRow + (((at >> 4) ^ turn(row)) << 4) + (at & 15);
  }
  // Requests them: address(row) is where a row lies; fetches j, j + step, ...
  template <class F>
  static __device__ __forceinline__ void request(uint8_t* rows, int j, int step, int lane, F&& address) {
    for (; j < kFetches; j += step) {
      const int row = j * kPerFetch + lane / kPieces;
      fetch_to_lds(lds_address(rows + j * 1024), (const char*)address(row) + ((lane % kPieces ^ turn(row)) << 4));
    }
  }
};

// Eight neighbouring channels of a row in LDS
template <typename T, int HD>
__device__ __forceinline__ void lds_load8(const uint8_t* rows, int row, int channel, bf16x8 (&part)[Parts<T>::N]) {
  using R = Rows<T, HD>;
  if constexpr (sizeof(T) == 2) {
    part[0] = *reinterpret_cast<const bf16x8*>(R::place(rows, row, channel * 2));
  } else {
    const f32x4 lo = *reinterpret_cast<const f32x4*>(R::place(rows, row, channel * 4)), hi = *reinterpret_cast<const f32x4*>(R::place(rows, row, channel * 4 + 16));
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    split_parts(x, part);
  }
}

// What a lane takes of a tile: keys, or values
template <int HD>
struct Operand {
  u32x4 codes[PackedLayout<HD>::kLoads];
  uint32_t scales;                                       // bytes: groups of the lane's key; channels of its value rows
};

// ---- logits of a tile of the cache
// The codes are made into bf16 operands, against the queries' rows as they are or their three parts.  The scaled matrix instruction takes codes as
// they lie and would save the conversions, but its other operand has eight bits a number, and two such numbers for a query leave off what
// is below 2^-13 of the largest of 32 channels.
template <typename T, int HD>
struct Queries {
  static constexpr int NF = HD / 16, PARTS = Parts<T>::N;
  bf16x8 qf[NF][PARTS];

  __device__ __forceinline__ void load(const uint8_t* rows, int m, int half) {
#pragma unroll
    for (int f = 0; f < NF; ++f) lds_load8<T, HD>(rows, m, 32 * (2 * (f >> 2) + half) + 8 * (f & 3), qf[f]);
  }
  // Logits of a tile in four steps, between which other work goes; the first sets s.
  template <int STEP>
  __device__ __forceinline__ void logits(const Operand<HD>& keys, int half, f32x16& s) const {
    if constexpr (STEP == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
    }
    if constexpr (STEP < PackedLayout<HD>::kLoads) {
      const float scale = scale_of_byte(keys.scales >> (8 * half), 2 * STEP);
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const bf16x8 kf = unpack8(keys.codes[STEP][st], scale);
#pragma unroll
        for (int n = PARTS - 1; n >= 0; --n) s = mfma(kf, qf[4 * STEP + st][n], s);
      }
    }
  }
};

// ---- a wavefront's tiles of the cache, every nw-th of [c, c_end), on their way through LDS of its own: two slots for key codes, two for value
// codes, four for scales.  A slot is requested again as soon as a lane's part of it is in registers, which is one tile ahead of their use
// for the keys; so two tiles are on their way at any time.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0, as in mfma_tile.h
// 64 lanes x 16 (or 4) bytes from base + off + AT to LDS at m0 + AT.  NT: past the caches
template <int AT, bool NT>
__device__ __forceinline__ void fetch_at(const char* base, uint32_t off) {
  if constexpr (NT) asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2 nt" :: "v"(off), "s"(base), "i"(AT) : "memory", "m0");
  else asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" :: "v"(off), "s"(base), "i"(AT) : "memory", "m0");
}
template <bool NT>
__device__ __forceinline__ void fetch4(const char* base, uint32_t off) {
  if constexpr (NT) asm volatile("global_load_lds_dword %0, %1 nt" :: "v"(off), "s"(base) : "memory", "m0");
  else asm volatile("global_load_lds_dword %0, %1" :: "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void fetch_goes_to(uint32_t lds) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" :: "s"(lds) : "memory", "m0"); }
#pragma clang diagnostic pop

template <int HD, bool NT>
struct Ring {
  using L = PackedLayout<HD>;
  static constexpr int kCodes = 16 * HD, kScales = 2 * HD;
  static constexpr int kValueSlots = 2 * kCodes, kScaleSlots = 4 * kCodes, kBytes = 4 * kCodes + 4 * kScales;
  static constexpr int kKeyFetches = L::kLoads + 1, kValueFetches = L::kLoads, kFetches = kKeyFetches + kValueFetches;
  const uint8_t* lds;
  uint32_t lds_at;                                       // the same as an LDS byte address, in a scalar register
  const char* tile;                                      // that is worked on
  int c, c_end, nw, lane, scale_slot;

  __device__ __forceinline__ bool has(int ahead) const { return c + ahead * nw < c_end; }
  // From this tile on; past the last one it may wrap round, and is not used.
  __device__ __forceinline__ int rows_left(int n_cached) const { return (int)((uint32_t)n_cached - (uint32_t)c * kTileKeys); }
  // AHEAD: of the tile; parity: of the tile's number among the wavefront's
  template <int AHEAD>
  __device__ __forceinline__ void fetch_keys(int parity) const {
    const char* t = tile + AHEAD * nw * L::kTile;
    const uint32_t lane16 = (uint32_t)lane * 16;
    fetch_goes_to(lds_at + ((parity + AHEAD) & 1) * kCodes);
    fetch_at<L::kKeys, NT>(t, lane16);
    if constexpr (HD == 128) fetch_at<L::kKeys + 1024, NT>(t, lane16);
    fetch_goes_to(lds_at + kScaleSlots + ((scale_slot + AHEAD) & 3) * kScales);
    if (HD == 128 || lane < 32) fetch4<NT>(t + L::kKeyScales, (uint32_t)lane * 4);
  }
  template <int AHEAD>
  __device__ __forceinline__ void fetch_values(int parity) const {
    const char* t = tile + AHEAD * nw * L::kTile + L::kValues;
    const uint32_t lane16 = (uint32_t)lane * 16;
    fetch_goes_to(lds_at + kValueSlots + ((parity + AHEAD) & 1) * kCodes);
    fetch_at<0, NT>(t, lane16);
    if constexpr (HD == 128) fetch_at<1024, NT>(t, lane16);
  }
  // Requests the first two tiles and waits for what was requested before.
  __device__ __forceinline__ void start() {
    in_issue_order();
    if (has(1)) {
      fetch_keys<0>(0);
      fetch_keys<1>(0);
      fetch_values<0>(0);
      fetch_values<1>(0);
      wait_vector_memory<2 * kFetches>();
    } else if (has(0)) {
      fetch_keys<0>(0);
      fetch_values<0>(0);
      wait_vector_memory<kFetches>();
    } else {
      wait_vector_memory<0>();
    }
    in_issue_order();
  }
  __device__ __forceinline__ void first_keys_arrived() const {
    in_issue_order();
    if (has(1)) wait_vector_memory<2 * kFetches - kKeyFetches>();
    else wait_vector_memory<kValueFetches>();
    in_issue_order();
  }
  // the values of this tile and the keys of the next one
  __device__ __forceinline__ void arrived() const {
    in_issue_order();
    if (has(2)) wait_vector_memory<kFetches>();          // requested after them: values of the next, keys of the one after it
    else if (has(1)) wait_vector_memory<kValueFetches>();
    else wait_vector_memory<0>();
    in_issue_order();
  }
  __device__ __forceinline__ Operand<HD> keys(int slot, int ahead) const { return read(slot * kCodes, ahead, 0); }
  __device__ __forceinline__ Operand<HD> values(int slot) const { return read(kValueSlots + slot * kCodes, 0, HD); }
  __device__ __forceinline__ Operand<HD> read(int codes, int ahead, int scales) const {
    Operand<HD> o;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) o.codes[i] = *reinterpret_cast<const u32x4*>(lds + codes + (i * 64 + lane) * 16);
    const uint8_t* at = lds + kScaleSlots + ((scale_slot + ahead) & 3) * kScales + scales + (lane & 31) * L::kGroups;
    if constexpr (HD == 128) o.scales = *reinterpret_cast<const uint32_t*>(at);
    else o.scales = *reinterpret_cast<const uint16_t*>(at);
    return o;
  }
};
static_assert(PackedLayout<128>::kKeyScales + 128 == PackedLayout<128>::kValueScales, "one request for both scales");

// Merge of the wavefronts: what one parks, [lane][register i][e] and one piece so that lanes rotate over the banks, and the columns'
// (reference, sum).
template <int HD> constexpr int park_row() { return 16 * (HD / 32) * 4 + 16; }
template <int HD> constexpr int park_bytes() { return 64 * park_row<HD>() + 64 * 4; }

// LDS of a workgroup: the query rows, the rows of the block's tiles, the rings.  What is parked later goes over all of it.
template <typename T, int HD> constexpr int workgroup_lds(int waves, int blk_tiles) {
  const int park = waves * park_bytes<HD>(), run = (1 + 2 * blk_tiles) * Rows<T, HD>::kBytes + waves * Ring<HD, false>::kBytes;
  return park > run ? park : run;
}
static_assert(workgroup_lds<__bf16, 128>(kPackedWavesBf16, 2) <= 160 * 1024 && workgroup_lds<float, 128>(kPackedWavesF32, 2) <= 160 * 1024, "LDS of a CU");

template <typename T, int HD, bool NT>
__global__ __launch_bounds__(Parts<T>::kWaves * kWave) void attn_packed_kernel(const PackedAttnParams p) {
  using L = PackedLayout<HD>;
  using R = Rows<T, HD>;
  constexpr int PARTS = Parts<T>::N, NE = L::kGroups, NF = HD / 16;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int half = lane >> 5, m = lane & 31;

  // columns of a KV head and split side by side on an XCD: they read the same tiles
  const int wg = xcd_contiguous_id(blockIdx.x, gridDim.x);
  const int pair = p.by_col_tiles.quotient(wg), ct = wg - pair * p.col_tiles;
  const int bg = p.by_split.quotient(pair), split = pair - bg * p.n_split;
  const int b = p.by_hkv.quotient(bg), g = bg - b * p.hkv;

  // The query rows, and with the last split the block's own keys and values, come once for all wavefronts, through LDS: as fragments that each
  // loads from memory they are 64 pieces of rows an instruction, 4000 cycles of the CU's address path.
  // Tiles of the block are taken by the first wavefronts, which have the fewest tiles of the cache.
  const int blk_tiles = split == p.n_split - 1 ? p.blk_tiles : 0;
  uint8_t* rest = smem + R::kBytes;
  R::request(smem, wave, nw, lane, [&](int r) {
    const int c = min(ct * kCols + r, p.cols - 1), cg = p.by_nq.quotient(c);
    return (const T*)p.q + b * p.q_sb + (g * p.group + cg) * p.q_sh + (c - cg * p.nq) * p.q_sr;
  });
  for (int t = 0; t < blk_tiles; ++t) {
    const size_t base = b * p.blk_sb + g * p.blk_sh;
    auto row = [&](int r) { return base + (size_t)min(t * kTileKeys + r, p.nq - 1) * p.blk_sr; };
    R::request(rest + 2 * t * R::kBytes, wave, nw, lane, [&](int r) { return (const T*)p.k_blk + row(r); });
    R::request(rest + (2 * t + 1) * R::kBytes, wave, nw, lane, [&](int r) { return (const T*)p.v_blk + row(r); });
  }

  Ring<HD, NT> ring;
  ring.lds = rest + blk_tiles * 2 * R::kBytes + wave * Ring<HD, NT>::kBytes;
  ring.lds_at = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(ring.lds));
  ring.c = split * p.tiles_per_split + nw - 1 - wave;
  ring.c_end = min(p.tiles, (split + 1) * p.tiles_per_split);
  ring.tile = in_scalars((const char*)p.cache + (size_t)bg * p.head_bytes + (size_t)ring.c * L::kTile);
  ring.nw = nw;
  ring.lane = lane;
  ring.scale_slot = 0;
  ring.start();
  bare_barrier();

  f32x16 acc[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  float m_ref = kNoMax, l_run = 0.f;

  for (int t = wave; t < blk_tiles; t += nw) {
    const uint8_t* rows = rest + 2 * t * R::kBytes;
    const int n = min(kTileKeys, p.nq - t * kTileKeys);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    if constexpr (sizeof(T) == 2) {
      bf16x8 kf[NF], qf[NF];                             // read before the first is used
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        kf[f] = *reinterpret_cast<const bf16x8*>(R::place(rows, m, 16 * (2 * f + half)));
        qf[f] = *reinterpret_cast<const bf16x8*>(R::place(smem, m, 16 * (2 * f + half)));
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < NF; ++f) s = mfma(kf[f], qf[f], s);
    } else {
#pragma unroll
      for (int f = 0; f < 2 * NF; ++f) {
        const f32x4 kf = *reinterpret_cast<const f32x4*>(R::place(rows, m, 16 * (2 * f + half))), qf = *reinterpret_cast<const f32x4*>(R::place(smem, m, 16 * (2 * f + half)));
#pragma unroll
        for (int x = 0; x < 4; ++x) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[x], qf[x], s, 0, 0, 0);
      }
    }
    // a lane takes HD / 32 neighbouring channels of each of its sixteen values
    typedef __attribute__((ext_vector_type(HD / 32))) T Few;
    Few v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = *reinterpret_cast<const Few*>(R::place(rows + R::kBytes, 8 * (r >> 2) + 4 * half + (r & 3), m * NE * (int)sizeof(T)));
    __builtin_amdgcn_sched_barrier(0);
    softmax_step<NE>(s, n, p.scale_log2, half, m_ref, l_run, acc);
    if (n < kTileKeys) {                                 // rows past the block are the last one again: as zeros
      asm volatile("");
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= n - 4 * half) v[r] = Few(0);
    }
    if constexpr (sizeof(T) == 2) {
      bf16x8 pb[2][1];
      prob_parts<1>(s, pb);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const bf16x8 vf = {v[8 * st][e], v[8 * st + 1][e], v[8 * st + 2][e], v[8 * st + 3][e], v[8 * st + 4][e], v[8 * st + 5][e], v[8 * st + 6][e], v[8 * st + 7][e]};
          acc[e] = mfma(vf, pb[st][0], acc[e]);
        }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)                       // the keys of a lane's register r are the two of a step
#pragma unroll
        for (int e = 0; e < NE; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[r][e], s[r], acc[e], 0, 0, 0);
    }
  }

  if (ring.has(0)) {
    Queries<T, HD> queries;
    queries.load(smem, m, half);
    float m_loc;                                         // of the tile whose logits are there
    // One tile: its softmax and its product with the values, and the next tile's logits.  While a matrix instruction waits, for the one before
    // it or for the unit, nothing of any wavefront is issued to the SIMD's vector units; so each is followed by as many vector instructions as
    // it takes, in this order (the barriers keep the compiler from gathering them).  Little overlaps all the same: a tile takes the sum of both times.
    auto step = [&](auto parity_tag, f32x16& s, f32x16& s_next) {
      constexpr int kParity = decltype(parity_tag)::value;
      ring.arrived();
      const Operand<HD> values = ring.values(kParity);
      const Operand<HD> keys = ring.keys(1 - kParity, 1);   // after the last tile: whatever is there, and its logits are not used
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (ring.has(3)) ring.template fetch_keys<3>(kParity);
      if (ring.has(2)) ring.template fetch_values<2>(kParity);
      in_issue_order();
      move_reference<NE>(m_loc, m_ref, l_run, acc);
      float l_loc = 0.f;
      auto numerators = [&](int from) {
#pragma unroll
        for (int i = from; i < from + 4; ++i) {
          s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2, -m_ref));
          l_loc += s[i];
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      __builtin_amdgcn_sched_barrier(0);
      queries.template logits<0>(keys, half, s_next);
      numerators(0);
      queries.template logits<1>(keys, half, s_next);
      numerators(4);
      queries.template logits<2>(keys, half, s_next);
      numerators(8);
      queries.template logits<3>(keys, half, s_next);
      numerators(12);
      l_run += l_loc;
      bf16x8 pb[2][PARTS];
      prob_parts<PARTS>(s, pb);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const bf16x8 vf = unpack8(values.codes[e >> 1][2 * (e & 1) + st], scale_of_byte(values.scales, e));
#pragma unroll
          for (int n = PARTS - 1; n >= 0; --n) acc[e] = mfma(vf, pb[st][n], acc[e]);
          __builtin_amdgcn_sched_barrier(0);
        }
      ring.c += nw;
      ring.tile += nw * L::kTile;
      ring.scale_slot = (ring.scale_slot + 1) & 3;
      m_loc = mask_max(s_next, ring.rows_left(p.n_cached), p.scale_log2, half);
    };
    f32x16 s0, s1;
    ring.first_keys_arrived();
    {
      const Operand<HD> keys = ring.keys(0, 0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (ring.has(2)) ring.template fetch_keys<2>(0);
      in_issue_order();
      queries.template logits<0>(keys, half, s0);
      queries.template logits<1>(keys, half, s0);
      queries.template logits<2>(keys, half, s0);
      queries.template logits<3>(keys, half, s0);
      m_loc = mask_max(s0, ring.rows_left(p.n_cached), p.scale_log2, half);
      if (wave >= blk_tiles) m_ref = fmaxf(kNoMax, fmaxf(m_loc, __shfl_xor(m_loc, 32)));   // nothing to rescale yet
    }
    while (true) {
      step(std::integral_constant<int, 0>{}, s0, s1);
      if (!ring.has(0)) break;
      step(std::integral_constant<int, 1>{}, s1, s0);
      if (!ring.has(0)) break;
    }
  }
  const float l_tot = l_run + __shfl_xor(l_run, 32);

  // Merge of the wavefronts: each parks its results and its columns' (reference, sum); wave w then folds four neighbouring channels a
  // lane, pieces w, w + nw, ... of a lane's results, of all of them.
  const bool stored = ct * kCols + m < p.cols;
  const int col = stored ? ct * kCols + m : 0, hg = p.by_nq.quotient(col), h = g * p.group + hg, row = col - hg * p.nq;
  const size_t slot = (size_t)(bg * p.col_tiles + ct) * p.n_split + split;
  // where the lane's columns go, worked out before the barriers
  uint64_t row_at = p.n_split == 1 ? (uint64_t)((T*)p.out + b * p.o_sb + h * p.o_sh + row * p.o_sr) : (uint64_t)(p.part_o + (slot * kCols + m) * HD);
  asm volatile("" : "+v"(row_at));
  constexpr int kPieces = 4 * NE, kPer = 4 / NE;         // registers of a piece
  uint8_t* mine = smem + wave * park_bytes<HD>();
  __syncthreads();                                       // all wavefronts are through with what lies there
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    f32x4 v;
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = acc[x % NE][u * kPer + x / NE];
    *reinterpret_cast<f32x4*>(mine + lane * park_row<HD>() + u * 16) = v;
  }
  if (lane < 32) {
    float* ml = reinterpret_cast<float*>(mine + 64 * park_row<HD>());
    ml[lane] = m_ref;
    ml[32 + lane] = l_tot;
  }
  __syncthreads();
  auto merge = [&](auto nw_tag) {
    constexpr int NW = decltype(nw_tag)::value;
    float f_w[NW], l_w[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float* of = reinterpret_cast<const float*>(smem + w * park_bytes<HD>() + 64 * park_row<HD>());
      f_w[w] = of[m];
      l_w[w] = of[32 + m];
    }
    f32x4 part[2][NW];
    auto request = [&](int u, f32x4 (&to)[NW]) {
#pragma unroll
      for (int w = 0; w < NW; ++w) to[w] = *reinterpret_cast<const f32x4*>(smem + w * park_bytes<HD>() + lane * park_row<HD>() + u * 16);
    };
    if (wave < kPieces) request(wave, part[0]);
    float m_tot = f_w[0], l_all = 0.f;
#pragma unroll
    for (int w = 1; w < NW; ++w) m_tot = fmaxf(m_tot, f_w[w]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      f_w[w] = __builtin_amdgcn_exp2f(f_w[w] - m_tot);
      l_all = __builtin_fmaf(l_w[w], f_w[w], l_all);
    }
    const float inv = 1.f / l_all;
    auto fold = [&](int u, const f32x4 (&of)[NW]) {
      f32x4 o = of[0] * f_w[0];
#pragma unroll
      for (int w = 1; w < NW; ++w) o += of[w] * f_w[w];
      const int i0 = u * kPer, ch = NE * (8 * (i0 >> 2) + 4 * half + (i0 & 3));
      if (p.n_split == 1) {
        typedef __attribute__((ext_vector_type(4))) T Four;
        Four y;
#pragma unroll
        for (int x = 0; x < 4; ++x) y[x] = (T)(o[x] * inv);
        if (stored) *reinterpret_cast<__attribute__((address_space(1))) Four*>(row_at + ch * sizeof(T)) = y;
      } else {
        *reinterpret_cast<__attribute__((address_space(1))) f32x4*>(row_at + ch * sizeof(float)) = o;
      }
    };
    for (int u = wave; u < kPieces; u += 2 * NW) {       // the next piece is requested before this one is folded
      if (u + NW < kPieces) request(u + NW, part[1]);
      fold(u, part[0]);
      if (u + 2 * NW < kPieces) request(u + 2 * NW, part[0]);
      if (u + NW < kPieces) fold(u + NW, part[1]);
    }
    if (p.n_split > 1 && wave == 0 && lane < 32) {
      p.part_ml[slot * 64 + lane] = m_tot;
      p.part_ml[slot * 64 + 32 + lane] = l_all;
    }
  };
  switch (nw) {
    case 1: merge(std::integral_constant<int, 1>{}); break;
    case 2: merge(std::integral_constant<int, 2>{}); break;
    case 3: merge(std::integral_constant<int, 3>{}); break;
    case 4: merge(std::integral_constant<int, 4>{}); break;
    case 5: merge(std::integral_constant<int, 5>{}); break;
    case 6: merge(std::integral_constant<int, 6>{}); break;
    case 7: merge(std::integral_constant<int, 7>{}); break;
    default: merge(std::integral_constant<int, 8>{}); break;
  }
}

// One thread folds the splits of four channels of a column.
template <typename T, int HD>
__global__ __launch_bounds__(256) void attn_packed_merge_kernel(const PackedAttnParams p) {
  const int unit = blockIdx.x / (kCols * HD / 4 / 256), at = (blockIdx.x % (kCols * HD / 4 / 256)) * 256 + threadIdx.x;
  const int m = at / (HD / 4), c4 = at % (HD / 4) * 4;
  const int bg = p.by_col_tiles.quotient(unit), ct = unit - bg * p.col_tiles;
  const int col = ct * kCols + m;
  if (col >= p.cols) return;
  const size_t slot = (size_t)unit * p.n_split;
  const RowPiece r = fold_splits<kCols>(p.part_ml + slot * 64 + m, p.part_o + (slot * kCols + m) * HD + c4, (size_t)kCols * HD, p.n_split, 0, 1);
  const int b = p.by_hkv.quotient(bg), g = bg - b * p.hkv, hg = p.by_nq.quotient(col), h = g * p.group + hg, row = col - hg * p.nq;
  store_piece<T>(r, (T*)p.out + b * p.o_sb + h * p.o_sh + row * p.o_sr + c4);
}

template <typename T, int HD, bool NT>
hipError_t launch_kernel(const PackedAttnParams& p, int units, hipStream_t s) {
  static LdsOptIn opt;
  const hipError_t e = opt.ensure(reinterpret_cast<const void*>(attn_packed_kernel<T, HD, NT>), workgroup_lds<T, HD>(Parts<T>::kWaves, 2));
  if (e != hipSuccess) return e;
  return launch(attn_packed_kernel<T, HD, NT>, dim3((uint32_t)units * p.n_split), dim3(p.waves * kWave), workgroup_lds<T, HD>(p.waves, p.blk_tiles), s, p);
}

template <typename T, int HD>
hipError_t launch_as(const PackedAttnParams& p, hipStream_t s) {
  const int units = p.batch * p.hkv * p.col_tiles;
  hipError_t e;
  if constexpr (sizeof(T) == 2) e = p.past_caches ? launch_kernel<T, HD, true>(p, units, s) : launch_kernel<T, HD, false>(p, units, s);
  else e = launch_kernel<T, HD, false>(p, units, s);
  if (e != hipSuccess || p.n_split == 1) return e;
  return launch(attn_packed_merge_kernel<T, HD>, dim3((uint32_t)units * (kCols * HD / 4 / 256)), dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_attn_packed(const PackedAttnParams& p, int dtype, int d, hipStream_t s) {
  if (dtype == 0) return d == 128 ? launch_as<__bf16, 128>(p, s) : launch_as<__bf16, 64>(p, s);
  return d == 128 ? launch_as<float, 128>(p, s) : launch_as<float, 64>(p, s);
}

}  // namespace sdllm
