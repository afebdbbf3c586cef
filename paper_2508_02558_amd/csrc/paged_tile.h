// What the kernels of the paged cache's attention share: which queries and keys a workgroup takes, and what a query row sees of a tile.
//
// The query rows of a KV head are columns: column c is query head c % G of the group and row c / G of the sequence, so that neighbours see nearly the same
// keys.  A workgroup takes a block of columns (an item) and all 32-key tiles that any of them sees, or a split of those tiles.  Lengths are
// known on the device only, so every wavefront works out the cut by itself: with W workgroups, n items and N tiles of all items together, a share is
// c tiles at most and an item with T tiles has ceil(T / c) splits.  c = ceil(N / (W - n)) is enough for their sum to be W at most, as it is below N / c + n; the
// least c that is, or near it, is found by halving.  Sums over the sequences, 64 of them at a time; nothing is kept between calls.
#pragma once

#include "mfma_tile.h"

namespace sdllm {

struct PagedItem {
  int b, g, blk;            // sequence, KV head, block of columns
  int split, n_split, slot; // slot: place of the split's partials
  int length, count, end;   // rows before the new ones, new ones, rows that can be seen
  int cols;                 // columns of the KV head
  int sink_end;             // first keys that any row of the block sees as such: [0, sink_end)
  int first, last;          // keys of the window of any row: [first, last]
  int least_last, most_first;   // keys [most_first, least_last] are in the window of every row
  bool past_caches;         // so many tiles are read in all that what is read does not stay in the caches anyway: tiles of 32 rows one stride apart are read past them
  int lead_tiles;           // tiles before the window's: of first keys, or (kSeeTree) of the cache
  int first_tile, tiles;    // first tile of the window; tiles in all
};

// Workgroup ids are dealt round-robin over the XCDs, and by each XCD over its shader engines, without regard to how long a workgroup takes.  So is the
// work: every XCD takes `chunk` neighbours, which read the same keys, of every 8 chunk ids, and every other turn goes backwards over XCDs and neighbours,
// so that ids in descending order of work come out even.  (Contiguous ranges, xcd_contiguous_id, give an XCD whole sequences: prompts of unlike lengths took 319
// us instead of 237.)  chunk is 4: causal, four sequences of 4096 rows x 28/4 heads 522 us with 2, 488 with 4, 481 with 8; 32 heads x 4096 rows 151, 161, 182.
__device__ __forceinline__ int chunked_id(const PagedAttnParams& p, int dealt, int n) {
  const int x = dealt % kNumXCDs, s = dealt / kNumXCDs, turn = p.by_chunk.quotient(s), e = s - turn * p.chunk;
  if (dealt >= p.by_chunk.quotient(n / kNumXCDs) * p.chunk * kNumXCDs) return dealt;
  return turn & 1 ? (turn * kNumXCDs + kNumXCDs - 1 - x) * p.chunk + p.chunk - 1 - e : (turn * kNumXCDs + x) * p.chunk + e;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Sum of x over the lanes up to this one, in registers (shuffles go through LDS)
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1, 2, 4, 8: within rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), kWave - 1); }

__device__ __forceinline__ int last_seen(const PagedAttnParams& p, int end, int place) {
  return p.right < 0 ? end - 1 : min(end - 1, place + p.right);
}
__device__ __forceinline__ int first_seen(const PagedAttnParams& p, int place) { return p.left < 0 ? 0 : max(0, place - p.left); }

// Blocks of columns of a KV head
__device__ __forceinline__ int blocks_of(const PagedAttnParams& p, int count) { return ceil_div(count * p.group, p.block_cols); }

// No block of the sequence has more tiles than this
template <int SEES>
__device__ __forceinline__ int most_tiles(const PagedAttnParams& p, int length, int count) {
  if (SEES == kSeeTree) return ceil_div(length, kTileKeys) + ceil_div(count, kTileKeys);
  const int all = ceil_div(min(length + count, p.cache.capacity), kTileKeys);
  if (p.left < 0 || p.right < 0) return all;
  const int rows = min(count, p.block_cols / p.group + 2);   // of a block
  return min(all, (p.left + p.right + rows) / kTileKeys + 2 + ceil_div(min(p.sinks, p.cache.capacity), kTileKeys));
}

// Rows and tiles of an item whose sequence, head and block are known
template <int SEES>
__device__ __forceinline__ void locate_item(const PagedAttnParams& p, PagedItem& w) {
  w.cols = w.count * p.group;
  w.end = SEES == kSeeTree ? w.length : min(w.length + w.count, p.cache.capacity);
  if (SEES == kSeeTree) {
    w.lead_tiles = ceil_div(w.length, kTileKeys);
    w.tiles = w.lead_tiles + ceil_div(w.count, kTileKeys);
    return;
  }
  const int c0 = w.blk * p.block_cols, c1 = min(c0 + p.block_cols, w.cols) - 1;
  const int p0 = w.length + p.by_group.quotient(c0), p1 = w.length + p.by_group.quotient(c1);
  w.first = first_seen(p, p0);
  w.most_first = first_seen(p, p1);
  w.least_last = last_seen(p, w.end, p0);
  w.last = last_seen(p, w.end, p1);
  w.sink_end = min(p.sinks, w.last + 1);
  w.first_tile = w.first / kTileKeys;
  w.lead_tiles = ceil_div(w.sink_end, kTileKeys);
  int window = 0;
  if (w.first <= w.last) {
    w.lead_tiles = min(w.lead_tiles, w.first_tile);
    window = w.last / kTileKeys - w.first_tile + 1;
  }
  w.tiles = w.lead_tiles + window;
}

// The item and split of this workgroup, the same for all of its threads; false: none
template <int SEES>
__device__ __forceinline__ bool find_item(const PagedAttnParams& p, int lane, PagedItem& w) {
  if (!p.part_o) {
    // Items as workgroups: `chunk` neighbouring blocks of a head, then those of the other heads, from the last blocks to the first: with all past keys to see the
    // last have the most tiles, and those that are not there come at the end.  (One head after another: causal, 32 heads x 4096 rows 257 us instead of 180, two
    // sequences of 2048 rows x 28/4 heads 114 instead of 78.)  The heads' order turns from chunk to chunk, or the ones whose sequences are long would stay
    // on a few XCDs (four sequences of 1024 to 4096 rows x 28/4 heads, a window of 1024 keys: 215 us, unturned 250).
    const int id = chunked_id(p, blockIdx.x, gridDim.x);
    const int unit = p.by_chunk.quotient(id), turn = p.by_heads.quotient(unit), place = unit + turn * p.turned;
    const int head = place - p.by_heads.quotient(place) * p.heads, rank = id + (turn - unit) * p.chunk;
    w.b = p.by_hkv.quotient(head);
    w.g = head - w.b * p.hkv;
    w.count = __builtin_amdgcn_readfirstlane(p.cache.count(w.b));
    w.length = __builtin_amdgcn_readfirstlane(p.cache.length(w.b));
    const int blocks = blocks_of(p, w.count);
    if (rank >= blocks) return false;
    w.blk = blocks - 1 - rank;
    w.split = 0;
    w.n_split = 1;
    w.slot = 0;
    locate_item<SEES>(p, w);
    w.past_caches = p.max_blocks == 1 && (int64_t)gridDim.x * w.tiles >= p.caches_tiles;   // a guess: as if all items were like this one
    return true;
  }
  struct Seq { int length, count, blocks, tiles; };
  auto sequence = [&](int b) {
    if (b >= p.batch) return Seq{0, 0, 0, 0};
    const int count = p.cache.count(b), length = p.cache.length(b);
    return Seq{length, count, blocks_of(p, count), most_tiles<SEES>(p, length, count)};
  };
  const Seq mine = sequence(lane);   // the first 64 sequences are looked at once
  auto sequence_at = [&](int b0) { return b0 == 0 ? mine : sequence(b0 + lane); };
  auto over_all = [&](auto f) {
    int n = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kWave) {
      const Seq s = sequence_at(b0);
      n += f(s, p.hkv * s.blocks);
    }
    return wave_sum(n);
  };
  const int items = over_all([](const Seq&, int heads) { return heads; });
  const int tiles = over_all([&](const Seq& s, int heads) { return heads * ((s.tiles >> p.tile_shift) + 1); });   // in units of 2^tile_shift, which add up in 32 bits
  // By floats: all that counts is that every wavefront finds the same number, and that the sum fits the grid.
  auto splits_at = [](const Seq& s, float per_tile) { return max(1, (int)ceilf((float)s.tiles * per_tile)); };
  auto used_at = [&](int share) {
    const float per_tile = __builtin_amdgcn_rcpf((float)share);
    return over_all([&](const Seq& s, int heads) { return heads * splits_at(s, per_tile); });
  };
  // The host launches more workgroups than there can be items: this share is enough, and the least that is lies between N / W and it.
  const float unit = (float)(1 << p.tile_shift), all = (float)tiles * unit;
  int share = max(p.least_tiles, (int)(all * __builtin_amdgcn_rcpf((float)(p.workgroups - items)) * 1.0001f) + 2), used = used_at(share);
  if (share > p.least_tiles) {
    int too_small = max(p.least_tiles - 1, (int)(all * __builtin_amdgcn_rcpf((float)p.workgroups) * 0.9999f - unit) - 1);
    for (int i = 0; i < 5 && share - too_small > 1; ++i) {
      const int middle = too_small + (share - too_small) / 2, u = used_at(middle);
      if (u <= p.workgroups) { share = middle; used = u; }
      else too_small = middle;
    }
  }
  while (used > p.workgroups) used = used_at(share += share / 8 + 1);   // not reached but by rounding
  if ((int)blockIdx.x >= used) return false;
  w.past_caches = p.max_blocks == 1 && (int64_t)tiles << p.tile_shift >= p.caches_tiles;
  const int id = chunked_id(p, blockIdx.x, used);
  int before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kWave) {
    const Seq s = sequence_at(b0);
    const int splits = splits_at(s, __builtin_amdgcn_rcpf((float)share)), here = p.hkv * s.blocks * splits, upto = wave_scan(here);
    const uint64_t past = __ballot(id < before + upto);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int blocks = __builtin_amdgcn_readlane(s.blocks, l);
      before += __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(here, l);
      w.n_split = __builtin_amdgcn_readlane(splits, l);
      w.b = b0 + l;
      // those of a head and split are neighbours: they read the same keys
      const int r = id - before, unit = r / blocks;
      w.blk = r - unit * blocks;
      w.g = unit / w.n_split;
      w.split = unit - w.g * w.n_split;
      w.slot = before + (w.g * blocks + w.blk) * w.n_split + w.split;
      w.count = __builtin_amdgcn_readlane(s.count, l);
      w.length = __builtin_amdgcn_readlane(s.length, l);
      locate_item<SEES>(p, w);
      if (w.split == 0 && threadIdx.x == 0) {
        int32_t* at = p.item_at + 2 * ((int64_t)(w.b * p.hkv + w.g) * p.max_blocks + w.blk);
        at[0] = w.slot;
        at[1] = w.n_split;
      }
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return false;
}

// One 32-key tile of an item.  Rows [lo, hi) of it are seen by some row of the block; the others may be anything, in pages of anybody.
struct PagedTile {
  bool own;      // kSeeTree: of the new rows
  int at;        // first key
  int lo, hi;
  bool full;     // every row of the block sees all 32
};

template <int SEES>
__device__ __forceinline__ PagedTile tile_of(const PagedAttnParams& p, const PagedItem& w, int t) {
  PagedTile x;
  if (SEES == kSeeTree) {
    x.own = t >= w.lead_tiles;
    x.at = (x.own ? t - w.lead_tiles : t) * kTileKeys;
    x.lo = 0;
    x.hi = min(kTileKeys, (x.own ? w.count : w.length) - x.at);
    x.full = x.hi == kTileKeys && !(x.own && p.mask);
    return x;
  }
  const bool lead = t < w.lead_tiles;
  x.own = false;
  x.at = (lead ? t : t - w.lead_tiles + w.first_tile) * kTileKeys;
  x.lo = lead || p.sinks > x.at ? 0 : max(0, w.first - x.at);
  x.hi = min(kTileKeys, (lead ? w.sink_end : w.last + 1) - x.at);
  x.full = (x.at >= w.most_first || x.at + kTileKeys <= p.sinks) && x.at + kTileKeys - 1 <= w.least_last;
  return x;
}

// What one query row sees
struct RowSight {
  uint64_t bits;       // kSeeTree: of the new rows
  int first, last;     // kSeeWindow
  bool none;           // no key at all
};

template <int SEES>
__device__ __forceinline__ RowSight sight_of(const PagedAttnParams& p, const PagedItem& w, int row) {
  RowSight r;
  r.bits = 0;
  r.first = r.last = 0;
  if (SEES == kSeeTree) {
    const uint64_t there = w.count >= 64 ? ~0ull : (1ull << w.count) - 1;
    r.bits = (p.mask ? p.mask[w.b * p.mask_stride + row] : ~0ull) & there;
    r.none = w.length == 0 && r.bits == 0;
  } else {
    r.first = first_seen(p, w.length + row);
    r.last = last_seen(p, w.end, w.length + row);
    r.none = r.last < 0 || (r.first > r.last && p.sinks == 0);
  }
  return r;
}

// Bits [0, n) of 32, for any n
__device__ __forceinline__ uint32_t bits_below(int n) { return (uint32_t)(0xffffffffull >> (32 - min(max(n, 0), 32))); }

// Bit r: the row sees key r of the tile
template <int SEES>
__device__ __forceinline__ uint32_t seen_bits(const PagedAttnParams& p, const PagedTile& x, const RowSight& r) {
  if (SEES == kSeeTree) return x.own ? (uint32_t)(r.bits >> x.at) : bits_below(x.hi);
  return bits_below(r.last + 1 - x.at) & (~bits_below(r.first - x.at) | bits_below(p.sinks - x.at));
}

// The page that holds a row, one of the pool's in any case
__device__ __forceinline__ int64_t page_of(const PagedCache& c, int b, int row) {
  return min(max(c.table[b * c.table_stride + (row >> c.page_shift)], 0), c.n_pages - 1);
}

// Bit `bit` of x as a mask of all bits: one instruction, and no comparison whose result would take a pair of scalar registers
__device__ __forceinline__ uint32_t bit_mask(uint32_t x, int bit) { return (uint32_t)((int32_t)(x << (31 - bit)) >> 31); }
__device__ __forceinline__ float or_minus_infinity(float s, uint32_t m) {
  return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) & m) | (0xff800000u & ~m));
}

// Values of a masked tile that are no numbers take no part in rows that do not see them, where zero times them would be NaN.  They are taken out of the
// operands, and a wavefront that met any goes over the tiles it looked at once more at the end, key by key, and adds them to the results of the rows that
// see them: to find out costs masked tiles three instructions a pair of values, the rest nothing but where it happens.
// `where(n)` is tile n of this wavefront's if its operands were looked at, or negative; `add(v_row, sees)` adds the infinities and NaN of one row of V.
template <int SEES, class Where, class Add>
__device__ __forceinline__ void add_specials(const PagedAttnParams& p, const PagedItem& w, const RowSight& sight, int esize, int tiles, const Where& where, const Add& add) {
  const PagedCache& c = p.cache;
  for (int n = 0; n < tiles; ++n) {
    const int t = where(n);
    if (t < 0) continue;
    const PagedTile x = tile_of<SEES>(p, w, t);
    const uint32_t seen = seen_bits<SEES>(p, x, sight);
    for (int r = x.lo; r < x.hi; ++r) {
      const int row = x.at + r;
      const char* v = SEES == kSeeTree && x.own
                          ? (const char*)p.v_blk + esize * (w.b * p.blk_sb + w.g * p.blk_sh + row * p.blk_sr)
                          : (const char*)p.v_pages + esize * (page_of(c, w.b, row) * c.sp + w.g * c.sh + (row & ((1 << c.page_shift) - 1)) * c.sr);
      add(v, (seen >> r & 1) != 0);
    }
  }
}

}  // namespace sdllm
