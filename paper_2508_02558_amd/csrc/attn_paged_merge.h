// Merge of the shares of the paged cache's attention: what the workgroups of an item left, folded with the usual rescaling, as a launch of its own.
// An item's first workgroup says where its partials are and how many (item_at).  Bound by round trips: the item's place, then everything else
// of several shares at once, with many shares by eight lanes that take every eighth each.  64 blocks of 256 columns x 128 in four shares (33 MB) 8.6 us, 128 of
// 16 columns 4.9.
#pragma once

#include "attn_merge.h"
#include "paged_math.h"

namespace sdllm {

constexpr int kPagedMergeThreads = 256;

// TPI adjacent lanes fold the shares of four channels of a column, NB shares at a time; blockIdx.x is the item, blockIdx.y a part of its results.
template <typename E, int HD, int C, int TPI, int NB>
__global__ __launch_bounds__(kPagedMergeThreads) void attn_paged_merge_kernel(const PagedAttnParams p) {
  using M = Math<E, HD, C>;
  const int item = blockIdx.x, tid = blockIdx.y * kPagedMergeThreads + threadIdx.x, sub = tid % TPI;
  const int at = tid / TPI, lane = at % kWave, i = at / kWave % M::kSlots, cols = at / (kWave * M::kSlots), col = cols * C + lane % C;
  const int head = p.by_blocks.quotient(item), blk = item - head * p.max_blocks;
  const int b = p.by_hkv.quotient(head), g = head - b * p.hkv;
  const int column = blk * p.block_cols + col;
  const int slot = p.item_at[2 * item], n_split = p.item_at[2 * item + 1];
  // an item that is not there has left nothing, not even its place
  if (column >= p.cache.count(b) * p.group || col >= p.block_cols || n_split < 2) return;
  const float* ml = p.part_ml + (int64_t)slot * 2 * p.block_cols + col;
  const mf32x4* po = reinterpret_cast<const mf32x4*>(partial_slot<M>(p, slot, cols, i, lane));
  const int64_t next = (int64_t)p.block_cols * HD / 4;
  RowPiece r;
  for (int s0 = sub; s0 < n_split; s0 += NB * TPI) {
    float m_s[NB], l_s[NB];
    mf32x4 o_s[NB];
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int64_t s = min(s0 + u * TPI, n_split - 1);   // past the end: left out below
      m_s[u] = ml[s * 2 * p.block_cols];
      l_s[u] = ml[s * 2 * p.block_cols + p.block_cols];
      o_s[u] = po[s * next];
    }
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      RowPiece x;
      x.m = m_s[u];
      x.l = l_s[u];
      x.o = o_s[u];
      if (s0 + u * TPI < n_split) merge_pieces(r, x);
    }
  }
#pragma unroll
  for (int o = 1; o < TPI; o <<= 1) {
    RowPiece other;
    other.m = __shfl_xor(r.m, o);
    other.l = __shfl_xor(r.l, o);
#pragma unroll
    for (int c = 0; c < 4; ++c) other.o[c] = __shfl_xor(r.o[c], o);
    merge_pieces(r, other);
  }
  if (sub != 0) return;
  const int row = p.by_group.quotient(column), h = g * p.group + column - row * p.group;
  if (r.m == -INFINITY) {   // the row sees nothing
    r.l = 1.f;
    r.o = mf32x4{0.f, 0.f, 0.f, 0.f};
  }
  store_piece<E>(r, (E*)p.out + b * p.o_sb + h * p.o_sh + row * p.o_sr + M::channel(i, lane));
}

template <typename E, int HD, int C, int TPI, int NB>
hipError_t launch_paged_merge_by(const PagedAttnParams& p, int most_cols, hipStream_t s) {
  const int items = p.batch * p.hkv * p.max_blocks, blocks = (most_cols + C - 1) / C;
  const dim3 grid((unsigned)items, (unsigned)(blocks * C * (HD / 4) * TPI / kPagedMergeThreads));
  return launch(attn_paged_merge_kernel<E, HD, C, TPI, NB>, grid, dim3(kPagedMergeThreads), 0, s, p);
}

template <typename E, int HD, int C>
hipError_t launch_paged_merge(const PagedAttnParams& p, hipStream_t s) {
  const int64_t cols = (int64_t)p.cache.rows * p.group;
  const int most_cols = cols < p.block_cols ? (int)cols : p.block_cols;
  const int items = p.batch * p.hkv * p.max_blocks;
  // Eight lanes where one would have many shares to fold one round after another (a token over one head x 30000 keys 17.6 us, with one lane 19.4; a tree of 64 rows
  // x 8/1 heads x 30000 keys 34.8, 47.2), unless the results need the machine's lanes themselves (two trees of 64 rows x 28/4 heads x 16000 keys 64.2, 56.1).
  return p.workgroups / items >= 16 && (int64_t)items * p.block_cols * (HD / 4) <= 2 * kNumCUs * kWave
             ? launch_paged_merge_by<E, HD, C, 8, 8>(p, most_cols, s) : launch_paged_merge_by<E, HD, C, 1, 8>(p, most_cols, s);
}

}  // namespace sdllm
