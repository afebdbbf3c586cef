// C-ABI entry points of the paged cache: argument checks, launch planning and dispatch.
#include <algorithm>

#include "api_checks.h"
#include "sdllm_bench.h"
#include "sdllm_internal.h"

using namespace sdllm;

namespace {

int32_t check_paged(const sdllm_paged_shape_t* shape) {
  if (!shape) return SDLLM_ERR_INVALID_ARG;
  const sdllm_paged_shape_t& s = *shape;
  if (s.batch < 1 || s.n_kv_heads < 1 || s.n_q_heads < 1 || s.n_q_heads % s.n_kv_heads != 0 || s.rows < 0 || s.n_pages < 0 || s.table_pages < 0 ||
      s.sinks < 0 || s.reserved != 0)
    return SDLLM_ERR_INVALID_ARG;
  if (s.dtype != SDLLM_BF16 && s.dtype != SDLLM_F32) return SDLLM_ERR_INVALID_ARG;
  if (!(s.softmax_scale >= 0.f) || !isfinite(s.softmax_scale)) return SDLLM_ERR_INVALID_ARG;
  if (s.table_stride < 0 || s.mask_stride < 0) return SDLLM_ERR_INVALID_ARG;
  const int es = elem_size(s.dtype);
  if (!strides_ok(s.q_stride, es) || !strides_ok(s.blk_stride, es) || !strides_ok(s.out_stride, es) || !strides_ok(s.page_stride, es))
    return SDLLM_ERR_INVALID_ARG;
  if (s.head_dim != 64 && s.head_dim != 128) return SDLLM_ERR_UNSUPPORTED;
  if (s.page_rows < 1) return SDLLM_ERR_INVALID_ARG;
  if (s.page_rows < 16 || s.page_rows > 256 || (s.page_rows & (s.page_rows - 1)) != 0) return SDLLM_ERR_UNSUPPORTED;
  if (s.rows > kPagedMax || (int64_t)s.table_pages * s.page_rows > kPagedMax) return SDLLM_ERR_UNSUPPORTED;
  return SDLLM_OK;
}

int32_t capacity_of(const sdllm_paged_shape_t& s) { return s.n_pages > 0 ? s.table_pages * s.page_rows : 0; }

// The pages, and the integers that say what is in them
int32_t fill_cache(const sdllm_paged_shape_t& s, const void* k_pages, const void* v_pages, const int32_t* table, const int32_t* lengths,
                   const int32_t* row_counts, PagedCache& c) {
  const int32_t capacity = capacity_of(s);
  if (!lengths) return SDLLM_ERR_INVALID_ARG;
  if (capacity > 0 && (!k_pages || !v_pages || !table || !aligned16(k_pages) || !aligned16(v_pages) || !row_stride_ok(s.page_stride, s.head_dim)))
    return SDLLM_ERR_INVALID_ARG;
  c.table = table; c.lengths = lengths; c.counts = row_counts;
  c.table_stride = s.table_stride;
  c.sp = s.page_stride[0]; c.sh = s.page_stride[1]; c.sr = s.page_stride[2];
  c.n_pages = s.n_pages;
  c.page_shift = __builtin_ctz((unsigned)s.page_rows);
  c.capacity = capacity;
  c.rows = s.rows;
  return SDLLM_OK;
}

// How a call is cut up (paged_tile.h): columns of a workgroup by the kernel, and how many workgroups there are for shares of the tiles.
int32_t plan_paged(const sdllm_paged_shape_t& s, bool tree, PagedPlan& pl) {
  const int64_t cols = (int64_t)s.rows * (s.n_q_heads / s.n_kv_heads);
  pl = PagedPlan{};
  const bool f32 = s.dtype == SDLLM_F32;
  const int64_t heads = (int64_t)s.batch * s.n_kv_heads;
  // 16 columns are enough for a token's heads and take less than 32 with half of them empty (a token of 4 sequences of 1000 keys x 28/4 heads 10.9 us, 11.8).
  // Up to 64 columns two blocks that read the same tiles, one of them from L2, are ahead of waves that share them (8 trees of 16 rows x 32/8 heads x 4096 rows
  // 33.2 us, shared 38.8), up to 128 where there are few heads (one tree of 32 rows x 32/8 heads x 8192 rows 21.5, shared 26.0; 8 trees 44.4, 40.0).
  pl.shared = !f32 && cols > (heads <= 16 ? 128 : 64);
  pl.block_cols = f32 || cols <= 16 ? 16 : !pl.shared ? 32 : cols <= 128 ? 128 : 256;
  // columns, blocks and threads of a launch (the merge's too) are counted in 32 bits
  if (cols > INT32_MAX - 256) return SDLLM_ERR_UNSUPPORTED;
  pl.max_blocks = (int)((cols + pl.block_cols - 1) / pl.block_cols);
  if (heads > INT32_MAX) return SDLLM_ERR_UNSUPPORTED;
  const int64_t items = heads * pl.max_blocks;
  const int chunks = std::max(1, (pl.max_blocks + 3) / 4);   // neighbours that are started together: four, or nearly
  pl.chunk = (pl.max_blocks + chunks - 1) / chunks;
  const int64_t whole = heads * chunks * pl.chunk;   // workgroups of items that are not cut
  if (whole > UINT32_MAX / (kGeneralMaxWaves * kWave)) return SDLLM_ERR_UNSUPPORTED;
  // tiles of an item, at most
  const int capacity = capacity_of(s);
  int64_t tiles = (capacity + kTileKeys - 1) / kTileKeys;
  if (tree) tiles += 2;
  else if (s.window_left >= 0 && s.window_right >= 0)
    tiles = std::min<int64_t>(tiles, ((int64_t)s.window_left + s.window_right + pl.block_cols) / kTileKeys + 2 + std::min(s.sinks, capacity) / kTileKeys);
  // With few items a workgroup has the eight wavefronts that a CU's LDS has room for, with many of them two of four wavefronts share it, one starting or
  // merging while the other streams.  Single tokens: 64 items of 4000 keys 26.6 us with eight, 28.1 with four; 128 of 1000 to 16000 keys 96.9, 93.9; 256 of
  // 2000 keys 49.7, 47.2.
  pl.waves = f32 ? paged_waves_f32(s.head_dim) : !pl.shared && items > 64 ? 4 : 8;
  const int64_t at_once = !f32 && pl.waves == 4 ? 2 * kNumCUs : kNumCUs;
  // Shares pay for a second launch, 4 to 5 us.  Up to 32 items leave most CUs idle without them: a tile for every wavefront is enough (us by tiles of a share:
  // 8 heads x 4096 keys, trees of 8 rows 13.3 with 8, 14.9 with 16, 18.8 with 48; 32 heads x 2000 keys, a token 12.2, 13.1, 15.5; 8 heads x 500 keys in fp32
  // 12.3 with 4, 15.2 with 8), where uncut items have four rounds of them at least (8 heads x 600 keys, a token: 10.4 with 8, 8.4 uncut; x 1000 keys 11.0, 11.0).
  // More items want larger ones: 64 heads x 1000 keys, a token 12.8 with 8, 11.9 with 24; 64 x 500 keys in fp32 17.8 with 4, 16.4 with 8.
  // Shared tiles: 8 heads x 1000 keys x 224 columns 18.8 us with 4, 18.4 with 8, 22.2 with 16, 25.7 with 32.
  const bool few = !pl.shared && items <= 32;
  pl.least_tiles = few ? pl.waves : pl.shared ? 8 : f32 ? 2 * pl.waves : 6 * pl.waves;
  // With items for half the CUs, workgroups that share tiles are better left whole: a second round of them costs more than uneven items do (256 columns x 2000
  // keys: 128 items 57.5 us cut, 66.3 whole; 144 items 91.4, 67.0).  Streaming ones fit in between (320 items of 2000 keys 63.0 cut, 59.9 whole, of 1 to 8000
  // keys 128, 151).  The rule counts items and does not know their lengths: with more of them, one sequence that is much longer than the others is not cut either
  // (trees of 20 rows x 32/8 heads, 100000 rows among sequences of 500: 128 items 134 us, 136 items 1630; single tokens x 32/8 heads likewise: 1024 items 146,
  // 1032 items 1237).
  pl.splits = items <= (pl.shared ? kNumCUs / 2 : 2 * at_once) && tiles > (few ? 4 * pl.waves - 1 : pl.least_tiles);
  pl.workgroups = pl.splits ? (int)std::max<int64_t>(at_once, 2 * items) : (int)whole;
  while (tiles >> pl.tile_shift >= 1 << 20) ++pl.tile_shift;   // items <= 1024
  return SDLLM_OK;
}

struct PagedBytes { size_t part_o, part_ml, items; size_t all() const { return part_o + part_ml + items; } };
PagedBytes paged_bytes(const sdllm_paged_shape_t& s, const PagedPlan& pl) {
  if (!pl.splits) return {};
  return {align_up((size_t)pl.workgroups * pl.block_cols * s.head_dim * sizeof(float)), align_up((size_t)pl.workgroups * pl.block_cols * 2 * sizeof(float)),
          align_up((size_t)s.batch * s.n_kv_heads * pl.max_blocks * 2 * sizeof(int32_t))};
}

int32_t check_op(const sdllm_paged_shape_t& s, bool tree) { return tree && s.rows > 64 ? SDLLM_ERR_UNSUPPORTED : SDLLM_OK; }

int32_t plan_of_op(const sdllm_paged_shape_t* s, int32_t op, PagedPlan& pl) {
  const bool tree = op == SDLLM_OP_TREE_ATTN_PAGED;
  if (!tree && op != SDLLM_OP_WINDOW_ATTN_PAGED) return SDLLM_ERR_INVALID_ARG;
  int32_t st = check_paged(s);
  if (st == SDLLM_OK) st = check_op(*s, tree);
  return st == SDLLM_OK ? plan_paged(*s, tree, pl) : st;
}

int32_t run_paged(const sdllm_paged_shape_t* shape, bool tree, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                  const int32_t* lengths, const int32_t* row_counts, const void* k_blk, const void* v_blk, const uint64_t* mask, void* out, void* ws,
                  size_t ws_bytes, void* stream) {
  int32_t st = check_paged(shape);
  if (st != SDLLM_OK) return st;
  const sdllm_paged_shape_t& s = *shape;
  PagedAttnParams p{};
  if ((st = fill_cache(s, k_pages, v_pages, table, lengths, row_counts, p.cache)) != SDLLM_OK) return st;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !row_stride_ok(s.q_stride, s.head_dim) || !row_stride_ok(s.out_stride, s.head_dim))
    return SDLLM_ERR_INVALID_ARG;
  if (tree && (!k_blk || !v_blk || !aligned16(k_blk) || !aligned16(v_blk) || !row_stride_ok(s.blk_stride, s.head_dim) ||
               (reinterpret_cast<uintptr_t>(mask) & 7u) != 0))
    return SDLLM_ERR_INVALID_ARG;
  if ((st = check_op(s, tree)) != SDLLM_OK) return st;
  // 16 rows are addressed from their first in 32 bits
  if (std::max(s.page_stride[2], tree ? s.blk_stride[2] : 0) > (int64_t)UINT32_MAX / 4 / 16 - 256) return SDLLM_ERR_UNSUPPORTED;
  PagedPlan pl;
  if ((st = plan_paged(s, tree, pl)) != SDLLM_OK) return st;
  const PagedBytes bytes = paged_bytes(s, pl);
  if (pl.splits && (!ws || ws_bytes < bytes.all() || (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0)) return SDLLM_ERR_WORKSPACE;
  if (s.rows == 0) return SDLLM_OK;
  p.q = q; p.k_pages = k_pages; p.v_pages = v_pages; p.k_blk = k_blk; p.v_blk = v_blk; p.mask = mask; p.out = out;
  p.mask_stride = s.mask_stride;
  p.q_sb = s.q_stride[0]; p.q_sh = s.q_stride[1]; p.q_sr = s.q_stride[2];
  p.blk_sb = s.blk_stride[0]; p.blk_sh = s.blk_stride[1]; p.blk_sr = s.blk_stride[2];
  p.o_sb = s.out_stride[0]; p.o_sh = s.out_stride[1]; p.o_sr = s.out_stride[2];
  p.batch = s.batch; p.hkv = s.n_kv_heads; p.group = s.n_q_heads / s.n_kv_heads;
  // limits that no row reaches are none: what is left of them adds up in 32 bits
  const int32_t capacity = p.cache.capacity;
  p.left = s.window_left >= capacity + s.rows ? -1 : s.window_left;
  p.right = s.window_right >= capacity ? -1 : s.window_right;
  p.sinks = std::min(s.sinks, capacity);
  p.scale_log2 = (s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)s.head_dim)) * kLog2e;
  p.block_cols = pl.block_cols; p.max_blocks = pl.max_blocks; p.workgroups = pl.workgroups; p.least_tiles = pl.least_tiles;
  p.tile_shift = pl.tile_shift;
  if (pl.splits) {
    p.part_o = (float*)ws;
    p.part_ml = (float*)((char*)ws + bytes.part_o);
    p.item_at = (int32_t*)((char*)ws + bytes.part_o + bytes.part_ml);
  }
  // Many keys are read past the caches (single tokens x 32/8 heads, MB: 65 19.9 us, through the caches 18.1; 131 27.9, 27.7; 262 47.3, 48.2; 524 89.5, 101.8)
  p.caches_tiles = (128 << 20) / (2 * kTileKeys * s.head_dim * elem_size(s.dtype));
  p.chunk = pl.chunk;
  p.heads = s.batch * s.n_kv_heads;
  p.turned = p.heads % 2 == 0 ? 5 : 0;
  p.by_chunk = Divisor((uint32_t)p.chunk); p.by_heads = Divisor((uint32_t)p.heads);
  p.by_group = Divisor((uint32_t)p.group); p.by_blocks = Divisor((uint32_t)p.max_blocks); p.by_hkv = Divisor((uint32_t)p.hkv);
  return launch_attn_paged(p, pl, tree ? kSeeTree : kSeeWindow, s.dtype, s.head_dim, (hipStream_t)stream) == hipSuccess ? SDLLM_OK : SDLLM_ERR_HIP;
}

}  // namespace

hipError_t sdllm::launch_attn_paged(const PagedAttnParams& p, const PagedPlan& pl, int sees, int dtype, int d, hipStream_t s) {
  return pl.shared ? launch_attn_paged_shared(p, pl, sees, d, s) : launch_attn_paged_stream(p, pl, sees, dtype, d, s);
}

extern "C" {

int32_t sdllm_paged_plan(const sdllm_paged_shape_t* shape, int32_t op, sdllm_paged_plan_t* plan) {
  PagedPlan pl;
  const int32_t st = plan_of_op(shape, op, pl);
  if (st != SDLLM_OK) return st;
  if (!plan) return SDLLM_ERR_INVALID_ARG;
  *plan = sdllm_paged_plan_t{pl.shared, pl.block_cols, pl.waves, pl.workgroups, pl.splits ? pl.least_tiles : 0};
  return SDLLM_OK;
}

int32_t sdllm_paged_workspace_bytes(const sdllm_paged_shape_t* shape, int32_t op, size_t* bytes) {
  PagedPlan pl;
  const int32_t st = plan_of_op(shape, op, pl);
  if (st != SDLLM_OK) return st;
  if (!bytes) return SDLLM_ERR_INVALID_ARG;
  *bytes = std::max(paged_bytes(*shape, pl).all(), kAlign);   // never zero, so callers can always allocate
  return SDLLM_OK;
}

int32_t sdllm_append_paged(const sdllm_qk_shape_t* qk, const sdllm_paged_shape_t* shape, const void* q_in, const void* k_in, const void* v_in,
                           const void* q_weight, const void* k_weight, const float* inv_freq, const int32_t* positions, const int32_t* pick,
                           const int32_t* lengths, const int32_t* row_counts, const int32_t* table, void* q_out, void* k_pages, void* v_pages,
                           void* stream) {
  int32_t st = check_qk_shape(qk);
  if (st != SDLLM_OK || (st = check_paged(shape)) != SDLLM_OK) return st;
  const sdllm_qk_shape_t& h = *qk;
  const sdllm_paged_shape_t& s = *shape;
  if (h.batch != s.batch || h.n_kv_heads != s.n_kv_heads || h.head_dim != s.head_dim || h.rows != s.rows || h.dtype != s.dtype) return SDLLM_ERR_INVALID_ARG;
  AppendParams p{};
  if ((st = fill_cache(s, k_pages, v_pages, table, lengths, row_counts, p.cache)) != SDLLM_OK) return st;
  if (h.rot_dim > 0 && !inv_freq) return SDLLM_ERR_INVALID_ARG;
  if (h.pos_stride < 0 || (pick && h.n_q_heads > 0)) return SDLLM_ERR_INVALID_ARG;
  if (h.rot_dim > 0 && !positions && (int64_t)p.cache.capacity + s.rows + h.pos_begin > (int64_t)INT32_MAX + 1) return SDLLM_ERR_INVALID_ARG;
  const int es = elem_size(s.dtype);
  auto input_ok = [&](const void* in, const int64_t* stride, const void* weight) {
    return in && aligned16(in) && aligned16(weight) && strides_ok(stride, es) && row_stride_ok(stride, s.head_dim);
  };
  if (!input_ok(k_in, h.k_in_stride, k_weight) || !v_in || !aligned16(v_in)) return SDLLM_ERR_INVALID_ARG;
  if (h.n_q_heads > 0 && (!input_ok(q_in, h.q_in_stride, q_weight) || !q_out || !aligned16(q_out) || !strides_ok(h.q_out_stride, es) ||
                          !row_stride_ok(h.q_out_stride, s.head_dim)))
    return SDLLM_ERR_INVALID_ARG;
  // a wavefront for each, in workgroups of four, their threads counted in 32 bits
  if ((int64_t)s.batch * s.rows > UINT32_MAX / kWave / 4 * 4) return SDLLM_ERR_UNSUPPORTED;
  if (s.rows == 0) return SDLLM_OK;
  QkParams& q = p.qk;
  q.q_in = q_in; q.k_in = k_in; q.q_out = q_out;
  q.q_weight = q_weight; q.k_weight = k_weight; q.inv_freq = inv_freq; q.positions = positions;
  q.pos_stride = h.pos_stride; q.pos_begin = h.pos_begin;
  q.qi_sb = h.q_in_stride[0]; q.qi_sh = h.q_in_stride[1]; q.qi_sr = h.q_in_stride[2];
  q.ki_sb = h.k_in_stride[0]; q.ki_sh = h.k_in_stride[1]; q.ki_sr = h.k_in_stride[2];
  q.qo_sb = h.q_out_stride[0]; q.qo_sh = h.q_out_stride[1]; q.qo_sr = h.q_out_stride[2];
  q.tokens = s.batch * s.rows; q.rows = s.rows; q.hq = h.n_q_heads; q.hkv = s.n_kv_heads;
  q.rot = h.rot_dim; q.adjacent = h.pairing == SDLLM_PAIR_ADJACENT; q.norm = h.norm == SDLLM_NORM_RMS; q.eps = h.eps;
  q.by_rows = Divisor((uint32_t)s.rows);
  p.v_in = v_in; p.pick = pick; p.k_pages = k_pages; p.v_pages = v_pages;
  return launch_append_paged(p, s.dtype, s.head_dim, (hipStream_t)stream) == hipSuccess ? SDLLM_OK : SDLLM_ERR_HIP;
}

int32_t sdllm_tree_attn_paged(const sdllm_paged_shape_t* shape, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                              const int32_t* lengths, const int32_t* row_counts, const void* k_blk, const void* v_blk, const uint64_t* mask, void* out,
                              void* ws, size_t ws_bytes, void* stream) {
  return run_paged(shape, true, q, k_pages, v_pages, table, lengths, row_counts, k_blk, v_blk, mask, out, ws, ws_bytes, stream);
}

int32_t sdllm_window_attn_paged(const sdllm_paged_shape_t* shape, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                                const int32_t* lengths, const int32_t* row_counts, void* out, void* ws, size_t ws_bytes, void* stream) {
  return run_paged(shape, false, q, k_pages, v_pages, table, lengths, row_counts, nullptr, nullptr, nullptr, out, ws, ws_bytes, stream);
}

}  // extern "C"
