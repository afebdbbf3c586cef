/*
 * sdllm.h - C ABI of the MI355X (gfx950) Sparse-dLLM block-step attention library.
 *
 * The library implements the per-layer hot path of Sparse-dLLM (delayed bidirectional sparse
 * caching for block-wise diffusion-LLM decoding): saliency scoring of the keys outside the
 * current block, max-pool smoothing, top-k retention, gather-compaction of the retained K/V rows
 * and unmasked attention of the block's queries over the compacted cache plus the block.
 *
 * Conventions for every entry point
 *   - plain C, no exceptions; the return value is a status code (SDLLM_OK == 0, errors < 0);
 *   - every data pointer is a DEVICE pointer on the current HIP device unless marked "host";
 *     the caller owns all buffers, the library never allocates, frees or synchronises;
 *   - work is only enqueued on `stream` (a hipStream_t passed as void*, NULL = default stream);
 *   - tensors are dense in their last axis (head_dim contiguous); the other axes are described
 *     by element strides {batch, head, row} in sdllm_shape_t.  Rows must be 16-byte aligned
 *     (base pointers and strides*sizeof(element) multiples of 16);
 *   - query head h reads KV head h / (n_q_heads / n_kv_heads);
 *   - on an argument error nothing is enqueued.
 *
 * Notation (the paper's): b block length, o offset of the block's first token, L sequence length,
 * N_pre = o, N_suf = L - o - b, N = N_pre + N_suf candidates, r retention ratio, s pool kernel.
 */
#ifndef SDLLM_H
#define SDLLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define SDLLM_OK 0
#define SDLLM_ERR_INVALID_ARG (-1) /* null pointer, bad size, r outside [0,1], even pool kernel, misalignment */
#define SDLLM_ERR_UNSUPPORTED (-2) /* a legal request this build has no kernel for */
#define SDLLM_ERR_WORKSPACE (-3)   /* workspace missing or too small (sdllm_workspace_bytes is always enough) */
#define SDLLM_ERR_HIP (-4)         /* a HIP launch reported an error */
#define SDLLM_ERR_STATIC_LIMIT (-5) /* sdllm_sparse_attn_noalloc: the request needs more than SDLLM_STATIC_SCRATCH_BYTES */

/* element types of Q/K/V/O (accumulation is always fp32) */
#define SDLLM_BF16 0
#define SDLLM_F32 1

/* how the per-candidate score is formed from the logits A = Q_b K_f^T / sqrt(d) (Sec. 3.3):
 * SOFTMAX_MEAN normalises each query row over all candidates first ("average attention scores",
 * the sentence introducing Alg. 1); LOGIT_MEAN averages the raw logits (Alg. 1 steps 5-6 literal). */
#define SDLLM_SOFTMAX_MEAN 0
#define SDLLM_LOGIT_MEAN 1

/* PER_SEGMENT pools and ranks prefix and suffix separately, each with its own quota;
 * JOINT pools and ranks the concatenated candidate array as one (Alg. 1 literal). */
#define SDLLM_PER_SEGMENT 0
#define SDLLM_JOINT 1

/* quota rounding: ceil(r*n) or floor(r*n) (Alg. 1 step 9), r*n evaluated in double with a 1e-9 guard */
#define SDLLM_CEIL 0
#define SDLLM_FLOOR 1

/* local aggregation (Sec. 3.3 third equation; AvgPool is the appendix ablation) */
#define SDLLM_MAX_POOL 0
#define SDLLM_AVG_POOL 1

/* which candidates may be evicted: both sides of the block (Alg. 1) or the prefix only, the
 * suffix being kept whole (Alg. 4, the prefix-sparse ablation) */
#define SDLLM_EVICT_BIDIRECTIONAL 0
#define SDLLM_EVICT_PREFIX_ONLY 1

/* cache states (Alg. 2 / Alg. 5) */
#define SDLLM_STATE_FULL 0
#define SDLLM_STATE_UPDATE 1
#define SDLLM_STATE_REUSE 2

/* operations for sdllm_workspace_bytes */
#define SDLLM_OP_SCORE_SELECT 0
#define SDLLM_OP_COMPACT_KV 1
#define SDLLM_OP_SPARSE_ATTN 2
#define SDLLM_OP_BLOCK_STEP 3
#define SDLLM_OP_SPARSE_ATTN_PACKED 4
#define SDLLM_OP_BLOCK_STEP_PACKED 5
/* for sdllm_paged_workspace_bytes */
#define SDLLM_OP_TREE_ATTN_PAGED 6
#define SDLLM_OP_WINDOW_ATTN_PAGED 7

typedef struct sdllm_shape {
  int32_t batch;       /* B >= 1 */
  int32_t n_q_heads;   /* Hq, multiple of n_kv_heads */
  int32_t n_kv_heads;  /* Hkv >= 1 */
  int32_t head_dim;    /* d in {64, 128} */
  int32_t seq_len;     /* L */
  int32_t block_off;   /* o, 0 <= o, o + b <= L */
  int32_t block_len;   /* b, 1 <= b <= 64 */
  int32_t dtype;       /* SDLLM_BF16 | SDLLM_F32 */
  int32_t pool_kernel; /* s, odd, >= 1 */
  int32_t score_mode;  /* SDLLM_SOFTMAX_MEAN | SDLLM_LOGIT_MEAN */
  int32_t select_mode; /* SDLLM_PER_SEGMENT | SDLLM_JOINT */
  int32_t k_rounding;  /* SDLLM_CEIL | SDLLM_FLOOR */
  int32_t pool_mode;   /* SDLLM_MAX_POOL | SDLLM_AVG_POOL */
  int32_t evict_scope; /* SDLLM_EVICT_BIDIRECTIONAL | SDLLM_EVICT_PREFIX_ONLY */
  float softmax_scale; /* 0 means 1/sqrt(head_dim) */
  int32_t reserved;    /* must be 0 */
  double retention;    /* r in [0, 1] */
  /* element strides {batch, head, row}; the last axis (head_dim) is contiguous */
  int64_t q_stride[3];     /* block queries            [B, Hq,  b, d] */
  int64_t kv_stride[3];    /* full-sequence K and V    [B, Hkv, L, d] */
  int64_t blk_stride[3];   /* block K_n and V_n        [B, Hkv, b, d] */
  int64_t cache_stride[3]; /* compacted K_c and V_c    [B, Hkv, >= k, d] */
  int64_t out_stride[3];   /* attention output         [B, Hq,  b, d] */
} sdllm_shape_t;

/* Static string for a status code.  Host only. */
const char* sdllm_error_string(int32_t status);

/* Library version, major*10000 + minor*100 + patch.  Host only. */
int32_t sdllm_version(void);

/*
 * Number of retained entries per (batch, KV head) row for this shape (Sec. 3.3: k = (L-b)*r;
 * Alg. 1 step 9).  All outputs are host pointers and may be NULL.  k_total is what
 * sdllm_score_select writes per row.  k_pre / k_suf are the prefix / suffix quotas in
 * PER_SEGMENT mode and -1 in JOINT mode, where the split depends on the data.  With
 * SDLLM_EVICT_PREFIX_ONLY the suffix quota is N_suf.
 */
int32_t sdllm_retained_count(const sdllm_shape_t* shape, int32_t* k_total, int32_t* k_pre, int32_t* k_suf);

/*
 * Bytes of device workspace `op` needs for this shape (host call).  n_cached is the number of
 * cache rows sdllm_sparse_attn will be given (ignored by the other ops; SDLLM_OP_BLOCK_STEP
 * covers every state of the step, including dense attention over all L keys).
 *
 * With that much, aligned to 256 bytes, a call runs the kernel and the key splits that its sizes choose.  Attention calls also
 * take less, down to an amount that depends on their sizes only and often is nothing: they then run fewer key splits or another kernel,
 * as small bf16 calls (head_dim 128, block of 32) of sdllm_sparse_attn do with a workspace that is not aligned to 16 bytes, and
 * the results differ by rounding.  sdllm_sparse_attn and state 2 of sdllm_block_step give the same bits for the same tensors if each
 * is given its full size.  The operations on a packed cache need all of theirs.
 */
int32_t sdllm_workspace_bytes(const sdllm_shape_t* shape, int32_t op, int32_t n_cached, size_t* bytes);

/* Cache state of step `step_in_block` (0-based) under delay x: 2 if i > x, 1 if i == x, else 0
 * (Alg. 2 for x = 1, Alg. 5 in general).  `state` is a host pointer. */
int32_t sdllm_cache_state(int32_t step_in_block, int32_t delay, int32_t* state);

/*
 * Alg. 1 steps 2-10: score every candidate key against the block's queries, smooth, keep the top
 * entries.  q_blk [B,Hq,b,d] (q_stride), k_full [B,Hkv,L,d] (kv_stride).
 *   idx_out    [B,Hkv,k_total] int32, contiguous: retained ABSOLUTE positions, ascending.  Ties in
 *              the pooled score go to the lower position.
 *   pooled_out optional [B,Hkv,N] fp32 contiguous, candidate-indexed (c < o -> position c,
 *              c >= o -> position c + b): the pooled score.  May be NULL.
 *   score_out  optional [B,Hkv,N] fp32: the score before pooling.  May be NULL.
 * A ranked segment (prefix, suffix, or the joint array) of more than 1 048 576 candidates returns
 * SDLLM_ERR_UNSUPPORTED.
 *   ws         workspace of at least sdllm_workspace_bytes(SDLLM_OP_SCORE_SELECT) bytes,
 *              256-byte aligned; contents undefined afterwards.
 */
int32_t sdllm_score_select(const sdllm_shape_t* shape, const void* q_blk, const void* k_full, int32_t* idx_out,
                           float* pooled_out, float* score_out, void* ws, size_t ws_bytes, void* stream);

/*
 * Alg. 1 steps 12-14: K_c[j] = K[idx[j]], V_c[j] = V[idx[j]] for j < k_total, per (batch, KV head).
 * k_full/v_full [B,Hkv,L,d] (kv_stride); idx [B,Hkv,k_total] int32 as written by
 * sdllm_score_select (values must lie in [0, L)); k_cache/v_cache [B,Hkv,>=k_total,d]
 * (cache_stride).  A byte copy: bit-exact.
 */
int32_t sdllm_compact_kv(const sdllm_shape_t* shape, const void* k_full, const void* v_full, const int32_t* idx,
                         void* k_cache, void* v_cache, void* stream);

/*
 * Alg. 3, cache_state == 2: out = softmax(scale * Q_n Concat(K_c,K_n)^T) Concat(V_c,V_n), no mask.
 * q_blk [B,Hq,b,d] (q_stride); k_cache/v_cache [B,Hkv,n_cached,d] (cache_stride), n_cached >= 0
 * (0: attention over the block only; the cache pointers may then be NULL); k_blk/v_blk
 * [B,Hkv,b,d] (blk_stride); out [B,Hq,b,d] (out_stride).  ws as for sdllm_score_select with
 * SDLLM_OP_SPARSE_ATTN and the same n_cached; less is taken where sdllm_workspace_bytes says so.
 */
int32_t sdllm_sparse_attn(const sdllm_shape_t* shape, const void* q_blk, const void* k_cache, const void* v_cache,
                          int32_t n_cached, const void* k_blk, const void* v_blk, void* out, void* ws,
                          size_t ws_bytes, void* stream);

/*
 * sdllm_sparse_attn for callers that cannot allocate or size a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and
 * results bit-identical to those with a full-sized workspace, but the split-KV partials live in an array of SDLLM_STATIC_SCRATCH_BYTES
 * that is part of the library's device image (every GPU the library runs on holds one copy until the
 * process ends).  The call allocates nothing and frees nothing.  A shape whose launch plan needs
 * more scratch than that returns SDLLM_ERR_STATIC_LIMIT and enqueues nothing (use sdllm_sparse_attn
 * with a workspace then).  With 7 or 8 query heads per KV head and up to 80 MB of keys and values, a kernel
 * whose partials do not fit gives way to a slower one that does without (the same happens in
 * sdllm_sparse_attn when the workspace is too small); its results differ by rounding.  All calls on one GPU
 * share that GPU's array: calls that overlap in time
 * on one GPU (different streams, or concurrently replayed graphs) race and are not allowed.  The
 * first call on each device resolves the array's address and must not be made under stream capture.
 */
#define SDLLM_STATIC_SCRATCH_BYTES (8u << 20)
int32_t sdllm_sparse_attn_noalloc(const sdllm_shape_t* shape, const void* q_blk, const void* k_cache,
                                  const void* v_cache, int32_t n_cached, const void* k_blk, const void* v_blk,
                                  void* out, void* stream);

/*
 * One denoising step of one layer (Alg. 2/5 -> Alg. 3 -> Alg. 1).  state = cache_state(step, delay).
 *   state 0: k_in/v_in are the full-sequence K,V [B,Hkv,L,d] (kv_stride); out = the block's rows
 *            of dense bidirectional attention over all L keys.  Cache untouched.
 *   state 1: as state 0, and the cache is rebuilt from this step's tensors: idx, k_cache, v_cache
 *            are written (sdllm_score_select + sdllm_compact_kv).
 *   state 2: k_in/v_in are the block's K_n,V_n [B,Hkv,b,d] (blk_stride); out = sparse attention
 *            over the cache (k_total rows per KV head, as sdllm_retained_count reports) + block.
 * idx [B,Hkv,k_total] int32; ws sized by SDLLM_OP_BLOCK_STEP.  `state_out` (host, may be NULL)
 * receives the state that was executed.  For fp32 tensors, head_dim 64, block lengths other than 32 and other shapes of
 * the general kernels that size lets state 1 keep its key-split partials until the compaction; a workspace
 * that holds the partials and the scoring buffers one after the other is accepted too (same results, one more launch).  For small
 * bf16 calls it holds all key splits that states 0 and 2 have a use for; less is accepted, with fewer of them (sdllm_workspace_bytes).
 */
int32_t sdllm_block_step(const sdllm_shape_t* shape, int32_t step_in_block, int32_t delay, const void* q_blk,
                         const void* k_in, const void* v_in, int32_t* idx, void* k_cache, void* v_cache, void* out,
                         void* ws, size_t ws_bytes, void* stream, int32_t* state_out);

/*
 * Full bidirectional attention of ALL L positions (Sec. 3.1: the mask predictor recomputes the whole
 * sequence; cache_state 0 and 1 of the cache-management appendix run it for the rows outside the
 * current block, whose block rows sdllm_block_step returns):
 *   out[b,h,i,:] = sum_j softmax_j(scale * <q[b,h,i], k[b,g(h),j]>) v[b,g(h),j],  i, j in [0, L), no mask.
 * q_full/out_full are [B,Hq,L,d] with element strides {batch, head, row} given by q_full_stride /
 * out_full_stride (host pointers to 3 values); k_full/v_full [B,Hkv,L,d] use shape->kv_stride.
 * Only batch, head counts, head_dim, seq_len, dtype, softmax_scale and kv_stride of `shape` are read
 * besides the usual validity checks.  No workspace.
 */
int32_t sdllm_dense_attn(const sdllm_shape_t* shape, const void* q_full, const int64_t* q_full_stride,
                         const void* k_full, const void* v_full, void* out_full, const int64_t* out_full_stride,
                         void* stream);

/*
 * ---- A cache of 4 bits a value
 *
 * The compacted cache in 4.25 bits a value instead of 16 or 32: written once per block, read at every step that reuses it.  A value is
 * one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (codes 0 to 7, sign in bit 3) times 2^e.  One e holds for a group of 32 values: 32
 * neighbouring channels of a key, or one channel of 32 value rows that follow each other in the cache (the last group of a head is filled up
 * with zeros).  e is the smallest integer in [-125, 125] for which all magnitudes of the group are below 7 2^e; a value becomes the nearest
 * number, of two equally near ones that with the even code, and the largest number past the end.  A group with an
 * infinity or a NaN reads as NaN as a whole.  Both types of tensors hold the numbers exactly.
 *
 * The cache is one buffer of sdllm_packed_cache_bytes, aligned to 16 bytes, for the rows [0, cache_rows) of every (batch, KV head); the caller
 * allocates it once for as many rows as it will need.  Per (batch, KV head), densely, ceil(cache_rows / 32) tiles of 34 d bytes:
 *   32 d/2 bytes  key codes    [d/32 groups g][32 rows][16 bytes]: channels 32 g .. 32 g + 31, the lower four bits first
 *   32 d/2 bytes  value codes  [d/64: i][2: h][32: m][2: j][8 bytes]: channel (d/32) m + 2 i + j; nibble 4 a + p is row 8 a + 4 h + p
 *   d bytes       key scales   [32 rows][d/32 groups]: e + 127, or 255 for NaN
 *   d bytes       value scales [d channels]
 * Rows past those written of the last tile hold zeros.
 *
 * These operations refuse shapes of 2^31 query heads or more in all (batch x n_q_heads), and caches of 2^63 bytes or more: SDLLM_ERR_UNSUPPORTED.
 */

/* Bytes of a packed cache for cache_rows >= 0 rows per (batch, KV head).  Reads batch, n_kv_heads and head_dim of `shape`.  Host call. */
int32_t sdllm_packed_cache_bytes(const sdllm_shape_t* shape, int32_t cache_rows, size_t* bytes);

/*
 * sdllm_compact_kv into a packed cache: its rows [0, k_total) become the rows idx[0..k_total) of k_full and v_full ([B,Hkv,L,d],
 * kv_stride).  cache_rows >= k_total.  idx as for sdllm_compact_kv.
 */
int32_t sdllm_compact_kv_packed(const sdllm_shape_t* shape, const void* k_full, const void* v_full, const int32_t* idx, void* cache,
                                int32_t cache_rows, void* stream);

/* The values of rows [0, n_cached) of a packed cache as rows of k_out and v_out, [B,Hkv,>= n_cached,d] (cache_stride), in the shape's type. */
int32_t sdllm_unpack_kv(const sdllm_shape_t* shape, const void* cache, int32_t cache_rows, int32_t n_cached, void* k_out, void* v_out,
                        void* stream);

/*
 * sdllm_sparse_attn over rows [0, n_cached) of a packed cache and the block's own k_blk/v_blk, which are not packed; n_cached may be 0 (the cache may
 * be NULL then).  Other arguments as there; ws of sdllm_workspace_bytes(SDLLM_OP_SPARSE_ATTN_PACKED) for the same n_cached, aligned to
 * 16 bytes.  The cache enters with its exact values; with bf16 tensors the softmax numerators are rounded to bf16 for the product with the values,
 * with fp32 tensors products and sums are fp32.
 */
int32_t sdllm_sparse_attn_packed(const sdllm_shape_t* shape, const void* q_blk, const void* cache, int32_t cache_rows, int32_t n_cached,
                                 const void* k_blk, const void* v_blk, void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * sdllm_block_step with a packed cache: states 0 and 1 are dense attention over k_in/v_in as there, state 1 packs the retained rows
 * (sdllm_score_select + sdllm_compact_kv_packed), state 2 is sdllm_sparse_attn_packed over k_total rows.  cache_rows >= k_total in states
 * 1 and 2.  ws of sdllm_workspace_bytes(SDLLM_OP_BLOCK_STEP_PACKED), aligned to 256 bytes.
 */
int32_t sdllm_block_step_packed(const sdllm_shape_t* shape, int32_t step_in_block, int32_t delay, const void* q_blk, const void* k_in,
                                const void* v_in, int32_t* idx, void* cache, int32_t cache_rows, void* out, void* ws, size_t ws_bytes,
                                void* stream, int32_t* state_out);

/*
 * ---- Norm of query and key heads and rotation by position
 *
 * What a projection goes through on its way to q_blk and k_in.  For each (batch, head, row):
 *   y = x / sqrt(mean(x^2) + eps) * weight     (SDLLM_NORM_RMS; a null weight is all ones)   or   y = x   (SDLLM_NORM_NONE),
 * then the pairs (a, b) of its first rot_dim channels are turned by t = position * inv_freq[f], f = 0 .. rot_dim/2 - 1:
 *   (a, b) -> (a cos t - b sin t, a sin t + b cos t),
 * pair f being channels (f, f + rot_dim/2) (SDLLM_PAIR_HALVES) or (2 f, 2 f + 1) (SDLLM_PAIR_ADJACENT).  fp32 throughout and one
 * rounding at the end; rows may be of any magnitude, also where x^2 is no number of fp32; t is formed and reduced in 64 bits.
 */
#define SDLLM_NORM_NONE 0
#define SDLLM_NORM_RMS 1
#define SDLLM_PAIR_HALVES 0
#define SDLLM_PAIR_ADJACENT 1

typedef struct sdllm_qk_shape {
  int32_t batch;       /* B >= 1 */
  int32_t n_q_heads;   /* >= 0 */
  int32_t n_kv_heads;  /* >= 0, not both 0, and no more than 2^30 together */
  int32_t head_dim;    /* 64 or 128 */
  int32_t rows;        /* n >= 0 positions */
  int32_t dtype;       /* SDLLM_BF16 | SDLLM_F32 */
  int32_t rot_dim;     /* a multiple of 16 in [0, head_dim]; 0: no rotation */
  int32_t pairing;     /* SDLLM_PAIR_HALVES | SDLLM_PAIR_ADJACENT */
  int32_t norm;        /* SDLLM_NORM_NONE | SDLLM_NORM_RMS */
  float eps;           /* >= 0 */
  int32_t pos_begin;   /* without `positions`: row i is at position pos_begin + i */
  int32_t reserved;    /* must be 0 */
  int64_t pos_stride;  /* elements between the batch's rows of `positions`; 0: the same for all */
  /* element strides {batch, head, row}; the last axis is contiguous */
  int64_t q_in_stride[3];  /* [B, Hq,  n, d] */
  int64_t k_in_stride[3];  /* [B, Hkv, n, d] */
  int64_t q_out_stride[3];
  int64_t k_out_stride[3];
} sdllm_qk_shape_t;

/*
 * q_in/k_in -> q_out/k_out; an output may be its input, with the same strides, and may overlap nothing else.  Tensors of no heads are not read (NULL).
 * q_weight/k_weight [d] in the tensors' type, 16-byte aligned, or NULL; inv_freq [rot_dim/2] fp32 (NULL if rot_dim is 0);
 * positions int32 [B, n], n contiguous (pos_stride between batches), of either sign, or NULL.
 */
int32_t sdllm_qk_norm_rope(const sdllm_qk_shape_t* shape, const void* q_in, const void* k_in, const void* q_weight, const void* k_weight,
                           const float* inv_freq, const int32_t* positions, void* q_out, void* k_out, void* stream);

/*
 * ---- Paged cache: sequences of unlike lengths
 *
 * Keys and values of a batch of sequences in pages of page_rows rows, handed out by the caller from one pool: row j of sequence b is row
 * j % page_rows of page table[b][j / page_rows].  sdllm_append_paged puts new rows there, normalised and turned on the way;
 * sdllm_tree_attn_paged attends from a block of rows, or a tree of drafted tokens, that are in no page yet; sdllm_window_attn_paged from rows that
 * are.  A step of a decoder calls them with the same `lengths`, `row_counts` and `table`:
 *   k_pages/v_pages [n_pages, Hkv, page_rows, d], page_stride between pages, heads and rows;
 *   table           int32 [B, table_pages], table_stride elements between sequences: pages of the pool.  Several sequences may name the same page
 *                   to share its rows.  Entries that no row in use falls in are not looked at.  An entry outside the pool is read as the nearest page of it, and not written to;
 *   lengths         int32 [B]: rows that sequence b has before the new ones, held to [0, table_pages * page_rows] (nothing if the pool is empty);
 *   row_counts      int32 [B]: new rows of sequence b, held to [0, rows]; NULL: `rows` each.  Rows from there on are not read, and outputs are left as they were there.
 * Integers are device memory, so that a captured graph takes those of its replay.  Pages are never allocated, moved or cleared.
 *
 * Both attentions run with fp32 sums; with bf16 tensors the softmax numerators are rounded to bf16 for the product with the values.  A row that sees no
 * key is zero.  What a row does not see takes no part in its result, whatever it holds (infinities and NaN included); an infinity that it
 * sees with a weight that fp32 holds as zero may make NaN.  Outputs and workspace may overlap
 * nothing else; calls that may run at the same time, on two streams or in two graphs, need a workspace each.
 * How a call is launched is planned on the host, from its sequences, heads and rows and from table_pages * page_rows, the most rows that a sequence can have: with
 * table_pages no larger than the call's longest sequence needs (table_stride as it is) a call over short sequences is often one launch where it would be two.
 * Work is cut into even shares where there are few blocks of query rows x heads (at most 128 of 128 or 256, 1024 of 16 or 32, 512 with fp32 tensors); with more of
 * them a sequence that is far longer than the others is better given a call of its own.
 */
typedef struct sdllm_paged_shape {
  int32_t batch;        /* B >= 1 sequences */
  int32_t n_q_heads;    /* Hq, multiple of n_kv_heads */
  int32_t n_kv_heads;   /* Hkv >= 1 */
  int32_t head_dim;     /* d in {64, 128} */
  int32_t rows;         /* n >= 0 new rows of a sequence, or the most that row_counts names; <= 64 for sdllm_tree_attn_paged, <= 2^29 */
  int32_t dtype;        /* SDLLM_BF16 | SDLLM_F32 */
  int32_t n_pages;      /* pages of the pool, >= 0 */
  int32_t page_rows;    /* 16, 32, 64, 128 or 256 */
  int32_t table_pages;  /* >= 0 entries of a sequence's row of the table; table_pages * page_rows <= 2^29 */
  int32_t window_left;  /* sdllm_window_attn_paged: keys before its own that a row sees; negative: all */
  int32_t window_right; /* ... and behind it; negative: all */
  int32_t sinks;        /* ... and first keys of the sequence that it sees besides, >= 0 */
  float softmax_scale;  /* 0 means 1/sqrt(head_dim) */
  int32_t reserved;     /* must be 0 */
  int64_t table_stride; /* elements between the sequences' rows of the table */
  int64_t mask_stride;  /* elements between the sequences' masks; 0: the same for all */
  /* element strides; the last axis (head_dim) is contiguous */
  int64_t q_stride[3];    /* {batch, head, row} of queries       [B, Hq,  n, d] */
  int64_t blk_stride[3];  /* of k_blk and v_blk                  [B, Hkv, n, d] */
  int64_t out_stride[3];  /* of the output                       [B, Hq,  n, d] */
  int64_t page_stride[3]; /* {page, head, row} of the pages      [n_pages, Hkv, page_rows, d] */
} sdllm_paged_shape_t;

/* Bytes of device workspace that SDLLM_OP_TREE_ATTN_PAGED or SDLLM_OP_WINDOW_ATTN_PAGED needs for this shape, whatever the lengths; the attentions take no less.
 * Host call. */
int32_t sdllm_paged_workspace_bytes(const sdllm_paged_shape_t* shape, int32_t op, size_t* bytes);

/*
 * sdllm_qk_norm_rope of queries and keys with the keys, and the values as they are, going to the pages: row i of sequence b to its cache row
 * lengths[b] + i.  Rows that the table has no room or no page for are not written.  q_in/q_out/weights/inv_freq as there (qk->k_out_stride is not read; n_q_heads may be 0);
 * v_in [B, Hkv, n, d] has the strides of k_in.  q_out may be q_in, with the same strides; nothing else may overlap.
 *   positions int32 [B, n] of the rows of q_in and k_in, n contiguous (qk->pos_stride between sequences), or NULL: lengths[b] + qk->pos_begin + i;
 *   pick      int32 [B, n], n contiguous, or NULL.  Row i that is appended is then row pick[b][i] of k_in and v_in (held to [0, n)), with
 *             that row's position if there are positions: what is left of a tree of drafted tokens.  Only with n_q_heads of 0.
 * Of `shape` the cache's fields are read; batch, n_kv_heads, head_dim, rows and dtype have to be those of qk.
 * Two rows of one call must not go to the same place.
 */
int32_t sdllm_append_paged(const sdllm_qk_shape_t* qk, const sdllm_paged_shape_t* shape, const void* q_in, const void* k_in, const void* v_in,
                           const void* q_weight, const void* k_weight, const float* inv_freq, const int32_t* positions, const int32_t* pick,
                           const int32_t* lengths, const int32_t* row_counts, const int32_t* table, void* q_out, void* k_pages, void* v_pages,
                           void* stream);

/*
 * out[b,h,i] = sum_j softmax_j(scale <q[b,h,i], k_j>) v_j over the lengths[b] cache rows of sequence b and those of its own new rows j that row i sees:
 * bit j of mask[b][i].  k_blk/v_blk [B, Hkv, n, d] (blk_stride) are the new rows' keys and values.  mask uint64 [B, n], n contiguous
 * (mask_stride between sequences); NULL: every row sees all new rows of its sequence, as a block of the paper does.  rows <= 64.
 * ws of sdllm_paged_workspace_bytes(SDLLM_OP_TREE_ATTN_PAGED), aligned to 256 bytes.
 */
int32_t sdllm_tree_attn_paged(const sdllm_paged_shape_t* shape, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                              const int32_t* lengths, const int32_t* row_counts, const void* k_blk, const void* v_blk, const uint64_t* mask,
                              void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * The same over the cache alone, for rows that have been appended: row i of sequence b is at place p = lengths[b] + i of its
 * lengths[b] + row_counts[b] rows and sees row j of them if j <= p + window_right and (j >= p - window_left or j < sinks), a negative
 * window_left or window_right being no limit.  {-1, 0, 0} is causal attention, {-1, -1, 0} full attention.  Pages of which
 * no row is seen are not read.  ws of sdllm_paged_workspace_bytes(SDLLM_OP_WINDOW_ATTN_PAGED), aligned to 256 bytes.
 */
int32_t sdllm_window_attn_paged(const sdllm_paged_shape_t* shape, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                                const int32_t* lengths, const int32_t* row_counts, void* out, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SDLLM_H */
