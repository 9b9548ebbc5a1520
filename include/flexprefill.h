/*
 * flexprefill.h -- C ABI of an MI355X (gfx950) implementation of FlexPrefill's
 * context-aware sparse prefill attention (Lai et al., "FlexPrefill: A Context-Aware
 * Sparse Attention Mechanism for Efficient Long-Sequence Inference", ICLR 2025).
 *
 * Two calls make up the method (Algorithm 1):
 *   fp_select       pattern search (Algorithm 2) + index search (Algorithm 3 for
 *                   vertical-slash heads, Algorithm 4 for query-aware heads),
 *                   producing per-head lists of key blocks for every query block;
 *   fp_sparse_attn  A(Q, K, V, S): causal attention restricted to those blocks
 *                   (Section 2, sparse attention with the mask M_S).
 *
 * Conventions shared by every entry point
 *  - Tensors are packed "THD": Q and O are [T][Hq][d], K and V are [T][Hkv][d],
 *    bf16 (raw 16-bit patterns), d contiguous, T = total tokens of all sequences.
 *    Sequence s occupies tokens [cu_seqlens[s], cu_seqlens[s+1]).
 *  - Query head h reads KV head h / (Hq / Hkv) (grouped-query attention).
 *  - Every device pointer is caller-owned device memory; the library never
 *    allocates, frees, or synchronises, and never throws across the ABI.
 *  - The compute calls enqueue kernel launches only (no memset or copy nodes, no host
 *    waits), so they can be captured into a HIP graph and replayed; the first call of
 *    fp_sparse_attn_noalloc on a device resolves its scratch address and belongs
 *    outside a capture.
 *  - All arguments are checked on the host before anything is enqueued; on a
 *    failed check the first failing status is returned and nothing is enqueued.
 *  - Work is enqueued on `stream` (a hipStream_t; NULL = the default stream) and
 *    completes asynchronously: outputs are valid once the caller has synchronised.
 *  - A launch failure returns FP_ERR_HIP; fp_last_error() then names it.
 *  - Calls that share a workspace or output buffers must not overlap in time.
 */
#ifndef FLEXPREFILL_H
#define FLEXPREFILL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fp_status {
  FP_OK = 0,
  FP_ERR_INVALID_ARG = 1,  /* null pointer, bad shape, out-of-range parameter */
  FP_ERR_UNSUPPORTED = 2,  /* valid but not implemented (e.g. head_dim 96)     */
  FP_ERR_WORKSPACE = 3,    /* workspace smaller than the *_workspace_size()   */
  FP_ERR_HIP = 4           /* a HIP runtime call or kernel launch failed       */
} fp_status;

/* Per-head pattern codes written to fp_indices.pattern. */
#define FP_PATTERN_QUERY_AWARE 0    /* Algorithm 4 ("query_specific")            */
#define FP_PATTERN_VERTICAL_SLASH 1 /* Algorithm 3                               */
#define FP_PATTERN_DENSE 2          /* gamma >= 1: every causal block, no search */

#define FP_MAX_BATCH 64             /* sequences per call                        */
#define FP_MAX_MIN_BUDGET 64        /* largest min_budget_blocks accepted        */

/* Problem shape. */
typedef struct fp_shape {
  int32_t batch;              /* number of packed sequences, 1..FP_MAX_BATCH          */
  const int32_t *cu_seqlens;  /* HOST array [batch+1]: cu[0] = 0, non-decreasing;    */
                              /* T = cu[batch]; every sequence has >= 1 token        */
  int32_t num_q_heads;        /* Hq >= 1                                              */
  int32_t num_kv_heads;       /* Hkv >= 1, Hq % Hkv == 0                              */
  int32_t head_dim;           /* d in {64, 128}                                       */
  int32_t block;              /* block_size: 128 (the paper's setting, Section 4.1)  */
                              /* or 64; at most 8192 blocks per sequence             */
} fp_shape;

/* Method parameters (Algorithm 1 inputs tau, gamma; Section 4.1 guards). */
typedef struct fp_params {
  float gamma;                /* cumulative-attention threshold, (0, 1]; gamma >= 1   */
                              /* selects every causal block (full attention)          */
  float tau;                  /* JS-distance threshold, [0, 1]; a head is query-aware */
                              /* iff D_JS < tau (so tau = 0 makes every head VS)      */
  int32_t min_budget_blocks;  /* each query-block row keeps >= min(m, I+1) key        */
                              /* blocks; 0..FP_MAX_MIN_BUDGET (paper: 1024 tokens = 8)*/
  float softmax_scale;        /* 0 => 1/sqrt(head_dim)                                */
  int32_t force_pattern;      /* -1 decide by JS; 0 force query-aware; 1 force VS     */
  int32_t max_budget_blocks;  /* 0: no cap; M >= 2 (and >= min_budget_blocks): every  */
                              /* row keeps <= M key blocks -- 0 and I, then the rest  */
                              /* in top-up order (appendix "maximum budget limit")    */
  int32_t qa_mode;            /* query-aware selection: 0 over the flattened pooled   */
                              /* map (Algorithm 4); 1 per query block, each row of    */
                              /* the map reaching gamma (appendix "flatten ablation") */
  int32_t vs_granularity;     /* vertical-slash lines: 0 token lines (Algorithm 3);   */
                              /* 1 block-pooled: key blocks and offset blocks of      */
                              /* lines are the selection units                        */
} fp_params;

/* Outputs of fp_select (caller-allocated device buffers; sizes from fp_indices_size).
 * Rows are (sequence s, query head h, query block I), I in [0, nb_s), nb_s = ceil(n_s/b).
 *   kb_idx : int32 [kb_idx_elems]; row (s,h,I) starts at
 *            h * TRI + tri_off[s] + I*(I+1)/2, where tri_off[s] = sum_{s'<s} nb_s'(nb_s'+1)/2
 *            and TRI = tri_off[batch]; it holds kb_cnt of that row key-block indices,
 *            strictly ascending, each in [0, I], always containing 0 and I.
 *   kb_cnt : int32 [kb_cnt_elems]; row (s,h,I) at h * NB + nb_off[s] + I,
 *            nb_off[s] = sum_{s'<s} nb_s', NB = nb_off[batch].
 *   pattern: uint8 [batch * Hq], FP_PATTERN_* per (s, h) at s*Hq + h.
 *   js     : float [batch * Hq], D_JS per (s, h) (negative when not computed).
 *   units  : int32 [batch * Hq * 2], per (s, h): {K, 0} for query-aware heads (units
 *            selected by Algorithm 4; with qa_mode 1 the sum over query blocks of
 *            their K), {K_v, K_s} for vertical-slash heads (lines, or blocks of lines
 *            with vs_granularity 1), {all, 0} when dense.
 *            Diagnostics only. */
typedef struct fp_indices {
  int32_t *kb_idx;
  int32_t *kb_cnt;
  uint8_t *pattern;
  float *js;
  int32_t *units;
  float softmax_scale;  /* HOST field: the scale the lists were selected with.  fp_select */
                        /* writes the scale it used (params->softmax_scale, or 1/sqrt(d) */
                        /* when that is 0); fp_sparse_attn attends with this scale (0 =>  */
                        /* 1/sqrt(d)), so selection and attention share one scale.        */
} fp_indices;

/* Element counts of fp_indices.kb_idx and .kb_cnt for `shape`.  Host only. */
fp_status fp_indices_size(const fp_shape *shape, size_t *kb_idx_elems, size_t *kb_cnt_elems);

/* Device workspace bytes needed by fp_select / fp_sparse_attn.  Host only.
 * fp_select: 0 when gamma >= 1 (every causal block is listed without any scoring).
 * fp_sparse_attn: the work order (16 bytes per query head and block), 8 counters, one
 * transposed copy of V (2 * Hkv * NB * block * d bytes, NB = sum of ceil(n_s / block)) and
 * the work order's sort keys and unsorted records (24 bytes per query head and block),
 * written at the start of every call. */
fp_status fp_select_workspace_size(const fp_shape *shape, const fp_params *params,
                                   size_t *bytes);
fp_status fp_attn_workspace_size(const fp_shape *shape, size_t *bytes);

/* Workspace bytes with which fp_sparse_attn runs short problems fastest: the size above,
 * which is always enough, and room for the partial results of rows whose lists are divided
 * among several workgroups.  More workspace than this is not used, and it never exceeds
 * FP_NOALLOC_SCRATCH_BYTES where the size above does not.  Host only.
 * Which rows are divided, and where, follows from the shape, the counts of listed blocks of
 * all rows of a KV group, and the workspace bytes up to this size.  It changes the low bits
 * of a divided row's output (bf16 weights taken against another reference maximum, float32
 * sums in another order; the error against exact results is the same), never from one call
 * to the next with the same arguments.  With exactly fp_attn_workspace_size bytes no row is
 * divided: an output row then depends on its own query, list, keys and values alone,
 * whatever else is in the batch. */
fp_status fp_attn_workspace_preferred(const fp_shape *shape, size_t *bytes);

/* Host-only argument check used by fp_select (params != NULL) and fp_sparse_attn
 * (params == NULL): shape, parameters and workspace size.  Touches no device. */
fp_status fp_validate(const fp_shape *shape, const fp_params *params, size_t ws_bytes);

/* Pattern search + index selection (Algorithm 1 up to S; Algorithms 2-4).
 * q: [T][Hq][d] bf16, k: [T][Hkv][d] bf16 (device).  ws: device workspace of
 * ws_bytes >= fp_select_workspace_size().  Enqueues the writes of every device buffer of
 * *out and sets out->softmax_scale on the host. */
fp_status fp_select(const fp_shape *shape, const void *q, const void *k,
                    const fp_params *params, fp_indices *out, void *ws,
                    size_t ws_bytes, void *stream);

/* Block-sparse causal attention O = A(Q, K, V, S) (Section 2): query i of block I
 * attends to keys j <= i whose key block is listed in row (s, h, I) of idx, with the
 * softmax scale idx->softmax_scale (0 => 1/sqrt(d); finite, >= 0).
 * q, o: [T][Hq][d] bf16; k, v: [T][Hkv][d] bf16; idx->kb_idx, idx->kb_cnt as written by
 * fp_select (pattern, js and units unused).  Listed blocks outside [0, I] are skipped; a
 * query row with no visible key gets O = 0. */
fp_status fp_sparse_attn(const fp_shape *shape, const void *q, const void *k,
                         const void *v, const fp_indices *idx, void *o, void *ws,
                         size_t ws_bytes, void *stream);

/* Size of the fixed device scratch array used by fp_sparse_attn_noalloc (one per GPU). */
#define FP_NOALLOC_SCRATCH_BYTES (64u << 20)

/* fp_sparse_attn without a workspace argument, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same arguments and checks as fp_sparse_attn, and the same result, bit for
 * bit, as fp_sparse_attn with fp_attn_workspace_preferred bytes or more; the workspace is a
 * fixed FP_NOALLOC_SCRATCH_BYTES device array inside the library (one per GPU, held until
 * the process ends), so the call itself allocates nothing.  Problems whose
 * fp_attn_workspace_size exceeds FP_NOALLOC_SCRATCH_BYTES are rejected with
 * FP_ERR_WORKSPACE before anything is enqueued (fp_last_error() says why).  Every call on
 * one GPU uses the same array: calls that overlap in time on one GPU (other streams, other
 * host threads) race and give undefined results. */
fp_status fp_sparse_attn_noalloc(const fp_shape *shape, const void *q, const void *k,
                                 const void *v, const fp_indices *idx, void *o, void *stream);

/* ---------------------------------------------------------------------------------------
 * After the prefill: a paged cache of keys and values, and the attention of the next tokens.
 *
 * A cache holds `layers` pools of `num_pages` pages of `page` tokens, shared by num_slots
 * sequences ("slots").  The bookkeeping is one for all layers and lives on the device, so the
 * calls of a decoding loop can be captured into a HIP graph: lengths and page numbers are read
 * by the kernels, and only the lists of slots are host arrays.
 *   k    : bf16 [layers][num_pages][Hkv][page][d]
 *   v    : bf16 [layers][num_pages][Hkv][page / 16][d][16] -- steps of 16 tokens, transposed:
 *          the operand of the matrix product that reads them, so a step is one contiguous copy
 *   meta : int32, fp_cache_meta_size elements, 8-byte aligned:
 *          state [8]                       pages in use, FP_CACHE_* error bits, 0, ...
 *          used  [2 * ceil(num_pages/64)]  bit p % 32 of word p / 32: page p is in use
 *          len   [num_slots]               tokens of a slot (0: empty)
 *          ref   [num_pages]               slots that hold a page
 *          table [num_slots][max_pages]    a slot's pages in order, -1 past its last one
 * Two slots may hold the same page (fp_cache_fork).  A page is written only while one slot holds
 * it: fp_cache_reserve first gives a slot that is about to grow a copy of a shared last page that
 * is not full.  Pages are handed out lowest number first, so the state after a series of calls
 * does not depend on how the GPU ordered their work.
 *
 * What only the device knows cannot be refused by the host.  A reserve that finds too few pages
 * or too short a table row changes nothing and sets an error bit in state[1]; while a bit is set
 * reserve, fork, truncate and compact do nothing.  Write finds its place from the length that
 * reserve, fork or truncate gave a slot, so once one of them has failed or has been left out
 * write does nothing either, and tokens that are there already stay.  The caller reads the word
 * when it synchronises anyway and clears it by storing 0. */
#define FP_CACHE_FULL 1       /* fp_cache_reserve: fewer free pages than the call needs        */
#define FP_CACHE_TOO_LONG 2   /* fp_cache_reserve: a slot would pass max_pages pages           */
#define FP_CACHE_SHARED 4     /* fp_cache_write: tokens on a page that is not the slot's alone */
                              /* (not reserved), which were left out                           */
#define FP_CACHE_SKIPPED 8    /* fp_cache_reserve, fp_cache_fork, fp_cache_truncate: left out  */
                              /* because of FP_CACHE_SHARED, and the writes after them         */

#define FP_MAX_CACHE_LIST 256         /* slots per call                                   */
#define FP_MAX_CACHE_PAGES (1 << 22)  /* largest num_pages                                */
#define FP_MAX_QUERIES 16             /* query tokens per sequence in fp_decode_attn      */

typedef struct fp_cache {
  int32_t layers;        /* >= 1                                                          */
  int32_t num_pages;     /* pages per layer, 1..FP_MAX_CACHE_PAGES                        */
  int32_t num_kv_heads;  /* Hkv, 1..1024                                                  */
  int32_t head_dim;      /* d in {64, 128}                                                */
  int32_t page;          /* tokens per page: 16, 32, 64, 128 or 256                       */
  int32_t num_slots;     /* 1..65536                                                      */
  int32_t max_pages;     /* pages a slot can hold: its capacity is max_pages * page       */
                         /* tokens, at most 2^26; num_slots * max_pages < 2^31            */
  void *k, *v;           /* device pools, 16-byte aligned                                 */
  int32_t *meta;         /* device bookkeeping                                            */
} fp_cache;

/* int32 elements of fp_cache.meta (k, v and meta are not looked at).  Host only. */
fp_status fp_cache_meta_size(const fp_cache *cache, size_t *elems);

/* Device workspace bytes of fp_cache_reserve and fp_cache_compact: the list of page copies
 * that the call makes, and for compact the new number of every page.  The workspace is 4-byte
 * aligned.  Host only. */
fp_status fp_cache_workspace_size(const fp_cache *cache, size_t *bytes);

/* Every slot empty, every page free, no error.  The pools are left as they are. */
fp_status fp_cache_init(const fp_cache *cache, void *stream);

/* Room for counts[i] >= 0 more tokens in slots[i], i < n (HOST arrays; 1 <= n <=
 * FP_MAX_CACHE_LIST, slots distinct): len grows by counts[i], and new pages, lowest free number
 * first, go to the slots in list order.  A slot that grows, whose last page is not full and
 * held by others too, gets a copy of it (in every layer) as its first new page; of several
 * such slots in the list, the last holder of a page keeps it.  The tokens themselves are
 * written by fp_cache_write.  All or nothing (see FP_CACHE_FULL, FP_CACHE_TOO_LONG). */
fp_status fp_cache_reserve(const fp_cache *cache, int32_t n, const int32_t *slots,
                           const int32_t *counts, void *ws, size_t ws_bytes, void *stream);

/* Keys and values of one layer for the last cu[i+1] - cu[i] tokens of slots[i] (HOST arrays,
 * cu [n+1], cu[0] = 0, non-decreasing): rows cu[i] .. cu[i+1]-1 of k and v, each [Hkv][d] bf16
 * contiguous, k_stride and v_stride elements from one token to the next (>= Hkv * d, a multiple
 * of 8; pointers 16-byte aligned).  Rows beyond a slot's length are left out.  Takes up to 2^24
 * pieces of 64 tokens and one KV head. */
fp_status fp_cache_write(const fp_cache *cache, int32_t layer, int32_t n, const int32_t *slots,
                         const int32_t *cu, const void *k, int64_t k_stride, const void *v,
                         int64_t v_stride, void *stream);

/* dst[i] becomes a copy of src[i] that shares its pages (HOST arrays; dst distinct, none of
 * them in src; src may repeat).  What dst[i] held before is given back. */
fp_status fp_cache_fork(const fp_cache *cache, int32_t n, const int32_t *src, const int32_t *dst,
                        void *stream);

/* slots[i] keeps its first min(len, lens[i]) tokens, lens[i] >= 0 (HOST arrays, slots
 * distinct); pages past them are given back, and are free once no slot holds them.  lens =
 * NULL frees the slots. */
fp_status fp_cache_truncate(const fp_cache *cache, int32_t n, const int32_t *slots,
                            const int32_t *lens, void *stream);

/* The pages in use become pages 0 .. state[0]-1: the k-th free page below that number takes the
 * content (in every layer), holders and place in every table of the k-th page in use at or above
 * it.  The pools can then be cut to state[0] pages, or another cache laid behind them.  Where
 * state[0] and the bitmap disagree (a caller's own bookkeeping) nothing moves. */
fp_status fp_cache_compact(const fp_cache *cache, void *ws, size_t ws_bytes, void *stream);

/* One batch of fp_decode_attn. */
typedef struct fp_decode {
  int32_t batch;               /* sequences, 1..FP_MAX_CACHE_LIST                            */
  const int32_t *slots;        /* HOST [batch]: the cache slot of a sequence, or -1: none    */
  int32_t num_q_heads;         /* Hq, a multiple of Hkv                                      */
  int32_t queries;             /* query tokens per sequence, 1..FP_MAX_QUERIES: its last     */
                               /* `queries` tokens, whose keys and values are in the cache   */
  int32_t groups;              /* 0, or groups of consecutive sequences that share a prefix  */
  const int32_t *group_start;  /* HOST [groups+1], 0 .. batch ascending (groups > 0)         */
  const int32_t *prefix_lens;  /* HOST [groups]: tokens at the start of every sequence of    */
                               /* the group that are the same (>= 0)                         */
  float softmax_scale;         /* 0 => 1/sqrt(d)                                             */
} fp_decode;

/* Device workspace bytes of fp_decode_attn: partial results of key ranges.  q, o and the workspace
 * are 16-byte aligned.  Host only. */
fp_status fp_decode_workspace_size(const fp_cache *cache, const fp_decode *batch, size_t *bytes);

/* Attention of each sequence's last `queries` tokens over the whole sequence: query t (of
 * `queries`) of a sequence of n tokens attends to its keys 0 .. n - queries + t.  Row b *
 * queries + t of q and o, each row [Hq][d] bf16 contiguous, q_stride elements from one row of q
 * to the next (>= Hq * d, a multiple of 8); rows of o are contiguous.  A query with no key (an
 * empty slot, slot -1, more queries than tokens) gets 0.  Only what the visible tokens hold
 * matters: what lies in a page past its tokens, or in tokens after a query, does not reach it.
 * The keys and values of a group's prefix are read once for all of its sequences, from the pages
 * of the first one that is not empty; if a sequence of the group is shorter, as much of the
 * prefix as every query of the group sees.
 * Scores, maxima, sums and O are float32.  The weights that multiply the values are rounded to
 * 2^-16 of themselves, over a prefix with more than 32 rows ((Hq / Hkv) * queries * sequences of
 * the group) to bf16, 2^-8, as in fp_sparse_attn; the sum is that of the rounded weights.  The same
 * call on the same state gives the same bits.  Where the keys are cut into ranges follows from the
 * lengths and groups of the whole batch, so the last bits of a row depend on the rest of it. */
fp_status fp_decode_attn(const fp_cache *cache, const fp_decode *batch, int32_t layer,
                         const void *q, int64_t q_stride, void *o, void *ws, size_t ws_bytes,
                         void *stream);

/* ---------------------------------------------------------------------------------------
 * Between a layer's projection and its attention: norms of query and key heads and their rotation
 * by position, by themselves (before fp_select and fp_sparse_attn) and on the way into the cache. */

#define FP_ROPE_HALF 0         /* pairs (i, i + rotary_dim / 2) of a head                       */
#define FP_ROPE_INTERLEAVED 1  /* pairs (2 i, 2 i + 1)                                          */

#define FP_ROPE_UNSCALED 0
#define FP_ROPE_LINEAR 1       /* every frequency divided by `factor`                           */
#define FP_ROPE_BASE 2         /* base * factor^(R / (R - 2)): the first frequency stays, the   */
                               /* last one is divided by `factor`                               */
#define FP_ROPE_PARTS 3        /* by the turns t = original_len f / 2 pi that a pair makes in   */
                               /* the original context: f g + (f / factor) (1 - g) with         */
                               /* g = clamp((t - low_turns) / (high_turns - low_turns), 0, 1)   */

typedef struct fp_rope_params {
  int32_t rotary_dim;    /* R: the first R elements of a head are rotated; a multiple of 16,    */
                         /* 16..128                                                             */
  int32_t layout;        /* FP_ROPE_HALF or FP_ROPE_INTERLEAVED                                 */
  int32_t scaling;       /* FP_ROPE_UNSCALED ..                                                 */
  double base;           /* f_i = base^(-2 i / R) radians per position, i < R / 2; > 0          */
  double factor;         /* >= 1 (scaling)                                                      */
  double original_len, low_turns, high_turns;   /* FP_ROPE_PARTS: > 0, >= 0, > low_turns        */
  double amplitude;      /* cosine and sine are multiplied by it; 0 => 1                        */
  const double *inv_freq;  /* HOST [R / 2], or NULL: the frequencies themselves (|f| <= 2^20),  */
                         /* unscaled; base is not looked at                                     */
} fp_rope_params;

/* Written by fp_rope_init; plain data, which may be copied. */
typedef struct fp_rope {
  int32_t rotary_dim, layout;
  float amplitude;
  int32_t reserved;
  uint64_t step[64];     /* per pair: turns per position as a fraction of 2^64                  */
} fp_rope;

/* Host only. */
fp_status fp_rope_init(const fp_rope_params *params, fp_rope *rope);

/* RMS norm over a head: x / sqrt(mean(x^2) + eps) * weight. */
typedef struct fp_head_norm {
  const void *q_weight, *k_weight;  /* device [d], 16-byte aligned, or NULL: 1                  */
  int32_t weight_f32;               /* the weights are float32, else bf16                       */
  float eps;                        /* >= 2^-126                                                */
} fp_head_norm;

/* Heads of `tokens` tokens normed (norm == NULL: not) and rotated by positions[token] (rope ==
 * NULL: not; positions is then not looked at).  q, q_out: [tokens][Hq][d] and k, k_out:
 * [tokens][Hkv][d] bf16, a token's heads contiguous, strides in elements from one token to the next
 * (>= heads * d, a multiple of 8; pointers 16-byte aligned); d in {64, 128}, rotary_dim <= d.  Hq or
 * Hkv may be 0, and its pointers NULL.  An output may be its own input (same pointer and stride),
 * and must not overlap an input otherwise.  positions: int32 on the device, of any sign and size.  Up to
 * 2^25 tokens, and 8192 heads of each kind.  A norm sums squares in float32, which those of elements below
 * 2^60 stay within.
 * Computed in float32 and rounded once; cosines and sines are off by at most 2^-22 (times the
 * amplitude) from those of the position times the frequency, a float64 number, whatever both are.  A NaN
 * or an infinity stays within its head (norm) or its pair. */
fp_status fp_rotate(int32_t tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                    const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                    const int32_t *positions, const fp_rope *rope, const fp_head_norm *norm,
                    void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride,
                    void *stream);

/* fp_cache_write of keys that are normed and rotated on the way, and of values as they are; the
 * queries of the same tokens are normed and rotated into q_out.  A token's position is its place in
 * the slot, so row cu[i] + j of a slot of n tokens has position n - (cu[i+1] - cu[i]) + j.  As in
 * fp_cache_write rows beyond a slot's length are left out (of q_out too), and nothing is done once
 * a reserve, fork or truncate has failed or been left out; keys and values of a page that other slots
 * hold too are left out (FP_CACHE_SHARED), the queries of those tokens are written.  q, q_out: rows [Hq][d] bf16, strides,
 * alignment and overlap as in fp_rotate; q == NULL with Hq 0: keys and values alone.  rope and norm
 * may be NULL.  Takes up to 2^24 / (Hkv + 8) pieces of 64 tokens. */
fp_status fp_cache_append(const fp_cache *cache, int32_t layer, int32_t n, const int32_t *slots,
                          const int32_t *cu, int32_t num_q_heads, const void *q, int64_t q_stride,
                          const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                          const fp_rope *rope, const fp_head_norm *norm, void *q_out,
                          int64_t q_out_stride, void *stream);

/* One batch of fp_chunk_attn. */
typedef struct fp_chunk {
  int32_t batch;               /* sequences, 1..FP_MAX_CACHE_LIST                            */
  const int32_t *slots;        /* HOST [batch]: the cache slot of a sequence, or -1: none    */
  const int32_t *cu;           /* HOST [batch+1], cu[0] = 0, non-decreasing: rows of q and o */
                               /* of a sequence, for its last cu[i+1] - cu[i] tokens, whose  */
                               /* keys and values are in the cache                           */
  int32_t num_q_heads;         /* Hq, a multiple of Hkv                                      */
  float softmax_scale;         /* 0 => 1/sqrt(d)                                             */
} fp_chunk;

/* Device workspace bytes of fp_chunk_attn: partial results of key ranges.  Host only. */
fp_status fp_chunk_workspace_size(const fp_cache *cache, const fp_chunk *batch, size_t *bytes);

/* Causal attention of chunks of new tokens over their sequences: query t of m = cu[i+1] - cu[i] of a
 * sequence of n tokens attends to its keys 0 .. n - m + t.  Rows, strides and alignment of q and o, rows
 * without a key and what of the cache reaches a row are as in fp_decode_attn.  Slots may repeat.
 * Scores, maxima, sums and O are float32; the weights that multiply the values are rounded to bf16, 2^-8,
 * and the sum is that of the rounded weights, as in fp_sparse_attn.  (fp_decode_attn rounds them to 2^-16
 * over a sequence's own keys: the same token comes out coarser here.)  Scores times the scale are to stay
 * below 2^29: from there on their rounding to float32 alone can make a row 0 or infinite.
 * The same call on the same state gives the same bits; where keys are cut into ranges follows from the
 * lengths of the whole batch, so the last bits of a row depend on the rest of it.
 * FP_ERR_UNSUPPORTED: more than 256 sequences, 8192 heads or 2^31 - 2^16 rows (tokens times Hq / Hkv) of
 * one sequence, or 5e14 places (rows / 128 times Hq times what a slot can hold). */
fp_status fp_chunk_attn(const fp_cache *cache, const fp_chunk *batch, int32_t layer, const void *q,
                        int64_t q_stride, void *o, void *ws, size_t ws_bytes, void *stream);

/* Static description of a status code. */
const char *fp_status_string(fp_status status);

/* Text of the last FP_ERR_HIP seen by this thread ("" if none). */
const char *fp_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FLEXPREFILL_H */
