// Internal declarations shared by the host orchestration and the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/flexprefill.h"

namespace fp {

// Longest key chunk owned by one workgroup of the representative-score kernels.  Short
// problems use chunks of 512 or 256 keys (SeqTable::ch_len) so that those kernels still
// get enough workgroups to fill the GPU.
constexpr int kScoreChunk = 1024;
constexpr int kScoreChunkMin = 256;
// workgroups of the line-sum kernel wanted before the chunk is shortened (4 per CU)
constexpr int kScoreWorkgroups = 1024;
constexpr int kHistBuckets = 2048;     // radix-select digit: 11 bits
constexpr int kHistCounts = 1024;      // last digit (10 bits), the only one with counts

// Per-call table of packed sequences, passed by value to every kernel.
struct SeqTable {
  int32_t n_seq;
  int32_t max_nb;
  int32_t cu[FP_MAX_BATCH + 1];       // token offsets
  int32_t nb_off[FP_MAX_BATCH + 1];   // prefix sums of nb_s = ceil(n_s / block)
  int32_t ch_len;                     // keys per score chunk: 1024, 512 or 256
  int32_t ch_off[FP_MAX_BATCH + 1];   // prefix sums of ceil(n_s / ch_len)
  int64_t tri_off[FP_MAX_BATCH + 1];  // prefix sums of nb_s (nb_s + 1) / 2
};

// Everything a kernel of the selection pipeline needs.
struct SelectArgs {
  SeqTable st;
  const uint16_t *q;       // [T][Hq][d] bf16
  const uint16_t *k;       // [T][Hkv][d] bf16
  int32_t hq, hkv, d, block;
  int32_t total_tokens;    // T
  int32_t nb_total;        // NB
  int64_t tri_total;       // TRI
  float scale;             // softmax scale
  float gamma, tau;
  int32_t min_budget;
  int32_t force_pattern;
  int32_t max_budget;      // 0 = no cap
  int32_t qa_mode;         // 0 flattened map (Algorithm 4), 1 per query block
  int32_t vs_granularity;  // 0 token lines (Algorithm 3), 1 block-pooled lines
  // set by the launcher: every selection problem in one workgroup (no histograms), and the
  // line marks made by convert_tiles itself (no vs_marks)
  int32_t small, marks_inline;
  // set by the launchers: the line pass merges the chunk statistics, pools Q, and the parts
  // it cuts a score chunk into
  int32_t merge_inline, pool_inline, line_parts;
  // workspace
  float2 *chunk_stats;     // [ch_total][Hq][block] (max, sum) in log2 units
  float2 *row_stats;       // [n_seq][Hq][block]
  float *kbar;             // [NB][Hkv][d]
  float *qbar;             // [NB][Hq][d]
  float *a_v;              // [Hq][T]
  float *a_s;              // [Hq][T]
  float *av_blk;           // [Hq][NB] a_v summed per key block (block-pooled lines)
  float *as_blk;           // [Hq][NB] a_s summed per offset block
  float *pat_logit;        // [Hq][NB] scale * q_bar . K_bar_J of the pattern search
  double *pat_ahat;        // [Hq][NB] a_hat[J] = a_v summed per key block
  uint8_t *vs_marks;       // [Hq][NB][4] per key block / diagonal: column, diagonal (full
                           // rows), diagonal (partial last row), diagonal + 1
  float *flat;             // [Hq][TRI]
  struct SelState *sel;    // [n_seq][Hq][2]
  uint32_t *hist_cnt;      // [n_seq][Hq][2][kHistCounts]
  unsigned long long *hist_mass;  // [n_seq][Hq][2][kHistBuckets]
  // outputs
  int32_t *kb_idx;
  int32_t *kb_cnt;
  uint8_t *pattern;
  float *js;
  int32_t *units;
};

// State of one cumulative-mass selection problem (one score vector).
struct SelState {
  unsigned long long total;       // fixed-point mass of all units
  unsigned long long thr;         // ceil(gamma * total)
  unsigned long long mass_above;  // mass of keys above the current digit range
  unsigned long long ticket;      // slices of the radix pass that are done, and (in the upper
                                  // 32 bits) the units that they counted above its range
  uint32_t cnt_above;             // number of keys above the current digit range
  uint32_t prefix;                // key bits fixed so far
  uint32_t key;                   // final threshold key
  int32_t idcut;                  // last id taken among key == `key`
  int32_t k;                      // units selected
  int32_t mode;                   // 0 active, 1 take all, 2 inactive (other pattern)
  int32_t n;                      // number of units
};

// The split grid is taken for at most this many tenths of a row per resident workgroup.
// Where the line lies (attention over selected lists, us, other grid -> split grid; single
// runs differ by 3-10%): block 128, head dim 128, 2.0 rows (32 heads, 4k tokens) 143 -> 121,
// 2.9 (6k) 251 -> 250, 3.4 (7k) 320 -> 318, 5.0 (10k) 516 -> 544; head dim 64, 3.0 rows (64
// heads, 4500) 208 -> 170, 3.6 (5500) 229 -> 194, 4.6 (7k) 375 -> 347, 6.2 (9500) 549 -> 549,
// so on the safe side there; block 64, head dim 128, 4.0 rows (32 heads, 8k) 282 -> 223, 4.8
// (9800) 460 -> 496; head dim 64, 4.6 (64 heads, 7k) 374 -> 293, 5.5 (8500) 517 -> 437, 6.9
// (10500) 586 -> 541.
constexpr int kSplitRows128 = 30;
constexpr int kSplitRows64 = 48;
// Shortest segment that a longer list is cut into: 3, 4 and 6 blocks measure the same within
// 3% (two heads of 64, 2k tokens: 29.9, 28.8, 28.4 us; 8 heads, 4k: 43.5, 44.6, 44.7).
constexpr int kSegBlocks = 4;
constexpr int kSplitUnits = 2816;   // units per KV group: 8 B of key slots (a power of two),
                                    // 32 B of records each in the sort's 128 KB of LDS

// Short attention problems: one workgroup per unit, a unit being a row's list or a segment
// of it (unit_cap = 0: not used).
struct SplitArgs {
  int4 *units;             // [Hkv][unit_cap] records {row, blocks, first block, second block}
  int4 *segs;              // [Hkv][unit_cap] {first list entry, first slot, segment, segments}
  int32_t *tickets;        // [slots] at a split row's first slot: its segments stored so far
  unsigned long long *partials;   // [slots] partial results of segments
  int32_t unit_cap;        // units per KV group, the unused last ones marked empty
  int32_t extra;           // units per KV group beyond its rows; 2 * extra slots
  int32_t all;             // `extra` covers every segment of kSegBlocks
  int32_t slots;           // resident workgroups of the chip
};

struct AttnArgs {
  SeqTable st;
  const uint16_t *q, *k, *v;
  uint16_t *o;
  const int32_t *kb_idx;
  const int32_t *kb_cnt;
  int32_t hq, hkv, d, block;
  int32_t nb_total;
  int64_t tri_total;
  float scale_log2;        // softmax scale * log2(e)
  int4 *items;             // [Hkv][G * NB] workspace: ordered item records per KV group
  int32_t *queue;          // [8] workspace: per-XCD work-queue counters
  int32_t mix;             // set by the launcher: an XCD's KV groups served interleaved
  uint16_t *vt;            // [Hkv][NB][B * d] workspace: V^T tiles per key block
  unsigned long long *sort_keys;  // [Hkv][G * NB] workspace: items' sort keys
  int4 *sort_recs;         // [Hkv][G * NB] workspace: item records in item-id order
  SplitArgs split;
};

// A cache as the kernels see it: fp_cache with the parts of its bookkeeping.
struct CacheView {
  uint16_t *k, *v;
  int32_t *state;              // [8]: pages in use, error bits
  unsigned long long *used;    // [words] one bit per page
  int32_t *len;                // [slots]
  int32_t *ref;                // [pages]
  int32_t *table;              // [slots][max_pages]
  int32_t layers, pages, hkv, d, page, page_shift, slots, max_pages, words;
};

// Slots of one call and a number for each, passed by value.
struct CacheList {
  int32_t n;
  int32_t slot[FP_MAX_CACHE_LIST];
  int32_t num[FP_MAX_CACHE_LIST + 1];
};

// Page copies that a call makes in every layer, made by its first launch (workspace).
struct PageCopies {
  int32_t *count;              // [4]: copies
  int32_t *src, *dst;          // [pages]
  int32_t *renamed;            // [pages] compact: new number of a page that moves
};

struct WriteArgs {
  CacheList list;              // num: row of a slot's first token; [n]: rows in all
  int32_t blk[FP_MAX_CACHE_LIST + 1];   // prefix sums of the 64-token blocks that a slot's
                                        // rows can touch
  const uint16_t *k, *v;
  int64_t k_stride, v_stride;
  int32_t layer;
};

struct ForkArgs {
  int32_t n;
  int32_t src[FP_MAX_CACHE_LIST], dst[FP_MAX_CACHE_LIST];
};

// fp_rope and fp_head_norm as the kernels see them.
struct RopeArgs {
  int32_t rotary;              // elements that are rotated; 0: none
  int32_t half;                // pairs (i, i + rotary / 2), else (2 i, 2 i + 1)
  int32_t normed, w_f32;       // heads are normed; the weights' type
  float amplitude, eps;
  const void *wq, *wk;         // weights [d], or null: 1
  uint64_t step[64];           // per pair: turns per position, times 2^64
};

struct RotateArgs {
  const uint16_t *q, *k;
  uint16_t *qo, *ko;
  int64_t q_stride, k_stride, qo_stride, ko_stride;
  const int32_t *positions;
  int32_t tokens, hq, hkv;
  int32_t groups, set;         // set by the launcher: waves that share the heads of a token, tokens of
                               // a wave
  RopeArgs rope;
};

struct AppendArgs {
  WriteArgs w;
  const uint16_t *q;           // or null
  uint16_t *qo;
  int64_t q_stride, qo_stride;
  int32_t hq;
  int32_t query_tokens, set;   // set by the launcher: positions of a part of the queries, tokens of a wave
  RopeArgs rope;
};

// What the joining launch of decode_attn knows of the call's plan (workspace).
struct DecodeJoin {
  int4 seq[FP_MAX_CACHE_LIST];     // per sequence: tokens, keys of the prefix, places of its own
                                   // keys and of the prefix
  int4 group[FP_MAX_CACHE_LIST];   // per sequence: group, its first sequence, its rows, many or not
  int32_t places_many, places_lean;
  int32_t clusters, width, lean;
};

struct DecodeArgs {
  const uint16_t *k, *v;       // pools of the layer
  const int32_t *len, *table;
  const uint16_t *q;
  uint16_t *o;
  int64_t q_stride;
  // partial results of key ranges: prefixes with many and with few rows, sequences' own keys
  float *part_many, *part_few, *part_own;
  DecodeJoin *join;
  int32_t any_prefix;          // some group may share a prefix
  int32_t any_many;            // ... with more than kDecodeFew rows
  int32_t tile_rows;           // query rows of a unit of the other work: 16 or 32
  int32_t tile_shift;          // its logarithm: 4 or 5
  int32_t pages, hkv, page_shift, max_pages;
  int32_t G, hq, nq, batch, groups;
  int32_t wgs;                 // workgroups that the key ranges are divided among
  float scale_log2;            // softmax scale * log2(e)
  int32_t slot[FP_MAX_CACHE_LIST];
  int32_t prefix[FP_MAX_CACHE_LIST];       // per group
  int16_t start[FP_MAX_CACHE_LIST + 1];    // per group: its first sequence
  uint8_t group[FP_MAX_CACHE_LIST];        // per sequence
};

struct ChunkArgs {
  const uint16_t *k, *v;       // pools of the layer
  const int32_t *len, *table;
  const uint16_t *q;
  uint16_t *o;
  int64_t q_stride;
  int32_t pages, hkv, page_shift, max_pages;
  int32_t G, hq, batch;
  int32_t wgs;                 // workgroups that the keys are divided among
  int32_t width;               // row tiles side by side, one for each workgroup of a cluster
  int32_t rows;                // rows of a row tile: 128 or, with workgroups of eight waves, 256
  int32_t records;             // what the join looks at: one for every segment or for every part
  int32_t by_segment;
  int32_t tile_rows;           // rows of a partial result: `rows`, fewer where no sequence has as many
  int32_t tiles;               // row tiles of all sequences and KV heads (0: too many for a grid)
  float scale_log2;            // softmax scale * log2(e)
  int4 *seg;                   // records: pieces of a segment (0: one or none) and its first part, its
                               // sequence, KV head and number
  float *part;                 // partial results, two for each workgroup
  int32_t slot[FP_MAX_CACHE_LIST];
  int32_t cu[FP_MAX_CACHE_LIST + 1];
  int32_t base[FP_MAX_CACHE_LIST];         // per sequence: records before its own (by_segment)
};

// Query rows of one unit of work on prefixes with many rows: 4 waves of 32.
constexpr int kDecodeRows = 128;
// Rows up to which a prefix is read like a sequence's own keys, in tiles of 16 or 32 rows.  Two such
// tiles for 64 rows (16 samples of 32k): 57 us, one tile of 128 rows half empty 40; five groups of 48
// rows (12 samples of 9k) 76 and 49.6.
constexpr int kDecodeFew = 32;
// Workgroups that fp_decode_attn divides its keys among: every one resident, two (head dim 128)
// or three (64) on each of 256 CUs.
constexpr int decode_wgs(int d) { return d == 64 ? 768 : 512; }

// Device address of the current device's fixed scratch array (fp_noalloc.hip).
hipError_t noalloc_scratch(void **out);

// Launchers (each returns the hipError_t of its launch).
hipError_t launch_sparse_attn(const AttnArgs &a, hipStream_t s);
hipError_t launch_select_pipeline(const SelectArgs &a, hipStream_t s);
hipError_t launch_dense_lists(const SelectArgs &a, hipStream_t s);
hipError_t launch_qa_rows(const SelectArgs &a, hipStream_t s);
hipError_t launch_cache_init(const CacheView &c, hipStream_t s);
hipError_t launch_cache_reserve(const CacheView &c, const CacheList &l, const PageCopies &w,
                                hipStream_t s);
hipError_t launch_cache_write(const CacheView &c, const WriteArgs &a, hipStream_t s);
hipError_t launch_cache_fork(const CacheView &c, const ForkArgs &a, hipStream_t s);
hipError_t launch_cache_truncate(const CacheView &c, const CacheList &l, hipStream_t s);
hipError_t launch_cache_compact(const CacheView &c, const PageCopies &w, hipStream_t s);
hipError_t launch_decode_attn(const DecodeArgs &a, int d, hipStream_t s);
hipError_t launch_chunk_attn(const ChunkArgs &a, int d, hipStream_t s);
hipError_t launch_rotate(const RotateArgs &a, int d, hipStream_t s);
hipError_t launch_cache_append(const CacheView &c, const AppendArgs &a, hipStream_t s);
// Workgroups of launch_cache_append per 64 positions of a slot.
int append_parts(const CacheView &c, int query_heads);

}  // namespace fp
