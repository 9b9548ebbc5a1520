// Host side of the C ABI: argument checks, workspace layout, launch order.
//
// Nothing here allocates device memory or synchronises: every call validates on the host,
// carves the caller's workspace, and enqueues kernels on the caller's stream.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "fp_internal.h"

namespace {

thread_local char g_last_error[256] = "";

constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct Dims {
  fp::SeqTable st;
  int64_t total_tokens;
  int64_t nb_total;
  int64_t tri_total;
  int64_t ch_total;
};

fp_status check_shape(const fp_shape *sh, Dims *dm) {
  if (!sh || !sh->cu_seqlens) return FP_ERR_INVALID_ARG;
  if (sh->batch < 1 || sh->num_q_heads < 1 || sh->num_kv_heads < 1 || sh->head_dim < 1 ||
      sh->block < 1)
    return FP_ERR_INVALID_ARG;
  if (sh->num_q_heads % sh->num_kv_heads != 0) return FP_ERR_INVALID_ARG;
  if (sh->batch > FP_MAX_BATCH) return FP_ERR_UNSUPPORTED;
  if (sh->head_dim != 64 && sh->head_dim != 128) return FP_ERR_UNSUPPORTED;
  if (sh->block != 128 && sh->block != 64) return FP_ERR_UNSUPPORTED;
  if (sh->num_kv_heads > 1024 || sh->num_q_heads > 8192) return FP_ERR_UNSUPPORTED;
  if (sh->cu_seqlens[0] != 0) return FP_ERR_INVALID_ARG;
  memset(dm, 0, sizeof(*dm));
  fp::SeqTable &st = dm->st;
  st.n_seq = sh->batch;
  // score chunk: the longest of 1024, 512, 256 keys that still gives the line-sum kernel
  // kScoreWorkgroups (sequence chunk, query head) workgroups
  st.ch_len = fp::kScoreChunkMin;
  for (int len = fp::kScoreChunk; len > fp::kScoreChunkMin; len /= 2) {
    int64_t chunks = 0;
    for (int s = 0; s < sh->batch; ++s)
      chunks += ((int64_t)sh->cu_seqlens[s + 1] - sh->cu_seqlens[s] + len - 1) / len;
    if (chunks * sh->num_q_heads >= fp::kScoreWorkgroups) {
      st.ch_len = len;
      break;
    }
  }
  int64_t nb_acc = 0, tri_acc = 0, ch_acc = 0;
  int max_nb = 0;
  for (int s = 0; s < sh->batch; ++s) {
    const int64_t n = (int64_t)sh->cu_seqlens[s + 1] - sh->cu_seqlens[s];
    if (n < 1) return FP_ERR_INVALID_ARG;
    const int64_t nb = (n + sh->block - 1) / sh->block;
    if (nb > 8192) return FP_ERR_UNSUPPORTED;   // up to 1M tokens (512k at block 64)
    st.cu[s] = sh->cu_seqlens[s];
    st.nb_off[s] = (int32_t)nb_acc;
    st.tri_off[s] = tri_acc;
    st.ch_off[s] = (int32_t)ch_acc;
    nb_acc += nb;
    tri_acc += nb * (nb + 1) / 2;
    ch_acc += (n + st.ch_len - 1) / st.ch_len;
    if (nb > max_nb) max_nb = (int)nb;
  }
  const int64_t T = sh->cu_seqlens[sh->batch];
  if (T > (int64_t)0x7FFFFFFF / 2) return FP_ERR_UNSUPPORTED;
  if (nb_acc > (1 << 20)) return FP_ERR_UNSUPPORTED;
  st.cu[sh->batch] = (int32_t)T;
  st.nb_off[sh->batch] = (int32_t)nb_acc;
  st.tri_off[sh->batch] = tri_acc;
  st.ch_off[sh->batch] = (int32_t)ch_acc;
  st.max_nb = max_nb;
  dm->total_tokens = T;
  dm->nb_total = nb_acc;
  dm->tri_total = tri_acc;
  dm->ch_total = ch_acc;
  // the flattened per-head index space must stay addressable with int32 offsets per head
  if (tri_acc * (int64_t)sh->num_q_heads > ((int64_t)1 << 40)) return FP_ERR_UNSUPPORTED;
  return FP_OK;
}

// A softmax scale argument: finite and >= 0 (0 selects 1 / sqrt(d)).
bool scale_ok(float s) { return s >= 0.f && !isnan(s) && !isinf(s); }
float resolved_scale(float s, int head_dim) {
  return s > 0.f ? s : 1.0f / sqrtf((float)head_dim);
}

fp_status check_params(const fp_shape *sh, const fp_params *p) {
  if (!(p->gamma > 0.f) || !(p->gamma <= 1.f) || isnan(p->gamma)) return FP_ERR_INVALID_ARG;
  if (!(p->tau >= 0.f) || !(p->tau <= 1.f)) return FP_ERR_INVALID_ARG;
  if (p->min_budget_blocks < 0) return FP_ERR_INVALID_ARG;
  if (p->min_budget_blocks > FP_MAX_MIN_BUDGET) return FP_ERR_UNSUPPORTED;
  if (!scale_ok(p->softmax_scale)) return FP_ERR_INVALID_ARG;
  if (p->force_pattern < -1 || p->force_pattern > 1) return FP_ERR_INVALID_ARG;
  if (p->max_budget_blocks < 0 || p->max_budget_blocks == 1) return FP_ERR_INVALID_ARG;
  if (p->max_budget_blocks > 0 && p->max_budget_blocks < p->min_budget_blocks)
    return FP_ERR_INVALID_ARG;
  if (p->qa_mode < 0 || p->qa_mode > 1) return FP_ERR_INVALID_ARG;
  if (p->vs_granularity < 0 || p->vs_granularity > 1) return FP_ERR_INVALID_ARG;
  (void)sh;
  return FP_OK;
}

// Workspace layout of fp_select; returns the total size, fills pointers when base != 0.
size_t select_layout(const fp_shape *sh, const Dims &dm, char *base, fp::SelectArgs *a) {
  const int64_t hq = sh->num_q_heads, hkv = sh->num_kv_heads, d = sh->head_dim, b = sh->block;
  const int64_t problems = (int64_t)sh->batch * hq * 2;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align_up(off + bytes);
    return base ? base + o : nullptr;
  };
  char *chunk_stats = take(sizeof(float2) * dm.ch_total * hq * b);
  char *row_stats = take(sizeof(float2) * sh->batch * hq * b);
  char *kbar = take(sizeof(float) * dm.nb_total * hkv * d);
  char *qbar = take(sizeof(float) * dm.nb_total * hq * d);
  char *a_v = take(sizeof(float) * hq * dm.total_tokens);
  char *a_s = take(sizeof(float) * hq * dm.total_tokens);
  char *av_blk = take(sizeof(float) * hq * dm.nb_total);
  char *as_blk = take(sizeof(float) * hq * dm.nb_total);
  char *pat_logit = take(sizeof(float) * hq * dm.nb_total);
  char *pat_ahat = take(sizeof(double) * hq * dm.nb_total);
  char *vs_marks = take(4 * hq * dm.nb_total);
  char *flat = take(sizeof(float) * hq * dm.tri_total);
  char *sel = take(sizeof(fp::SelState) * problems);
  char *hist_cnt = take(sizeof(uint32_t) * problems * fp::kHistCounts);
  char *hist_mass = take(sizeof(unsigned long long) * problems * fp::kHistBuckets);
  if (a) {
    a->chunk_stats = (float2 *)chunk_stats;
    a->row_stats = (float2 *)row_stats;
    a->kbar = (float *)kbar;
    a->qbar = (float *)qbar;
    a->a_v = (float *)a_v;
    a->a_s = (float *)a_s;
    a->av_blk = (float *)av_blk;
    a->as_blk = (float *)as_blk;
    a->pat_logit = (float *)pat_logit;
    a->pat_ahat = (double *)pat_ahat;
    a->vs_marks = (uint8_t *)vs_marks;
    a->flat = (float *)flat;
    a->sel = (fp::SelState *)sel;
    a->hist_cnt = (uint32_t *)hist_cnt;
    a->hist_mass = (unsigned long long *)hist_mass;
  }
  return off;
}

// attention workspace: ordered item records [Hq][NB] int4, 8 queue counters, then the V^T
// tiles [Hkv][NB][block * d] bf16
// Attention workspace: ordered item records (16 B per query head and block), 8 queue
// counters, V^T tiles, and the items' sort keys (8 B) and records in id order (16 B).
size_t attn_layout(const fp_shape *sh, const Dims &dm) {
  const size_t items = (size_t)dm.nb_total * sh->num_q_heads;
  return align_up(16 * items) + align_up(8 * sizeof(int32_t)) +
         align_up(2 * (size_t)dm.nb_total * sh->num_kv_heads * sh->block * sh->head_dim) +
         align_up(8 * items) + align_up(16 * items);
}

// Split plan of a short attention problem in `room` (room_bytes of device workspace after the
// `base` bytes of attn_layout; null: any size): fills *out (unit_cap = 0 when the problem is
// not short, or the room too small) and returns the bytes it takes.  A plan never takes more
// than the fixed scratch array leaves after `base`, so that fp_sparse_attn_noalloc cuts the
// same rows as fp_sparse_attn with all the room it can use.
size_t plan_split(const fp::SeqTable &st, int hq, int hkv, int d, int block, size_t base,
                  char *room, size_t room_bytes, fp::SplitArgs *out) {
  *out = fp::SplitArgs{};
  const int nb_total = st.nb_off[st.n_seq], G = hq / hkv;
  // resident workgroups of 256 CUs: two (head dim 128) or three waves per SIMD
  const int slots = (d == 64 ? 768 : 512) * 128 / block;
  const int64_t n_g = (int64_t)G * nb_total;
  if (10 * n_g * hkv > (int64_t)(block == 64 ? fp::kSplitRows64 : fp::kSplitRows128) * slots)
    return 0;
  // units that cutting rows of I + 1 blocks into segments of kSegBlocks can add at most
  int64_t most = 0;
  for (int s = 0; s < st.n_seq; ++s)
    for (int I = 0, nb = st.nb_off[s + 1] - st.nb_off[s]; I < nb; ++I) most += I / fp::kSegBlocks;
  most *= G;
  const int64_t part = (int64_t)block * (d + 4) * 4;   // O, then two floats per lane of a row
  auto layout = [&](int64_t extra, fp::SplitArgs *a) {
    const int64_t cap = n_g + extra, n_slot = 2 * extra * hkv;
    const size_t o1 = align_up(16 * cap * hkv), o2 = o1 + align_up(16 * cap * hkv),
                 o3 = o2 + align_up(4 * n_slot);
    if (a) {
      a->units = (int4 *)room;
      a->segs = (int4 *)(room + o1);
      a->tickets = (int32_t *)(room + o2);
      a->partials = (unsigned long long *)(room + o3);
      a->unit_cap = (int)cap;
      a->extra = (int)extra;
      a->all = extra == most;
      a->slots = slots;
    }
    return o3 + part * n_slot;
  };
  // Units beyond the rows: 0.7 of a resident workgroup each, i.e. segments of the group's
  // blocks over 0.7 of its workgroups.  More cuts cost partial results, fewer leave long
  // segments: at 1, 0.85, 0.7, 0.6, 0.5 the attention of 32 heads takes 126, 120, 119, 123,
  // 124 us at 4k tokens and 55, -, 45, 43, 45 at 1500, of 8 heads on own lists 40, 39, 40, 43,
  // 44 at 4k, of dense 2k 66, 64, 62, 65, 65.
  const int64_t share = (7 * (int64_t)slots / 10 + hkv - 1) / hkv;
  int64_t extra = share < most ? share : most;
  if (n_g + extra > fp::kSplitUnits) return 0;
  // as much of the plan as the room holds
  if (!room) room_bytes = SIZE_MAX;
  if (base <= (size_t)FP_NOALLOC_SCRATCH_BYTES)
    room_bytes = std::min(room_bytes, (size_t)FP_NOALLOC_SCRATCH_BYTES - base);
  extra = (int64_t)std::min<size_t>((size_t)extra, room_bytes / (size_t)(2 * hkv * part));
  while (extra > 0 && layout(extra, nullptr) > room_bytes) --extra;
  if (layout(extra, nullptr) > room_bytes) return 0;
  if (room) layout(extra, out);
  return layout(extra, nullptr);
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void *p) { return ((uintptr_t)p & 3) == 0; }

// Sizes of a cache; `view` (or null) gets the kernels' view of it.
fp_status check_cache(const fp_cache *c, fp::CacheView *view) {
  if (!c) return FP_ERR_INVALID_ARG;
  if (c->layers < 1 || c->num_pages < 1 || c->num_kv_heads < 1 || c->head_dim < 1 ||
      c->page < 1 || c->num_slots < 1 || c->max_pages < 1)
    return FP_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FP_ERR_UNSUPPORTED;
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1))) return FP_ERR_UNSUPPORTED;
  if (c->num_pages > FP_MAX_CACHE_PAGES || c->num_kv_heads > 1024 || c->num_slots > 65536)
    return FP_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page > ((int64_t)1 << 26)) return FP_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->num_slots > 0x7FFFFFFF) return FP_ERR_UNSUPPORTED;
  if (!view) return FP_OK;
  if (!c->k || !c->v || !c->meta || !aligned16(c->k) || !aligned16(c->v) ||
      ((uintptr_t)c->meta & 7))
    return FP_ERR_INVALID_ARG;
  fp::CacheView &w = *view;
  w.k = (uint16_t *)c->k;
  w.v = (uint16_t *)c->v;
  w.layers = c->layers;
  w.pages = c->num_pages;
  w.hkv = c->num_kv_heads;
  w.d = c->head_dim;
  w.page = c->page;
  w.page_shift = __builtin_ctz((unsigned)c->page);
  w.slots = c->num_slots;
  w.max_pages = c->max_pages;
  w.words = (c->num_pages + 63) / 64;
  w.state = c->meta;
  w.used = (unsigned long long *)(c->meta + 8);
  w.len = c->meta + 8 + 2 * (size_t)w.words;
  w.ref = w.len + w.slots;
  w.table = w.ref + w.pages;
  return FP_OK;
}

// Workspace of reserve and compact: the number of copies, their pages, and every page's new
// number.
size_t copies_layout(const fp_cache *c, char *base, fp::PageCopies *w) {
  const size_t list = align_up(4 * (size_t)c->num_pages);
  if (w) {
    w->count = (int32_t *)base;
    w->src = (int32_t *)(base + kAlign);
    w->dst = (int32_t *)(base + kAlign + list);
    w->renamed = (int32_t *)(base + kAlign + 2 * list);
  }
  return kAlign + 3 * list;
}

// Slot numbers of one call, distinct and in range; `seen` holds the slots so far.  Only the words
// that the cache's slots need are cleared: these calls are made several times a layer.
struct SlotSet {
  uint64_t bits[65536 / 64];
  explicit SlotSet(const fp_cache *c) { memset(bits, 0, ((size_t)c->num_slots + 63) / 64 * 8); }
  bool add(int32_t s) {
    const uint64_t bit = (uint64_t)1 << (s & 63);
    const bool fresh = !(bits[s >> 6] & bit);
    bits[s >> 6] |= bit;
    return fresh;
  }
  bool has(int32_t s) const { return bits[s >> 6] >> (s & 63) & 1; }
};

fp_status check_slots(const fp_cache *c, int32_t n, const int32_t *slots, SlotSet *seen) {
  if (n < 1 || !slots) return FP_ERR_INVALID_ARG;
  if (n > FP_MAX_CACHE_LIST) return FP_ERR_UNSUPPORTED;
  for (int i = 0; i < n; ++i) {
    if (slots[i] < 0 || slots[i] >= c->num_slots) return FP_ERR_INVALID_ARG;
    if (seen && !seen->add(slots[i])) return FP_ERR_INVALID_ARG;
  }
  return FP_OK;
}

// Units of a decoding batch: query rows, tiles of kDecodeRows rows, workspace.
struct DecodeDims {
  int G;                       // query heads per KV head
  int rows;                    // rows of a sequence and KV head
  int tile_rows, tiles;        // their row tiles
  bool many, few;              // some group has a prefix to share, with that many rows
  size_t bytes_many, bytes_few, bytes_own;   // workspace: partial results
  size_t bytes() const {
    return align_up(sizeof(fp::DecodeJoin)) + bytes_many + bytes_few + bytes_own;
  }
};

fp_status check_decode(const fp_cache *c, const fp_decode *b, DecodeDims *dm) {
  const fp_status st = check_cache(c, nullptr);
  if (st != FP_OK) return st;
  if (!b || !b->slots || b->batch < 1 || b->num_q_heads < 1 || b->queries < 1 || b->groups < 0)
    return FP_ERR_INVALID_ARG;
  if (b->num_q_heads % c->num_kv_heads) return FP_ERR_INVALID_ARG;
  if (b->batch > FP_MAX_CACHE_LIST || b->queries > FP_MAX_QUERIES || b->num_q_heads > 8192)
    return FP_ERR_UNSUPPORTED;
  if (!scale_ok(b->softmax_scale)) return FP_ERR_INVALID_ARG;
  for (int i = 0; i < b->batch; ++i)
    if (b->slots[i] < -1 || b->slots[i] >= c->num_slots) return FP_ERR_INVALID_ARG;
  dm->G = b->num_q_heads / c->num_kv_heads;
  dm->rows = dm->G * b->queries;
  dm->tile_rows = dm->rows > 16 ? 32 : 16;
  dm->many = dm->few = false;
  // cost of all key ranges, in tiles of 64 keys: an int32 in the kernels
  const int64_t most = ((int64_t)c->max_pages * c->page + 63) / 64;
  int64_t cost = 0;
  if (b->groups > 0) {
    if (!b->group_start || !b->prefix_lens || b->groups > b->batch) return FP_ERR_INVALID_ARG;
    if (b->group_start[0] != 0 || b->group_start[b->groups] != b->batch)
      return FP_ERR_INVALID_ARG;
    for (int g = 0; g < b->groups; ++g) {
      const int m = b->group_start[g + 1] - b->group_start[g];
      if (m < 1 || m > b->batch || b->prefix_lens[g] < 0) return FP_ERR_INVALID_ARG;
      if (m > 1 && b->prefix_lens[g] > 0) {
        (m * dm->rows > fp::kDecodeFew ? dm->many : dm->few) = true;
        if (m * dm->rows > 16 && m * dm->rows <= fp::kDecodeFew) dm->tile_rows = 32;
        cost += ((int64_t)m * dm->rows / 16 + 1) *
                (std::min(most, ((int64_t)b->prefix_lens[g] + 63) / 64) + 8);
      }
    }
  }
  dm->tiles = (dm->rows + dm->tile_rows - 1) / dm->tile_rows;
  cost += (int64_t)b->batch * dm->tiles * (most + 8);   // 8: more than a segment's fixed cost
  if (cost * c->num_kv_heads > 0x7FFFFFFF) return FP_ERR_UNSUPPORTED;
  const size_t wgs = fp::decode_wgs(c->head_dim), row = 4 * (size_t)(c->head_dim + 2);
  const size_t own = wgs + (size_t)b->batch * c->num_kv_heads * dm->tiles;
  dm->bytes_own = align_up(own * dm->tile_rows * row);
  // a group's row tiles start at (its first row) / (rows of a tile) + its number
  auto prefixes = [&](bool any, int tile) -> size_t {
    if (!any) return 0;
    const size_t tiles = (size_t)b->batch * dm->rows / tile + b->groups + 1;
    return align_up((wgs + c->num_kv_heads * tiles) * tile * row);
  };
  dm->bytes_few = prefixes(dm->few, dm->tile_rows);
  dm->bytes_many = prefixes(dm->many, fp::kDecodeRows);
  return FP_OK;
}

fp_status hip_fail(hipError_t e, const char *what) {
  snprintf(g_last_error, sizeof(g_last_error), "%s: %s", what, hipGetErrorString(e));
  return FP_ERR_HIP;
}

}  // namespace

extern "C" {

fp_status fp_indices_size(const fp_shape *shape, size_t *kb_idx_elems, size_t *kb_cnt_elems) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  if (!kb_idx_elems || !kb_cnt_elems) return FP_ERR_INVALID_ARG;
  *kb_idx_elems = (size_t)(dm.tri_total * shape->num_q_heads);
  *kb_cnt_elems = (size_t)(dm.nb_total * shape->num_q_heads);
  return FP_OK;
}

fp_status fp_select_workspace_size(const fp_shape *shape, const fp_params *params,
                                   size_t *bytes) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  if (!params || !bytes) return FP_ERR_INVALID_ARG;
  if ((st = check_params(shape, params)) != FP_OK) return st;
  *bytes = params->gamma >= 1.f ? 0 : select_layout(shape, dm, nullptr, nullptr);
  return FP_OK;
}

fp_status fp_attn_workspace_size(const fp_shape *shape, size_t *bytes) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  if (!bytes) return FP_ERR_INVALID_ARG;
  *bytes = attn_layout(shape, dm);
  return FP_OK;
}

fp_status fp_attn_workspace_preferred(const fp_shape *shape, size_t *bytes) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  if (!bytes) return FP_ERR_INVALID_ARG;
  fp::SplitArgs sp;
  const size_t base = attn_layout(shape, dm);
  *bytes = base + plan_split(dm.st, shape->num_q_heads, shape->num_kv_heads, shape->head_dim,
                             shape->block, base, nullptr, 0, &sp);
  return FP_OK;
}

fp_status fp_validate(const fp_shape *shape, const fp_params *params, size_t ws_bytes) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  if (params) {
    if ((st = check_params(shape, params)) != FP_OK) return st;
    const size_t need = params->gamma >= 1.f ? 0 : select_layout(shape, dm, nullptr, nullptr);
    if (ws_bytes < need) return FP_ERR_WORKSPACE;
  } else {
    if (ws_bytes < attn_layout(shape, dm)) return FP_ERR_WORKSPACE;
  }
  return FP_OK;
}

fp_status fp_select(const fp_shape *shape, const void *q, const void *k, const fp_params *params,
                    fp_indices *out, void *ws, size_t ws_bytes, void *stream) {
  fp_status st = fp_validate(shape, params, ws_bytes);
  if (st != FP_OK) return st;
  if (!q || !k || !out || !out->kb_idx || !out->kb_cnt || !out->pattern || !out->js ||
      !out->units)
    return FP_ERR_INVALID_ARG;
  Dims dm;
  check_shape(shape, &dm);
  fp::SelectArgs a;
  memset(&a, 0, sizeof(a));
  a.st = dm.st;
  a.q = (const uint16_t *)q;
  a.k = (const uint16_t *)k;
  a.hq = shape->num_q_heads;
  a.hkv = shape->num_kv_heads;
  a.d = shape->head_dim;
  a.block = shape->block;
  a.total_tokens = (int32_t)dm.total_tokens;
  a.nb_total = (int32_t)dm.nb_total;
  a.tri_total = dm.tri_total;
  a.scale = resolved_scale(params->softmax_scale, shape->head_dim);
  a.gamma = params->gamma;
  a.tau = params->tau;
  a.min_budget = params->min_budget_blocks;
  a.force_pattern = params->force_pattern;
  a.max_budget = params->max_budget_blocks;
  a.qa_mode = params->qa_mode;
  a.vs_granularity = params->vs_granularity;
  a.kb_idx = out->kb_idx;
  a.kb_cnt = out->kb_cnt;
  a.pattern = out->pattern;
  a.js = out->js;
  a.units = out->units;
  out->softmax_scale = a.scale;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (params->gamma >= 1.f) {
    e = fp::launch_dense_lists(a, s);
    return e == hipSuccess ? FP_OK : hip_fail(e, "fp_select(dense)");
  }
  if (!ws) return FP_ERR_INVALID_ARG;
  select_layout(shape, dm, (char *)ws, &a);
  e = fp::launch_select_pipeline(a, s);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_select");
}

fp_status fp_sparse_attn(const fp_shape *shape, const void *q, const void *k, const void *v,
                         const fp_indices *idx, void *o, void *ws, size_t ws_bytes,
                         void *stream) {
  fp_status st = fp_validate(shape, nullptr, ws_bytes);
  if (st != FP_OK) return st;
  if (!q || !k || !v || !o || !idx || !idx->kb_idx || !idx->kb_cnt || !ws)
    return FP_ERR_INVALID_ARG;
  if (!scale_ok(idx->softmax_scale)) return FP_ERR_INVALID_ARG;
  Dims dm;
  check_shape(shape, &dm);
  fp::AttnArgs a;
  memset(&a, 0, sizeof(a));
  a.st = dm.st;
  a.q = (const uint16_t *)q;
  a.k = (const uint16_t *)k;
  a.v = (const uint16_t *)v;
  a.o = (uint16_t *)o;
  a.kb_idx = idx->kb_idx;
  a.kb_cnt = idx->kb_cnt;
  a.hq = shape->num_q_heads;
  a.hkv = shape->num_kv_heads;
  a.d = shape->head_dim;
  a.block = shape->block;
  a.nb_total = (int32_t)dm.nb_total;
  a.tri_total = dm.tri_total;
  a.scale_log2 = resolved_scale(idx->softmax_scale, shape->head_dim) * 1.4426950408889634f;
  a.items = (int4 *)ws;
  a.queue = (int32_t *)((char *)ws + align_up(16 * dm.nb_total * shape->num_q_heads));
  a.vt = (uint16_t *)((char *)a.queue + align_up(8 * sizeof(int32_t)));
  a.sort_keys = (unsigned long long *)((char *)a.vt +
                                       align_up(2 * (size_t)dm.nb_total * shape->num_kv_heads *
                                                shape->block * shape->head_dim));
  a.sort_recs = (int4 *)((char *)a.sort_keys + align_up(8 * dm.nb_total * shape->num_q_heads));
  const size_t base = attn_layout(shape, dm);
  plan_split(dm.st, a.hq, a.hkv, a.d, a.block, base, (char *)ws + base, ws_bytes - base,
             &a.split);
  hipError_t e = fp::launch_sparse_attn(a, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_sparse_attn");
}

fp_status fp_sparse_attn_noalloc(const fp_shape *shape, const void *q, const void *k,
                                 const void *v, const fp_indices *idx, void *o, void *stream) {
  Dims dm;
  fp_status st = check_shape(shape, &dm);
  if (st != FP_OK) return st;
  const size_t need = attn_layout(shape, dm);
  if (need > (size_t)FP_NOALLOC_SCRATCH_BYTES) {
    snprintf(g_last_error, sizeof(g_last_error),
             "fp_sparse_attn_noalloc: the problem needs %zu workspace bytes, more than the "
             "fixed scratch of %zu",
             need, (size_t)FP_NOALLOC_SCRATCH_BYTES);
    return FP_ERR_WORKSPACE;
  }
  if (!q || !k || !v || !o || !idx || !idx->kb_idx || !idx->kb_cnt) return FP_ERR_INVALID_ARG;
  if (!scale_ok(idx->softmax_scale)) return FP_ERR_INVALID_ARG;
  void *ws = nullptr;
  const hipError_t e = fp::noalloc_scratch(&ws);
  if (e != hipSuccess) return hip_fail(e, "fp_sparse_attn_noalloc(scratch)");
  return fp_sparse_attn(shape, q, k, v, idx, o, ws, (size_t)FP_NOALLOC_SCRATCH_BYTES, stream);
}

fp_status fp_cache_meta_size(const fp_cache *cache, size_t *elems) {
  const fp_status st = check_cache(cache, nullptr);
  if (st != FP_OK) return st;
  if (!elems) return FP_ERR_INVALID_ARG;
  *elems = 8 + 2 * (((size_t)cache->num_pages + 63) / 64) + (size_t)cache->num_slots +
           (size_t)cache->num_pages + (size_t)cache->num_slots * cache->max_pages;
  return FP_OK;
}

fp_status fp_cache_workspace_size(const fp_cache *cache, size_t *bytes) {
  const fp_status st = check_cache(cache, nullptr);
  if (st != FP_OK) return st;
  if (!bytes) return FP_ERR_INVALID_ARG;
  *bytes = copies_layout(cache, nullptr, nullptr);
  return FP_OK;
}

fp_status fp_cache_init(const fp_cache *cache, void *stream) {
  fp::CacheView c;
  const fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  const hipError_t e = fp::launch_cache_init(c, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_init");
}

fp_status fp_cache_reserve(const fp_cache *cache, int32_t n, const int32_t *slots,
                           const int32_t *counts, void *ws, size_t ws_bytes, void *stream) {
  fp::CacheView c;
  fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  SlotSet seen(cache);
  if ((st = check_slots(cache, n, slots, &seen)) != FP_OK) return st;
  if (!counts) return FP_ERR_INVALID_ARG;
  fp::CacheList l;
  l.n = n;
  for (int i = 0; i < n; ++i) {
    if (counts[i] < 0) return FP_ERR_INVALID_ARG;
    l.slot[i] = slots[i];
    l.num[i] = counts[i];
  }
  if (!ws || !aligned4(ws)) return FP_ERR_INVALID_ARG;
  if (ws_bytes < copies_layout(cache, nullptr, nullptr)) return FP_ERR_WORKSPACE;
  fp::PageCopies w;
  copies_layout(cache, (char *)ws, &w);
  const hipError_t e = fp::launch_cache_reserve(c, l, w, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_reserve");
}

fp_status fp_cache_write(const fp_cache *cache, int32_t layer, int32_t n, const int32_t *slots,
                         const int32_t *cu, const void *k, int64_t k_stride, const void *v,
                         int64_t v_stride, void *stream) {
  fp::CacheView c;
  fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  SlotSet seen(cache);
  if ((st = check_slots(cache, n, slots, &seen)) != FP_OK) return st;
  if (layer < 0 || layer >= cache->layers || !cu || cu[0] != 0) return FP_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cache->num_kv_heads * cache->head_dim;
  fp::WriteArgs a;
  a.list.n = n;
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t m = (int64_t)cu[i + 1] - cu[i];
    if (m < 0) return FP_ERR_INVALID_ARG;
    a.list.slot[i] = slots[i];
    a.list.num[i] = cu[i];
    a.blk[i] = (int32_t)blocks;
    if (m > 0) blocks += (m + 62) / 64 + 1;   // 64-token blocks that m tokens can touch
  }
  if (cu[n] == 0) return FP_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v) || k_stride < row || v_stride < row ||
      k_stride % 8 || v_stride % 8)
    return FP_ERR_INVALID_ARG;
  if (blocks * cache->num_kv_heads >= (1 << 24)) return FP_ERR_UNSUPPORTED;   // grid size
  a.list.num[n] = cu[n];
  a.blk[n] = (int32_t)blocks;
  a.k = (const uint16_t *)k;
  a.v = (const uint16_t *)v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.layer = layer;
  const hipError_t e = fp::launch_cache_write(c, a, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_write");
}

fp_status fp_cache_fork(const fp_cache *cache, int32_t n, const int32_t *src, const int32_t *dst,
                        void *stream) {
  fp::CacheView c;
  fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  SlotSet seen(cache);
  if ((st = check_slots(cache, n, dst, &seen)) != FP_OK) return st;
  if ((st = check_slots(cache, n, src, nullptr)) != FP_OK) return st;
  fp::ForkArgs a;
  a.n = n;
  for (int i = 0; i < n; ++i) {
    if (seen.has(src[i])) return FP_ERR_INVALID_ARG;
    a.src[i] = src[i];
    a.dst[i] = dst[i];
  }
  const hipError_t e = fp::launch_cache_fork(c, a, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_fork");
}

fp_status fp_cache_truncate(const fp_cache *cache, int32_t n, const int32_t *slots,
                            const int32_t *lens, void *stream) {
  fp::CacheView c;
  fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  SlotSet seen(cache);
  if ((st = check_slots(cache, n, slots, &seen)) != FP_OK) return st;
  fp::CacheList l;
  l.n = n;
  for (int i = 0; i < n; ++i) {
    if (lens && lens[i] < 0) return FP_ERR_INVALID_ARG;
    l.slot[i] = slots[i];
    l.num[i] = lens ? lens[i] : 0;
  }
  const hipError_t e = fp::launch_cache_truncate(c, l, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_truncate");
}

fp_status fp_cache_compact(const fp_cache *cache, void *ws, size_t ws_bytes, void *stream) {
  fp::CacheView c;
  const fp_status st = check_cache(cache, &c);
  if (st != FP_OK) return st;
  if (!ws || !aligned4(ws)) return FP_ERR_INVALID_ARG;
  if (ws_bytes < copies_layout(cache, nullptr, nullptr)) return FP_ERR_WORKSPACE;
  fp::PageCopies w;
  copies_layout(cache, (char *)ws, &w);
  const hipError_t e = fp::launch_cache_compact(c, w, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_cache_compact");
}

fp_status fp_decode_workspace_size(const fp_cache *cache, const fp_decode *batch,
                                   size_t *bytes) {
  DecodeDims dm;
  const fp_status st = check_decode(cache, batch, &dm);
  if (st != FP_OK) return st;
  if (!bytes) return FP_ERR_INVALID_ARG;
  *bytes = dm.bytes();
  return FP_OK;
}

fp_status fp_decode_attn(const fp_cache *cache, const fp_decode *batch, int32_t layer,
                         const void *q, int64_t q_stride, void *o, void *ws, size_t ws_bytes,
                         void *stream) {
  DecodeDims dm;
  fp_status st = check_decode(cache, batch, &dm);
  if (st != FP_OK) return st;
  fp::CacheView c;
  if ((st = check_cache(cache, &c)) != FP_OK) return st;
  if (layer < 0 || layer >= cache->layers || !q || !o || !ws || !aligned16(q) || !aligned16(o) ||
      !aligned16(ws))
    return FP_ERR_INVALID_ARG;
  if (q_stride < (int64_t)batch->num_q_heads * c.d || q_stride % 8) return FP_ERR_INVALID_ARG;
  if (ws_bytes < dm.bytes()) return FP_ERR_WORKSPACE;
  fp::DecodeArgs a;
  memset(&a, 0, sizeof(a));
  const int64_t pool = (int64_t)layer * c.pages * c.hkv * c.page * c.d;
  a.k = c.k + pool;
  a.v = c.v + pool;
  a.len = c.len;
  a.table = c.table;
  a.q = (const uint16_t *)q;
  a.o = (uint16_t *)o;
  a.q_stride = q_stride;
  a.join = (fp::DecodeJoin *)ws;
  char *part = (char *)ws + align_up(sizeof(fp::DecodeJoin));
  a.part_many = (float *)part;
  a.part_few = (float *)(part + dm.bytes_many);
  a.part_own = (float *)(part + dm.bytes_many + dm.bytes_few);
  a.any_prefix = dm.many || dm.few;
  a.any_many = dm.many;
  a.tile_rows = dm.tile_rows;
  a.tile_shift = dm.tile_rows == 32 ? 5 : 4;
  a.pages = c.pages;
  a.hkv = c.hkv;
  a.page_shift = c.page_shift;
  a.max_pages = c.max_pages;
  a.G = dm.G;
  a.hq = batch->num_q_heads;
  a.nq = batch->queries;
  a.batch = batch->batch;
  a.wgs = fp::decode_wgs(c.d);
  a.scale_log2 = resolved_scale(batch->softmax_scale, c.d) * 1.4426950408889634f;
  for (int i = 0; i < batch->batch; ++i) a.slot[i] = batch->slots[i];
  if (batch->groups > 0) {
    a.groups = batch->groups;
    for (int g = 0; g < batch->groups; ++g) {
      a.start[g] = (int16_t)batch->group_start[g];
      a.prefix[g] = batch->prefix_lens[g];
      for (int i = batch->group_start[g]; i < batch->group_start[g + 1]; ++i)
        a.group[i] = (uint8_t)g;
    }
  } else {
    a.groups = 1;              // one group with nothing shared
  }
  a.start[a.groups] = (int16_t)batch->batch;
  const hipError_t e = fp::launch_decode_attn(a, c.d, (hipStream_t)stream);
  return e == hipSuccess ? FP_OK : hip_fail(e, "fp_decode_attn");
}

const char *fp_status_string(fp_status status) {
  switch (status) {
    case FP_OK: return "FP_OK";
    case FP_ERR_INVALID_ARG: return "FP_ERR_INVALID_ARG: invalid argument";
    case FP_ERR_UNSUPPORTED: return "FP_ERR_UNSUPPORTED: configuration not supported";
    case FP_ERR_WORKSPACE: return "FP_ERR_WORKSPACE: workspace too small";
    case FP_ERR_HIP: return "FP_ERR_HIP: HIP runtime error";
  }
  return "unknown fp_status";
}

const char *fp_last_error(void) { return g_last_error; }

}  // extern "C"
