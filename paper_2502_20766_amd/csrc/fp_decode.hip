// Attention of the next tokens over a paged cache: o = softmax(c q K^T) V for the last
// `queries` tokens of every sequence of a batch, with the keys and values that a group of
// sequences shares at its start read once for the whole group.
//
// Split softmax: over a range R of keys, with reference m and weights w_j = exp2(s_j - m),
//   O_R = sum w_j v_j,  l_R = sum w_j;   o = (sum_R 2^(m_R - M) O_R) / (sum_R 2^(m_R - M) l_R).
// The ranges are cut as follows.  A segment is the work of one KV head and one tile of query
// rows over one run of keys: the prefix of a group (rows: all query heads of the KV head, all
// queries, all sequences of the group) or the rest of one sequence (rows: its own).  Segments,
// one after the other in tiles of 64 keys, form a line that is cut into equal parts, one for
// each workgroup, so every workgroup has the same work whatever the lengths.  A piece (the part
// of a segment in one workgroup) leaves O_R, m_R and l_R in float32; a last launch joins the
// pieces of each row in the order of the line.  A segment in one piece whose rows have no
// prefix is finished on the spot. Where the cuts fall follows from the lengths alone, so
// results do not depend on timing.
//
// Segments with few rows are bound by the bytes of their keys, prefixes with many by their
// products, so there are two ways to take a piece (lean_pieces, many_pieces) and two lines.
// One launch takes both: the resident workgroups are divided between the lines by their work,
// so that neither waits for the other.  Workgroups that take the row tiles of one prefix go
// through the same keys side by side (a cluster), so that those come from memory once.
#include <type_traits>

#include "fp_attn_dev.h"
#include "fp_internal.h"
#include "fp_paged_dev.h"

namespace fp {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxList = FP_MAX_CACHE_LIST;
// Places of the line, beside its tiles, that a segment takes: starting and ending a piece costs
// a workgroup about as much as this many tiles.  At 1, 2, 3, 4: 64 sequences of 3 to 32000 tokens
// 90.2, 86.8, 87.4, 88.2 us; 16 samples of 32k 41.2, 40.0, 40.6, 41.0; 256 samples of 128k 588, 574,
// 579, 586; 60 sequences of 60k with four queries at head dim 64 327, 306, 308, 305.
constexpr int kSegCost = 2;

static_assert(kThreads == kMaxList, "the plan has one thread per sequence");

// Entries of the lean line: group g is entry g, sequence b is kOwn + b.
constexpr int kOwn = kMaxList, kEnd = 2 * kMaxList;

// The lines of a call.  Starts are the places where the segments of a group's prefix and of a
// sequence's own keys begin; an entry without keys has the start of the next one.
struct Plan {
  int len[kMaxList];                      // tokens of a sequence (0: no sequence)
  int prefix[kMaxList];                   // per group: keys read once, a multiple of 16
  int lead[kMaxList];                     // per group: a sequence whose pages hold them
  int live[kMaxList];
  int many[kMaxList + 1];                 // line of many rows: groups, the end
  int lean[2 * kMaxList + 1];             // the other: groups, sequences (from kOwn), the end
  int scan[3][4];
  int rows_lo, rows_hi;                   // fewest and most row tiles of a group of many rows
  int first;                              // entry that this workgroup's part begins in
};

__device__ __forceinline__ int tiles_of(int keys) { return (keys + kKeys - 1) / kKeys; }

__device__ __forceinline__ int group_rows(const DecodeArgs &a, int g) {
  return (a.start[g + 1] - a.start[g]) * a.nq * a.G;
}

// Groups whose prefix is taken as one of many rows.
__device__ __forceinline__ bool is_many(const DecodeArgs &a, int g) {
  return group_rows(a, g) > kDecodeFew;
}

// Row tiles: of kDecodeRows rows for prefixes of many, of a.tile_rows (16 or 32) else.
__device__ __forceinline__ int many_tiles(int rows) {
  return (rows + kDecodeRows - 1) / kDecodeRows;
}
__device__ __forceinline__ int lean_tiles(const DecodeArgs &a, int rows) {
  return (rows + a.tile_rows - 1) >> a.tile_shift;
}

// Number of the partial result of row tile 0 and KV head 0 of a prefix, less its workgroup's: a
// group's row tiles start at (its first row) / (rows of a tile) + its number, which leaves each
// group as many as it has.
__device__ __forceinline__ int prefix_base(const DecodeArgs &a, int g, bool many) {
  const int first = a.start[g] * a.nq * a.G;
  return ((many ? first / kDecodeRows : first >> a.tile_shift) + g) * a.hkv;
}

// A line of `total` places in `wgs` equal parts, the first total % wgs of them one place
// longer.
struct Cut {
  int per, rem;
  __device__ __forceinline__ Cut(int total, int wgs) : per(total / wgs), rem(total % wgs) {}
  __device__ __forceinline__ int begin(int w) const { return per * w + min(w, rem); }
  __device__ __forceinline__ int owner(int x) const {
    const int longer = rem * (per + 1);
    return x < longer ? x / (per + 1) : rem + (x - longer) / per;
  }
};

// Inclusive prefix sum over the wave: within rows of 16 lanes, then the rows' sums handed on.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 to rows 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31 to rows 2, 3
  return x;
}

// Least x of the wave, in every lane.
__device__ __forceinline__ int wave_min(int x) {
  constexpr int none = 0x7FFFFFFF;
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));   // row_shr 1
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));   // row_bcast 15
  x = min(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));   // row_bcast 31
  return __builtin_amdgcn_readlane(x, 63);
}

// How the workgroups are divided: `clusters` times `width` of them take the line of many rows,
// a cluster one part of it and each of its workgroups one row tile; `lean` the other line.
struct Shares {
  int clusters, width, lean;
};

// This workgroup's part of its line.
struct Part {
  int many;             // which line
  int lo, hi;           // places; lo == hi: none
  int wg;               // number of the part
  int tile;             // many: row tile, when the cluster has one for each
};

// What a place of the lean line counts against one of the other: more than one where products
// bound the prefixes (several row tiles), less where their bytes do.
// Several row tiles, at 0.8, 1, 1.2, 1.4, 1.6: 256 samples of 128k 578, 575, 563, 569, 571 us; 60
// sequences of 60k with four queries at head dim 64 327, 328, 303, 304, 303; 100 samples of 60k
// (best) 154, 137, 139, 141, 142.
// One, at 0.6, 0.7, 0.8, 0.9, 1, 1.2: 16 samples of 32k 42.4, 41.1, 40.5, 40.2, 40.5, 41.4; drafts
// at head dim 64 51.7, 47.9, 47.9, 47.6, 48.6, 48.4; 20 sequences of 10k and 500 to 6000 of their
// own 45.8, 44.3, 43.6, 44.6, 45.2, 49.0.
constexpr float kLeanProducts = 1.2f, kLeanBytes = 0.85f;

// Work of the lines (`many` per row tile) in shares of a.wgs workgroups.
__device__ __forceinline__ Shares divide(int wgs, int many, int width, int lean,
                                         float lean_cost) {
  Shares r = {0, width, 0};
  if (many > 0) {
    const float work = (float)many * width;
    const int most = (wgs - (lean > 0 ? 1 : 0)) / width;
    r.clusters = (int)((float)wgs / width * (work / (work + lean_cost * lean)) + 0.5f);
    // two places at least to a part, so that short prefixes leave fewer pieces: 4 sequences of 20k
    // that share 64 rows 28.7 -> 23.1 us; three places: 20.7, but others 10% more
    r.clusters = max(1, min(min(r.clusters, most), many / 2));
  }
  r.lean = min(wgs - r.clusters * width, lean);
  return r;
}

// Fills the plan and finds this workgroup's part and the entry it begins in.
__device__ __forceinline__ Part make_plan(const DecodeArgs &a, Plan &p) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int len = 0, g = 0;
  int rows = 0, want = 0;                 // of group t; read with the rest, before any barrier
  if (a.any_prefix && t < a.groups) {
    rows = group_rows(a, t);
    want = a.prefix[t];
  }
  if (t < a.batch) {
    g = a.group[t];
    if (a.slot[t] >= 0) len = min(max(a.len[a.slot[t]], 0), a.max_pages << a.page_shift);
    p.len[t] = len;
  }
  int cost[3] = {0, 0, 0};                // groups of many rows, of few, own keys
  int width = 1, keys = 0;
  float lean_cost = kLeanProducts;
  if (a.any_prefix) {
    if (t < a.groups) {
      p.prefix[t] = 0x7FFFFFFF;
      p.lead[t] = kMaxList - 1;
      p.live[t] = 0;
    }
    if (t == 0) {
      p.rows_lo = 0x7FFFFFFF;
      p.rows_hi = 0;
    }
    __syncthreads();
    const unsigned long long any = __ballot(len > 0);
    if (any) {
      // a wave whose sequences are all of one group takes their least length by lane moves
      const int lead = __builtin_ctzll(any), g0 = __builtin_amdgcn_readlane(g, lead);
      if (__ballot(len > 0 && g != g0)) {
        if (len > 0) {
          atomicMin(&p.prefix[g], max(len - a.nq, 0));
          atomicMin(&p.lead[g], t);
          atomicAdd(&p.live[g], 1);
        }
      } else {
        const int least = wave_min(len > 0 ? max(len - a.nq, 0) : 0x7FFFFFFF);
        if (lane == lead) {
          atomicMin(&p.prefix[g], least);
          atomicMin(&p.lead[g], t);
          atomicAdd(&p.live[g], __popcll(any));
        }
      }
    }
    __syncthreads();
    int tiles = 0;
    // one sequence alone has nothing to share
    if (t < a.groups && p.live[t] >= 2) keys = min(p.prefix[t], want) & ~15;
    if (keys > 0) {
      const bool many = rows > kDecodeFew;
      tiles = many ? many_tiles(rows) : lean_tiles(a, rows);
      cost[many ? 0 : 1] = a.hkv * (tiles_of(keys) + kSegCost);
      if (many) {
        atomicMin(&p.rows_lo, tiles);
        atomicMax(&p.rows_hi, tiles);
      }
    }
    if (t < a.groups) p.prefix[t] = keys;
    __syncthreads();
    // a cluster per part where all prefixes have the same number of row tiles
    if (p.rows_lo == p.rows_hi && p.rows_hi <= a.wgs / 4) width = p.rows_hi;
    else cost[0] *= tiles;
    if (p.rows_hi <= 1) lean_cost = kLeanBytes;
    cost[1] *= tiles;
  } else if (t < a.groups) {
    p.prefix[t] = 0;
  }
  if (len > 0)
    cost[2] = a.hkv * lean_tiles(a, a.G * a.nq) *
              (tiles_of(len - (a.any_prefix ? p.prefix[g] : 0)) + kSegCost);
  int start[3], total[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    start[i] = wave_scan(cost[i]);
    if (lane == 63) p.scan[i][w] = start[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    start[i] -= cost[i];
    total[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < w) start[i] += p.scan[i][j];
      total[i] += p.scan[i][j];
    }
  }
  start[2] += total[1];
  p.many[t] = start[0];
  p.lean[t] = start[1];
  p.lean[kOwn + t] = start[2];
  const int places = total[1] + total[2];
  if (t == 0) {
    p.many[kMaxList] = total[0];
    p.lean[kEnd] = places;
  }
  const Shares sh = divide(a.wgs, total[0], width, places, lean_cost);
  // Workgroups of one XCD (every eighth) take neighbouring parts, which share keys, unless
  // there is not work for all.
  const int crowd = sh.clusters * sh.width, used = crowd + sh.lean;
  int wg = blockIdx.x;
  if (8 * used > 7 * a.wgs) wg = (wg & 7) * (a.wgs / 8) + (wg >> 3);
  Part r = {wg < crowd, 0, 0, 0, 0};
  if (r.many) {
    r.wg = wg / sh.width;
    r.tile = wg - r.wg * sh.width;
    const Cut cut(total[0], sh.clusters);
    r.lo = cut.begin(r.wg);
    r.hi = cut.begin(r.wg + 1);
    if (start[0] <= r.lo && r.lo < start[0] + cost[0]) p.first = t;
  } else if (wg < used) {
    r.wg = wg - crowd;
    const Cut cut(places, sh.lean);
    r.lo = cut.begin(r.wg);
    r.hi = cut.begin(r.wg + 1);
    if (start[1] <= r.lo && r.lo < start[1] + cost[1]) p.first = t;
    if (start[2] <= r.lo && r.lo < start[2] + cost[2]) p.first = kOwn + t;
  }
  __syncthreads();
  if (blockIdx.x == 0) {                  // what the joining launch needs of this
    DecodeJoin &j = *a.join;
    if (t < a.batch) {
      const int prefix = len > 0 ? p.prefix[g] : 0;
      const bool many = is_many(a, g);
      j.seq[t] = make_int4(len, prefix, start[2], many ? p.many[g] : p.lean[g]);
      j.group[t] = make_int4(g, a.start[g], group_rows(a, g), many);
    }
    if (t == 0) {
      j.places_many = total[0];
      j.places_lean = places;
      j.clusters = sh.clusters;
      j.width = sh.width;
      j.lean = sh.lean;
    }
  }
  r.many = __builtin_amdgcn_readfirstlane(r.many);
  r.lo = __builtin_amdgcn_readfirstlane(r.lo);
  r.hi = __builtin_amdgcn_readfirstlane(r.hi);
  r.wg = __builtin_amdgcn_readfirstlane(r.wg);
  r.tile = sh.width > 1 ? __builtin_amdgcn_readfirstlane(r.tile) : -1;
  return r;
}

// A run of tiles of one segment in one workgroup; every field is wave-uniform.
struct Piece {
  int entry;            // of the plan
  int end;              // place of the line where the segment ends
  int row;              // cache slot whose pages are read
  int head;             // KV head
  int t0, t1;           // tiles [t0, t1); t0 == t1: none
  int key0, limit;      // the segment's keys: first, and first one past
  int row0, rows;       // rows of this row tile: row0 .. row0 + rows - 1 of the segment's
  int token0;           // query token of the segment's first row
  int vis;              // keys that the first query of a sequence sees
  int slot;             // partial result
  int whole;            // the piece is all that its rows have
  int once;             // one row tile: no other workgroup reads these keys
};

// The piece at place x of the workgroup's part, which lies in entry `e` or a later one.
template <bool MANY>
__device__ __forceinline__ Piece piece_at(const DecodeArgs &a, const Plan &p, int e, int x,
                                          const Part &part) {
  const int *starts = MANY ? p.many : p.lean;
  while (starts[e + 1] <= x)
    if (++e == a.groups && !MANY) e = kOwn;   // (the entries between are empty)
  Piece r;
  r.entry = __builtin_amdgcn_readfirstlane(e);
  const bool shared = MANY || r.entry < kOwn;
  const int b = r.entry - kOwn;
  const int g = shared ? r.entry : a.group[b];
  const int prefix = __builtin_amdgcn_readfirstlane(p.prefix[g]);
  int rows, base, whole = 0;
  const int per = MANY ? kDecodeRows : a.tile_rows;
  if (shared) {
    r.row = a.slot[__builtin_amdgcn_readfirstlane(p.lead[g])];
    r.key0 = 0;
    r.limit = r.vis = prefix;
    rows = group_rows(a, g);
    r.token0 = a.start[g] * a.nq;
    base = prefix_base(a, g, MANY);
  } else {
    r.row = a.slot[b];
    r.key0 = prefix;
    r.limit = __builtin_amdgcn_readfirstlane(p.len[b]);
    r.vis = r.limit - a.nq + 1;
    rows = a.G * a.nq;
    r.token0 = b * a.nq;
    base = b * a.hkv * lean_tiles(a, rows);
    whole = prefix == 0;
  }
  const bool cluster = MANY && part.tile >= 0;
  const int tiles = cluster ? 1 : MANY ? many_tiles(rows) : lean_tiles(a, rows);
  const int n = tiles_of(r.limit - r.key0);
  const int start = __builtin_amdgcn_readfirstlane(starts[r.entry]);
  const int seg = (x - start) / (n + kSegCost);         // (KV head, row tile) of the entry
  const int at = start + seg * (n + kSegCost) + kSegCost;   // place of its first tile
  r.once = rows <= per;
  r.head = tiles == 1 ? seg : seg / tiles;
  r.row0 = (cluster ? part.tile : seg - r.head * tiles) * per;
  r.rows = min(rows - r.row0, per);
  r.t0 = max(x - at, 0);
  r.t1 = max(min(part.hi - at, n), r.t0);
  r.end = at + n;
  // (a cluster's row tiles are as many as its workgroups)
  r.slot = cluster ? (part.wg + seg) * many_tiles(rows) + part.tile + base : part.wg + base + seg;
  r.whole = whole && r.t0 == 0 && r.t1 == n;
  return r;
}

// A weight as the sum of two bf16 numbers, both above zero if it is: both multiply the same value,
// and an infinite one would meet a zero or the other sign in a second number that is what rounding
// the first one left.  So the first is the largest bf16 number below the weight; the second, up to
// 2^-7 of it, is rounded to 2^-9 of itself.
__device__ __forceinline__ void split_weight(float w, __bf16 &top, __bf16 &low) {
  const uint32_t below = __builtin_elementwise_sub_sat(__float_as_uint(w), 1u) & 0xFFFF0000u;
  top = __builtin_bit_cast(__bf16, (uint16_t)(below >> 16));
  low = (__bf16)(w - __uint_as_float(below));
}

// Largest x, and sum, over the four lanes that share lane % 16.
__device__ __forceinline__ float quad_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return wave_pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return wave_pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// ---- few rows: RT tiles of 16 query rows.  The four waves of a workgroup take 16 keys each of
// every tile and need each other only at the end of a piece, where their results are joined in
// LDS.  Per wave and step, on v_mfma_f32_16x16x32_bf16:
//   S^T (16 keys x 16 rows) = K Q^T, D / 32 products; lane (row r = lane % 16, g = lane / 16) holds
//   the scores of keys 4 g .. 4 g + 3;
//   O^T += V^T P^T, D / 16 products.  The 32 places of a product's inner dimension are the 16 keys
//   twice: a weight is the sum of two bf16 numbers (error 2^-16, see split_weight), the second one in
//   places where V^T is repeated.  That costs no product, and the keys' bytes bound the kernel anyway.
// Measured: 64 sequences of 3 to 32000 tokens, 32 query and 8 KV heads of 128, 507 MB of keys
// and values in 83 us, 6.1 TB/s (a copy of 1 GiB moves 5.3); pages of 16 and of 64 tokens the
// same.  With 32-row products instead (one wave 32 keys, weights in one piece, joined in pairs)
// the same bytes took 189 us.  256 sequences of 100 tokens, two tiles a segment: 27 us for 105
// MB.
template <int D, int RT>
__device__ __forceinline__ void lean_pieces(const DecodeArgs &a, const Plan &plan, uint8_t *lds0,
                                            uint8_t *lds1, float2 (*s_ml)[16],
                                            const Part &part) {
  using S = PagedGeo<D>;
  constexpr int KS = D / 32, DB = D / 16;
  // K and V of wave w's even (0) or odd steps; at the end of a piece the last one holds the
  // wave's O (16 x D floats)
  auto lds = [&](int w, int odd) { return (odd ? lds1 : lds0) + w * 2 * S::STEP; };
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int r16 = lane & 15, g4 = lane >> 4;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  const Loader<D> load(w, lane);
  uint32_t kaddr[KS];                     // this lane's K fragments: key r16, chunks 4 k + g4
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = r16 * S::RB + swz_k<D>(4 * k + g4, r16) * 16;
  const uint32_t vaddr = S::STEP + 16 * vt_unit(r16, g4 >> 1) + 8 * (g4 & 1);

  Piece cur = piece_at<false>(a, plan, plan.first, part.lo, part);
  if (cur.t0 == cur.t1) return;           // the part ends before the segment's first tile
  int buf = 0;
  load.issue(a, cur, cur.t0, load.page(a, cur, cur.t0), lds(w, 0), lds(w, 0) + S::STEP);
  int page_next = load.page(a, cur, min(cur.t0 + 1, cur.t1 - 1));
  while (true) {
    // ---- this lane's rows (16 i + r16), their queries and how many keys they see
    bf16x8 qf[RT][KS];
    int lim[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int srow = cur.row0 + min(16 * i + r16, cur.rows - 1);
      const int tok = srow / a.G;
      lim[i] = cur.entry < kOwn ? cur.limit : cur.vis + tok;
      const uint16_t *qp = a.q + (int64_t)(cur.token0 + tok) * a.q_stride +
                           (cur.head * a.G + srow - tok * a.G) * D + 8 * g4;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[i][k] = *reinterpret_cast<const bf16x8 *>(qp + 32 * k);
    }
    // the next piece, if this part of the line goes on past the segment
    Piece nxt;
    nxt.t0 = nxt.t1 = 0;
    int page_piece = 0;
    if (cur.end < part.hi) {
      nxt = piece_at<false>(a, plan, cur.entry, cur.end, part);
      page_piece = load.page(a, nxt, nxt.t0);
    }
    const bool more = nxt.t0 < nxt.t1;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(qf[i][k]));
    f32x4 oacc[RT][DB];
    float m_ref[RT], mc[RT], m_trig[RT], l_run[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[i][db] = f32x4{};
      m_ref[i] = m_trig[i] = -INFINITY;
      mc[i] = l_run[i] = 0.f;
    }

    for (int t = cur.t0; t < cur.t1; ++t) {
      wait_copies();                      // this wave's keys are here
      uint8_t *next = lds(w, buf ^ 1);
      if (t + 1 < cur.t1) {
        load.issue(a, cur, t + 1, page_next, next, next + S::STEP);
        page_next = load.page(a, cur, min(t + 2, cur.t1 - 1));
      } else if (more) {
        load.issue(a, nxt, nxt.t0, page_piece, next, next + S::STEP);
        page_next = load.page(a, nxt, min(nxt.t0 + 1, nxt.t1 - 1));
      }
      uint8_t *step = lds(w, buf);
      buf ^= 1;
      const int k0 = cur.key0 + kKeys * t + 16 * w;
      if (k0 >= cur.limit) continue;
      const bool edge = k0 + 16 > cur.vis;
      bool odd = false;
      if (edge) odd = settle<D>(step + S::STEP, k0, cur.limit, cur.vis, lane);
      bf16x8 kf[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[k] = *reinterpret_cast<const bf16x8 *>(step + kaddr[k]);
      bf16x8 pf[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        f32x4 s = f32x4{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k], qf[i][k], s, 0, 0, 0);
        // (On every step: with a branch for the steps off the edges the times are the same, 4 short
        // sequences 0.5 us more.)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = k0 + 4 * g4 + e < lim[i] ? s[e] : -INFINITY;
        const float mt = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        // the reference moves only when a score rises 2^kLazy above it in weight
        if (__ballot(mt > m_trig[i])) {
          const float m_new = fmaxf(m_ref[i], quad_max(mt));
          const float f =
              m_ref[i] == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref[i] - m_new) * c);
          l_run[i] *= f;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[i][db] *= f;
          m_ref[i] = m_new;
          const bool none = m_new == -INFINITY;
          mc[i] = none ? 0.f : m_new * c;
          m_trig[i] = none ? -INFINITY : m_new + lazy_raw;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float wt = __builtin_amdgcn_exp2f(fmaf(s[e], c, -mc[i]));
          __bf16 top, low;
          split_weight(wt, top, low);
          pf[i][e] = top;
          pf[i][4 + e] = low;
        }
        const bf16x8 pair[1] = {pf[i]};
        l_run[i] = sum_weights(pair, l_run[i]);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(step + vaddr + 512 * db);
        const bf16x8 vf = __builtin_shufflevector(v, v, 0, 1, 2, 3, 0, 1, 2, 3);
#pragma unroll
        for (int i = 0; i < RT; ++i)
          oacc[i][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[i], oacc[i][db], 0, 0, 0);
      }
      if (odd) {                          // the values that settle took out
        for (int key = max(cur.vis, k0); key < min(cur.limit, k0 + 16); ++key) {
          const int pg = min(max(a.table[(int64_t)cur.row * a.max_pages + (key >> a.page_shift)],
                                 0), a.pages - 1);
          const uint16_t *vp =
              a.v + ((((int64_t)pg * a.hkv + cur.head) << a.page_shift) +
                     (key & ((1 << a.page_shift) - 1) & ~15)) * D + (key & 15) + 64 * g4;
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            float wt = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (k0 + 4 * g4 + e == key) wt = (float)pf[i][e] + (float)pf[i][4 + e];
            wt = quad_sum(wt);
            if (key >= lim[i]) continue;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t x = vp[16 * (16 * db + e)];
                if ((x & 0x7F80) == 0x7F80)
                  oacc[i][db][e] = fmaf(wt, __uint_as_float(x << 16), oacc[i][db][e]);
              }
          }
        }
      }
    }

    // ---- the waves' results joined: each leaves O in its last step's LDS, 16-byte chunks of a row
    // swizzled by the row; thread (row tid / 16, i = tid % 16) sums chunks i, i + 16
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      if (16 * i >= cur.rows) break;
      if (i) wg_barrier();
      float *box = reinterpret_cast<float *>(lds(w, buf ^ 1));
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<f32x4 *>(box + r16 * D + 4 * ((4 * db + g4) ^ r16)) = oacc[i][db];
      const float l = quad_sum(l_run[i]);
      if (g4 == 0) s_ml[w][r16] = make_float2(m_ref[i], l);
      wg_barrier();
      const int row = tid >> 4, ch = tid & 15;
      if (16 * i + row < cur.rows) {
        float2 ml[4];
        float m = -INFINITY, l_tot = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          ml[j] = s_ml[j][row];
          m = fmaxf(m, ml[j].x);
        }
        f32x4 sum[D / 64];
#pragma unroll
        for (int q = 0; q < D / 64; ++q) sum[q] = f32x4{};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f = ml[j].y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml[j].x - m) * c);
          l_tot = fmaf(f, ml[j].y, l_tot);
          const float *from = reinterpret_cast<const float *>(lds(j, buf ^ 1)) + row * D;
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(from + 4 * ((ch + 16 * q) ^ row));
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[q][e] = fmaf(f, x[e], sum[q][e]);
          }
        }
        const int srow = cur.row0 + 16 * i + row;
        if (cur.whole) {
          const int tok = srow / a.G;
          const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
          uint16_t *op = a.o + ((int64_t)(cur.token0 + tok) * a.hq + cur.head * a.G + srow -
                                tok * a.G) * D + 4 * ch;
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (__bf16)(sum[q][e] * inv);
            *reinterpret_cast<bf16x4 *>(op + 64 * q) = o;
          }
        } else {
          float *to = (cur.entry < kOwn ? a.part_few : a.part_own) +
                      (int64_t)cur.slot * a.tile_rows * (D + 2);
          const int at = 16 * i + row;
          if (ch == 0)
            *reinterpret_cast<float2 *>(to + a.tile_rows * D + 2 * at) = make_float2(m, l_tot);
#pragma unroll
          for (int q = 0; q < D / 64; ++q)
            *reinterpret_cast<f32x4 *>(to + at * D + 4 * ch + 64 * q) = sum[q];
        }
      }
    }
    if (!more) return;
    wg_barrier();                         // read before the next copy arrives there
    cur = nxt;
  }
}

// ---- many rows: tiles of 128, 32 per wave.  The 64 keys of a tile go through LDS (double
// buffered, each wave bringing 16) and are read by all four waves; the products are those of
// the prefill, on v_mfma_f32_32x32x16_bf16: S^T = K Q^T with K rows permuted so that a lane's
// scores are the consecutive keys that P^T of O^T += V^T P^T needs, one update of the reference
// for 64 keys.  A weight is one bf16 number, as there, its error 2^-8 in O and in the sum alike;
// the error of the result, 1.6e-3 in norm against 64 bits, is that of its rounding all the same.  Two
// numbers would be half as many products again: 40.3 -> 40.8 us for 64 rows (16 samples of 32k), where
// the keys' bytes bound most of it, 48.2 -> 53.4 for 96 rows (drafts at head dim 64).
// All rows see all keys of a prefix. Measured: 256 samples of a 131072-token prompt, 32
// query and 8 KV heads of 128, 550 GFLOP in 535 to 570 us (by the clock that the power limit
// leaves), 1.03 to 0.96 PFLOP/s where a product of 8192^3 reaches 1.34: the matrix pipe is busy
// 55% of cycles, the vector unit 40%, at 1.7 GHz.  With 64 rows (16 samples of 32k, two of the
// waves idle) 30 to 35 us for 141 MB that come from memory, of which the plan and the first tile
// are 8.
template <int D>
__device__ __forceinline__ void many_pieces(const DecodeArgs &a, const Plan &plan, uint8_t *lds0,
                                            uint8_t *lds1, const Part &part) {
  using S = PagedGeo<D>;
  constexpr int KS = D / 16, DB = D / 32, TILE = 4 * S::STEP;
  // K and V of even tiles in lds0, of odd ones in lds1
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  const Loader<D> load(w, lane);
  auto issue = [&](const Piece &r, int t, int pg, uint8_t *into) {
    uint8_t *k = into + w * S::STEP;
    load.issue(a, r, t, pg, k, k + TILE);
  };
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;
  const uint32_t vaddr = TILE + 16 * vt_unit(lr, lh);

  Piece cur = piece_at<true>(a, plan, plan.first, part.lo, part);
  if (cur.t0 == cur.t1) return;
  // Of the two workgroups of a CU at head dim 128 the one started first is served first, and ended
  // 10% before the other, whose work is as long.  The second (the grid's second half: the first
  // fills every CU once) is put ahead in two of four tiles, except in clusters, which go at the
  // pace of all: 16 samples of 32k 40.8 -> 40.0 us; with clusters too 256 samples of 128k take 574
  // instead of 553, 100 of 60k 147 instead of 143.  Three workgroups at head dim 64: no difference.
  const bool second = D == 128 && part.tile < 0 && 2 * (int)blockIdx.x >= a.wgs;
  int odd = 0;
  issue(cur, cur.t0, load.page(a, cur, cur.t0), lds0);
  int page_next = load.page(a, cur, min(cur.t0 + 1, cur.t1 - 1));
  while (true) {
    const bool active = 32 * w < cur.rows;
    const int row = 32 * w + lr;
    const int srow = cur.row0 + min(row, cur.rows - 1);
    const int tok = srow / a.G;
    const uint16_t *qp = a.q + (int64_t)(cur.token0 + tok) * a.q_stride +
                         (cur.head * a.G + srow - tok * a.G) * D + 8 * lh;
    bf16x8 qf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const bf16x8 *>(qp + 16 * k);
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(qf[k]));
    f32x16 oacc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) oacc[i] = f32x16{};
    float m_ref = -INFINITY, mc = 0.f, m_trig = -INFINITY, l_run = 0.f;
    Piece nxt;
    nxt.t0 = nxt.t1 = 0;
    if (cur.end < part.hi) nxt = piece_at<true>(a, plan, cur.entry, cur.end, part);
    const bool more = nxt.t0 < nxt.t1;

    auto step = [&](uint8_t *tile, uint8_t *next, const int t) {
      const int k0 = cur.key0 + kKeys * t;
      if (second && (t & 2)) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
      wait_copies();                                     // this wave's part of tile t is here
      const bool edge = k0 + kKeys > cur.limit;
      if (edge)
        settle<D>(tile + TILE + w * S::STEP, k0 + 16 * w, cur.limit, cur.limit, lane);
      wg_barrier();                                      // ... and every wave's
      if (t + 1 < cur.t1) {
        issue(cur, t + 1, page_next, next);
        page_next = load.page(a, cur, min(t + 2, cur.t1 - 1));
      } else if (more) {
        issue(nxt, nxt.t0, load.page(a, nxt, nxt.t0), next);
        page_next = load.page(a, nxt, min(nxt.t0 + 1, nxt.t1 - 1));
      }
      if (!active) return;
      f32x16 sacc[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        bf16x8 kf[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k)
          kf[k] = *reinterpret_cast<const bf16x8 *>(tile + kaddr[k] + b * 32 * S::RB);
        sacc[b] = f32x16{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
          sacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[k], sacc[b], 0, 0, 0);
      }
      if (edge) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (k0 + 32 * b + 16 * (v >> 3) + 8 * lh + (v & 7) >= cur.limit)
              sacc[b][v] = -INFINITY;
      }
      float mt = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sacc[b][v]);
      if (__ballot(mt > m_trig)) {
        const float m_new = fmaxf(m_ref, wave_pair_max(mt));
        const float f = m_ref == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        l_run *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) oacc[i] *= f;
        m_ref = m_new;
        const bool none = m_new == -INFINITY;
        mc = none ? 0.f : m_new * c;
        m_trig = none ? -INFINITY : m_new + lazy_raw;
      }
      bf16x8 pf[4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          pf[2 * b + (v >> 3)][v & 7] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sacc[b][v], c, -mc));
      l_run = sum_weights(pf, l_run);
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const bf16x8 vf =
              *reinterpret_cast<const bf16x8 *>(tile + vaddr + db * 1024 + t4 * S::STEP);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t4], oacc[db], 0, 0, 0);
        }
    };
    // (in pairs: a branch on the buffer in every step would move O from register to register)
    int t = cur.t0;
    if (odd) step(lds1, lds0, t++);
    for (; t + 2 <= cur.t1; t += 2) {
      step(lds0, lds1, t);
      step(lds1, lds0, t + 1);
    }
    odd = t < cur.t1;
    if (odd) step(lds0, lds1, t);

    // ---- lane holds row `row`, d = 32 db + 8 (v / 4) + 4 lh + v % 4
    const float l = wave_pair_sum(l_run);
    if (row < cur.rows) {
      float *to = a.part_many + (int64_t)cur.slot * kDecodeRows * (D + 2);
      if (lh == 0)
        *reinterpret_cast<float2 *>(to + kDecodeRows * D + 2 * row) = make_float2(m_ref, l);
      to += row * D + 4 * lh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4 *>(to + 32 * db + 8 * g) =
              make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2],
                          oacc[db][4 * g + 3]);
    }
    if (!more) return;
    cur = nxt;
  }
}

// RT: row tiles of 16 of a piece with few rows.  MANY: the batch may have prefixes with many.
template <int D, int RT, bool MANY>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(PagedGeo<D>::OCC, PagedGeo<D>::OCC)))
void decode_fwd(DecodeArgs a) {
  // two arrays, so that the compiler sees that reads of one do not wait for copies into the
  // other
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[8 * PagedGeo<D>::STEP];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[8 * PagedGeo<D>::STEP];
  __shared__ Plan plan;
  __shared__ float2 s_ml[4][16];
  const Part part = make_plan(a, plan);
  if (part.lo == part.hi) return;
  if (MANY && part.many) many_pieces<D>(a, plan, lds0, lds1, part);
  else lean_pieces<D, RT>(a, plan, lds0, lds1, s_ml, part);
}

// ---- Joins the pieces of a row: WPR waves, each with every 64 / (D / 4) * WPR-th group of pieces,
// D / 4 lanes to a piece, 16 bytes each, four loads in flight (two: 13.2 us instead of 10.2 for
// 1024 rows of 65 pieces; eight: the same there, 12.0 instead of 10.0 for 6144 rows of 12).
// Latency bound up to a few hundred rows (4.4 us for 32), then by the bytes of the pieces, which
// are read once: as ordinary loads the call with 16 samples of 32k takes 46.0 us, as these 44.3,
// drafts at head dim 64 54.4 and 53.3.  (Nontemporal stores of the pieces: 45.1 and 54.6 in a row,
// 3 us more for a call by itself.)  128 references at once instead of 64, eight waves a row: the same.
template <int D, int WPR>
__global__ __launch_bounds__(kThreads) void decode_join(DecodeArgs a) {
  constexpr int LPP = D / 4;              // lanes per piece
  constexpr int PPW = 64 / LPP;           // pieces at once in a wave
  __shared__ f32x4 s_sum[4][LPP];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, part = w % WPR;
  const int64_t id = (int64_t)blockIdx.x * (4 / WPR) + w / WPR;
  if (WPR == 1 && id >= (int64_t)a.batch * a.nq * a.hq) return;
  const int token = (int)(id / a.hq), qh = (int)(id - (int64_t)token * a.hq);
  const int b = token / a.nq, t = token - b * a.nq, head = qh / a.G, kk = qh - head * a.G;
  const DecodeJoin &j = *a.join;
  const int4 seq = j.seq[b];              // tokens, prefix, places of own keys and of the prefix
  const int4 grp = j.group[b];            // group, its first sequence, its rows, whether many
  const int len = seq.x, prefix = seq.y;
  uint16_t *op = a.o + id * D;
  const float c = a.scale_log2;
  // pieces of the row's two segments: its own keys (1) and the prefix (0)
  int count[2] = {0, 0}, stride[2] = {0, 0}, ml_at[2] = {0, 0};
  const float *from[2] = {a.part_own, a.part_own};
  if (len > 0) {
    const int per = a.tile_rows, r = t * a.G + kk, row = r & (per - 1);
    const int tiles = lean_tiles(a, a.G * a.nq), n = tiles_of(len - prefix);
    const int seg = head * tiles + (r >> a.tile_shift);
    const int at = seq.z + seg * (n + kSegCost) + kSegCost;
    const Cut cut(j.places_lean, j.lean);
    const int first = cut.owner(at);
    count[1] = cut.owner(at + n - 1) - first + 1;
    stride[1] = per * (D + 2);
    ml_at[1] = per * D + 2 * row - row * D;
    from[1] = a.part_own + (int64_t)(first + b * a.hkv * tiles + seg) * stride[1] + row * D;
  }
  if (prefix > 0) {
    const int g = grp.x, many = grp.w;
    const int per = many ? kDecodeRows : a.tile_rows, width = many ? j.width : 1;
    const int r = ((b - grp.y) * a.nq + t) * a.G + kk;
    const int tile = many ? r / kDecodeRows : r >> a.tile_shift, row = r & (per - 1);
    const int tiles = width > 1 ? 1 : many ? many_tiles(grp.z) : lean_tiles(a, grp.z);
    const int n = tiles_of(prefix);
    const int seg = head * tiles + (width > 1 ? 0 : tile);
    const int at = seq.w + seg * (n + kSegCost) + kSegCost;
    const Cut cut(many ? j.places_many : j.places_lean, many ? j.clusters : j.lean);
    const int first = cut.owner(at);
    count[0] = cut.owner(at + n - 1) - first + 1;
    stride[0] = width * per * (D + 2);
    ml_at[0] = per * D + 2 * row - row * D;
    const int slot = (first + seg) * width + (width > 1 ? tile : 0) + prefix_base(a, g, many);
    from[0] = (many ? a.part_many : a.part_few) + (int64_t)slot * per * (D + 2) + row * D;
  }
  const int n = count[0] + count[1];
  if (prefix == 0 && n == 1) return;      // finished by its workgroup
  auto piece = [&](int i) {
    return i < count[0] ? from[0] + (int64_t)i * stride[0]
                        : from[1] + (int64_t)(i - count[0]) * stride[1];
  };
  float m = -INFINITY, l = 0.f;
  f32x4 acc = f32x4{};
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int k = min(64, n - i0);
    constexpr int U = 4;                  // loads in flight
    f32x4 x[U];
    auto fetch = [&](int i) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(
            piece(i0 + min(i + u * WPR * PPW + lane / LPP, k - 1)) + 4 * (lane % LPP)));
    };
    fetch(part * PPW);                    // beside the references, not after them
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < k)
      ml = *reinterpret_cast<const float2 *>(piece(i0 + lane) +
                                             ml_at[i0 + lane < count[0] ? 0 : 1]);
    float top = fmaxf(m, ml.x);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float old = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
    // (a sum of 0: no key seen; a NaN has to come through, whatever its reference)
    const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml.x - top) * c);
    float sum = f * ml.y;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    l = l * old + sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= old;
    m = top;
    for (int i = part * PPW; i < k; i += U * WPR * PPW) {
      float fi[U];
      if (i != part * PPW) fetch(i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = i + u * WPR * PPW + lane / LPP;
        fi[u] = __shfl(f, at & 63);       // (by all lanes)
        if (at >= k) fi[u] = 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (fi[u] != 0.f) acc[e] = fmaf(fi[u], x[u][e], acc[e]);
    }
  }
#pragma unroll
  for (int d = LPP; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
  if constexpr (WPR > 1) {
    if (lane < LPP) s_sum[w][lane] = acc;
    __syncthreads();
    if (part != 0) return;
    if (lane < LPP) {
      acc = f32x4{};
#pragma unroll
      for (int i = 0; i < WPR; ++i) acc += s_sum[w + i][lane];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < LPP) {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4 *>(op + 4 * lane) = o;
  }
}

template <int D>
hipError_t launch(const DecodeArgs &a, hipStream_t s) {
  if (a.any_many && a.tile_rows == 16) decode_fwd<D, 1, true><<<a.wgs, kThreads, 0, s>>>(a);
  else if (a.any_many) decode_fwd<D, 2, true><<<a.wgs, kThreads, 0, s>>>(a);
  else if (a.tile_rows == 16) decode_fwd<D, 1, false><<<a.wgs, kThreads, 0, s>>>(a);
  else decode_fwd<D, 2, false><<<a.wgs, kThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // four waves a row while there are few: 512 rows of 66 pieces 7.8 us, one wave each 9.4; 2048
  // rows of up to 20 pieces 8.8 and 6.1
  const int rows = a.batch * a.nq * a.hq;
  if (rows <= 512) decode_join<D, 4><<<rows, kThreads, 0, s>>>(a);
  else decode_join<D, 1><<<(rows + 3) / 4, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_attn(const DecodeArgs &a, int d, hipStream_t s) {
  return d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace fp
