// Causal attention of chunks of new tokens over a paged cache: o = softmax(c q K^T) V, where query t of
// m of a sequence of n tokens sees its keys 0 .. n - m + t.
//
// The rows of a sequence and KV head are its queries times the query heads of that KV head, a token's
// heads one after the other, in tiles of 128 rows: keys are so read once for all heads that share
// them, and few of a tile's rows end within another key tile than its last one.  Tiles of 64 keys go
// through LDS, double buffered; a wave has 32 rows, and its products are those of the prefill, on
// v_mfma_f32_32x32x16_bf16: S^T = K Q^T with K rows permuted so that a lane's scores are the
// consecutive keys that P^T of O^T += V^T P^T needs, one update of the reference for 64 keys.
//
// How the work is divided.  Row tiles of about equal length, or short ones, are not cut: a workgroup has
// one with all of its keys, the longest ones of a sequence first.  Else a segment is a.width row tiles of
// one sequence and KV head that lie side by side, with the keys that the last of them sees.  Segments, one
// after the other, form a line whose places are rows of keys; it is cut into equal parts, one for each
// cluster of a.width workgroups, each of which takes one of the row tiles.  The workgroups of a cluster go
// through the same keys at the same time, so those come from memory, and mostly from the XCD's L2, once.
// A piece (a part's share of a segment) that is not all of it leaves O, its reference and its sum in
// float32, and a last launch joins the pieces of a row in the order of the line.  All of it follows from
// the lengths alone, so results do not depend on timing.
//
// The weights that multiply the values are rounded to one bf16 number, 2^-8, in O and in the sum alike: against
// 64 bits the result is off by 1.65e-3 in norm, with weights in float32 by 1.64e-3, since it is rounded to bf16
// itself.  A second number for what the first leaves (as for the few rows of decode_attn) would be half as
// many products again.
//
// Bounds: products and softmax for chunks (4096 tokens after 127k, 32 heads of 128: 8.0 ms, 1.09 PFLOP/s, at
// the clock of the power limit; four whole prompts of 1001-9001 tokens, 64 heads of 64: 630 us), memory for
// single tokens (43 of them beside five chunks, over up to 20k tokens: 289 us, 3.2 TB/s), latency for short
// ones (three of up to 112 tokens: 10.7 us).
#include <algorithm>
#include <type_traits>

#include "fp_attn_dev.h"
#include "fp_chunk_plan.h"
#include "fp_internal.h"
#include "fp_paged_dev.h"

namespace fp {
namespace {

constexpr int kJoinThreads = 256;

// A score that is the reference of its row has a weight of 2^-kBelow.  No weight is then above 2^-26, and
// those of the 2^26 tokens that a slot holds at most do not sum to more than 1: sums of the largest values of
// their type stay within float32 until they are divided.  The smallest normal bf16 number is 2^-92 of the
// reference's weight: keys that count less than that are lost.
constexpr float kBelow = kLazy + 26.f;

// Row tiles are not cut where the longest sequence has at most so many key tiles more than SHARES times a
// workgroup's equal share of all of them (two, one for row tiles of 256): the device then hands out whole
// row tiles, and whoever is done first takes the next.  Four whole prompts at head dim 64 720 -> 664 us, 59
// chunks over 500 tokens 30 -> 22; but 8 sequences of 20 tiles 22 -> 29, 48 of which one has 300 285 -> 459.
// (With 1 in place of 2: 41 sequences of 20 tiles 39 us instead of 35.)  Of 256: a prompt of 20000 tokens
// 3425 -> 3319; with 2 in place of 1 2048 tokens after 30001 857 -> 888, 12 prompts on a small rank 69 -> 82.
constexpr int kWholeTiles = 14;

// The line: places where the segments of a sequence begin, in (key, query head) pairs: a key tile is 64 G
// places, so that the places of a sequence's segments are an arithmetic series.
struct Plan {
  int64_t start[kMaxList + 1];
  int64_t scan[kMaxList / 64];
  int tiles[kMaxList / 64], longest[kMaxList / 64];
  int len[kMaxList];                      // tokens of a sequence (0: no slot)
  int64_t lo, hi;                         // this workgroup's part
  Segment first;                          // the segment that its uncut start lies in
};

// Inclusive prefix sum over the wave: within rows of 16 lanes, then the rows' sums handed on.
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  auto add = [&](auto ctrl, auto rows, auto zero) {
    constexpr int c = decltype(ctrl)::value, m = decltype(rows)::value;
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)x, c, m, 0xf, decltype(zero)::value);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), c, m, 0xf, decltype(zero)::value);
    x += (int64_t)(((uint64_t)hi << 32) | lo);
  };
  using std::integral_constant;
  typedef integral_constant<int, 0xf> All;
  add(integral_constant<int, 0x111>{}, All{}, std::true_type{});          // row_shr 1
  add(integral_constant<int, 0x112>{}, All{}, std::true_type{});
  add(integral_constant<int, 0x114>{}, All{}, std::true_type{});
  add(integral_constant<int, 0x118>{}, All{}, std::true_type{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}, std::false_type{});  // row_bcast 15
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}, std::false_type{});  // row_bcast 31
  return x;
}

// Inclusive prefix sum over the wave, or the largest value in its last lane.
template <bool MAX>
__device__ __forceinline__ int wave_fold(int x) {
  auto step = [&](auto ctrl, auto rows) {
    const int y = __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xf,
                                              false);
    x = MAX ? max(x, y) : x + y;
  };
  using std::integral_constant;
  typedef integral_constant<int, 0xf> All;
  step(integral_constant<int, 0x111>{}, All{});
  step(integral_constant<int, 0x112>{}, All{});
  step(integral_constant<int, 0x114>{}, All{});
  step(integral_constant<int, 0x118>{}, All{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return x;
}

// Fills the plan and finds this workgroup's part.  That may be one row tile with all of its
// keys, of which the device then starts as many as there are, one after the other; `parts` is 0.
template <class G, int SHARES>
__device__ __forceinline__ Part make_plan(const ChunkArgs &a, Plan &plan, int &parts) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int len = 0, m = 0;
  if (t < a.batch) {
    const int slot = a.slot[t];
    m = a.cu[t + 1] - a.cu[t];
    if (slot >= 0) len = min(max(a.len[slot], 0), a.max_pages << a.page_shift);
  }
  if (t < kMaxList) plan.len[t] = len;
  const Series<G> series(a, a.width, m, len);
  const int64_t whole = series.whole(), cost = whole * a.hkv;
  const int64_t sum = wave_scan(cost);
  if (lane == 63 && w < kMaxList / 64) plan.scan[w] = sum;
  const int tiles = (int)((uint32_t)(m * a.G + G::ROWS - 1) / G::ROWS);
  const int tiles_sum = wave_fold<false>(tiles);
  const int longest_here = wave_fold<true>(m > 0 ? (len + G::KEYS - 1) / G::KEYS : 0);
  if (lane == 63 && w < kMaxList / 64) {
    plan.tiles[w] = tiles_sum;
    plan.longest[w] = longest_here;
  }
  __syncthreads();
  int64_t start = sum - cost, total = 0;
#pragma unroll
  for (int j = 0; j < kMaxList / 64; ++j) {
    if (j < w) start += plan.scan[j];
    total += plan.scan[j];
  }
  Part r;
  r.width = a.width;
  int first = tiles_sum - tiles, longest = 0;
  for (int j = 0; j < kMaxList / 64; ++j) {
    if (j < w) first += plan.tiles[j];
    longest = max(longest, plan.longest[j]);
  }
  // (in float: all workgroups compute the same)
  if (a.tiles > 0 &&
      longest - kWholeTiles <=
          SHARES * ((float)total * a.width / ((float)(G::KEYS * a.G) * a.wgs))) {
    const int tile = blockIdx.x / a.hkv, head = blockIdx.x - tile * a.hkv;
    if (t == 0) plan.hi = 0;
    __syncthreads();
    if (first <= tile && tile < first + tiles) {     // the last ones, which see most, before the others
      plan.first = {t, head, tiles - 1 - (tile - first), 0, INT64_MAX};
      plan.hi = INT64_MAX;
    }
    __syncthreads();
    parts = 0;
    r.p = blockIdx.x;
    r.tile = 0;
    r.width = 1;
    r.lo = 0;
    r.hi = plan.hi;
    return r;
  }
  if (t < kMaxList) plan.start[t] = start;
  if (t == 0) plan.start[kMaxList] = total;
  parts = parts_of<G>(a, total);
  r = place_of(a, blockIdx.x, parts);
  if (r.p < parts) {
    const Cut cut(total, parts);
    // its two ends, each by the thread of the sequence that it lies in
    for (int i = 0; i < 2; ++i) {
      const int64_t at = cut.begin(r.p + i);
      if (at >= total) {
        if (t == 0) plan.hi = total;
      } else if (start <= at && at < start + cost) {
        const Segment s = segment_at(series, whole, t, start, at);
        (i ? plan.hi : plan.lo) = snap<G>(a, at, s.start, s.end);
        if (i == 0) plan.first = s;
      }
    }
  }
  __syncthreads();
  if (r.p < parts) {
    r.lo = plan.lo;
    r.hi = plan.hi;
  }
  return r;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// The segment after `s`, which is not the line's last.
template <class G>
__device__ __forceinline__ Segment after(const ChunkArgs &a, const Plan &plan, const Segment &s) {
  Segment r = {s.seq, s.head, s.seg + 1, s.end, 0};
  Series<G> series(a, a.width, a.cu[s.seq + 1] - a.cu[s.seq], uniform(plan.len[s.seq]));
  if (r.seg == series.n) {
    r.seg = 0;
    if (++r.head == a.hkv) {
      r.head = 0;
      while (uniform(plan.start[r.seq + 1]) <= r.start) ++r.seq;
      series = Series<G>(a, a.width, a.cu[r.seq + 1] - a.cu[r.seq], uniform(plan.len[r.seq]));
    }
  }
  r.end = r.start + series.end(r.seg) - series.begin(r.seg);
  return r;
}

// What the join needs: of a segment that goes on in later parts, how many pieces it has and its first part.
// With `by_segment` there is a record for every segment, from the part that it begins in, else one for
// every part, of the segment that begins in it and goes on.
template <class G>
__device__ __forceinline__ void record(const ChunkArgs &a, const Plan &plan, const Part &part, int parts,
                                       const Piece &p, bool last) {
  const int pieces = pieces_of<G>(a, plan.start[kMaxList], parts, part, p);
  const int4 rec = make_int4(pieces | part.p << 16, p.s.seq, p.s.head, p.s.seg);
  if (a.by_segment) {
    if (p.here && p.begins) a.seg[record_of<G>(a, p)] = rec;
  } else if (last) {
    a.seg[part.p] = rec;
  }
}

// Scores of keys that a row does not see, among N blocks of 32: -infinity from key `room` on.  (The least
// of a score and + or - infinity: comparisons would take as many scalar registers as there are.)
template <int N>
__device__ __forceinline__ void mask(f32x16 *s, int room) {
  const float end = (float)room - 0.5f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      s[i][v] = fminf(s[i][v], (end - (32 * i + 16 * (v >> 3) + (v & 7))) * INFINITY);
}

// Values among keys [key, end) that are not finite, times their weights, into O of the rows that see
// them.  `qp`: the lane's half of its row's query.
template <int D>
__device__ __forceinline__ void late_values(const ChunkArgs &a, const Source &src, int key, int end,
                                            int lim, const uint16_t *qp, float c, float mc, int lh,
                                            f32x16 (&oacc)[D / 32]) {
  for (; key < end; ++key) {
    const int pg =
        min(max(a.table[(int64_t)src.row * a.max_pages + (key >> a.page_shift)], 0), a.pages - 1);
    const int64_t head = (((int64_t)pg * a.hkv + src.head) << a.page_shift) * D;
    const int in = key & ((1 << a.page_shift) - 1);
    const uint16_t *kp = a.k + head + in * D + 8 * lh, *vp = a.v + head + (in & ~15) * D + (in & 15);
    float s = 0.f;
    for (int d = 0; d < D; d += 16)
      for (int e = 0; e < 8; ++e)
        s = fmaf(__uint_as_float((uint32_t)qp[d + e] << 16), __uint_as_float((uint32_t)kp[d + e] << 16),
                 s);
    s = wave_pair_sum(s);
    const float wt = (float)(__bf16)__builtin_amdgcn_exp2f(fmaf(s, c, -mc));
    if (key >= lim) continue;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const uint32_t x = vp[16 * (32 * db + 8 * (v >> 2) + 4 * lh + (v & 3))];
        if ((x & 0x7F80) == 0x7F80) oacc[db][v] = fmaf(wt, __uint_as_float(x << 16), oacc[db][v]);
      }
  }
}

// The rows of a lane: to their place in o (`out`, a row of [d]), divided by the sum, or to the partial
// result `part`.  The lane holds d = 32 db + 8 (v / 4) + 4 lh + v % 4 of row `row` of the tile.
template <int D>
__device__ __forceinline__ void finish(const ChunkArgs &a, bool whole, bool any,
                                       const f32x16 (&oacc)[D / 32], float m_ref, float l, float *part,
                                       int row, int lh, int64_t out) {
  if (whole) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *op = a.o + out * D + 4 * lh;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (__bf16)(oacc[db][4 * g + e] * inv);
        *reinterpret_cast<bf16x4 *>(op + 32 * db + 8 * g) = o;
      }
    return;
  }
  if (lh == 0) *reinterpret_cast<float2 *>(part + a.tile_rows * D + 2 * row) = make_float2(m_ref, l);
  part += row * D + 4 * lh;
  if (any) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4 *>(part + 32 * db + 8 * g) =
            make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2],
                        oacc[db][4 * g + 3]);
  }
}

// ---- Row tiles of 128: four waves of 32 rows, several workgroups to a CU.
template <int D>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(PagedGeo<D>::OCC, PagedGeo<D>::OCC)))
void chunk_fwd(ChunkArgs a) {
  using S = PagedGeo<D>;
  using G = Geo<4, kKeys>;
  constexpr int KS = D / 16, DB = D / 32, TILE = 4 * S::STEP;
  // K and V of even tiles in lds0, of odd ones in lds1: two arrays, so that the compiler sees that
  // reads of one do not wait for copies into the other
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[2 * TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[2 * TILE];
  __shared__ Plan plan;
  // the piece at hand, each wave's own copy: what is looked at after its tiles would else take scalar
  // registers meanwhile
  __shared__ Piece s_piece[4];
  __shared__ int s_odd[2];                // piece with late values that are not finite, by its parity
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  if (tid < 2) s_odd[tid] = 0;
  int parts;
  const Part part = make_plan<G, 2>(a, plan, parts);
  const bool keeps = parts > 0 && part.tile == 0 && tid == 0;    // writes the part's record
  if (parts == 0 && tid == 0 && (int)blockIdx.x < a.records)
    a.seg[blockIdx.x] = make_int4(0, 0, 0, 0);         // (there are at least as many workgroups)
  if (part.lo >= part.hi) {
    if (keeps && !a.by_segment && part.p < a.wgs / a.width) a.seg[part.p] = make_int4(0, 0, 0, 0);
    return;
  }
  const Loader<D, G::KEYS> load(w, lane);
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;
  const uint32_t vaddr = TILE + 16 * vt_unit(lr, lh);
  Segment next = plan.first;
  next = {uniform(next.seq), uniform(next.head), uniform(next.seg), uniform(next.start),
          uniform(next.end)};
  if (next.end <= part.lo) next = after<G>(a, plan, next);
  int worked = 1;
  while (true) {
    s_piece[w] = piece_of<G>(a, next, uniform(plan.len[next.seq]), part);
    asm volatile("" ::: "memory");
    const Piece &me = s_piece[w];
    const Source src = {uniform(me.src.row), uniform(me.src.head), 0, uniform(me.src.limit),
                        uniform(me.src.once)};
    const int t0 = uniform(me.t0), t1 = uniform(me.t1);
    const int32_t *table = a.table + (int64_t)src.row * a.max_pages;
    const int64_t in_page = ((int64_t)src.head << a.page_shift) * D;
    const int64_t page_size = ((int64_t)a.hkv << a.page_shift) * D;
    // this wave's 16 keys of tile t: the table's entry, a tile ahead, and their copies
    auto page = [&](int t) {
      return table[min(G::KEYS * t + 16 * w, src.limit - 1) >> a.page_shift];
    };
    auto issue = [&](int t, int pg, uint8_t *into) {
      const int key = G::KEYS * t + 16 * w;
      if (key >= src.limit) return;       // past the sequence: those keys are masked
      pg = min(max(uniform(pg), 0), a.pages - 1);
      load.copy(a.k, a.v, pg * page_size + in_page + (key & ((1 << a.page_shift) - 1)) * D, src.once,
                into + w * S::STEP, into + w * S::STEP + TILE);
    };
    int page_next = 0;
    if (t0 < t1) {
      wg_barrier();                       // (other waves may still read the last piece's tiles)
      issue(t0, page(t0), lds0);
      page_next = page(min(t0 + 1, t1 - 1));
    }
    const int row0 = uniform(me.row0), seq = uniform(me.s.seq), vis = uniform(me.vis);
    const bool active = 32 * w < uniform(me.rows);
    const int row = 32 * w + lr;
    const int srow = min(row0 + row, (a.cu[seq + 1] - a.cu[seq]) * a.G - 1);
    const int tok = srow / a.G;
    const int lim = vis + tok;            // keys that this lane's row sees
    const int seen = max(vis + row0 / a.G, 0);
    // keys that the wave's first row sees, and its last
    const int lim_w = vis + (row0 + 32 * w) / a.G;
    const int lim_all = vis + min(row0 + 32 * w + 31, (a.cu[seq + 1] - a.cu[seq]) * a.G - 1) / a.G;
    const uint16_t *qp = a.q + (int64_t)(a.cu[seq] + tok) * a.q_stride +
                         (int64_t)(src.head * a.G + srow - tok * a.G) * D + 8 * lh;
    bf16x8 qf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const bf16x8 *>(qp + 16 * k);
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(qf[k]));
    f32x16 oacc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) oacc[i] = f32x16{};
    float m_ref = -INFINITY, mc = 0.f, m_trig = -INFINITY, l_run = 0.f;

    auto step = [&](uint8_t *tile, uint8_t *next, const int t) {
      const int k0 = G::KEYS * t;
      wait_copies();                                   // this wave's part of tile t is here
      const bool edge = k0 + G::KEYS > seen;           // some row does not see all of it
      if (edge && settle<D>(tile + TILE + w * S::STEP, k0 + 16 * w, src.limit, seen, lane) &&
          lane == 0)
        s_odd[worked & 1] = worked;
      wg_barrier();                                    // ... and every wave's
      if (t + 1 < t1) {
        issue(t + 1, page_next, next);
        page_next = page(min(t + 2, t1 - 1));
      }
      if (!active) return;
      if (k0 >= lim_all) return;
      f32x16 sacc[2] = {f32x16{}, f32x16{}};
      // Fragments are read eight products before their use, in this order (left alone the compiler keeps
      // registers for one pair and waits for each: three short sequences 13.4 us against 13.1, 48 chunks
      // and single tokens 292 against 287).
      constexpr int KA = 4, VA = 8;
      bf16x8 kf[KA][2], vf[VA];
      auto read_k = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          kf[k % KA][i] = *reinterpret_cast<const bf16x8 *>(tile + kaddr[k] + i * 32 * S::RB);
      };
      auto read_v = [&](int n) {
        vf[n % VA] = *reinterpret_cast<const bf16x8 *>(tile + vaddr + n % DB * 1024 + n / DB * S::STEP);
      };
#pragma unroll
      for (int k = 0; k < KA; ++k) read_k(k);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          sacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k % KA][i], qf[k], sacc[i], 0, 0, 0);
        if (k + KA < KS) read_k(k + KA);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (k0 + kKeys > lim_w) mask<2>(sacc, lim - k0 - 8 * lh);
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sacc[i][v]);
      // The reference moves only when a score rises 2^kLazy above it in weight; its own weight is 2^-kBelow.
      if (__ballot(mt > m_trig)) {
        const float m_new = fmaxf(m_ref, wave_pair_max(mt));
        const float f = m_ref == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        l_run *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) oacc[i] *= f;
        m_ref = m_new;
        const bool none = m_new == -INFINITY;
        mc = none ? 0.f : fmaf(m_new, c, kBelow);
        m_trig = none ? -INFINITY : m_new + lazy_raw;
      }
      bf16x8 pf[4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          pf[2 * i + (v >> 3)][v & 7] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sacc[i][v], c, -mc));
      l_run = sum_weights(pf, l_run);
#pragma unroll
      for (int n = 0; n < VA; ++n) read_v(n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 4 * DB; ++n) {
        oacc[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n % VA], pf[n / DB], oacc[n % DB], 0, 0, 0);
        if (n + VA < 4 * DB) read_v(n + VA);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // (in pairs: a branch on the buffer in every step would move O from register to register)
    for (int t = t0; t < t1; t += 2) {
      step(lds0, lds1, t);
      if (t + 1 < t1) step(lds1, lds0, t + 1);
    }
    asm volatile("" ::: "memory");

    // ---- values that settle took out, for the rows that see them: a weight above zero makes its
    // element what they are, so that it need not be the same to the last bit
    if (t0 < t1) {
      if (s_odd[worked & 1] == worked && active)
        late_values<D>(a, src, max(seen, G::KEYS * t0), min(src.limit, G::KEYS * t1), lim, qp, c, mc, lh,
                       oacc);
      ++worked;
    }
    const int rows = uniform(me.rows);
    const bool begins = uniform(me.begins), whole = begins && uniform(me.ends);

    const float l = wave_pair_sum(l_run);
    if (row < rows)
      finish<D>(a, whole, t0 < t1, oacc, m_ref, l,
                a.part + (int64_t)((2 * part.p + begins) * a.width + part.tile) * a.tile_rows * (D + 2),
                row, lh, (int64_t)(a.cu[seq] + tok) * a.hq + src.head * a.G + srow - tok * a.G);
    next = {seq, src.head, uniform(me.s.seg), uniform(me.s.start), uniform(me.s.end)};
    const bool last = next.end >= part.hi;
    if (keeps) record<G>(a, plan, part, parts, me, last);
    if (last) return;
    next = after<G>(a, plan, next);
  }
}

// ---- Row tiles of 256, head dim 128: eight waves of 32 rows, two on each SIMD.  Half a tile, 32 keys, at
// a time, three of them at work together: S of half h + 1, the weights of half h and O += V P of half
// h - 1 do not depend on each other, so that a wave keeps the matrix and the vector pipe busy at once
// (both run side by side without loss: a product of 32 cycles with three multiply-adds and an exponential
// takes 1.5 cycles more than alone).
//
// K of a tile is looked at a half before V, so tiles t - 1 to t + 1 are in use in step t and the next one
// is on its way: four tiles of LDS each, 128 KB, one barrier a step.
struct Wide {
  using S = PagedGeo<128>;
  using G = Geo<8, 64>;
  static constexpr int D = 128, KS = D / 16, DB = D / 32, TILE = 4 * S::STEP, RING = 4;
  // one object, of whose parts the compiler does not think that reads must wait for copies into others
  struct Shared {
    uint8_t k[RING][TILE], v[RING][TILE];
    Plan plan;
    Piece piece[8];                       // see chunk_fwd
    int odd[2];                           // piece with late values that are not finite, by its parity
  };
};

__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void chunk_wide(ChunkArgs a) {
  using S = Wide::S;
  using G = Wide::G;
  constexpr int D = Wide::D, KS = Wide::KS, DB = Wide::DB, RING = Wide::RING;
  __shared__ __attribute__((aligned(1024))) Wide::Shared sh;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  if (tid < 2) sh.odd[tid] = 0;
  int parts;
  const Part part = make_plan<G, 1>(a, sh.plan, parts);
  const bool keeps = parts > 0 && part.tile == 0 && tid == 0;    // writes the part's record
  if (parts == 0 && tid == 0 && (int)blockIdx.x < a.records)
    a.seg[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (part.lo >= part.hi) {
    if (keeps && !a.by_segment && part.p < a.wgs / a.width) a.seg[part.p] = make_int4(0, 0, 0, 0);
    return;
  }
  const int w4 = w & 3;                   // of the eight waves four bring the keys, four the values
  const Loader<D, G::KEYS> load(w4, lane);
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;
  const uint32_t vaddr = 16 * vt_unit(lr, lh);

  Segment next = sh.plan.first;
  next = {uniform(next.seq), uniform(next.head), uniform(next.seg), uniform(next.start),
          uniform(next.end)};
  if (next.end <= part.lo) next = after<G>(a, sh.plan, next);
  int worked = 1;
  while (true) {
    sh.piece[w] = piece_of<G>(a, next, uniform(sh.plan.len[next.seq]), part);
    asm volatile("" ::: "memory");
    const Piece &me = sh.piece[w];
    const Source src = {uniform(me.src.row), uniform(me.src.head), 0, uniform(me.src.limit),
                        uniform(me.src.once)};
    const int t0 = uniform(me.t0), t1 = uniform(me.t1);
    const int32_t *table = a.table + (int64_t)src.row * a.max_pages;
    const int64_t in_page = ((int64_t)src.head << a.page_shift) * D;
    const int64_t page_size = ((int64_t)a.hkv << a.page_shift) * D;
    // this wave's 16 keys or values of tile t: the table's entry, and the copy
    auto page = [&](int t) {
      return table[min(G::KEYS * t + 16 * w4, max(src.limit - 1, 0)) >> a.page_shift];
    };
    auto offset = [&](int t, int pg) {
      pg = min(max(uniform(pg), 0), a.pages - 1);
      return pg * page_size + in_page + ((G::KEYS * t + 16 * w4) & ((1 << a.page_shift) - 1)) * D;
    };
    auto copy_k = [&](int t, int pg) {
      if (w < 4 && t < t1 && G::KEYS * t + 16 * w4 < src.limit)
        load.copy_k(a.k + offset(t, pg), src.once, sh.k[t & (RING - 1)] + w4 * S::STEP);
    };
    auto copy_v = [&](int t, int pg) {
      if (w >= 4 && t < t1 && G::KEYS * t + 16 * w4 < src.limit)
        load.copy_v(a.v + offset(t, pg), src.once, sh.v[t & (RING - 1)] + w4 * S::STEP);
    };
    const int row0 = uniform(me.row0), seq = uniform(me.s.seq), vis = uniform(me.vis);
    const bool active = 32 * w < uniform(me.rows);
    const int row = 32 * w + lr;
    const int srow = min(row0 + row, (a.cu[seq + 1] - a.cu[seq]) * a.G - 1), tok = srow / a.G;
    const uint16_t *qp = a.q + (int64_t)(a.cu[seq] + tok) * a.q_stride +
                         (int64_t)(src.head * a.G + srow - tok * a.G) * D + 8 * lh;
    const int seen = max(vis + row0 / a.G, 0);         // keys that the tile's first row sees
    // keys of this part that the wave's first row sees, and this lane's row
    const int lim_w = min(vis + (row0 + 32 * w) / a.G, G::KEYS * t1);
    const int lim = min(vis + tok, G::KEYS * t1);
    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
    float m_ref = -INFINITY, mc = 0.f, m_trig = -INFINITY, l_run = 0.f;

    if (t0 < t1) {
      wg_barrier();                       // (other waves may still read the last piece's tiles)
      const int pg0 = page(t0), pg1 = page(t0 + 1), pg2 = page(t0 + 2);
      copy_k(t0, pg0);
      copy_v(t0, pg0);
      copy_k(t0 + 1, pg1);
      copy_v(t0 + 1, pg1);
      copy_k(t0 + 2, pg2);
      int pg_v = pg2, pg_k = page(t0 + 3);
      bf16x8 qf[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const bf16x8 *>(qp + 16 * k);
#pragma unroll
      for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(qf[k]));

      auto scores = [&](int half, f32x16 &to) {
        const uint8_t *tile = sh.k[(half >> 1) & (RING - 1)] + (half & 1) * 32 * S::RB;
        to = f32x16{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
          to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              *reinterpret_cast<const bf16x8 *>(tile + kaddr[k]), qf[k], to, 0, 0, 0);
      };
      auto values = [&](int half, const bf16x8 (&p)[2]) {
        const uint8_t *tile = sh.v[(half >> 1) & (RING - 1)] + (half & 1) * 2 * S::STEP + vaddr;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int db = 0; db < DB; ++db)
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                *reinterpret_cast<const bf16x8 *>(tile + db * 1024 + t * S::STEP), p[t], oacc[db], 0,
                0, 0);
      };
      auto weights = [&](const f32x16 &s, bf16x8 (&to)[2]) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          to[v >> 3][v & 7] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[v], c, -mc));
        l_run = sum_weights(to, l_run);
      };
      auto largest = [&](const f32x16 &of) {
        float mt = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) mt = fmaxf(mt, of[v]);
        return mt;
      };
      // What the new scores `of` (of `half`, the largest mt) do to the reference, as in chunk_fwd.  O has
      // one half less than the sum, in the reference that was: it follows a half later (`pending`).
      bool pending = false;
      float alpha = 1.f;
      auto settle_ref = [&](int half, f32x16 &of, float mt) {
        if (32 * half + 32 > lim_w) {     // keys that some row of the wave does not see
          mask<1>(&of, lim - 32 * half - 8 * lh);
          mt = largest(of);
        }
        const bool moves = __ballot(mt > m_trig);
        if (moves || pending) {
          if (pending) {
#pragma unroll
            for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
          }
          const float m_new = moves ? fmaxf(m_ref, wave_pair_max(mt)) : m_ref;
          alpha = m_ref == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
          l_run *= alpha;
          m_ref = m_new;
          const bool none = m_new == -INFINITY;
          mc = none ? 0.f : fmaf(m_new, c, kBelow);
          m_trig = none ? -INFINITY : m_new + lazy_raw;
          pending = moves;
        }
      };
      // Half h: S of h + 1 (sn), weights of h (pn) from its scores (s), O += V P of h - 1 (p), dealt out
      // over 16 places, each a product, the read of the fragment three places on, and a share of the
      // vector instructions, which the compiler keeps in this order.
      bf16x8 frag[4];
      auto read_frag = [&](int h, int place) {         // of half h, or of the next one (place >= 16)
        h += place >> 4;
        place &= 15;
        const int of = place < KS ? h + 1 : h - 1, slot = (of >> 1) & (RING - 1);
        return *reinterpret_cast<const bf16x8 *>(
            place < KS ? sh.k[slot] + (of & 1) * 32 * S::RB + kaddr[place & 7]
                       : sh.v[slot] + ((of & 1) * 2 + (place - KS) / DB) * S::STEP +
                             (place - KS) % DB * 1024 + vaddr);
      };
      auto half = [&](int h, const f32x16 &s, f32x16 &sn, const bf16x8 (&p)[2], bf16x8 (&pn)[2]) {
        float mt = -INFINITY, ex[16];
        sn = f32x16{};
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          frag[(q + 3) & 3] = read_frag(h, q + 3);
          f32x16 &acc = q < KS ? sn : oacc[(q - KS) % DB];
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[q & 3], q < KS ? qf[q & 7] : p[(q - KS) / DB & 1],
                                                        acc, 0, 0, 0);
          ex[q] = __builtin_amdgcn_exp2f(fmaf(s[q], c, -mc));
          if (q % 2 == 0 && q >= 2) {
            pn[(q - 2) >> 3][(q - 2) & 7] = (__bf16)ex[q - 2];
            pn[(q - 1) >> 3][(q - 1) & 7] = (__bf16)ex[q - 1];
          }
          if (q >= 10) {                  // (the scores are there two places after their last product)
#pragma unroll
            for (int v = (q - 10) * 3; v < (q - 9) * 3 && v < 16; ++v) mt = fmaxf(mt, sn[v]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        pn[1][6] = (__bf16)ex[14];
        pn[1][7] = (__bf16)ex[15];
        l_run = sum_weights(pn, l_run);
        asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(mt));   // (before the branch that follows)
        settle_ref(h + 1, sn, mt);
      };
      // K of tile t + 1 and V of tile t are here; the next ones are sent for.
      auto arrive = [&](int t) {
        wait_copies();
        if (w >= 4 && G::KEYS * (t + 1) > seen &&
            settle<D>(sh.v[t & (RING - 1)] + w4 * S::STEP, G::KEYS * t + 16 * w4, src.limit, seen,
                      lane) &&
            lane == 0)
          sh.odd[worked & 1] = worked;
        wg_barrier();
        const int k = pg_k, v = pg_v;
        pg_v = pg_k;
        pg_k = page(t + 4);
        copy_k(t + 3, k);
        copy_v(t + 2, v);
      };
      // scores and weights of even halves and of odd ones
      f32x16 s0, s1;
      bf16x8 p0[2], p1[2];
      arrive(t0);
      if (active) {
        scores(2 * t0, s0);
        settle_ref(2 * t0, s0, largest(s0));
        scores(2 * t0 + 1, s1);
        weights(s0, p0);
        settle_ref(2 * t0 + 1, s1, largest(s1));
#pragma unroll
        for (int q = 0; q < 3; ++q) frag[q] = read_frag(2 * t0 + 1, q);
        half(2 * t0 + 1, s1, s0, p0, p1);
      }
      for (int t = t0 + 1; t < t1; ++t) {
        arrive(t);
        if (active) {
          half(2 * t, s0, s1, p1, p0);
          half(2 * t + 1, s1, s0, p0, p1);
        }
      }
      if (active) values(2 * t1 - 1, p1);              // (no score of the half after it moved anything)
      asm volatile("" ::: "memory");
      if (sh.odd[worked & 1] == worked && active)
        late_values<D>(a, src, max(seen, G::KEYS * t0), min(src.limit, G::KEYS * t1), lim, qp, c, mc, lh,
                       oacc);
      ++worked;
    }
    const bool begins = uniform(me.begins), whole = begins && uniform(me.ends);
    const float l = wave_pair_sum(l_run);
    if (row < uniform(me.rows))
      finish<D>(a, whole, t0 < t1, oacc, m_ref, l,
                a.part + (int64_t)((2 * part.p + begins) * a.width + part.tile) * a.tile_rows * (D + 2),
                row, lh, (int64_t)(a.cu[seq] + tok) * a.hq + src.head * a.G + srow - tok * a.G);
    next = {seq, src.head, uniform(me.s.seg), uniform(me.s.start), uniform(me.s.end)};
    const bool last = next.end >= part.hi;
    if (keeps) record<G>(a, sh.plan, part, parts, me, last);
    if (last) return;
    next = after<G>(a, sh.plan, next);
  }
}

// ---- Joins the pieces of a segment that begins in part p and ends in a later one; blockIdx.y is a
// record and a row tile of its segment, of which the workgroups blockIdx.x share the rows.  D / 4 lanes to
// a row, 16 bytes each.  Up to kFewPieces pieces: 32 rows at a time, all their loads in flight together.
// More: WPR waves to a row, each with every 64 / (D / 4) * WPR-th group of pieces, four loads in flight.
constexpr int kFewPieces = 4;

template <int D, int WPR>
__global__ __launch_bounds__(kJoinThreads) void chunk_join(ChunkArgs a) {
  constexpr int LPP = D / 4;              // lanes per piece
  constexpr int PPW = 64 / LPP;           // pieces at once in a wave
  constexpr int U = 4;                    // loads in flight
  __shared__ f32x4 s_sum[4][LPP];
  const int at = blockIdx.y / a.width, j = blockIdx.y - at * a.width;
  const int4 rec = a.seg[at];
  const int n = rec.x & 0xFFFF, p = rec.x >> 16;
  if (n == 0) return;
  const int b = rec.y, first = (rec.w * a.width + j) * a.rows;    // the tile's first row
  const int rows = min((a.cu[b + 1] - a.cu[b]) * a.G - first, a.rows);
  const int64_t size = (int64_t)a.tile_rows * (D + 2);
  auto piece = [&](int i) {
    const int q = min(i, n - 1);
    return a.part + ((int64_t)(q == 0 ? 2 * p + 1 : 2 * (p + q)) * a.width + j) * size;
  };
  auto store = [&](int r, const f32x4 &acc, float l, int lane) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int srow = first + r, tok = srow / a.G;
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4 *>(
        a.o + ((int64_t)(a.cu[b] + tok) * a.hq + rec.z * a.G + srow - tok * a.G) * D + 4 * lane) = o;
  };
  const float c = a.scale_log2;
  // What a piece (its reference and sum) counts beside the largest reference.  A sum of 0 is that of a
  // piece without a key that the row sees, whose O may not be there.  All others count: NaN comes through
  // whatever its reference, infinity however small its weight.
  auto factor = [&](float2 ml, float top) {
    return ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml.x - top) * c);
  };
  if (n <= kFewPieces) {
    constexpr int AT_ONCE = kJoinThreads / LPP, PER = 32 / AT_ONCE;
    const int lane = threadIdx.x % LPP, group = threadIdx.x / LPP;
    for (int r0 = 32 * blockIdx.x; r0 < rows; r0 += 32 * gridDim.x) {
      int row[PER];
      float2 ml[PER][kFewPieces];
      f32x4 x[PER][kFewPieces], acc[PER];
      float l[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        row[i] = min(r0 + AT_ONCE * i + group, rows - 1);
#pragma unroll
        for (int q = 0; q < kFewPieces; ++q)
          ml[i][q] = q < n ? *reinterpret_cast<const float2 *>(piece(q) + a.tile_rows * D + 2 * row[i])
                           : make_float2(-INFINITY, 0.f);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int q = 0; q < kFewPieces; ++q)
          if (q < n)
            x[i][q] = __builtin_nontemporal_load(
                reinterpret_cast<const f32x4 *>(piece(q) + row[i] * D + 4 * lane));
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < kFewPieces; ++q) top = fmaxf(top, ml[i][q].x);
        l[i] = 0.f;
        acc[i] = f32x4{};
#pragma unroll
        for (int q = 0; q < kFewPieces; ++q) {
          ml[i][q].x = factor(ml[i][q], top);
          l[i] = fmaf(ml[i][q].x, ml[i][q].y, l[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int q = 0; q < kFewPieces; ++q)
          if (q < n && ml[i][q].y != 0.f)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(ml[i][q].x, x[i][q][e], acc[i][e]);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (r0 + AT_ONCE * i + group < rows) store(row[i], acc[i], l[i], lane);
    }
    return;
  }
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, part = w % WPR;
  for (int r0 = blockIdx.x * (4 / WPR); r0 < rows; r0 += gridDim.x * (4 / WPR)) {
    const int r = r0 + w / WPR;           // (with WPR == 4 all waves have the same)
    if (WPR == 1 && r >= rows) break;
    const int ml_at = a.tile_rows * D + 2 * r;
    float top_all = -INFINITY, l = 0.f;
    f32x4 acc = f32x4{};
    for (int i0 = 0; i0 < n; i0 += 64) {
      const int k = min(64, n - i0);
      f32x4 x[U];
      auto fetch = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          x[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(
              piece(i0 + min(i + u * WPR * PPW + lane / LPP, k - 1)) + r * D + 4 * (lane % LPP)));
      };
      fetch(part * PPW);                  // beside the references, not after them
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < k) ml = *reinterpret_cast<const float2 *>(piece(i0 + lane) + ml_at);
      float top = fmaxf(top_all, ml.x);
#pragma unroll
      for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
      const float old = top_all == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top_all - top) * c);
      const float f = ml.y == 0.f ? -1.f : factor(ml, top);      // (-1: nothing to add)
      float sum = ml.y == 0.f ? 0.f : f * ml.y;
#pragma unroll
      for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
      l = l * old + sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= old;
      top_all = top;
      for (int i = part * PPW; i < k; i += U * WPR * PPW) {
        float fi[U];
        if (i != part * PPW) fetch(i);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = i + u * WPR * PPW + lane / LPP;
          fi[u] = __shfl(f, at & 63);     // (by all lanes)
          if (at >= k) fi[u] = -1.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fi[u] < 0.f)) acc[e] = fmaf(fi[u], x[u][e], acc[e]);
      }
    }
#pragma unroll
    for (int d = LPP; d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
    if constexpr (WPR > 1) {
      __syncthreads();                    // the sums of the row before are read
      if (lane < LPP) s_sum[w][lane] = acc;
      __syncthreads();
      if (part == 0 && lane < LPP) {
        acc = f32x4{};
#pragma unroll
        for (int i = 0; i < WPR; ++i) acc += s_sum[w + i][lane];
      }
    }
    if (part == 0 && lane < LPP) store(r, acc, l, lane);
  }
}

template <int D>
hipError_t launch(const ChunkArgs &a, hipStream_t s) {
  const bool wide = D == 128 && a.rows == 256;
  if (wide) chunk_wide<<<std::max(a.wgs, a.tiles), 512, 0, s>>>(a);
  else chunk_fwd<D><<<std::max(a.wgs, a.tiles), 256, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  // (a cache whose slots are so short is never cut)
  const bool short_slots = (int64_t)a.max_pages << a.page_shift <= kWholeTiles * kKeys;
  if (e != hipSuccess || (a.tiles > 0 && short_slots)) return e;
  // 32 rows to a workgroup where there are many tiles, few of them cut into many pieces; else four, or one
  const int tiles = a.records * a.width, few = a.tile_rows <= 32 ? 1 : 4;
  const int per = (int64_t)tiles * a.tile_rows > 8192 * few ? 32 : few;
  const dim3 grid((a.tile_rows + per - 1) / per, tiles);
  if (a.tile_rows <= 32) chunk_join<D, 4><<<grid, kJoinThreads, 0, s>>>(a);
  else chunk_join<D, 1><<<grid, kJoinThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkArgs &a, int d, hipStream_t s) {
  return d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace fp
