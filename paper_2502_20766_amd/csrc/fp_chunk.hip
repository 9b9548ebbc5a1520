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
// How the work is divided.  A segment is a.width row tiles of one sequence and KV head that lie side by
// side, with the keys that the last of them sees.  Segments, one after the other, form a line whose
// places are rows of keys; it is cut into equal parts, one for each cluster of a.width workgroups, each of
// which takes one of the row tiles.  The workgroups of a cluster go through the same keys at the same
// time, so those come from memory, and mostly from the XCD's L2, once.  A piece (a part's share of a
// segment) that is not all of it leaves O, its reference and its sum in float32, and a last launch joins
// the pieces of a row in the order of the line.  The cuts follow from the lengths alone, so results do
// not depend on timing.
#include <type_traits>

#include "fp_attn_dev.h"
#include "fp_internal.h"
#include "fp_paged_dev.h"

namespace fp {
namespace {

constexpr int kMaxList = FP_MAX_CACHE_LIST;
constexpr int kJoinThreads = 256;

// A workgroup of `WAVES` waves: 32 rows each, and 16 keys of a tile that each brings.
template <int WAVES>
struct Geo {
  static constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES, KEYS = 16 * WAVES;
  static_assert(THREADS >= kMaxList, "the plan has one thread per sequence");
};

// Key tiles that a segment takes of the line beside its own: the cost of starting and ending a piece.
constexpr int kSegCost = 2;
// Fewest key tiles of a part.
constexpr int kPartTiles = 4;

// The line: places where the segments of a sequence begin, in (key, query head) pairs: a key tile is 64 G
// places, so that the places of a sequence's segments are an arithmetic series.
struct Plan {
  int64_t start[kMaxList + 1];
  int64_t scan[kMaxList / 64];
  int len[kMaxList];                      // tokens of a sequence (0: no slot)
  int first;                              // sequence that this workgroup's part begins in
};

// A line of `total` places in `parts` equal parts, the first total % parts of them one place longer.
struct Cut {
  int64_t per, rem;
  __device__ __forceinline__ Cut(int64_t total, int parts) : per(total / parts) {
    rem = total - per * parts;
  }
  __device__ __forceinline__ int64_t begin(int p) const { return per * p + min((int64_t)p, rem); }
  __device__ __forceinline__ int owner(int64_t x) const {
    const int64_t longer = rem * (per + 1);
    return (int)(x < longer ? x / (per + 1) : rem + (x - longer) / per);
  }
};

// A sequence's segments of one KV head: segment i takes fixed + (i + 1) * step places.
template <class G>
struct Series {
  int64_t fixed, step;
  int n;
  __device__ __forceinline__ Series(const ChunkArgs &a, int m, int len) {
    const int64_t base = len > m ? len - m : 0;
    const int span = a.width * G::ROWS;
    n = (int)(((int64_t)m * a.G + span - 1) / span);
    fixed = a.G * (int64_t)(G::KEYS * kSegCost + (len > 0 ? G::KEYS + base : 0));
    step = len > 0 ? span : 0;
  }
  __device__ __forceinline__ int64_t begin(int64_t i) const {
    return i * fixed + step * (i * (i + 1) / 2);
  }
};

struct Part {
  int p, tile;          // number of the part, row tile of its segments
  int64_t lo, hi;       // places; lo == hi: none
};

// Fills the plan and finds this workgroup's part.
template <class G>
__device__ __forceinline__ Part make_plan(const ChunkArgs &a, Plan &plan, int &parts) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int64_t cost = 0;
  if (t < a.batch) {
    const int slot = a.slot[t], m = a.cu[t + 1] - a.cu[t];
    const int len = slot < 0 ? 0 : min(max(a.len[slot], 0), a.max_pages << a.page_shift);
    plan.len[t] = len;
    const Series<G> series(a, m, len);
    cost = series.begin(series.n) * a.hkv;
  }
  int64_t sum = cost;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 63 && w < kMaxList / 64) plan.scan[w] = sum;
  __syncthreads();
  int64_t start = sum - cost, total = 0;
#pragma unroll
  for (int j = 0; j < kMaxList / 64; ++j) {
    if (j < w) start += plan.scan[j];
    total += plan.scan[j];
  }
  if (t < kMaxList) plan.start[t] = start;
  if (t == 0) plan.start[kMaxList] = total;
  const int most = a.wgs / a.width;
  const int64_t want = total / (kPartTiles * G::KEYS * (int64_t)a.G);
  parts = (int)min(max(want, (int64_t)1), (int64_t)most);
  // Workgroups of one XCD (every eighth) take neighbouring parts; where there is not work for all, the
  // clusters are dealt out over the XCDs.
  const int x = blockIdx.x & 7, y = blockIdx.x >> 3, room = a.wgs / 8 / a.width;
  Part r;
  if (8 * parts * a.width > 7 * a.wgs || parts > 8 * room) {
    const int wg = x * (a.wgs / 8) + y;
    r.p = wg / a.width;
    r.tile = wg - r.p * a.width;
  } else {
    const int c = y / a.width;
    r.p = c < room ? c * 8 + x : most;
    r.tile = y - c * a.width;
  }
  r.lo = r.hi = 0;
  if (r.p < parts) {
    const Cut cut(total, parts);
    r.lo = cut.begin(r.p);
    r.hi = cut.begin(r.p + 1);
    if (start <= r.lo && r.lo < start + cost) plan.first = t;
  }
  __syncthreads();
  return r;
}

// Where a piece's keys lie, as Loader needs it.
struct Source {
  int row;              // cache slot whose pages are read
  int head;             // KV head
  int key0, limit;      // keys: first, and the sequence's tokens
  int once;             // no other workgroup reads these keys
};

// A run of key tiles of one row tile in one workgroup; every field is wave-uniform.
struct Piece {
  Source src;
  int t0, t1;           // tiles [t0, t1) of its keys that this row tile sees
  int row0, rows;       // rows of the sequence and KV head: first, and how many (0: none)
  int seq, seg;         // sequence, and segment of it and the KV head
  int vis;              // keys that the sequence's first query sees (may be negative)
  int begins, ends;     // the part has the segment's first tile, its last
  int64_t end;          // place of the line where the segment ends
  int64_t last;         // place of the segment's last tile
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// The piece at place x of the workgroup's part, which lies in sequence `e` or a later one.
template <class G>
__device__ __forceinline__ Piece piece_at(const ChunkArgs &a, const Plan &plan, int e, int64_t x,
                                          const Part &part) {
  while (plan.start[e + 1] <= x) ++e;
  Piece r;
  r.seq = uniform(e);
  const int len = uniform(plan.len[r.seq]), m = a.cu[r.seq + 1] - a.cu[r.seq];
  const Series<G> series(a, m, len);
  const int64_t whole = series.begin(series.n);        // places of one KV head
  const int64_t y = uniform(x - plan.start[r.seq]);
  const int head = uniform((int)(y / whole));
  const int64_t z = y - head * whole;
  int lo = 0, hi = series.n;                           // begin(lo) <= z < begin(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (series.begin(mid) <= z) lo = mid;
    else hi = mid;
  }
  r.seg = uniform(lo);
  const int64_t start = x - z + series.begin(lo);
  r.end = x - z + series.begin(lo + 1);
  const int rows = m * a.G, span = a.width * G::ROWS;
  r.src.row = a.slot[r.seq];
  r.src.head = head;
  r.src.key0 = 0;
  r.src.limit = len;
  r.src.once = rows <= G::ROWS;
  r.vis = len - m + 1;
  // tiles that the segment's last row sees, and those in this part
  const int tile = G::KEYS * a.G;
  auto tiles_of = [&](int end) {
    const int keys = len > 0 ? max(r.vis + (end - 1) / a.G, 0) : 0;
    return (keys + G::KEYS - 1) / G::KEYS;
  };
  const int all = tiles_of(min((lo + 1) * span, rows));
  const int64_t first = start + kSegCost * (int64_t)tile;
  r.last = first + (int64_t)tile * all - 1;
  const int t0 = part.lo <= first ? 0 : (int)min((part.lo - first) / tile, (int64_t)all);
  const int t1 = part.hi >= r.end ? all
                 : part.hi <= first ? 0 : (int)min((part.hi - first) / tile, (int64_t)all);
  // (rows without a key belong to the part where they begin)
  const bool here = all > 0 ? t0 < t1 : part.lo <= start;
  r.row0 = lo * span + part.tile * G::ROWS;
  r.rows = here ? max(min(rows - r.row0, G::ROWS), 0) : 0;
  r.t0 = t0;
  r.t1 = r.rows > 0 ? max(min(t1, tiles_of(r.row0 + r.rows)), t0) : t0;
  r.begins = t0 == 0;
  r.ends = t1 == all || !here;
  return r;
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

template <int D, int WAVES>
__global__ __launch_bounds__((Geo<WAVES>::THREADS))
__attribute__((amdgpu_waves_per_eu(PagedGeo<D>::OCC, PagedGeo<D>::OCC)))
void chunk_fwd(ChunkArgs a) {
  using S = PagedGeo<D>;
  using G = Geo<WAVES>;
  constexpr int KS = D / 16, DB = D / 32, TILE = WAVES * S::STEP;
  // K and V of even tiles in lds0, of odd ones in lds1: two arrays, so that the compiler sees that
  // reads of one do not wait for copies into the other
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[2 * TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[2 * TILE];
  __shared__ Plan plan;
  // the piece at hand, each wave's own copy: what is looked at after its tiles would else take scalar
  // registers meanwhile
  __shared__ Piece s_piece[WAVES];
  __shared__ int s_odd[2];                // piece with late values that are not finite, by its parity
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  if (tid < 2) s_odd[tid] = 0;
  int parts;
  const Part part = make_plan<G>(a, plan, parts);
  const bool keeps = part.tile == 0 && tid == 0;       // writes the part's record
  if (part.lo == part.hi) {
    if (keeps && part.p < a.wgs / a.width) a.seg[part.p] = make_int4(0, 0, 0, 0);
    return;
  }
  const Loader<D, G::KEYS> load(w, lane);
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;
  const uint32_t vaddr = TILE + 16 * vt_unit(lr, lh);
  int e = plan.first, worked = 1;
  int64_t x = part.lo;
  while (true) {
    s_piece[w] = piece_at<G>(a, plan, e, x, part);
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
    const int row0 = uniform(me.row0), seq = uniform(me.seq), vis = uniform(me.vis);
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
#pragma unroll
      for (int sub = 0; sub < G::KEYS / kKeys; ++sub) {
        const int ks = k0 + kKeys * sub;
        if (ks >= lim_all) return;
        f32x16 sacc[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          bf16x8 kf[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            kf[i] = *reinterpret_cast<const bf16x8 *>(tile + kaddr[k] + (2 * sub + i) * 32 * S::RB);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            sacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[k], sacc[i], 0, 0, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS - 6; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
        if (ks + kKeys > lim_w) {
          // (the least of a score and + or - infinity: comparisons would take scalar registers)
          const float room = (float)(lim - ks - 8 * lh) - 0.5f;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              sacc[i][v] = fminf(sacc[i][v], (room - (32 * i + 16 * (v >> 3) + (v & 7))) * INFINITY);
        }
        float mt = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sacc[i][v]);
        // The reference moves only when a score rises 2^kLazy above it in weight, and has a weight of
        // 2^-kLazy, so that no weight is above 1: sums of large values do not pass float32 before they
        // are divided.
        if (__ballot(mt > m_trig)) {
          const float m_new = fmaxf(m_ref, wave_pair_max(mt));
          const float f = m_ref == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
          l_run *= f;
#pragma unroll
          for (int i = 0; i < DB; ++i) oacc[i] *= f;
          m_ref = m_new;
          const bool none = m_new == -INFINITY;
          mc = none ? 0.f : fmaf(m_new, c, kLazy);
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
        for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const bf16x8 vf =
                *reinterpret_cast<const bf16x8 *>(tile + vaddr + db * 1024 + (4 * sub + t4) * S::STEP);
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t4], oacc[db], 0, 0, 0);
          }
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

    // ---- lane holds row `row`, d = 32 db + 8 (v / 4) + 4 lh + v % 4
    const float l = wave_pair_sum(l_run);
    if (whole) {
      if (row < rows) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t *op = a.o + ((int64_t)(a.cu[seq] + tok) * a.hq + src.head * a.G + srow - tok * a.G) * D +
                       4 * lh;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (__bf16)(oacc[db][4 * g + e] * inv);
            *reinterpret_cast<bf16x4 *>(op + 32 * db + 8 * g) = o;
          }
      }
    } else if (row < rows) {
      float *to = a.part + (int64_t)((2 * part.p + begins) * a.width + part.tile) *
                               a.tile_rows * (D + 2);
      if (lh == 0)
        *reinterpret_cast<float2 *>(to + a.tile_rows * D + 2 * row) = make_float2(m_ref, l);
      to += row * D + 4 * lh;
      if (t0 < t1) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4 *>(to + 32 * db + 8 * g) =
                make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2],
                            oacc[db][4 * g + 3]);
      }
    }
    e = seq;
    x = uniform(me.end);
    if (x >= part.hi) {
      if (keeps) {                        // a segment that goes on in later parts
        int4 rec = make_int4(0, seq, src.head, me.seg);
        if (begins && !whole) rec.x = Cut(plan.start[kMaxList], parts).owner(me.last) - part.p + 1;
        a.seg[part.p] = rec;
      }
      return;
    }
  }
}

// ---- Joins the pieces of a row of a segment that begins in part p and ends in a later one: WPR waves,
// each with every 64 / (D / 4) * WPR-th group of pieces, D / 4 lanes to a piece, 16 bytes each, four loads
// in flight.
template <int D, int WPR>
__global__ __launch_bounds__(kJoinThreads) void chunk_join(ChunkArgs a) {
  constexpr int LPP = D / 4;              // lanes per piece
  constexpr int PPW = 64 / LPP;           // pieces at once in a wave
  constexpr int U = 4;                    // loads in flight
  __shared__ f32x4 s_sum[4][LPP];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, part = w % WPR;
  const int tile_at = blockIdx.y, p = tile_at / a.width, j = tile_at - p * a.width;
  const int4 rec = a.seg[p];
  const int n = rec.x;
  if (n == 0) return;
  const int r = blockIdx.x * (4 / WPR) + w / WPR;      // row of the tile
  const int b = rec.y, m = a.cu[b + 1] - a.cu[b];
  const int srow = (rec.w * a.width + j) * a.rows + r;
  const bool live = r < a.tile_rows && srow < m * a.G;
  if (WPR == 1 && !live) return;
  const int64_t size = (int64_t)a.tile_rows * (D + 2);
  auto piece = [&](int i) {
    const int q = min(i, n - 1);
    return a.part + ((int64_t)(q == 0 ? 2 * p + 1 : 2 * (p + q)) * a.width + j) * size;
  };
  const int row = live ? r : 0, ml_at = a.tile_rows * D + 2 * row;
  const float c = a.scale_log2;
  float top_all = -INFINITY, l = 0.f;
  f32x4 acc = f32x4{};
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int k = min(64, n - i0);
    f32x4 x[U];
    auto fetch = [&](int i) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(
            piece(i0 + min(i + u * WPR * PPW + lane / LPP, k - 1)) + row * D + 4 * (lane % LPP)));
    };
    fetch(part * PPW);                    // beside the references, not after them
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < k) ml = *reinterpret_cast<const float2 *>(piece(i0 + lane) + ml_at);
    float top = fmaxf(top_all, ml.x);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float old = top_all == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top_all - top) * c);
    // (a sum of 0: no key seen; a NaN has to come through, whatever its reference)
    const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml.x - top) * c);
    float sum = f * ml.y;
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
  if (lane < LPP && live) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int tok = srow / a.G;
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4 *>(a.o + ((int64_t)(a.cu[b] + tok) * a.hq + rec.z * a.G + srow -
                                       tok * a.G) * D + 4 * lane) = o;
  }
}

template <int D, int WAVES>
hipError_t launch(const ChunkArgs &a, hipStream_t s) {
  chunk_fwd<D, WAVES><<<a.wgs, Geo<WAVES>::THREADS, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tiles = a.wgs / a.width * a.width;
  if (a.tile_rows <= 32) chunk_join<D, 4><<<dim3(a.tile_rows, tiles), kJoinThreads, 0, s>>>(a);
  else chunk_join<D, 1><<<dim3(a.tile_rows / 4, tiles), kJoinThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkArgs &a, int d, hipStream_t s) {
  if (d == 64) return launch<64, 4>(a, s);
  return a.rows == 256 ? launch<128, 8>(a, s) : launch<128, 4>(a, s);
}

}  // namespace fp
