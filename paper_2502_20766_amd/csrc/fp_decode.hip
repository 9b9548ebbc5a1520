// Attention of the next tokens over a paged cache: o = softmax(c q K^T) V for the last `queries`
// tokens of every sequence of a batch, with the keys and values that a group of sequences shares
// at its start read once for the whole group.
//
// Split softmax: over a range R of keys, with reference m and weights w_j = exp2(s_j - m),
//   O_R = sum w_j v_j,  l_R = sum w_j;   o = (sum_R 2^(m_R - M) O_R) / (sum_R 2^(m_R - M) l_R).
// The ranges are cut as follows.  A segment is the work of one KV head and up to 128 query rows
// over one run of keys: the prefix of a group (rows: all query heads of the KV head, all queries,
// all sequences of the group) or the rest of one sequence (rows: its own).  All segments, one
// after the other in tiles of 64 keys, form a line that is cut into equal parts, one for each
// resident workgroup, so every workgroup has the same number of tiles whatever the lengths.
// Prefixes with more than 64 rows, whose products and not bytes are what costs, form a line and a
// launch of their own.  A piece (the part of a segment in one workgroup) leaves O_R, m_R and l_R
// in float32; a last launch joins the pieces of each row in the order of the line.  A segment in one piece whose
// rows have no prefix is finished on the spot.  Where the cuts fall follows from the lengths
// alone, so results do not depend on timing.
//
// One workgroup is four waves.  The 64 keys of a tile go through LDS (double buffered, by DMA,
// each wave bringing 16 keys, which always lie in one page); with more than 64 rows each wave
// has 32 rows of its own, with fewer two waves, or two pairs of waves, take 32 keys each and join
// in LDS at the end of the piece.  The products are those of the prefill: S^T = K Q^T with K rows permuted so that a
// lane's scores are the consecutive keys that P^T of O^T += V^T P^T needs.
#include <type_traits>

#include "fp_attn_dev.h"
#include "fp_internal.h"

namespace fp {
namespace {

constexpr int kKeys = 64;                 // keys per tile
constexpr int kThreads = 256;
constexpr int kMaxList = FP_MAX_CACHE_LIST;
constexpr float kLazy = 8.f;              // rise (log2 units) that moves a row's reference

static_assert(kThreads == kMaxList, "the plan has one thread per sequence");

// The line of a call: lengths, prefixes, and where each group's prefix and each sequence's own
// keys start on it.
struct Plan {
  int len[kMaxList];                      // tokens of a sequence (0: no sequence)
  int prefix[kMaxList];                   // per group: keys read once, a multiple of 16
  int lead[kMaxList];                     // per group: sequence whose pages hold them
  int live[kMaxList];
  int cum[2 * kMaxList + 1];              // starts: groups, then sequences at kMaxList + b
  int cum_many[kMaxList + 1];             // starts of the groups on the other line
  int scan[4];
};

__device__ __forceinline__ int tiles_of(int keys) { return (keys + kKeys - 1) / kKeys; }

__device__ __forceinline__ int row_tiles(int rows) { return (rows + kDecodeRows - 1) / kDecodeRows; }

__device__ __forceinline__ int group_rows(const DecodeArgs &a, int g) {
  return (a.start[g + 1] - a.start[g]) * a.nq * a.G;
}

// Groups whose prefix is on the line of many rows.
__device__ __forceinline__ bool is_many(const DecodeArgs &a, int g) {
  return group_rows(a, g) > kDecodeFew;
}

// Partial results of prefixes: on the line of many rows, row tile 0 of group g and KV head 0 is
// number (first row of g) / kDecodeRows + g, times Hkv; on the other, one row tile each.
__device__ __forceinline__ int prefix_base(const DecodeArgs &a, int g, bool many) {
  return (many ? a.start[g] * a.nq * a.G / kDecodeRows + g : g) * a.hkv;
}

// Exclusive prefix sum over the workgroup's 256 threads, and the total.
__device__ __forceinline__ int scan256(int x, int *part, int &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  __syncthreads();
  if (lane == 63) part[w] = sum;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < w) base += part[i];
    total += part[i];
  }
  return base + sum - x;
}

// Fills the plan; every workgroup of both launches does so for itself.
__device__ __forceinline__ void make_plan(const DecodeArgs &a, Plan &p) {
  const int t = threadIdx.x;
  if (t < a.groups) {
    p.prefix[t] = 0x7FFFFFFF;
    p.lead[t] = 0x7FFFFFFF;
    p.live[t] = 0;
  }
  __syncthreads();
  int len = 0, g = 0;
  if (t < a.batch) {
    g = a.group[t];
    if (a.slot[t] >= 0) len = min(max(a.len[a.slot[t]], 0), a.max_pages << a.page_shift);
    p.len[t] = len;
    if (len > 0) {
      atomicMin(&p.prefix[g], max(len - a.nq, 0));
      atomicMin(&p.lead[g], t);
      atomicAdd(&p.live[g], 1);
    }
  }
  __syncthreads();
  int cost = 0, cost_many = 0;
  if (t < a.groups) {
    // one sequence alone has nothing to share
    const int keys = p.live[t] >= 2 ? min(p.prefix[t], a.prefix[t]) & ~15 : 0;
    p.prefix[t] = keys;
    (is_many(a, t) ? cost_many : cost) = a.hkv * row_tiles(group_rows(a, t)) * tiles_of(keys);
  }
  int total_many, total_g, total;
  const int at_many = scan256(cost_many, p.scan, total_many);   // (publishes p.prefix)
  const int at_g = scan256(cost, p.scan, total_g);
  cost = 0;
  if (t < a.batch && len > 0)
    cost = a.hkv * row_tiles(a.G * a.nq) * tiles_of(len - p.prefix[g]);
  const int at_s = scan256(cost, p.scan, total);
  p.cum_many[t] = at_many;
  p.cum[t] = at_g;
  p.cum[kMaxList + t] = total_g + at_s;
  if (t == 0) {
    p.cum_many[kMaxList] = total_many;
    p.cum[2 * kMaxList] = total_g + total;
  }
  __syncthreads();
}

// The line of `total` tiles cut for `wgs` workgroups: [first, first of the next).
__device__ __forceinline__ int cut(int64_t total, int wgs, int w) {
  return (int)(total * w / wgs);
}
// The workgroup that has tile x.
__device__ __forceinline__ int owner(int64_t total, int wgs, int x) {
  return (int)((((int64_t)x + 1) * wgs - 1) / total);
}

// A run of tiles of one segment in one workgroup.
struct Piece {
  int end;              // first place of the line past it
  int row;              // cache slot whose pages are read
  int head;             // KV head
  int t0, t1, n;        // tiles [t0, t1) of the segment's n
  int key0, limit;      // first key, and the first one past the segment
  int row0, rows;       // rows of this row tile: row0 .. row0 + rows - 1 of the segment's
  int token0;           // query token of the segment's first row
  int vis;              // keys that the first query of a sequence sees
  int shared;           // a group's prefix
  int slot;             // partial result
  int whole;            // the piece is all that its rows have
};

template <bool MANY>
__device__ __forceinline__ Piece piece_at(const DecodeArgs &a, const Plan &p, int x, int hi,
                                          int wg) {
  const int *cum = MANY ? p.cum_many : p.cum;
  int lo = 0, up = MANY ? kMaxList : 2 * kMaxList;   // cum[lo] <= x < cum[up]
  while (up - lo > 1) {
    const int mid = (lo + up) / 2;
    if (cum[mid] <= x) lo = mid;
    else up = mid;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Piece r;
  r.shared = MANY || lo < kMaxList;
  const int e = r.shared ? lo : lo - kMaxList;
  const int g = r.shared ? e : a.group[e];
  const int prefix = p.prefix[g];
  int rows, base;
  if (r.shared) {
    r.row = a.slot[min(p.lead[e], kMaxList - 1)];
    r.key0 = 0;
    r.limit = r.vis = prefix;
    rows = group_rows(a, e);
    r.token0 = a.start[e] * a.nq;
    base = prefix_base(a, e, MANY);
  } else {
    r.row = a.slot[e];
    r.key0 = prefix;
    r.limit = p.len[e];
    r.vis = r.limit - a.nq + 1;
    rows = a.G * a.nq;
    r.token0 = e * a.nq;
    base = e * a.hkv * row_tiles(rows);
  }
  r.n = tiles_of(r.limit - r.key0);
  const int rt = row_tiles(rows);
  const int off = x - cum[lo];
  const int seg = off / r.n;               // (KV head, row tile) of the segment
  r.head = seg / rt;
  r.row0 = (seg - r.head * rt) * kDecodeRows;
  r.rows = min(rows - r.row0, kDecodeRows);
  r.t0 = off - seg * r.n;
  r.t1 = min(r.n, r.t0 + hi - x);
  r.end = x + r.t1 - r.t0;
  r.slot = wg + base + seg;
  r.whole = !r.shared && prefix == 0 && r.t0 == 0 && r.t1 == r.n;
  return r;
}

__device__ __forceinline__ Piece uniform(const Piece &r) {
  Piece u;
  u.end = __builtin_amdgcn_readfirstlane(r.end);
  u.row = __builtin_amdgcn_readfirstlane(r.row);
  u.head = __builtin_amdgcn_readfirstlane(r.head);
  u.t0 = __builtin_amdgcn_readfirstlane(r.t0);
  u.t1 = __builtin_amdgcn_readfirstlane(r.t1);
  u.n = __builtin_amdgcn_readfirstlane(r.n);
  u.key0 = __builtin_amdgcn_readfirstlane(r.key0);
  u.limit = __builtin_amdgcn_readfirstlane(r.limit);
  u.row0 = __builtin_amdgcn_readfirstlane(r.row0);
  u.rows = __builtin_amdgcn_readfirstlane(r.rows);
  u.token0 = __builtin_amdgcn_readfirstlane(r.token0);
  u.vis = __builtin_amdgcn_readfirstlane(r.vis);
  u.shared = __builtin_amdgcn_readfirstlane(r.shared);
  u.slot = __builtin_amdgcn_readfirstlane(r.slot);
  u.whole = __builtin_amdgcn_readfirstlane(r.whole);
  return u;
}

template <int D>
struct DecGeo {
  static constexpr int OCC = D == 64 ? 3 : 2;      // workgroups per CU = waves per SIMD
  static constexpr int RB = 2 * D;                 // bytes per key row
  static constexpr int BYTES = kKeys * RB;         // a tile of K or of V
  static constexpr int DMA = BYTES / 4 / 1024;     // 1 KB copies per wave and tile
  static constexpr int CPR = RB / 16;
  static constexpr int RPI = 1024 / RB;            // key rows per copy
};

// MANY: the line of prefixes with more than kDecodeFew rows, every wave with rows of its own and
// both 32-key halves of a tile under one update of the reference.  Otherwise halves are taken one
// at a time, by different waves where there are rows for two of them or for one.
template <int D, bool MANY>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(DecGeo<D>::OCC, DecGeo<D>::OCC)))
void decode_fwd(DecodeArgs a) {
  constexpr int NB = MANY ? 2 : 1;        // 32-key halves under one update
  using S = DecGeo<D>;
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * S::BYTES];   // [2 tiles][K, V]
  __shared__ Plan plan;
  __shared__ float2 s_ml[2][64];
  __shared__ Piece s_next;
  __shared__ int s_odd[2][4];             // per tile buffer: a wave's keys hold such a value
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  make_plan(a, plan);
  const int total =
      __builtin_amdgcn_readfirstlane(MANY ? plan.cum_many[kMaxList] : plan.cum[2 * kMaxList]);
  // workgroups of one XCD (every eighth) take neighbouring parts of the line, which share keys;
  // with fewer tiles than workgroups, one tile each
  const int wgs = min(a.wgs, total);
  int wg = blockIdx.x;
  if (wgs == a.wgs) wg = (wg & 7) * (a.wgs / 8) + (wg >> 3);
  if (wg >= wgs) return;
  const int hi = cut(total, wgs, wg + 1);

  // DMA offsets of this wave's 16 keys: K rows with swizzled chunks, V^T in fragment order
  uint32_t koff[S::DMA];
#pragma unroll
  for (int i = 0; i < S::DMA; ++i) {
    const int r = 16 * w + i * S::RPI + lane / S::CPR;
    koff[i] = (i * S::RPI + lane / S::CPR) * S::RB + swz_k<D>(lane % S::CPR, r) * 16 - i * 1024;
  }
  const int vd = 8 * (lane >> 4) + (lane & 7), vh = ((lane >> 3) ^ (lane >> 4)) & 1;
  const uint32_t voff = (2 * vd + vh) * 16;
  const uint32_t vaddr = 16 * vt_unit(lr, lh);
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;

  // table entry of this wave's 16 keys of tile t; loaded a tile ahead and first looked at in
  // `issue`, so that nothing waits for it
  auto page_of = [&](const Piece &r, int t) {
    const int key = min(r.key0 + kKeys * t + 16 * w, r.limit - 1);
    return a.table[(int64_t)r.row * a.max_pages + (key >> a.page_shift)];
  };
  auto issue = [&](const Piece &r, int t, int pg, int into) {
    const int key = r.key0 + kKeys * t + 16 * w;
    if (key >= r.limit) return;           // past the segment: those keys are masked
    pg = min(max(__builtin_amdgcn_readfirstlane(pg), 0), a.pages - 1);
    const int64_t off = ((((int64_t)pg * a.hkv + r.head) << a.page_shift) +
                         (key & ((1 << a.page_shift) - 1))) * D;
    const __amdgpu_buffer_rsrc_t rk = uniform_rsrc(a.k + off, 16 * S::RB);
    const __amdgpu_buffer_rsrc_t rv = uniform_rsrc(a.v + off, 16 * S::RB);
    uint8_t *dst = lds + into * 2 * S::BYTES + w * 16 * S::RB;
    dma_slots<0, S::DMA>(rk, (__attribute__((address_space(3))) void *)dst, koff);
    dma_slots<0, S::DMA>(rv, (__attribute__((address_space(3))) void *)(dst + S::BYTES), voff);
  };
  auto barrier = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  Piece cur = uniform(piece_at<MANY>(a, plan, cut(total, wgs, wg), hi, wg));
  int buf = 0;
  issue(cur, cur.t0, page_of(cur, cur.t0), 0);
  int page_next = page_of(cur, min(cur.t0 + 1, cur.t1 - 1));
  while (true) {
    // ---- rows of this wave, and the half of a tile that it takes (both with `four`)
    const bool four = MANY || cur.rows > 64;
    const int rb = four ? w : cur.rows > 32 ? w >> 1 : 0;
    const bool active = four ? 32 * w < cur.rows : cur.rows > 32 || w < 2;
    const int half = w & 1;
    const int row = 32 * rb + lr;                       // within the row tile
    const int srow = cur.row0 + min(row, cur.rows - 1); // within the segment
    const int tok = srow / a.G;
    const int kk = srow - tok * a.G;
    const int64_t token = cur.token0 + tok;
    bf16x8 qf[KS];
    {
      const uint16_t *qp = a.q + token * a.q_stride + (cur.head * a.G + kk) * D + 8 * lh;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const bf16x8 *>(qp + 16 * k);
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(qf[k]));
    const int lim = cur.shared ? cur.limit : cur.vis + tok;   // keys that this lane's row sees
    f32x16 oacc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) oacc[i] = f32x16{};
    float m_ref = -INFINITY, mc = 0.f, m_trig = -INFINITY, l_run = 0.f;
    const bool more = cur.end < hi;
    if (more) {                           // published by the first tile's barrier
      const Piece nxt = piece_at<MANY>(a, plan, cur.end, hi, wg);
      if (tid == 0) s_next = nxt;
    }

    // NB 32-key halves of the tile in `buf`, from half h0 on
    auto compute = [&](int h0, int k0) {
      const uint8_t *ks = lds + buf * 2 * S::BYTES + h0 * 32 * S::RB;
      const uint8_t *vs = lds + (buf * 2 + 1) * S::BYTES + h0 * 32 * S::RB + vaddr;
      k0 += 32 * h0;
      f32x16 sacc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        bf16x8 kf[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k)
          kf[k] = *reinterpret_cast<const bf16x8 *>(ks + kaddr[k] + b * 32 * S::RB);
        sacc[b] = f32x16{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
          sacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[k], sacc[b], 0, 0, 0);
      }
      const bool edge = k0 + 32 * NB > cur.vis;         // some row does not see every key
      if (edge) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (k0 + 32 * b + 16 * (v >> 3) + 8 * lh + (v & 7) >= lim) sacc[b][v] = -INFINITY;
      }
      float mt = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sacc[b][v]);
      // the reference moves only when a score rises 2^kLazy above it in weight
      if (__ballot(mt > m_trig)) {
        const float m_new = fmaxf(m_ref, wave_pair_max(mt));
        const float a2 = m_ref == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        l_run *= a2;
#pragma unroll
        for (int i = 0; i < DB; ++i) oacc[i] *= a2;
        m_ref = m_new;
        const bool none = m_new == -INFINITY;
        mc = none ? 0.f : m_new * c;
        m_trig = none ? -INFINITY : m_new + lazy_raw;
      }
      // Weights: with few rows the keys' bytes bound the kernel, and a weight is the sum of two
      // bf16 numbers, its error 2^-17; with many the products do, and it is one, as in the prefill,
      // its error 2^-8 in O and in the sum alike.
      bf16x8 pf[2 * NB], pl[2 * NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float wt = __builtin_amdgcn_exp2f(fmaf(sacc[b][v], c, -mc));
          const __bf16 top = (__bf16)wt;
          pf[2 * b + (v >> 3)][v & 7] = top;
          if constexpr (!MANY) pl[v >> 3][v & 7] = (__bf16)(wt - (float)top);
        }
      l_run = sum_weights(pf, l_run);
      if constexpr (!MANY) l_run = sum_weights(pl, l_run);
#pragma unroll
      for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const bf16x8 vf = *reinterpret_cast<const bf16x8 *>(vs + db * 1024 + t * 32 * D);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t], oacc[db], 0, 0, 0);
          if constexpr (!MANY)
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl[t], oacc[db], 0, 0, 0);
        }
      if (!MANY && edge && (s_odd[buf][0] | s_odd[buf][1] | s_odd[buf][2] | s_odd[buf][3])) {
        // the values that settle_edge took out, for the rows that see them
        const int32_t *table = a.table + (int64_t)cur.row * a.max_pages;
        for (int key = max(cur.vis, k0); key < min(cur.limit, k0 + 32 * NB); ++key) {
          float wt = 0.f;
#pragma unroll
          for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (k0 + 16 * t + 8 * lh + e == key) wt = (float)pf[t][e];
          wt = wave_pair_sum(wt);
          if (key >= lim) continue;
          const int pg = min(max(table[key >> a.page_shift], 0), a.pages - 1);
          const uint16_t *vp = a.v + ((((int64_t)pg * a.hkv + cur.head) << a.page_shift) +
                                      (key & ((1 << a.page_shift) - 1) & ~15)) * D + (key & 15);
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const uint32_t x = vp[16 * (32 * db + 8 * (v >> 2) + 4 * lh + (v & 3))];
              if ((x & 0x7F80) == 0x7F80) oacc[db][v] = fmaf(wt, __uint_as_float(x << 16), oacc[db][v]);
            }
        }
      }
    };
    // This wave's 16 keys of a tile that some row does not see whole, before the others read
    // them.  Values past the segment may hold anything, NaN among it, which a weight of zero
    // would not cancel: they become zero.  So do infinities and NaN of tokens that only later
    // queries see; the rows that see them take them separately (s_odd).
    auto settle_edge = [&](int k0) {
      uint8_t *vs = lds + (buf * 2 + 1) * S::BYTES + w * 32 * D;
      bool odd = false;
      for (int i = 0; i < 2 * D / 64; ++i) {
        const int u = 64 * i + lane;      // unit (d, vh) of the step, see voff
        const int key = k0 + 16 * w + 8 * (((u >> 3) ^ (u >> 4)) & 1);
        s16x8 x = *reinterpret_cast<const s16x8 *>(vs + 16 * u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool out = key + e >= cur.limit;
          const bool late = key + e >= cur.vis && (x[e] & 0x7F80) == 0x7F80;
          odd |= late && !out;
          if (out || late) x[e] = 0;
        }
        *reinterpret_cast<s16x8 *>(vs + 16 * u) = x;
      }
      const bool any = __ballot(odd) != 0;
      if (lane == 0) s_odd[buf][w] = any;
    };

    for (int t = cur.t0; t < cur.t1; ++t) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's part of tile t is here
      const int k0 = cur.key0 + kKeys * t;
      if (k0 + kKeys > cur.vis) settle_edge(k0);
      barrier();                                         // ... and every wave's
      if (t + 1 < cur.t1) {
        issue(cur, t + 1, page_next, buf ^ 1);
        page_next = page_of(cur, min(t + 2, cur.t1 - 1));
      } else if (more) {
        const Piece nxt = uniform(s_next);
        issue(nxt, nxt.t0, page_of(nxt, nxt.t0), buf ^ 1);
        page_next = page_of(nxt, min(nxt.t0 + 1, nxt.t1 - 1));
      }
      if constexpr (MANY) {
        if (active) compute(0, k0);
      } else if (active) {
        for (int h = four ? 0 : half; h < (four ? 2 : half + 1); ++h)
          if (k0 + 32 * h < cur.limit) compute(h, k0);
      }
      buf ^= 1;
    }

    // ---- the two key halves of a row joined in LDS (in the tile just used)
    float l_tot = wave_pair_sum(l_run);
    if (!MANY && !four) {
      barrier();
      float *box = reinterpret_cast<float *>(lds + (buf ^ 1) * 2 * S::BYTES) +
                   (w >> 1) * 64 * 16 * DB;
      if (active && half == 1) {
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) box[(16 * i + v) * 64 + lane] = oacc[i][v];
        s_ml[w >> 1][lane] = make_float2(m_ref, l_tot);
      }
      barrier();
      if (active && half == 0) {
        const float2 other = s_ml[w >> 1][lane];
        const float m_new = fmaxf(m_ref, other.x);
        const float f0 = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        const float f1 =
            other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((other.x - m_new) * c);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            oacc[i][v] = fmaf(f1, box[(16 * i + v) * 64 + lane], f0 * oacc[i][v]);
        l_tot = f0 * l_tot + f1 * other.y;
        m_ref = m_new;
      }
    }
    // ---- lane holds row `row`, d = 32 db + 8 (v / 4) + 4 lh + v % 4
    if (active && (four || half == 0) && row < cur.rows) {
      if (cur.whole) {
        const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
        uint16_t *op = a.o + (token * a.hq + cur.head * a.G + kk) * D + 4 * lh;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 ov;
#pragma unroll
            for (int e = 0; e < 4; ++e) ov[e] = (__bf16)(oacc[db][4 * g + e] * inv);
            *reinterpret_cast<bf16x4 *>(op + 32 * db + 8 * g) = ov;
          }
      } else {
        const int slot_rows =
            MANY ? kDecodeRows : cur.shared ? kDecodeFew : min(a.G * a.nq, kDecodeRows);
        float *to = (MANY ? a.part_many : cur.shared ? a.part_few : a.part_own) +
                    (int64_t)cur.slot * slot_rows * (D + 2);
        if (lh == 0) *reinterpret_cast<float2 *>(to + slot_rows * D + 2 * row) =
            make_float2(m_ref, l_tot);
        to += row * D + 4 * lh;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4 *>(to + 32 * db + 8 * g) =
                make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2],
                            oacc[db][4 * g + 3]);
      }
    }
    if (!more) return;
    cur = uniform(s_next);
    barrier();                            // read by all before it is written again
  }
}

// Joins the pieces of every row: one wave per row, D / 64 elements per lane; lane i first takes
// the reference and weight sum of piece i.
template <int D>
__global__ __launch_bounds__(kThreads) void decode_join(DecodeArgs a) {
  __shared__ Plan plan;
  make_plan(a, plan);
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (int64_t)a.batch * a.nq * a.hq) return;
  const int token = (int)(id / a.hq), qh = (int)(id - (int64_t)token * a.hq);
  const int b = token / a.nq, head = qh / a.G, kk = qh - head * a.G;
  const int g = a.group[b], prefix = plan.prefix[g], len = plan.len[b];
  uint16_t *op = a.o + id * D;
  constexpr int E = D / 64;
  const float c = a.scale_log2;
  if (len == 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) op[lane * E + e] = 0;
    return;
  }
  const bool many = is_many(a, g);
  // segment of the row and its pieces, for the prefix (kind 0) and its own keys (1)
  int first[2], count[2], row[2];
  int64_t slot[2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const int rows = kind == 0 ? group_rows(a, g) : a.G * a.nq;
    const int r = kind == 0 ? ((b - a.start[g]) * a.nq + token - b * a.nq) * a.G + kk
                            : (token - b * a.nq) * a.G + kk;
    const int n = tiles_of(kind == 0 ? prefix : len - prefix);
    const int rt = row_tiles(rows), seg = head * rt + r / kDecodeRows;
    const bool line = kind == 0 && many;
    const int total = line ? plan.cum_many[kMaxList] : plan.cum[2 * kMaxList];
    const int wgs = min(a.wgs, total);
    const int x =
        (line ? plan.cum_many[g] : plan.cum[kind == 0 ? g : kMaxList + b]) + seg * n;
    first[kind] = n ? owner(total, wgs, x) : 0;
    count[kind] = n ? owner(total, wgs, x + n - 1) - first[kind] + 1 : 0;
    row[kind] = r % kDecodeRows;
    slot[kind] = (kind == 0 ? prefix_base(a, g, many) : b * a.hkv * rt) + seg;
  }
  if (prefix == 0 && count[1] == 1) return;       // finished by its workgroup
  const int own_rows = min(a.G * a.nq, kDecodeRows);
  const int n = count[0] + count[1];
  // partial i of the row: its floats, and its reference and weight sum
  auto part = [&](int i, const float *&ml) {
    const int kind = i >= count[0];
    const int slot_rows = kind ? own_rows : many ? kDecodeRows : kDecodeFew;
    const float *base = (kind ? a.part_own : many ? a.part_many : a.part_few) +
                        (slot[kind] + first[kind] + (kind ? i - count[0] : i)) * slot_rows * (D + 2);
    ml = base + slot_rows * D + 2 * row[kind];
    return base + row[kind] * D;
  };
  float m = -INFINITY, l = 0.f, acc[E] = {};
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int k = min(64, n - i0);
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < k) {
      const float *at;
      part(i0 + lane, at);
      ml = *reinterpret_cast<const float2 *>(at);
    }
    float top = fmaxf(m, ml.x);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float old = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml.x - top) * c);
    float sum = f * ml.y;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    l = l * old + sum;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= old;
    m = top;
    for (int i = 0; i < k; ++i) {
      const float *unused;
      const float *at = part(i0 + i, unused) + lane * E;
      const float fi = __shfl(f, i);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(fi, at[e], acc[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e)
    op[lane * E + e] = __builtin_bit_cast(uint16_t, (__bf16)(acc[e] * inv));
}

template <int D>
hipError_t launch(const DecodeArgs &a, hipStream_t s) {
  if (a.any_many) {
    decode_fwd<D, true><<<a.wgs, kThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  decode_fwd<D, false><<<a.wgs, kThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)a.batch * a.nq * a.hq;
  decode_join<D><<<(int)((rows + 3) / 4), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_attn(const DecodeArgs &a, int d, hipStream_t s) {
  return d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace fp
