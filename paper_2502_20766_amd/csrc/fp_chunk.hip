// Causal attention of chunks of new tokens over a paged cache: o = softmax(c q K^T) V, where query t of
// m of a sequence of n tokens sees its keys 0 .. n - m + t.
//
// The rows of a sequence and KV head are its queries times the query heads of that KV head, a token's
// heads one after the other, in tiles of 128 rows: keys are so read once for all heads that share
// them, and few of a tile's rows end within another key tile than its last one.  Tiles of 64 keys go
// through LDS, double buffered; a wave has 32 rows, and its products are those of the prefill, on
// v_mfma_f32_32x32x16_bf16: S^T = K Q^T with K rows permuted so that a lane's scores are the
// consecutive keys that P^T of O^T += V^T P^T needs, one update of the reference for 64 keys.
#include <type_traits>

#include "fp_attn_dev.h"
#include "fp_internal.h"
#include "fp_paged_dev.h"

namespace fp {
namespace {

constexpr int kThreads = 256;

// The rows of one row tile and the keys that they see; every field is wave-uniform.
struct Piece {
  int row;              // cache slot whose pages are read
  int head;             // KV head
  int t0, t1;           // tiles [t0, t1) of its keys
  int key0, limit;      // keys: first, and the sequence's tokens
  int row0, rows;       // rows of the sequence and KV head: first, and how many
  int token0;           // row of q of the sequence's first query
  int vis;              // keys that the sequence's first query sees (may be negative)
  int seen;             // keys that the first row of the tile sees
  int once;
};

// Scores of 64 keys for the rows of a wave, its weights and O.
template <int D>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(PagedGeo<D>::OCC, PagedGeo<D>::OCC)))
void chunk_fwd(ChunkArgs a) {
  using S = PagedGeo<D>;
  constexpr int KS = D / 16, DB = D / 32, TILE = 4 * S::STEP;
  // K and V of even tiles in lds0, of odd ones in lds1: two arrays, so that the compiler sees that
  // reads of one do not wait for copies into the other
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[2 * TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[2 * TILE];
  __shared__ int s_seq, s_odd[2];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const float c = a.scale_log2;
  const float lazy_raw = fminf(kLazy / c, 3.0e38f);
  // ---- the tile: KV head blockIdx.x % hkv of the row tile blockIdx.x / hkv
  const int item = blockIdx.x / a.hkv;
  if (tid < a.batch && a.tile[tid] <= item && item < a.tile[tid + 1]) s_seq = tid;
  if (tid < 2) s_odd[tid] = 0;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(s_seq);
  const int m = a.cu[b + 1] - a.cu[b];
  Piece cur;
  cur.row = a.slot[b];
  cur.head = blockIdx.x - item * a.hkv;
  cur.key0 = 0;
  cur.limit = cur.row < 0 ? 0 : min(max(a.len[cur.row], 0), a.max_pages << a.page_shift);
  cur.limit = __builtin_amdgcn_readfirstlane(cur.limit);
  cur.row0 = (item - a.tile[b]) * kChunkRows;
  cur.rows = min(m * a.G - cur.row0, kChunkRows);
  cur.token0 = a.cu[b];
  cur.vis = cur.limit - m + 1;
  cur.seen = max(cur.vis + cur.row0 / a.G, 0);
  const int last = max(cur.vis + (cur.row0 + cur.rows - 1) / a.G, 0);   // keys of the last row
  cur.t0 = 0;
  cur.t1 = (last + kKeys - 1) / kKeys;
  cur.once = m * a.G <= kChunkRows;

  const Loader<D> load(w, lane);
  auto issue = [&](int t, int pg, uint8_t *into) {
    uint8_t *k = into + w * S::STEP;
    load.issue(a, cur, t, pg, k, k + TILE);
  };
  const int kr = (lr & ~12) | ((lr >> 1) & 4) | ((lr << 1) & 8);
  uint32_t kaddr[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) kaddr[k] = kr * S::RB + swz_k<D>(2 * k + lh, kr) * 16;
  const uint32_t vaddr = TILE + 16 * vt_unit(lr, lh);

  const bool active = 32 * w < cur.rows;
  const int row = 32 * w + lr;
  const int srow = cur.row0 + min(row, cur.rows - 1);
  const int tok = srow / a.G;
  const int64_t at = (int64_t)(cur.head * a.G + srow - tok * a.G) * D;
  const int lim = cur.vis + tok;          // keys that this lane's row sees
  const int lim_w = __builtin_amdgcn_readfirstlane(cur.vis + (cur.row0 + 32 * w) / a.G);
  int page_next = 0;
  if (cur.t0 < cur.t1) {
    issue(cur.t0, load.page(a, cur, cur.t0), lds0);
    page_next = load.page(a, cur, min(cur.t0 + 1, cur.t1 - 1));
  }
  const uint16_t *qp = a.q + (int64_t)(cur.token0 + tok) * a.q_stride + at + 8 * lh;
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
    const int k0 = kKeys * t;
    wait_copies();                                     // this wave's part of tile t is here
    const bool edge = k0 + kKeys > cur.seen;           // some row does not see all of it
    if (edge &&
        settle<D>(tile + TILE + w * S::STEP, k0 + 16 * w, cur.limit, cur.seen, lane) && lane == 0)
      s_odd[t & 1] = t + 1;
    wg_barrier();                                      // ... and every wave's
    if (t + 1 < cur.t1) {
      issue(t + 1, page_next, next);
      page_next = load.page(a, cur, min(t + 2, cur.t1 - 1));
    }
    if (!active) return;
    f32x16 sacc[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bf16x8 kf[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k)
        kf[k] = *reinterpret_cast<const bf16x8 *>(tile + kaddr[k] + i * 32 * S::RB);
      sacc[i] = f32x16{};
#pragma unroll
      for (int k = 0; k < KS; ++k)
        sacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[k], sacc[i], 0, 0, 0);
    }
    if (k0 + kKeys > lim_w) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (k0 + 32 * i + 16 * (v >> 3) + 8 * lh + (v & 7) >= lim) sacc[i][v] = -INFINITY;
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
            *reinterpret_cast<const bf16x8 *>(tile + vaddr + db * 1024 + t4 * S::STEP);
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t4], oacc[db], 0, 0, 0);
      }
    if (edge && s_odd[t & 1] == t + 1) {                    // the values that settle took out
      for (int key = max(cur.seen, k0); key < min(cur.limit, k0 + kKeys); ++key) {
        const int pg = min(max(a.table[(int64_t)cur.row * a.max_pages + (key >> a.page_shift)], 0),
                           a.pages - 1);
        const uint16_t *vp = a.v + ((((int64_t)pg * a.hkv + cur.head) << a.page_shift) +
                                    (key & ((1 << a.page_shift) - 1) & ~15)) * D + (key & 15);
        float wt = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (k0 + 16 * i + 8 * lh + e == key) wt = (float)pf[i][e];
        wt = wave_pair_sum(wt);
        if (key >= lim) continue;
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
  // (in pairs: a branch on the buffer in every step would move O from register to register)
  int t = cur.t0;
  for (; t + 2 <= cur.t1; t += 2) {
    step(lds0, lds1, t);
    step(lds1, lds0, t + 1);
  }
  if (t < cur.t1) step(lds0, lds1, t);

  // ---- lane holds row `row`, d = 32 db + 8 (v / 4) + 4 lh + v % 4
  const float l = wave_pair_sum(l_run);
  if (row < cur.rows) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *op = a.o + (int64_t)(cur.token0 + tok) * a.hq * D + at + 4 * lh;
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
}

template <int D>
hipError_t launch(const ChunkArgs &a, hipStream_t s) {
  chunk_fwd<D><<<a.tile[a.batch] * a.hkv, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkArgs &a, int d, hipStream_t s) {
  return d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace fp
