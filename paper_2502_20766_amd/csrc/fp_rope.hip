// Norms of query and key heads and the rotation by their positions, by themselves and on the way into
// the paged cache.
//
// y = x rsqrt(mean(x^2) + eps) w over a head (or y = x), then for pair i of the first R elements, at
// position p with frequency f_i:
//   (u, v) -> A (u cos p f_i - v sin p f_i, v cos p f_i + u sin p f_i).
// All in float32, rounded once.  The angle is held as a fraction of a turn: p times round(2^64 f_i /
// 2 pi), modulo 2^64, which is off by at most 2^-34 of a turn at any position; its upper 32 bits give a
// quadrant and an angle within pi / 4, of which sine and cosine are the Taylor series.
//
// Memory bounds it: every head is read and written once, by 16-byte chunks, and nothing else is read but a
// position a token (131072 tokens of 40 heads of 128 with norms 494 us, 5.4 TB/s; appends of 64k tokens 256
// us, 5.3 TB/s).  Small calls take the time of a launch, 8-11 us.
#include <algorithm>
#include <type_traits>

#include "fp_cache_dev.h"

namespace fp {
namespace {

constexpr int kThreads = 256;

// D / 16 lanes have a head, each two 16-byte chunks of it: both elements of the pairs that it turns.
template <int D>
struct Lane {
  static constexpr int PER = D / 16;      // lanes per head
  static constexpr int HEADS = 64 / PER;  // heads per wave
  int a, b;                               // chunks
  bool turns;                             // they are rotated
  __device__ __forceinline__ Lane(int j, int rotary) {
    const int r = rotary / 16;
    turns = j < r;
    a = turns ? j : j + r;
    b = a + (turns ? r : PER - r);
  }
};

// Cosine and sine of the lane's eight pairs at position `pos`.
template <int D, bool HALF>
__device__ __forceinline__ void turn_of(const RopeArgs &r, const Lane<D> &l, int pos, float (&cs)[8],
                                        float (&sn)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int pair = HALF ? 8 * l.a + e : e < 4 ? 4 * l.a + e : 4 * l.b + e - 4;
    const uint64_t turns = (uint64_t)(int64_t)pos * r.step[l.turns ? pair : 0];
    const uint32_t u = (uint32_t)(turns >> 32);
    const uint32_t quad = (u + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(u - (quad << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float x2 = x * x;
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880.f, -1.f / 5040.f),
                                               1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f),
                                  -0.5f), 1.f);
    const float cq = quad & 1 ? s : c, sq = quad & 1 ? c : s;
    cs[e] = r.amplitude * ((quad + 1) & 2 ? -cq : cq);
    sn[e] = r.amplitude * (quad & 2 ? -sq : sq);
  }
}

__device__ __forceinline__ void widen(Unit x, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(x[i] << 16);
    y[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ Unit narrow(const float (&y)[8]) {
  Unit x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __bf16 lo = (__bf16)y[2 * i], hi = (__bf16)y[2 * i + 1];
    x[i] = __builtin_bit_cast(uint16_t, lo) | (uint32_t)__builtin_bit_cast(uint16_t, hi) << 16;
  }
  return x;
}

// Sum over the D / 16 lanes of a head.
template <int D>
__device__ __forceinline__ float head_sum(float x) {
  auto moved = [](float v, auto ctrl) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value,
                                                       0xf, 0xf, true));
  };
  x += moved(x, std::integral_constant<int, 0xB1>{});     // lanes 1 0 3 2 of four
  x += moved(x, std::integral_constant<int, 0x4E>{});     // lanes 2 3 0 1
  if constexpr (D == 128) x += moved(x, std::integral_constant<int, 0x141>{});   // 7 - i of eight
  return x;
}

__device__ __forceinline__ void weights(const RopeArgs &r, const void *w, int chunk, float (&y)[8]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = 1.f;
  } else if (r.w_f32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = ((const float *)w)[8 * chunk + e];
  } else {
    widen(((const Unit *)w)[chunk], y);
  }
}

// The lane's part of a head, in place.  `w`: the norm's weights or null.
template <int D, bool NORM, bool HALF>
__device__ __forceinline__ void turn(const RopeArgs &r, const Lane<D> &l, const void *w,
                                     const float (&cs)[8], const float (&sn)[8], Unit &a, Unit &b) {
  float x[8], y[8];
  widen(a, x);
  widen(b, y);
  if constexpr (NORM) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
    const float inv = __builtin_amdgcn_rsqf(fmaf(head_sum<D>(sum), 1.f / D, r.eps));
    float wx[8], wy[8];
    weights(r, w, l.a, wx);
    weights(r, w, l.b, wy);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] *= inv * wx[e];
      y[e] *= inv * wy[e];
    }
  }
  if (l.turns) {
    if constexpr (HALF) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = x[e], v = y[e];
        x[e] = u * cs[e] - v * sn[e];
        y[e] = v * cs[e] + u * sn[e];
      }
    } else {
      auto pairs = [&](float (&z)[8], int first) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = z[2 * e], v = z[2 * e + 1];
          z[2 * e] = u * cs[first + e] - v * sn[first + e];
          z[2 * e + 1] = v * cs[first + e] + u * sn[first + e];
        }
      };
      pairs(x, 0);
      pairs(y, 4);
    }
  }
  a = narrow(x);
  b = narrow(y);
}

// Heads of one token, by a wave: chunks of 64 / (D / 16) heads, kBatch at a time, whose loads are in flight
// together (9001 tokens of 34 heads 36.1 us; one at a time 37.4, four at a time 37.2).  `from` and `to`: a
// head's places, `weight` its norm's weights; `first` runs once the first loads are on their way.  A lane
// has head `mine` of each chunk, and loads another in its place where there is none.
constexpr int kBatch = 2;

template <int D, bool NORM, bool HALF, class From, class To, class Weight, class First>
__device__ __forceinline__ void turn_heads(const RopeArgs &r, const Lane<D> &l, int heads, int mine,
                                           int chunk0, int chunk_step, const float (&cs)[8],
                                           const float (&sn)[8], const From &from, const To &to,
                                           const Weight &weight, const First &first) {
  using L = Lane<D>;
  for (int h0 = chunk0 * L::HEADS, begun = 0; h0 < heads; h0 += kBatch * chunk_step * L::HEADS) {
    Unit x[kBatch], y[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i * chunk_step * L::HEADS;
      if (h >= heads) break;
      const Unit *at = (const Unit *)from(min(h + mine, heads - 1));
      x[i] = at[l.a];
      y[i] = at[l.b];
    }
    if (!begun) first();
    begun = 1;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i * chunk_step * L::HEADS;
      if (h >= heads) break;
      const int head = min(h + mine, heads - 1);
      turn<D, NORM, HALF>(r, l, weight(head), cs, sn, x[i], y[i]);
      if (h + mine < heads) {
        Unit *at = (Unit *)to(head);
        at[l.a] = x[i];
        at[l.b] = y[i];
      }
    }
  }
}

// Of what has fewer heads than a wave holds it takes `set` tokens, the lane that of number `token` of them
// and its head `head`.
template <int D>
struct Place {
  int token, head;
  __device__ __forceinline__ Place(int set, int heads) {
    const int i = (threadIdx.x & 63) / Lane<D>::PER;
    token = set > 1 ? i / heads : 0;
    head = i - token * heads;
    if (set > 1 && token >= set) token = 0, head = heads;
  }
};

template <int D>
int set_of(int heads) {
  return std::max(1, Lane<D>::HEADS / heads);
}

// ---- rotate: a wave takes one token, or of few tokens a chunk of the heads (a.groups waves to a token),
// or of few heads several tokens (33348 tokens of 3 heads of 64 31.4 us a token at a time, 12.9 five).
template <int D, bool NORM, bool HALF>
__global__ __launch_bounds__(kThreads) void rotate_heads(RotateArgs a) {
  using L = Lane<D>;
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int64_t unit = wave / a.groups, token0 = unit * a.set;
  if (token0 >= a.tokens) return;
  const int heads = a.hq + a.hkv;
  Place<D> place(a.set, heads);
  if (token0 + place.token >= a.tokens) place.token = 0, place.head = heads;
  const int64_t token = token0 + place.token;
  const L l(lane % L::PER, a.rope.rotary);
  const int pos = a.positions ? a.positions[token] : 0;
  float cs[8], sn[8];
  turn_heads<D, NORM, HALF>(
      a.rope, l, heads, place.head, (int)(wave - unit * a.groups), a.groups, cs, sn,
      [&](int h) {
        return h < a.hq ? a.q + token * a.q_stride + h * D : a.k + token * a.k_stride + (h - a.hq) * D;
      },
      [&](int h) {
        return h < a.hq ? a.qo + token * a.qo_stride + h * D
                        : a.ko + token * a.ko_stride + (h - a.hq) * D;
      },
      [&](int h) { return h < a.hq ? a.rope.wq : a.rope.wk; },
      [&]() { turn_of<D, HALF>(a.rope, l, pos, cs, sn); });
}

// ---- append: as cache_write, a workgroup has the new tokens among 64 positions of one slot, and of
// them one KV head or a part of the queries (x.query_tokens positions, all heads: eight, or more of few
// heads, so that a wave has two chunks).
template <int D>
int query_tokens(int heads) {
  int n = 8;
  while (2 * n <= std::min(64, 8 * set_of<D>(heads))) n *= 2;
  return n;
}

template <int D, bool NORM, bool HALF>
__global__ __launch_bounds__(kThreads) void cache_append(CacheView c, AppendArgs x) {
  using L = Lane<D>;
  constexpr int CPR = D / 8;                 // 16-byte chunks per row
  constexpr int KU = 64 * L::PER / kThreads, VU = 64 * CPR / kThreads;
  const WriteArgs &a = x.w;
  __shared__ __attribute__((aligned(16))) uint16_t tile[64][D + 8];
  __shared__ int s_i, s_page[4];
  const int per = c.hkv + (x.q ? 64 / x.query_tokens : 0);
  const int blk = blockIdx.x / per, h = blockIdx.x - blk * per, tid = threadIdx.x;
  if (tid < a.list.n && a.blk[tid] <= blk && blk < a.blk[tid + 1]) s_i = tid;
  const int error = c.state[1];
  __syncthreads();
  const int i = __builtin_amdgcn_readfirstlane(s_i);
  if (error & (FP_CACHE_FULL | FP_CACHE_TOO_LONG | FP_CACHE_SKIPPED)) return;
  const int row0 = a.list.num[i], n = a.list.num[i + 1] - row0;
  const int slot = a.list.slot[i];
  const int len = min(c.len[slot], c.max_pages << c.page_shift);
  const int start = len - n;                 // position of the first row
  const int p0 = (max(start, 0) & ~63) + 64 * (blk - a.blk[i]);
  const int lo = max(start, p0), end = min(len, p0 + 64);
  if (lo >= end) return;
  float cs[8], sn[8];
  if (h >= c.hkv) {                          // queries
    const int lane = tid & 63;
    const L l(lane % L::PER, x.rope.rotary);
    const int t0 = max(p0 + x.query_tokens * (h - c.hkv), lo);
    const int t1 = min(p0 + x.query_tokens * (h - c.hkv + 1), end);
    const Place<D> place(x.set, x.hq);
    for (int t = t0 + x.set * (tid >> 6); t < t1; t += x.set * (kThreads / 64)) {
      const bool mine = t + place.token < t1;
      const int at = mine ? t + place.token : t;
      const int64_t row = row0 + (at - start);
      turn_heads<D, NORM, HALF>(
          x.rope, l, x.hq, mine ? place.head : x.hq, 0, 1, cs, sn,
          [&](int qh) { return x.q + row * x.q_stride + qh * D; },
          [&](int qh) { return x.qo + row * x.qo_stride + qh * D; }, [&](int) { return x.rope.wq; },
          [&]() { turn_of<D, HALF>(x.rope, l, at, cs, sn); });
    }
    return;
  }
  auto tile_of = [&](int p, int t) {         // element offset of position t's 16-token step
    return ((((int64_t)a.layer * c.pages + p) * c.hkv + h) << c.page_shift) * D +
           (int64_t)(t & (c.page - 1) & ~15) * D;
  };
  const L l(tid % L::PER, x.rope.rotary);
  Unit ka[KU], kb[KU], vx[VU];
#pragma unroll
  for (int j = 0; j < KU; ++j) {
    // (lanes of rows that are not written load the nearest one, so that sums over lanes are whole)
    const int t = min(max(p0 + (tid + kThreads * j) / L::PER, lo), end - 1);
    const Unit *from = (const Unit *)(a.k + (row0 + (int64_t)(t - start)) * a.k_stride + h * D);
    ka[j] = __builtin_nontemporal_load(from + l.a);
    kb[j] = __builtin_nontemporal_load(from + l.b);
  }
#pragma unroll
  for (int j = 0; j < VU; ++j) {
    const int u = tid + kThreads * j, t = p0 + u / CPR;
    if (t < lo || t >= end) continue;
    vx[j] = __builtin_nontemporal_load(
        (const Unit *)(a.v + (row0 + (int64_t)(t - start)) * a.v_stride + h * D + u % CPR * 8));
  }
  if (tid < 4) s_page[tid] = step_page(c, slot, p0 + 16 * tid, lo, end);
#pragma unroll
  for (int j = 0; j < VU; ++j) {
    const int u = tid + kThreads * j, r = u / CPR, t = p0 + r;
    if (t >= lo && t < end) *(Unit *)&tile[r][u % CPR * 8] = vx[j];
  }
#pragma unroll
  for (int j = 0; j < KU; ++j) {
    const int t = p0 + (tid + kThreads * j) / L::PER;
    turn_of<D, HALF>(x.rope, l, t, cs, sn);
    turn<D, NORM, HALF>(x.rope, l, x.rope.wk, cs, sn, ka[j], kb[j]);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < KU; ++j) {
    const int r = (tid + kThreads * j) / L::PER, t = p0 + r, p = s_page[r >> 4];
    if (t < lo || t >= end || p < 0) continue;
    Unit *to = (Unit *)(c.k + tile_of(p, t) + (t & 15) * D);
    __builtin_nontemporal_store(ka[j], to + l.a);
    __builtin_nontemporal_store(kb[j], to + l.b);
  }
  write_values<D>(c, tile, s_page, p0, lo, end, tile_of);
}

}  // namespace

int append_parts(const CacheView &c, int heads) {
  if (heads == 0) return c.hkv;
  return c.hkv + 64 / (c.d == 64 ? query_tokens<64>(heads) : query_tokens<128>(heads));
}

namespace {

template <int D, bool NORM, bool HALF>
hipError_t rotate(const RotateArgs &a, hipStream_t s) {
  RotateArgs b = a;
  const int chunks = (a.hq + a.hkv + Lane<D>::HEADS - 1) / Lane<D>::HEADS;
  b.set = set_of<D>(a.hq + a.hkv);
  b.groups = a.tokens <= 1024 ? chunks : 1;
  const int64_t waves = ((int64_t)a.tokens + b.set - 1) / b.set * b.groups;
  rotate_heads<D, NORM, HALF><<<(unsigned)((waves + 3) / 4), kThreads, 0, s>>>(b);
  return hipGetLastError();
}

template <int D, bool NORM, bool HALF>
hipError_t append(const CacheView &c, const AppendArgs &a, hipStream_t s) {
  AppendArgs b = a;
  b.set = a.q ? set_of<D>(a.hq) : 1;
  b.query_tokens = a.q ? query_tokens<D>(a.hq) : 64;
  const int per = append_parts(c, a.q ? a.hq : 0);
  cache_append<D, NORM, HALF><<<a.w.blk[a.w.list.n] * per, kThreads, 0, s>>>(c, b);
  return hipGetLastError();
}

template <int D>
hipError_t rotate(const RotateArgs &a, hipStream_t s) {
  if (a.rope.normed) return a.rope.half ? rotate<D, true, true>(a, s) : rotate<D, true, false>(a, s);
  return a.rope.half ? rotate<D, false, true>(a, s) : rotate<D, false, false>(a, s);
}

template <int D>
hipError_t append(const CacheView &c, const AppendArgs &a, hipStream_t s) {
  if (a.rope.normed)
    return a.rope.half ? append<D, true, true>(c, a, s) : append<D, true, false>(c, a, s);
  return a.rope.half ? append<D, false, true>(c, a, s) : append<D, false, false>(c, a, s);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a, int d, hipStream_t s) {
  return d == 64 ? rotate<64>(a, s) : rotate<128>(a, s);
}

hipError_t launch_cache_append(const CacheView &c, const AppendArgs &a, hipStream_t s) {
  return c.d == 64 ? append<64>(c, a, s) : append<128>(c, a, s);
}

}  // namespace fp
