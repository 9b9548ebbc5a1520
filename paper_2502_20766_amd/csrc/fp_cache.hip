// The paged cache of keys and values: bookkeeping of its pages, and the copies that move tokens
// and pages.
//
// All bookkeeping is on the device (fp_cache.meta), so that a decoding loop needs no host wait
// and can be captured into a graph.  Free pages are a bitmap beside the reference counts: pages
// are taken lowest number first by counting bits, and given back by clearing them, in any order
// with the same result, so no list has to be kept in order.
#include "fp_internal.h"

namespace fp {
namespace {

constexpr int kPlanThreads = 1024;   // the single workgroup that hands out pages
constexpr int kCopyUnits = 1024;     // 16-byte units of a page copied by one workgroup at a time
constexpr int kCopyGrid = 2048;      // workgroups of a copy whose length the host cannot know

// 16 bytes as a vector: arrays of a struct of four words were kept in scratch memory, which
// cost a short copy 13 us.
typedef uint32_t Unit __attribute__((ext_vector_type(4)));

// Exclusive prefix sum over the workgroup (kPlanThreads threads) and the total; `part` is an
// int of LDS per wave.
__device__ __forceinline__ int block_scan(int x, int *part, int &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  __syncthreads();                   // earlier reads of `part` are done
  if (lane == 63) part[w] = sum;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    const int y = part[i];
    if (i < w) base += y;
    total += y;
  }
  return base + sum - x;
}

__device__ __forceinline__ int pages_of(int tokens, int shift) {
  return (int)(((unsigned)tokens + (1u << shift) - 1) >> shift);
}

// One holder less of each page listed (-1: none) for the entries of a thread; neighbours that
// name the same page share an atomic, and all of a thread's are in flight together.  Bits of
// pages without holders are cleared; returns how many there are.
template <int kBatch>
__device__ __forceinline__ int drop_pages(const CacheView &c, const int (&page)[kBatch]) {
  int less[kBatch], before[kBatch], run = 0, gone = 0;
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    run = page[i] >= 0 && page[i] < c.pages ? run + 1 : 0;
    const bool last = i + 1 == kBatch || page[i + 1] != page[i];
    less[i] = last ? run : 0;
    if (last) run = 0;
  }
#pragma unroll
  for (int i = 0; i < kBatch; ++i)
    if (less[i]) before[i] = atomicSub(c.ref + page[i], less[i]);
#pragma unroll
  for (int i = 0; i < kBatch; ++i)
    if (less[i] && before[i] == less[i]) {
      atomicAnd(c.used + (page[i] >> 6), ~(1ull << (page[i] & 63)));
      ++gone;
    }
  return gone;
}

// state[0] less `gone` summed over the workgroup's waves.
__device__ __forceinline__ void count_freed(const CacheView &c, int gone) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) gone += __shfl_xor(gone, d);
  if ((threadIdx.x & 63) == 0 && gone) atomicSub(c.state, gone);
}

// A call that would have changed a slot's length is left out because an error bit is set.  If no
// bit that stops writes is among them, this one is set: a write finds its place from the length,
// and would land on tokens that are there already.
__device__ __forceinline__ void left_out(const CacheView &c, int error) {
  if (error == FP_CACHE_SHARED) atomicOr(c.state + 1, FP_CACHE_SKIPPED);
}

__global__ __launch_bounds__(256) void cache_init(CacheView c) {
  const int64_t n_zero = 8 + 2 * (int64_t)c.words + c.slots + c.pages;
  const int64_t n = n_zero + (int64_t)c.slots * c.max_pages;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    c.state[i] = i < n_zero ? 0 : -1;
}

// ---- reserve: one workgroup decides, a second launch makes the copies.
//
// Slot i of the list needs ceil((len + num) / page) - ceil(len / page) pages, and one more when
// its last page is not full and another slot will still hold it: with r holders, the first r -
// 1 such slots of the list take copies.  The free pages, in ascending order, go to the slots in
// list order; rank r among the free pages belongs to the slot whose range of the prefix sums
// holds r, found by bisection. Latency bound (one workgroup, a chain of about six loads): 4.8
// us for 64 slots and one token each, 6.0 for 860 new pages, 7.2 with 31 copies.
__global__ __launch_bounds__(kPlanThreads) void cache_reserve(CacheView c, CacheList l,
                                                              PageCopies w) {
  __shared__ int part[kPlanThreads / 64];
  __shared__ int s_slot[FP_MAX_CACHE_LIST], s_held[FP_MAX_CACHE_LIST];
  __shared__ int s_begin[FP_MAX_CACHE_LIST + 1], s_tail[FP_MAX_CACHE_LIST];
  __shared__ int s_copy[FP_MAX_CACHE_LIST];      // index of the slot's copy, or -1
  __shared__ int s_base[kPlanThreads];
  __shared__ unsigned long long s_free[kPlanThreads];
  const int tid = threadIdx.x;
  const int used_pages = c.state[0], error = c.state[1];
  if (error != 0) {
    if (tid == 0) {
      w.count[0] = 0;
      left_out(c, error);
    }
    return;
  }
  const bool mine = tid < l.n;
  const int64_t room = (int64_t)c.max_pages << c.page_shift;
  int slot = 0, len = 0, num = 0, held = 0, tail = -1, refs = 0;
  bool bad = false;
  if (mine) {
    slot = l.slot[tid];
    num = l.num[tid];
    len = c.len[slot];
    bad = len < 0 || (int64_t)len + num > room;
    if (!bad) {
      held = pages_of(len, c.page_shift);
      if (num > 0 && (len & (c.page - 1))) {
        tail = c.table[(int64_t)slot * c.max_pages + held - 1];
        if ((unsigned)tail < (unsigned)c.pages) refs = c.ref[tail];
        else tail = -1;
      }
    }
    s_tail[tid] = tail;
  }
  int copy = 0;
  if (__syncthreads_or(refs > 1)) {
    if (refs > 1) {
      int before = 0;
      for (int j = 0; j < tid; ++j) before += s_tail[j] == tail;
      copy = refs - before > 1;
    }
  }
  const int need = mine && !bad ? pages_of(len + num, c.page_shift) - held + copy : 0;
  int total, copies;
  const int begin = block_scan(need, part, total);
  const int at = block_scan(copy, part, copies);
  const int too_long = __syncthreads_or(bad) ? FP_CACHE_TOO_LONG : 0;
  const int full = total > c.pages - used_pages ? FP_CACHE_FULL : 0;
  if (too_long | full) {
    if (tid == 0) {
      c.state[1] = too_long | full;
      w.count[0] = 0;
    }
    return;
  }
  if (mine) {
    s_slot[tid] = slot;
    s_held[tid] = held - copy;
    s_begin[tid] = begin;
    s_copy[tid] = copy ? at : -1;
    c.len[slot] = len + num;
    if (copy) {
      w.src[at] = tail;
      atomicSub(c.ref + tail, 1);
    }
  }
  if (tid == 0) {
    s_begin[l.n] = total;
    c.state[0] = used_pages + total;
    w.count[0] = copies;
  }
  // free pages, 64 to a word, kPlanThreads words at a time; a wave takes a word, a lane a page
  for (int w0 = 0, taken = 0; taken < total && w0 < c.words; w0 += kPlanThreads) {
    const int word = w0 + tid;
    unsigned long long fr = 0;
    if (word < c.words) {
      fr = ~c.used[word];
      const int left = c.pages - word * 64;
      if (left < 64) fr &= (1ull << left) - 1;
    }
    int found;
    const int base = block_scan(__popcll(fr), part, found) + taken;
    s_base[tid] = base;
    s_free[tid] = fr;
    __syncthreads();
    const int lane = tid & 63;
    for (int i = tid >> 6; i < min(kPlanThreads, c.words - w0); i += kPlanThreads / 64) {
      const unsigned long long f = s_free[i];
      const int first = s_base[i];
      if (f == 0 || first >= total) continue;
      const int rank = first + __popcll(f & ((1ull << lane) - 1));
      const bool take = (f >> lane & 1) && rank < total;
      if (take) {
        const int p = (w0 + i) * 64 + lane;
        int lo = 0, hi = l.n;              // s_begin[lo] <= rank < s_begin[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (s_begin[mid] <= rank) lo = mid;
          else hi = mid;
        }
        const int j = rank - s_begin[lo];
        c.table[(int64_t)s_slot[lo] * c.max_pages + s_held[lo] + j] = p;
        c.ref[p] = 1;
        if (j == 0 && s_copy[lo] >= 0) w.dst[s_copy[lo]] = p;
      }
      const unsigned long long got = __ballot(take);
      if (lane == 0) c.used[w0 + i] |= got;
    }
    taken += found;
  }
}

// The page copies of a list in every layer.  blockIdx.x is a part (kCopyUnits 16-byte units) of
// a page of K or V in one layer, blockIdx.y and every gridDim.y-th after it a copy.  16-byte loads
// and stores, four in flight per thread; memory bound: compaction reads and writes 3.15 GB (1500
// pages of 64 tokens in four layers) in 619 us, 5.1 TB/s; a few pages take 4.3 us.  Compaction moves
// each page once and past the caches (with its plan 634 -> 620 us for those pages); copies of a
// shared page read it several times (reserve with 31 copies, and the writes: 46 -> 55 us that way).
// Of such a page the whole is copied, 65 MB for 31 of 128 tokens in four layers: 13.6 us.
template <bool kOnce>
__device__ __forceinline__ void copy_pages(const CacheView &c, const PageCopies &w) {
  const int units = c.hkv * c.page * c.d / 8;
  const int parts = (units + kCopyUnits - 1) / kCopyUnits;
  const int pool = blockIdx.x / parts;                   // layer and K or V
  uint16_t *base = (pool & 1 ? c.v : c.k) + (int64_t)(pool >> 1) * c.pages * units * 8;
  const int u0 = (blockIdx.x - pool * parts) * kCopyUnits + threadIdx.x;
  const int n = w.count[0];
  for (int i = blockIdx.y; i < n; i += gridDim.y) {
    const int src = w.src[i], dst = w.dst[i];
    if ((unsigned)src >= (unsigned)c.pages || (unsigned)dst >= (unsigned)c.pages) continue;
    const Unit *from = (const Unit *)base + (int64_t)src * units;
    Unit *to = (Unit *)base + (int64_t)dst * units;
    Unit x[kCopyUnits / 256];
#pragma unroll
    for (int j = 0; j < kCopyUnits / 256; ++j)
      if (u0 + 256 * j < units)
        x[j] = kOnce ? __builtin_nontemporal_load(from + u0 + 256 * j) : from[u0 + 256 * j];
#pragma unroll
    for (int j = 0; j < kCopyUnits / 256; ++j)
      if (u0 + 256 * j < units) {
        if (kOnce) __builtin_nontemporal_store(x[j], to + u0 + 256 * j);
        else to[u0 + 256 * j] = x[j];
      }
  }
}

dim3 copy_grid(const CacheView &c, int most) {
  const int units = c.hkv * c.page * c.d / 8;
  const int64_t x = (int64_t)c.layers * 2 * ((units + kCopyUnits - 1) / kCopyUnits);
  const int64_t y = x < kCopyGrid ? (kCopyGrid + x - 1) / x : 1;
  return dim3((unsigned)x, (unsigned)(y < most ? y : most));
}

__global__ __launch_bounds__(256) void cache_copy(CacheView c, PageCopies w) {
  copy_pages<false>(c, w);
}

// ---- write: a workgroup writes the new tokens among 64 positions of one slot and KV head.
// Keys are rows, copied as they are; values go through LDS and leave as 16-byte units of eight
// tokens of one head dimension.  A unit that also holds older tokens is written element by
// element.  Memory bound for long pieces (110k tokens, 8 KV heads of 128, 900 MB read and
// written in two layers: 84 us a layer, 5.4 TB/s), latency bound for one token a slot (5.4 us
// for 64 slots).  What passes through is not read again soon, so loads and stores are nontemporal:
// that call 195.7 -> 178.3 us, with loads or stores alone 192.5 and 183.1 (and 210 after a call
// that left the caches full of its writes, where both take 183).
template <int D>
__global__ __launch_bounds__(256) void cache_write(CacheView c, WriteArgs a) {
  constexpr int CPR = D / 8;                 // 16-byte chunks per row
  __shared__ __attribute__((aligned(16))) uint16_t tile[64][D + 8];
  __shared__ int s_i, s_page[4];
  // neighbouring workgroups take the KV heads of the same rows
  const int blk = blockIdx.x / c.hkv, h = blockIdx.x - blk * c.hkv, tid = threadIdx.x;
  // the slot whose blocks hold this one: one thread's
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
  auto tile_of = [&](int p, int t) {         // element offset of position t's 16-token step
    return ((((int64_t)a.layer * c.pages + p) * c.hkv + h) << c.page_shift) * D +
           (int64_t)(t & (c.page - 1) & ~15) * D;
  };
  Unit kx[64 * CPR / 256], vx[64 * CPR / 256];
#pragma unroll
  for (int i = 0; i < 64 * CPR / 256; ++i) {
    const int u = tid + 256 * i, r = u / CPR, ch = u % CPR, t = p0 + r;
    if (t < lo || t >= end) continue;
    const int64_t row = row0 + (t - start);
    kx[i] = __builtin_nontemporal_load((const Unit *)(a.k + row * a.k_stride + h * D + ch * 8));
    vx[i] = __builtin_nontemporal_load((const Unit *)(a.v + row * a.v_stride + h * D + ch * 8));
  }
  // pages of the four 16-token steps, or -1 for one that is not this slot's alone
  if (tid < 4) {
    const int t = p0 + 16 * tid;
    int p = -1;
    if (t < end && t + 16 > lo) {
      p = c.table[(int64_t)slot * c.max_pages + (t >> c.page_shift)];
      if ((unsigned)p >= (unsigned)c.pages || c.ref[p] != 1) {
        p = -1;
        atomicOr(c.state + 1, FP_CACHE_SHARED);
      }
    }
    s_page[tid] = p;
  }
#pragma unroll
  for (int i = 0; i < 64 * CPR / 256; ++i) {
    const int u = tid + 256 * i, r = u / CPR, ch = u % CPR, t = p0 + r;
    if (t >= lo && t < end) *(Unit *)&tile[r][ch * 8] = vx[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64 * CPR / 256; ++i) {
    const int u = tid + 256 * i, r = u / CPR, ch = u % CPR, t = p0 + r, p = s_page[r >> 4];
    if (t < lo || t >= end || p < 0) continue;
    __builtin_nontemporal_store(kx[i], (Unit *)(c.k + tile_of(p, t) + (t & 15) * D + ch * 8));
  }
  for (int u = tid; u < 8 * D; u += 256) {   // 8 half steps x D
    const int half = u & 1, d = (u >> 1) % D, step = (u >> 1) / D;
    const int r = 16 * step + 8 * half, t = p0 + r;
    if (t + 8 <= lo || t >= end) continue;
    const int p = s_page[step];
    if (p < 0) continue;
    uint16_t *to = c.v + tile_of(p, t) + d * 16 + 8 * half;
    if (t >= lo && t + 8 <= end) {
      Unit x;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[j] = tile[r + 2 * j][d] | (uint32_t)tile[r + 2 * j + 1][d] << 16;
      __builtin_nontemporal_store(x, (Unit *)to);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (t + j >= lo && t + j < end) to[j] = tile[r + j][d];
    }
  }
}

// ---- fork: a thread takes one place of the tables of kBatch sources to their copies.  A source
// keeps its pages throughout, so a page is never free in between, whatever the order of the
// counts. Neighbours that share a page share its atomics: samples of one prompt hold mostly the
// same.
template <int kBatch>
__global__ __launch_bounds__(256) void cache_fork(CacheView c, ForkArgs a) {
  const int first = blockIdx.y * kBatch, n = min(a.n - first, kBatch);
  const int j = blockIdx.x * 256 + threadIdx.x;
  const int error = c.state[1];
  if (error != 0) {
    if (j == 0 && blockIdx.y == 0) left_out(c, error);
    return;
  }
  int gone = 0;
  if (j < c.max_pages) {
    int now[kBatch], old[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      now[i] = i < n ? c.table[(int64_t)a.src[first + i] * c.max_pages + j] : -1;
      old[i] = i < n ? c.table[(int64_t)a.dst[first + i] * c.max_pages + j] : -1;
    }
    int more = 0;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const bool change = now[i] != old[i];
      if (change) c.table[(int64_t)a.dst[first + i] * c.max_pages + j] = now[i];
      else old[i] = -1;
      more += change;
      if (i + 1 == kBatch || now[i + 1] != now[i]) {
        if (more && (unsigned)now[i] < (unsigned)c.pages) atomicAdd(c.ref + now[i], more);
        more = 0;
      }
    }
    gone = drop_pages(c, old);
  }
  count_freed(c, gone);
  if (blockIdx.x == 0 && threadIdx.x < n)
    c.len[a.dst[first + threadIdx.x]] = c.len[a.src[first + threadIdx.x]];
}

// ---- truncate: a thread gives back one place of the tables of kBatch slots
template <int kBatch>
__global__ __launch_bounds__(256) void cache_truncate(CacheView c, CacheList l) {
  const int first = blockIdx.y * kBatch, n = min(l.n - first, kBatch);
  const int j = blockIdx.x * 256 + threadIdx.x;
  const int error = c.state[1];
  if (error != 0) {
    if (j == 0 && blockIdx.y == 0) left_out(c, error);
    return;
  }
  int gone = 0;
  if (j < c.max_pages) {
    int old[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      old[i] = i < n && j >= pages_of(l.num[first + i], c.page_shift)
                   ? c.table[(int64_t)l.slot[first + i] * c.max_pages + j]
                   : -1;
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (old[i] >= 0) c.table[(int64_t)l.slot[first + i] * c.max_pages + j] = -1;
    gone = drop_pages(c, old);
  }
  count_freed(c, gone);
  if (blockIdx.x == 0 && threadIdx.x < n) {
    int32_t *len = c.len + l.slot[first + threadIdx.x];
    *len = min(*len, l.num[first + threadIdx.x]);
  }
}

// ---- compact: one workgroup pairs holes with the pages behind them, a second launch copies the
// pages and renames them in the tables.  Sources lie at or above state[0] and targets below, so
// no copy reads what another writes.
__global__ __launch_bounds__(kPlanThreads) void cache_compact_plan(CacheView c, PageCopies w) {
  __shared__ int part[kPlanThreads / 64];
  __shared__ int s_base[kPlanThreads];
  __shared__ unsigned long long s_bits[kPlanThreads];
  const int tid = threadIdx.x, lane = tid & 63;
  const int n_used = c.state[0];
  if (c.state[1] != 0 || n_used < 0 || n_used > c.pages) {
    if (tid == 0) w.count[0] = 0;
    return;
  }
  int holes = 0;
  for (int pass = 0; pass < 2; ++pass) {     // free pages below n_used, then used ones above
    int seen = 0;
    const int first_word = pass == 0 ? 0 : n_used / 64;
    const int end_word = pass == 0 ? (n_used + 63) / 64 : c.words;
    for (int w0 = first_word; w0 < end_word; w0 += kPlanThreads) {
      const int word = w0 + tid;
      unsigned long long bits = 0;
      if (word < end_word) {
        bits = c.used[word];
        const int below = min(max(n_used - word * 64, 0), 64);
        const unsigned long long mask = below == 64 ? ~0ull : (1ull << below) - 1;
        bits = pass == 0 ? ~bits & mask : bits & ~mask;
        const int left = c.pages - word * 64;
        if (left < 64) bits &= (1ull << left) - 1;
      }
      int found;
      s_base[tid] = block_scan(__popcll(bits), part, found) + seen;
      s_bits[tid] = bits;
      __syncthreads();
      for (int i = tid >> 6; i < min(kPlanThreads, end_word - w0); i += kPlanThreads / 64) {
        const unsigned long long b = s_bits[i];
        if (!(b >> lane & 1)) continue;
        const int p = (w0 + i) * 64 + lane;
        const int rank = s_base[i] + __popcll(b & ((1ull << lane) - 1));
        if (pass == 0) {
          w.dst[rank] = p;
        } else if (rank < holes) {
          w.src[rank] = p;
          w.renamed[p] = w.dst[rank];
        }
      }
      seen += found;
      __syncthreads();
    }
    if (pass == 0) {
      holes = seen;
      if (holes == 0) break;
    } else if (seen != holes) {
      holes = 0;                             // the bitmap and state[0] disagree: nothing moves
    }
  }
  if (tid == 0) w.count[0] = holes;
  if (holes == 0) return;
  for (int word = tid; word < c.words; word += kPlanThreads) {
    const int below = min(max(n_used - word * 64, 0), 64);
    c.used[word] = below == 64 ? ~0ull : (1ull << below) - 1;
  }
}

__global__ __launch_bounds__(256) void cache_compact_move(CacheView c, PageCopies w) {
  const int n = w.count[0], n_used = c.state[0];
  if (n == 0) return;
  const int64_t me = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const int64_t all = (int64_t)gridDim.x * gridDim.y * 256;
  for (int64_t i = me; i < n; i += all) {
    c.ref[w.dst[i]] = c.ref[w.src[i]];
    c.ref[w.src[i]] = 0;
  }
  for (int64_t i = me; i < (int64_t)c.slots * c.max_pages; i += all) {
    const int p = c.table[i];
    if (p >= n_used && p < c.pages) c.table[i] = w.renamed[p];
  }
  copy_pages<true>(c, w);
}

}  // namespace

hipError_t launch_cache_init(const CacheView &c, hipStream_t s) {
  cache_init<<<1024, 256, 0, s>>>(c);
  return hipGetLastError();
}

hipError_t launch_cache_reserve(const CacheView &c, const CacheList &l, const PageCopies &w,
                                hipStream_t s) {
  cache_reserve<<<1, kPlanThreads, 0, s>>>(c, l, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  cache_copy<<<copy_grid(c, l.n), 256, 0, s>>>(c, w);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheView &c, const WriteArgs &a, hipStream_t s) {
  const int grid = a.blk[a.list.n] * c.hkv;
  if (c.d == 64) cache_write<64><<<grid, 256, 0, s>>>(c, a);
  else cache_write<128><<<grid, 256, 0, s>>>(c, a);
  return hipGetLastError();
}

// Table rows that one thread takes a place of in fork and truncate.  Slots of one prompt share most
// pages and so atomics, of which long tables have many; but a thread's rows come one after the
// other.  Fork and free, in us, at 4, 8 and 16 rows: 60 slots with 133 places 12.2, 14.3, 17.4; 100
// with 480 15.6, 14.8, 18.1; 100 with 1900 19.6, 16.5, 17.9; 100 with 3800 23.5, 19.0, 19.6; 100 and
// 40 with 8200 30.7, 22.5, 21.3; 30 with 7500 14.2 throughout.
static int table_rows(const CacheView &c, int n) {
  const int64_t places = (int64_t)n * c.max_pages;
  if (n <= 32 || places <= 1 << 14) return 4;
  return places <= 1 << 19 ? 8 : 16;
}

// Workgroups of fork and truncate: 256 places of the tables, `rows` slots of the list.
static dim3 table_grid(const CacheView &c, int n, int rows) {
  return dim3((c.max_pages + 255) / 256, (n + rows - 1) / rows);
}

hipError_t launch_cache_fork(const CacheView &c, const ForkArgs &a, hipStream_t s) {
  const int rows = table_rows(c, a.n);
  const dim3 grid = table_grid(c, a.n, rows);
  if (rows == 4) cache_fork<4><<<grid, 256, 0, s>>>(c, a);
  else if (rows == 8) cache_fork<8><<<grid, 256, 0, s>>>(c, a);
  else cache_fork<16><<<grid, 256, 0, s>>>(c, a);
  return hipGetLastError();
}

hipError_t launch_cache_truncate(const CacheView &c, const CacheList &l, hipStream_t s) {
  const int rows = table_rows(c, l.n);
  const dim3 grid = table_grid(c, l.n, rows);
  if (rows == 4) cache_truncate<4><<<grid, 256, 0, s>>>(c, l);
  else if (rows == 8) cache_truncate<8><<<grid, 256, 0, s>>>(c, l);
  else cache_truncate<16><<<grid, 256, 0, s>>>(c, l);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheView &c, const PageCopies &w, hipStream_t s) {
  cache_compact_plan<<<1, kPlanThreads, 0, s>>>(c, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  cache_compact_move<<<copy_grid(c, (c.pages + 1) / 2), 256, 0, s>>>(c, w);
  return hipGetLastError();
}

}  // namespace fp
