// Device helpers shared by the attention kernels that read the paged cache: copies of a tile's keys
// and values into LDS, values that no row may see, waits and barriers.
//
// `Args` below has k, v (pools of the layer), table, pages, hkv, page_shift and max_pages; `Piece` has
// row (the cache slot read), head (KV head), key0 and limit (first key and one past the last) and once
// (no other workgroup reads these keys).
#pragma once

#include "fp_attn_dev.h"

namespace fp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kKeys = 64;                 // keys per tile
constexpr float kLazy = 8.f;              // rise (log2 units) that moves a row's reference

template <int D>
struct PagedGeo {
  static constexpr int OCC = D == 64 ? 3 : 2;      // workgroups per CU = waves per SIMD
  static constexpr int RB = 2 * D;                 // bytes per key row
  static constexpr int STEP = 16 * RB;             // bytes of 16 keys, of K or of V
  static constexpr int DMA = STEP / 1024;          // 1 KB copies of them
  static constexpr int CPR = RB / 16;              // 16-byte chunks per key row
  static constexpr int RPI = 1024 / RB;            // key rows per copy
};

// A wave's 16 keys of a tile, which always lie in one page, brought into LDS by DMA: K
// row-major with 16-byte chunks swizzled as in the prefill, V^T in the fragment order of
// vt_unit.  KEYS: keys of a tile, 16 for each wave.
template <int D, int KEYS = kKeys>
struct Loader {
  using S = PagedGeo<D>;
  uint32_t koff[S::DMA], voff;
  int w;
  __device__ __forceinline__ Loader(int w, int lane) : w(w) {
#pragma unroll
    for (int i = 0; i < S::DMA; ++i) {
      const int r = i * S::RPI + lane / S::CPR;
      koff[i] = r * S::RB + swz_k<D>(lane % S::CPR, r) * 16 - i * 1024;
    }
    const int d = 8 * (lane >> 4) + (lane & 7), half = ((lane >> 3) ^ (lane >> 4)) & 1;
    voff = (2 * d + half) * 16;
  }
  // Table entry of the keys of tile t; loaded a tile ahead and first looked at in `issue`, so
  // that nothing waits for it.
  template <class Args, class Piece>
  __device__ __forceinline__ int page(const Args &a, const Piece &r, int t) const {
    const int key = min(r.key0 + KEYS * t + 16 * w, r.limit - 1);
    return a.table[(int64_t)r.row * a.max_pages + (key >> a.page_shift)];
  }
  template <class Args, class Piece>
  __device__ __forceinline__ void issue(const Args &a, const Piece &r, int t, int pg, uint8_t *k,
                                        uint8_t *v) const {
    const int key = r.key0 + KEYS * t + 16 * w;
    if (key >= r.limit) return;           // past the segment: those keys are masked
    pg = min(max(__builtin_amdgcn_readfirstlane(pg), 0), a.pages - 1);
    const int64_t off = ((((int64_t)pg * a.hkv + r.head) << a.page_shift) +
                         (key & ((1 << a.page_shift) - 1))) * D;
    copy(a.k, a.v, off, r.once, k, v);
  }
  // The copies of 16 keys and values, `off` elements into the pools.
  __device__ __forceinline__ void copy(const uint16_t *kp, const uint16_t *vp, int64_t off, int once,
                                       uint8_t *k, uint8_t *v) const {
    // Keys that are read once pass the caches by: 64 sequences of 3 to 32000 tokens 98.5 -> 87.3
    // us, 16 samples of 32k 43.8 -> 40.9, drafts at head dim 64 53.8 -> 48.8, and 130 -> 88, 58 ->
    // 44, 68 -> 52 after a call that left the caches full of its own writes.  For prefixes of
    // several row tiles 560 -> 582 (256 samples of 128k).
    copy_k(kp + off, once, k);
    copy_v(vp + off, once, v);
  }
  __device__ __forceinline__ void copy_k(const uint16_t *from, int once, uint8_t *to) const {
    const auto r = uniform_rsrc(from, S::STEP);
    const auto dst = (__attribute__((address_space(3))) void *)to;
    if (once) dma_slots<0, S::DMA, 2>(r, dst, koff);
    else dma_slots<0, S::DMA>(r, dst, koff);
  }
  __device__ __forceinline__ void copy_v(const uint16_t *from, int once, uint8_t *to) const {
    const auto r = uniform_rsrc(from, S::STEP);
    const auto dst = (__attribute__((address_space(3))) void *)to;
    if (once) dma_slots<0, S::DMA, 2>(r, dst, voff);
    else dma_slots<0, S::DMA>(r, dst, voff);
  }
};

// 16 keys of V^T in LDS, of which some row does not see all.  Values past the segment may hold
// anything, NaN among it, which a weight of zero would not cancel: they become zero.  So do
// infinities and NaN of tokens that only later queries see; returns whether there were any, and
// the rows that see them then take them separately.
template <int D>
__device__ __forceinline__ bool settle(uint8_t *v, int key0, int limit, int vis, int lane) {
  bool odd = false;
  for (int i = 0; i < 2 * D / 64; ++i) {
    const int u = 64 * i + lane;          // unit (d, half), see Loader::voff
    const int key = key0 + 8 * (((u >> 3) ^ (u >> 4)) & 1);
    s16x8 x = *reinterpret_cast<const s16x8 *>(v + 16 * u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool out = key + e >= limit;
      const bool late = key + e >= vis && (x[e] & 0x7F80) == 0x7F80;
      odd |= late && !out;
      if (out || late) x[e] = 0;
    }
    *reinterpret_cast<s16x8 *>(v + 16 * u) = x;
  }
  return __ballot(odd) != 0;
}

// Waits for this wave's copies into LDS (and its other loads and stores).  The builtin, unlike
// the same instruction in an asm statement, also tells the compiler, which would else wait for
// them where their LDS is first read, after the next copies have been issued, and so for those
// too.
__device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0)
  asm volatile("" ::: "memory");
}

// Workgroup barrier that orders LDS accesses only: it waits for no copy and no store in flight.
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace
}  // namespace fp
