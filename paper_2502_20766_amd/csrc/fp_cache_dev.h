// Device helpers of the calls that write tokens into the paged cache.
#pragma once

#include "fp_internal.h"

namespace fp {
namespace {

// 16 bytes as a vector: arrays of a struct of four words were kept in scratch memory, which
// cost a short copy 13 us.
typedef uint32_t Unit __attribute__((ext_vector_type(4)));

// Page of the 16-token step at position t of a slot that is written from lo to end, or -1 for one
// that has none of those tokens or is not this slot's alone (which sets the error bit).
__device__ __forceinline__ int step_page(const CacheView &c, int slot, int t, int lo, int end) {
  if (t >= end || t + 16 <= lo) return -1;
  const int p = c.table[(int64_t)slot * c.max_pages + (t >> c.page_shift)];
  if ((unsigned)p < (unsigned)c.pages && c.ref[p] == 1) return p;
  atomicOr(c.state + 1, FP_CACHE_SHARED);
  return -1;
}

// Values of positions lo .. end-1 among the 64 from p0, from rows of LDS to their pages (s_page, one
// for each 16-token step; -1: left out): 16-byte units of eight tokens of one head dimension.  A unit
// that also holds older tokens is written element by element.  256 threads.
template <int D, class TileOf>
__device__ __forceinline__ void write_values(const CacheView &c, const uint16_t (*tile)[D + 8],
                                             const int *s_page, int p0, int lo, int end,
                                             const TileOf &tile_of) {
  for (int u = threadIdx.x; u < 8 * D; u += 256) {   // 8 half steps x D
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

}  // namespace
}  // namespace fp
