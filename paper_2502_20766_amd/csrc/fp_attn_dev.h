// Device helpers shared by the attention kernels: vector types, exchanges between the two lanes
// of a query row, LDS swizzles of K and V^T tiles, and 16-byte DMAs into LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float wave_pair_max(float x) {
  // lanes l and l^32 exchange values; max of both halves of the swap is symmetric
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float wave_pair_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// acc + the sum of N 16-key steps' bf16 weights -- exactly the values the P V products
// use -- two per v_dot2_f32_bf16 against (1, 1), steps in order.
template <int N>
__device__ __forceinline__ float sum_weights(const bf16x8 (&pf)[N], float acc) {
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bf16x2 pair = {pf[i][2 * e], pf[i][2 * e + 1]};
      acc = __builtin_amdgcn_fdot2_f32_bf16(pair, one, acc, false);
    }
  return acc;
}

// 16-byte chunk swizzles (XOR, so the same function maps logical <-> physical).
// K: the 32 rows read by one half-wave at the same chunk land on distinct banks.
template <int D>
__device__ __forceinline__ int swz_k(int y, int r) {
  if constexpr (D == 128) return y ^ (r & 15);
  else return y ^ ((r >> 1) & 7);
}
// V^T: 16-byte unit of (head dim d, key half lh) inside one 16-key step of 2 d units per d.
// The 16 lanes that read one step at the same lh (d = d0 .. d0 + 15) land in 16 distinct
// 16-byte bank groups, and so do each 8 of them; the placement is additive in d / 32 and
// in the step, so a lane's reads differ only by immediate offsets.
__device__ __forceinline__ int vt_unit(int d, int lh) {
  return 16 * (d >> 3) + 8 * (lh ^ ((d >> 3) & 1)) + (d & 7);
}

// Buffer descriptor over [base, base + nrec) with out-of-range reads returning zero.  The
// inputs are made wave-uniform first so the descriptor always lives in scalar registers
// (a descriptor the compiler believes divergent would be issued once per distinct lane
// value in a loop).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const void *base, int nrec) {
  const uint64_t p = (uint64_t)(uintptr_t)base;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)(uintptr_t)(((uint64_t)hi << 32) | lo),
                                           (short)0, __builtin_amdgcn_readfirstlane(nrec),
                                           0x00020000);
}

// Wave-wide 16-byte DMAs into LDS slots I .. N-1, slot i at i * 1024 past `dst` (the
// immediate offset moves the source address by the same amount), with a per-lane offset
// per slot (K) or one shared by all slots (V^T).  POLICY: cache policy bits of the load (2:
// nontemporal).
template <int I, int N, int POLICY = 0>
__device__ __forceinline__ void dma_slots(__amdgpu_buffer_rsrc_t r,
                                          __attribute__((address_space(3))) void *dst,
                                          const uint32_t *voff) {
  if constexpr (I < N) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff[I], 0, I * 1024, POLICY);
    dma_slots<I + 1, N, POLICY>(r, dst, voff);
  }
}
template <int I, int N, int POLICY = 0>
__device__ __forceinline__ void dma_slots(__amdgpu_buffer_rsrc_t r,
                                          __attribute__((address_space(3))) void *dst,
                                          uint32_t voff) {
  if constexpr (I < N) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, 0, I * 1024, POLICY);
    dma_slots<I + 1, N, POLICY>(r, dst, voff);
  }
}

}  // namespace
}  // namespace fp
