// Device helpers of the attention kernels over quantised caches, one wave per work
// item: LDS DMA into a ring of the wave's own, reductions over the four groups of 16
// lanes, and the masks of the step's positions.
#pragma once

#include "common.h"

namespace sdv {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

template <bool X>
struct Kind {
  static constexpr bool value = X;
};
template <int X>
struct Int {
  static constexpr int value = X;
};

// LDS DMA of 1 KB: lane l copies 16 bytes from base + off into LDS bytes lds +
// 16 l (lds wave-uniform).  From inline assembly, so that the compiler adds no
// waits of its own.  The base is copied by a scalar instruction first: that is the
// wait state between the write of M0 and the load, and the load's base is never a
// register that a vector instruction (a lane's read, a spill's) wrote just before,
// which would take five.
__device__ __forceinline__ void ring_dma(const void* base, uint32_t off, uint32_t lds) {
  uint64_t from;
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt"
               : "=&s"(from)
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base)
               : "m0", "memory");
}

__device__ __forceinline__ float max_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Positions that position `lane` (< G) sees of the step's own (bit a: position
// a): in a chain itself and those before it, in a tree itself and its
// ancestors, by pointer jumping over the parents.
__device__ __forceinline__ uint64_t position_mask(const int32_t* __restrict__ parent, int G) {
  const int lane = threadIdx.x & 63;
  if (parent == nullptr) return lane >= 63 ? ~0ull : (2ull << lane) - 1ull;
  int p = 0;
  if (lane > 0 && lane < G) {
    const int pp = parent[lane - 1];
    p = (pp >= -1 && pp < lane - 1) ? pp + 1 : 0;
  }
  uint64_t m = 1ull | (1ull << lane);
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const uint32_t lo = __shfl((uint32_t)m, p), hi = __shfl((uint32_t)(m >> 32), p);
    m |= ((uint64_t)hi << 32) | lo;
    p = __shfl(p, p);
  }
  return m;
}

// Bit i: whether key `off` + i (counted from the first of the step's positions)
// is seen: all keys before them, then the positions of `sees`, none after.
__device__ __forceinline__ uint64_t keys_seen(uint64_t sees, int off) {
  const uint64_t up = off < 64 ? sees >> (off & 63) : 0ull;
  const int n = -off;
  const uint64_t down = n < 64 ? (sees << (n & 63)) | ((1ull << (n & 63)) - 1ull) : ~0ull;
  return off >= 0 ? up : down;
}

}  // namespace sdv
