// Pieces that the attention kernels share: LDS transpose reads, barriers and
// waits that leave copies in flight, the placement of V rows in LDS.
#pragma once

#include "common.h"

namespace sr {

constexpr float kLog2e = 1.4426950408889634f;

// Work-group barrier after this wave's LDS reads and writes complete; vector
// memory loads issued before it stay in flight (__syncthreads would wait for
// them too).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

// gfx950 LDS transpose read (ds_read_b64_tr_b16).  Every lane names 8 bytes
// (four bf16); within each group of 16 lanes, element e of lane i's result
// is element (i & 3) of the four named by lane 4 e + (i >> 2).
__device__ __forceinline__ i16x4 lds_read_tr16(const bf16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
}
// LDS byte address of a shared-memory pointer.
__device__ __forceinline__ uint32_t lds_addr(const bf16_t* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const bf16_t*)(p);
}
// Transpose reads at byte offsets LO and HI from each of N LDS addresses,
// complete on return (issue and wait are one block).  Unlike the builtin,
// after which the compiler waits for every copy into LDS still in flight
// (vmcnt 0), they leave the next tile's copies flying.
template <int N, int LO, int HI>
__device__ __forceinline__ void lds_read_tr16_pairs(const uint32_t (&a)[N], i16x4 (&lo)[N], i16x4 (&hi)[N]) {
  static_assert(N == 2 || N == 4, "pairs");
  if constexpr (N == 2) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
        "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1])
        : "v"(a[0]), "v"(a[1]), "n"(LO), "n"(HI)
        : "memory");
  } else if constexpr (N == 4) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1]), "=&v"(lo[2]), "=&v"(hi[2]), "=&v"(lo[3]),
          "=&v"(hi[3])
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(LO), "n"(HI)
        : "memory");
  }
}

// the value of lane l ^ 32
__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// two transpose reads as one MFMA operand (the 16-bit words reinterpreted
// as a whole vector)
__device__ __forceinline__ bf16x8 tr16_pair(i16x4 lo, i16x4 hi) {
  const i16x8 w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, w);
}

// Wait until at most N vector-memory operations of this wave are in flight.
template <int N>
__device__ __forceinline__ void vm_wait() {
  if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  else if constexpr (N == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if constexpr (N == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else static_assert(N < 0, "add this wait count");
}

// 16-byte chunk slot of chunk c of key k (k = key index within a 32-key V
// block) in the LDS copy: XOR-swizzled so that the transpose reads of a
// wave (four consecutive keys per lane group, two chunks each) spread over
// the banks.
template <int CPK>
__device__ __forceinline__ int vslot(int k, int c) {
  if constexpr (CPK == 16) return c ^ (((k & 3) << 1) | (((k >> 2) & 1) << 3));
  else return c ^ ((k & 3) << 1);
}

}  // namespace sr
