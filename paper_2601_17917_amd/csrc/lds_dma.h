// Building blocks of the bf16 attention kernels: transfers global -> LDS, counted waits, scalar addresses, packing.
#pragma once
#include "common.h"

namespace sdllm {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;   // scalar (constant-cache) loads
typedef s16x4 __attribute__((address_space(3))) * lds_s16x4_ptr;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  // one v_cvt_pk_bf16_f32 (round to nearest even)
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// One 16-byte-per-lane global -> LDS transfer (the data never passes through registers): lane i's
// 16 bytes land at lds_addr + 16*i.  Issued through inline assembly so that the compiler's
// wait-count insertion does not serialise a multi-stage pipeline; completion is tracked by hand
// with s_waitcnt vmcnt(n) before the workgroup barrier (transfers complete in issue order).
__device__ __forceinline__ void dma16_sbase(unsigned lds_addr, const void* sbase, unsigned voff) {
  // the base is the same in every lane; say so, so that it is held in a scalar register pair
  const unsigned long long p = reinterpret_cast<unsigned long long>(sbase);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)p);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
  const unsigned long long pu = ((unsigned long long)hi << 32) | lo;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(pu) : "memory", "m0");
}
// One 16-row slab of one tensor: NT transfers of 1 KiB to consecutive KiB of LDS from one scalar
// base.  m0 (the LDS base of a transfer) is written once: the instruction's immediate offset moves
// the LDS address and the global address alike, so transfer j carries offset j KiB and its lane offset
// voffj has those j KiB taken off beforehand.  One wait state separates the write of m0 from the
// first transfer that reads it.
// ONCE: every byte of K/V is read by exactly one workgroup of the launch (one query tile per K/V head and
// split); the transfers then carry the nontemporal hint (cfg3A 31.1 -> 28.6 us).  Where query tiles share a
// K/V stream through L2 the hint costs 4-6 %, so it is left off there.
template <int NT, bool ONCE>
__device__ __forceinline__ void dma_slab(unsigned lds_addr, const void* sbase, const unsigned (&voffj)[4]) {
  static_assert(NT == 2 || NT == 4, "transfers per slab");
  if constexpr (NT == 4 && ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %1 nt\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024 nt\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048 nt\n\t"
                 "global_load_lds_dwordx4 %5, %1 offset:3072 nt"
                 :: "s"(lds_addr), "s"(sbase), "v"(voffj[0]), "v"(voffj[1]), "v"(voffj[2]), "v"(voffj[3]) : "memory", "m0");
  else if constexpr (NT == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %1\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:2048\n\t"
                 "global_load_lds_dwordx4 %5, %1 offset:3072"
                 :: "s"(lds_addr), "s"(sbase), "v"(voffj[0]), "v"(voffj[1]), "v"(voffj[2]), "v"(voffj[3]) : "memory", "m0");
  else if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %1 nt\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024 nt"
                 :: "s"(lds_addr), "s"(sbase), "v"(voffj[0]), "v"(voffj[1]) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %2, %1\n\t"
                 "global_load_lds_dwordx4 %3, %1 offset:1024"
                 :: "s"(lds_addr), "s"(sbase), "v"(voffj[0]), "v"(voffj[1]) : "memory", "m0");
}
template <bool ONCE>
__device__ __forceinline__ void dma16_vaddr(unsigned lds_addr, const void* vaddr) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt"
                 :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(vaddr) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(vaddr) : "memory", "m0");
}
// A pointer that is the same in every lane, moved into a scalar register pair (64-bit address
// arithmetic with products is done on the vector ALU; everything derived from the result would
// otherwise stay there too)
template <typename T>
__device__ __forceinline__ const T* uniform_ptr(const T* p) {
  const unsigned long long v = reinterpret_cast<unsigned long long>(p);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
  return reinterpret_cast<const T*>(((unsigned long long)hi << 32) | lo);
}
// s_waitcnt vmcnt(n) only (expcnt / lgkmcnt fields left at "no wait")
template <int N> __device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit field");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

}  // namespace sdllm
