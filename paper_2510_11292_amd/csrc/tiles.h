// What the matrix-core attention kernels share: operand types, copies of rows to LDS
// and how rows lie there.
#pragma once

#include "common.h"

namespace louiskv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Waits for every copy and LDS access of the wave, then for the block's waves.
__device__ __forceinline__ void sync_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 64 lanes copy 16 bytes each from base + off (per lane) to LDS lds + 16 * lane.  The
// copy reads M0 one wait state after its write at the earliest.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}

// The same for rows that are read once and would only push others out of the caches.
__device__ __forceinline__ void stream_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}

typedef __attribute__((address_space(3))) char* lds_ptr;
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(lds_ptr)p; }

// Rows lie in LDS with their 16-byte pieces permuted, piece c of row r at
// c ^ swizzle(r).  Sixteen consecutive rows put a piece in sixteen different places
// (the key reads, a lane a row).  bfloat16, 16 pieces: four consecutive rows put a
// run of four pieces in four different ones (the transposing value reads).
// float32, 32 pieces: rows four apart put a run of eight in different halves of the
// banks (the value reads of the two halves of a wave).
template <class T>
__device__ __forceinline__ int swizzle(int r) {
  if constexpr (sizeof(T) == 2) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3;
}

}  // namespace louiskv
