// attention_lds.h -- tiles in LDS and what brings them there: shared by the attention
// kernels, forward and backward.
#pragma once

#include "internal.h"

namespace lvsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base,
                                                            uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0,
                                           bytes, 0x00020000);
}

// LDS tile layout ("slabs").  A BLOCK x 128 tile (one key block) is stored
// as 4 slabs of 32 columns; a slab row is 64 bytes (4 chunks of 16 bytes) and
// rows follow each other, so tile byte (slab, row, chunk) =
// slab*BLOCK*64 + row*64 + chunk*16.
// The chunk is XORed with x(row) = -(row/4) mod 4.  With 64 banks of 4 bytes:
//   - ds_read_b128 is served 16 lanes at a time, lanes 0-3, 12-15 and 20-27
//     together (then 4-11, 16-19 and 28-31; the same from lane 32 on): rows
//     0-3 and 12-15 at one logical chunk c and rows 4-11 at c ^ 1, which x
//     sends to four different bank quarters;
//   - ds_read_b64_tr_b16 (served 32 lanes at a time) reads 8 consecutive rows
//     x 2 chunks of a 32-byte half: rows 4..7 take the other half's banks.
// Both are free of bank conflicts, and every fragment address an unrolled loop
// needs is one of three per-lane bases plus an immediate offset.
constexpr int SLAB_ROW = 64;
__device__ __forceinline__ int xsw(int row) { return -(row >> 2) & 3; }

// One wave load (1 KiB) of a K or V tile into LDS at byte address lds_dst:
// `rsrc` starts at the tile's first row, `voff` = the lane's part of the
// global byte offset plus the load's uniform part (LoadPlan).  Rows at or
// past N fall outside the buffer resource and read as zeros.  The loads are
// issued from inline assembly so the compiler does not track them: they are
// waited for explicitly (vmcnt(0) plus a barrier) at the end of the step, and
// no compiler-inserted wait can stall the phases in between.  The nop is the
// wait state gfx9 needs between an SALU write of M0 and an LDS-DMA
// instruction (the compiler cannot see into the statement to add it).
__device__ __forceinline__ void issue_load(uint32_t lds_dst, __amdgpu_buffer_rsrc_t rsrc,
                                           uint32_t voff, uint32_t soff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, %3 offen lds"
      :
      : "s"(lds_dst), "v"(voff), "s"(rsrc), "s"(soff)
      : "memory", "m0");
}

// The same for 64 words of 4 bytes, one a lane.
__device__ __forceinline__ void issue_load_dword(uint32_t lds_dst, __amdgpu_buffer_rsrc_t rsrc,
                                                 uint32_t voff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %1, %2, 0 offen lds"
      :
      : "s"(lds_dst), "v"(voff), "s"(rsrc)
      : "memory", "m0");
}

__device__ __forceinline__ void wait_loads_and_sync() {
  __builtin_amdgcn_s_waitcnt(0);  // vmcnt(0) expcnt(0) lgkmcnt(0)
  __syncthreads();
}

__device__ __forceinline__ bf16x8 join(i16x4 lo, i16x4 hi) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace lvsa
