// What the tiles of a product (tile.h) that are fed from a ring of chunks in LDS
// share (wide.h, ring4.h): a workgroup of four wavefronts forms a 32 T x 32 T
// tile of D, a wavefront 16 T x 16 T of it.
//
// One wavefront a SIMD keeps the matrix unit busy by itself: the operands that
// come next are read from LDS, and a later chunk is loaded from memory, between
// the matrix instructions of the present ones, a few at a time (loads that come
// in bursts hold up the wavefront that issues them: 2850 against 2430 cycles a
// chunk of 16-bit operands at T = 8).  One barrier a chunk, in its middle, where
// every wavefront has its last operands of the chunk in registers: the chunk's
// place in the ring is free from there on.  The accumulators are tied to the
// accumulation registers in the instruction; left to the compiler they are moved
// about between matrix instructions.
#pragma once

#include "tile.h"

namespace rrf {
namespace ops {

typedef __amdgpu_buffer_rsrc_t rsrc_t;

// A buffer from p on; accesses past its size read zeros.
__device__ __forceinline__ rsrc_t rsrc_of(const void* p, int64_t size = 0xffffffff) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)size, 0x27000);
}

__device__ __forceinline__ void mfma_acc(f4_t& c, i4_t a, i4_t b) {
  asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// s_waitcnt for at most N outstanding vector memory accesses and no LDS ones.
template <int N>
__device__ __forceinline__ void wait_mem() {
  static_assert(N >= 0 && N < 64, "counter of six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

}  // namespace ops
}  // namespace rrf
