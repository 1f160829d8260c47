// Products D = U V^T of two operands that are both contiguous along the
// contracted index, on the 16-bit and the 4-bit matrix instructions.
//
// An operand row is cut into chunks of 128 bytes: 64 values of 16 bits or 256
// of 4 bits.  A workgroup holds BM rows of U and BN rows of V of one chunk in
// LDS (a ring of them), loaded straight from memory to LDS in 16-byte packs, and
// the packs of a row are permuted (pack p at p ^ (row % 8)), so that the 16
// lanes which read one pack column of 16 rows touch all banks.  The
// permutation is applied to the address that a lane loads from: the LDS side
// of such a load is fixed.
//
// MFMA 16x16x32 (16 bits) and 16x16x128 (4 bits) read their operands alike:
// lane l holds the 16-byte pack l / 16 of row l % 16; item i of the result is
// D[4 (l / 16) + i][l % 16].
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../rrf_internal.h"

namespace rrf {
namespace ops {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef int i4_t __attribute__((ext_vector_type(4)));
typedef int i8_t __attribute__((ext_vector_type(8)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef _Float16 h4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b4_t __attribute__((ext_vector_type(4)));

constexpr int kChunkBytes = 128;

enum class Kind { kF16, kBF16 };

template <Kind KIND>
__device__ __forceinline__ f4_t mfma16(i4_t a, i4_t b, f4_t c) {
  if constexpr (KIND == Kind::kF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, a),
                                                  __builtin_bit_cast(h8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, a),
                                                   __builtin_bit_cast(b8_t, b), c, 0, 0, 0);
}

// Position of pack p of row r in a chunk's LDS image, in bytes.
__device__ __forceinline__ int pack_at(int r, int p) { return r * kChunkBytes + ((p ^ (r & 7)) << 4); }

// A product's operands, whose values are sums of two 16-bit parts: u + ul times
// v + vl is taken as u v + ul v + u vl.
struct Operands {
  const char *u, *ul, *v, *vl;
  int nk;           // chunks of a row
  int64_t ldu, ldv; // row pitch in bytes
  int rows_u, rows_v;
};

// Workgroups go to the eight dies in turn, each with a cache of its own: the
// place in the order of tiles that gives a die consecutive tiles.
__device__ __forceinline__ int die_order(int w, int n) {
  const int die = w & 7, q = n >> 3, r = n & 7;
  return die * q + min(die, r) + (w >> 3);
}

// Tile w of ti x tj in bands of eight along i, so that consecutive tiles are
// near each other in both directions (256 x 256 tiles of 4096 x 11008, K =
// 4096, one plane each: 303 -> 287 us with die_order).
__device__ __forceinline__ void band_tile(int w, int ti, int tj, int& bi, int& bj) {
  const int band = w / (8 * tj), wide = min(8, ti - 8 * band), o = w - band * 8 * tj;
  bi = 8 * band + o % wide;
  bj = o / wide;
}

}  // namespace ops
}  // namespace rrf
