// Microscaled 4-bit matrices: their memory layout and the conversions that the
// kernels share.
//
// A K x N matrix is kept column by column.  A column is padded with zeros to
// kp = 256 ceil(K / 256) rows and holds kp / 2 bytes of codes (row 2 r in the
// low half of byte r) and kp / 32 bytes of scales, one for every 32 rows.  A
// code is a sign bit and a 3-bit e2m1 magnitude of {0, 1/2, 1, 3/2, 2, 3, 4,
// 6}; a scale byte s stands for 2^(s - 127), 255 for NaN.
#pragma once

#include "tile.h"
#include "types.h"

namespace rrf {
namespace ops {

constexpr int kMxBlock = 32;
constexpr int kMxPad = 256;

inline int64_t mx_rows(int64_t k) { return round_up(k, kMxPad); }

// 2^(s - 127) in binary32 (2^-127 is subnormal), NaN for 255.
__device__ __forceinline__ float mx_scale(unsigned s) {
  const unsigned bits = s == 0 ? 0x00400000u : s << 23;
  return __builtin_bit_cast(float, s == 255 ? 0x7fc00000u : bits);
}

// Codes 2 B and 2 B + 1 of a word of eight, in binary32.
typedef float f2_t __attribute__((ext_vector_type(2)));
template <int B>
__device__ __forceinline__ f2_t mx_pair(unsigned word) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, B);
}
__device__ __forceinline__ void mx_decode8(unsigned word, float scale, float (&v)[8]) {
  const f2_t a = mx_pair<0>(word), b = mx_pair<1>(word), c = mx_pair<2>(word), d = mx_pair<3>(word);
  v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
  v[4] = c[0] * scale; v[5] = c[1] * scale; v[6] = d[0] * scale; v[7] = d[1] * scale;
}

// A real number as a sum of bfloat16 parts: 8 bits each, truncated (rounding
// could overflow), so binary32 takes three, binary16 two.  Exact down to 2^-110 in
// magnitude; the last part of what is smaller falls below bfloat16's least
// number, 2^-133, and the value is cut to a multiple of that.  (The matrix
// instruction takes subnormal operands as they are.)
template <typename T> constexpr int parts_of() { return sizeof(T) == 4 ? 3 : 2; }
template <> constexpr int parts_of<bf16_t>() { return 1; }

template <int P>
__device__ __forceinline__ void split_bf16(float x, unsigned short (&out)[P]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const unsigned bits = __builtin_bit_cast(unsigned, x);
    out[p] = (unsigned short)(bits >> 16);
    const float h = __builtin_bit_cast(float, bits & 0xffff0000u);
    x = h == x ? 0.f : x - h;     // an infinity has no rest
  }
}

}  // namespace ops
}  // namespace rrf
