// Products with microscaled 4-bit matrices.
//
// rrf_mx4_product: both operands in 4 bits, on the scaled matrix instruction
// (16x16x128, one scale byte per lane for its 32 values): tiles from a ring in
// LDS (ring4.h), or for up to 64 columns of B from memory straight into
// registers.
// rrf_mx4_apply: a 4-bit matrix or its transpose times real columns.  A 4-bit
// value is a bfloat16 number exactly, and a real one is the exact sum of one
// (bf16), two (f16) or three (f32) bfloat16 parts (below 2^-110 up to 2^-133:
// mx4.h), so every product is exact and the result has the error of binary32
// sums alone.

#include "mx4.h"
#include "cost.h"
#include "ring4.h"
#include "store.h"

#include <algorithm>

namespace rrf {
namespace ops {
namespace {

// Rows i .. i + 3 of column j of C, in one store whatever its alignment.
template <typename T>
__device__ __forceinline__ void store4(T* C, int64_t ldc, int64_t i, int64_t j, int64_t rows, f4_t v) {
  struct Four { T v[4]; };
  T* p = C + j * ldc + i;
  if (i + 4 <= rows) {
    Four o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o.v[r] = (T)v[r];
    *reinterpret_cast<Four*>(p) = o;
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (i + r < rows) p[r] = (T)v[r];
  }
}

// --- both operands in 4 bits -------------------------------------------------------

template <typename T>
struct MxArgs {
  Mx4Operands op;        // u: the first operand (M columns), v: the second (N)
  int ti, tj;            // tiles of C
  T* C; int64_t ldc;
};

// 32 TS x 32 TS tiles of C.
template <typename T, int TS, int S>
__global__ __launch_bounds__(256) void mx4_product_kernel(MxArgs<T> p) {
  typedef Mx4Tile<TS, S> MT;
  __shared__ __attribute__((aligned(1024))) char lds[MT::kLds];
  static_assert(4 * kStoreLds<TS> <= MT::kLds, "LDS");
  int bi, bj;
  band_tile(die_order(blockIdx.x, gridDim.x), p.ti, p.tj, bi, bj);
  const int i0 = bi * MT::BM, j0 = bj * MT::BN;
  f4_t acc[TS][TS];
  MT::run(p.op, i0, j0, lds, acc);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  store_tile<T, TS, false>(acc, p.C, p.ldc, i0 + (wv & 1) * 16 * TS, j0 + (wv >> 1) * 16 * TS, p.op.rows_u, p.op.rows_v,
                           lane, lds + wv * kStoreLds<TS>, [](float, float v) __attribute__((always_inline)) { return v; });
}

// Partial 16 x 16 tiles of W wavefronts added up in order: tile y of NT goes to
// wavefront y % W, which calls emit(y, sum).  part: W * NT * 64 values.
template <int W, int NT, typename EMIT>
__device__ __forceinline__ void add_partials(f4_t* part, const f4_t (&acc)[NT], EMIT emit) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int y = 0; y < NT; ++y) part[(wv * NT + y) * 64 + lane] = acc[y];
  __syncthreads();
#pragma unroll
  for (int y = 0; y < NT; ++y)
    if (wv == y % W) {
      f4_t s = part[y * 64 + lane];
#pragma unroll
      for (int w = 1; w < W; ++w) s += part[(w * NT + y) * 64 + lane];
      emit(y, s);
    }
}

// Up to 16 NT columns of B: a workgroup of eight wavefronts takes 16 rows of C
// and splits the contraction.  The 16 bytes that a lane loads of its column
// are the matrix instruction's operand as they are, so nothing passes through
// LDS but the eight partial sums.  Bound by the memory's latency and rate:
// up to six chunks (12 KB a wavefront) are in flight.
template <typename T, int NT>
__global__ __launch_bounds__(512) void mx4_product_few_kernel(MxArgs<T> p) {
  constexpr int kFlight = NT == 1 ? 6 : NT == 2 ? 4 : 2;
  __shared__ f4_t part[8 * NT * 64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int64_t i0 = (int64_t)blockIdx.x * 16;
  const int64_t pitch = (int64_t)p.op.nk * kChunkBytes, spitch = (int64_t)p.op.nk * 8;
  const int64_t row = min(i0 + m16, (int64_t)p.op.rows_u - 1);
  const char *u = p.op.u + row * pitch + g * 16, *su = p.op.su + row * spitch;
  const char *v[NT], *sv[NT];
#pragma unroll
  for (int y = 0; y < NT; ++y) {
    const int64_t c = min(16 * y + m16, p.op.rows_v - 1);
    v[y] = p.op.v + c * pitch + g * 16;
    sv[y] = p.op.sv + c * spitch;
  }
  f4_t acc[NT];
#pragma unroll
  for (int y = 0; y < NT; ++y) acc[y] = f4_t{0.f, 0.f, 0.f, 0.f};
  const int per = (p.op.nk + 7) >> 3, c0 = wv * per, c1 = min(p.op.nk, c0 + per);
  const i8_t zero = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int c = c0; c < c1; c += kFlight) {
    i4_t a[kFlight][2], b[kFlight][NT][2];
    uint2 ka[kFlight], kb[kFlight][NT];
#pragma unroll
    for (int q = 0; q < kFlight; ++q) {
      const int64_t cc = min(c + q, c1 - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) a[q][h] = *reinterpret_cast<const i4_t*>(u + cc * kChunkBytes + h * 64);
      ka[q] = *reinterpret_cast<const uint2*>(su + cc * 8);
#pragma unroll
      for (int y = 0; y < NT; ++y) {
#pragma unroll
        for (int h = 0; h < 2; ++h) b[q][y][h] = *reinterpret_cast<const i4_t*>(v[y] + cc * kChunkBytes + h * 64);
        kb[q][y] = *reinterpret_cast<const uint2*>(sv[y] + cc * 8);
      }
    }
#pragma unroll
    for (int q = 0; q < kFlight; ++q)
      if (c + q < c1) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          i8_t x = zero;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = a[q][h][e];
          const int sa = (int)((h ? ka[q].y : ka[q].x) >> (8 * g));
#pragma unroll
          for (int y = 0; y < NT; ++y) {
            i8_t z = zero;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = b[q][y][h][e];
            acc[y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                x, z, acc[y], 4, 4, 0, sa, 0, (int)((h ? kb[q][y].y : kb[q][y].x) >> (8 * g)));
          }
        }
      }
  }
  add_partials<8, NT>(part, acc, [&](int y, f4_t s) __attribute__((always_inline)) {
    const int64_t j = 16 * y + m16;
    if (j < p.op.rows_v) store4(p.C, p.ldc, i0 + 4 * g, j, p.op.rows_u, s);
  });
}

template <typename T, int TS, int S>
void launch_tiles(MxArgs<T> p, hipStream_t st) {
  p.ti = (int)ceil_div(p.op.rows_u, 32 * TS);
  p.tj = (int)ceil_div(p.op.rows_v, 32 * TS);
  mx4_product_kernel<T, TS, S><<<(unsigned)((int64_t)p.ti * p.tj), 256, 0, st>>>(p);
}

template <typename T>
rrf_status product_typed(int64_t M, int64_t N, int64_t k, const void* a, const void* sa, const void* b,
                         const void* sb, void* C, int64_t ldc, hipStream_t st) {
  MxArgs<T> p{{(const char*)a, (const char*)sa, (const char*)b, (const char*)sb, (int)(mx_rows(k) / kMxPad),
               (int)M, (int)N}, 0, 0, (T*)C, ldc};
  const unsigned rows16 = (unsigned)ceil_div(M, 16);
  if (N <= 16) {
    mx4_product_few_kernel<T, 1><<<rows16, 512, 0, st>>>(p);
  } else if (N <= 32) {
    mx4_product_few_kernel<T, 2><<<rows16, 512, 0, st>>>(p);
  } else if (N <= 64) {
    mx4_product_few_kernel<T, 4><<<rows16, 512, 0, st>>>(p);
  } else {
    switch (choose_product(M, N, p.op.nk)) {
      case 0: launch_tiles<T, 2, 4>(p, st); break;
      case 1: launch_tiles<T, 4, 2>(p, st); break;
      case 2: launch_tiles<T, 6, 2>(p, st); break;
      default: launch_tiles<T, 8, 2>(p, st); break;
    }
  }
  return status_of(hipGetLastError());
}

// --- a 4-bit matrix times real columns -----------------------------------------------

template <typename T>
struct ApplyArgs {
  const unsigned char *codes, *scales;
  int64_t k, m;          // the 4-bit matrix is k x m
  int chunks;            // of 256 rows a column
  const T* B; int64_t ldb;
  int64_t n;
  T* C; int64_t ldc;
  int64_t rows;          // of C
  int ti;
  int splits;            // of the contraction
  float* part;           // their sums, [split][column of C][row]
};

// Eight codes of a word times a scale, as bfloat16: pairs of consecutive ones.
__device__ __forceinline__ void mx_decode8_bf16(unsigned w, float scale, unsigned (&o)[4]) {
  o[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  o[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  o[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  o[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
}

// Eight consecutive values of a column of B from l on, zero past L; raw as
// loaded.
template <typename T> struct Raw8 { T v[8]; };
// In one or two loads whatever their alignment, which the hardware allows.
template <typename T>
__device__ __forceinline__ Raw8<T> load_pack8(const T* p) {
  return *reinterpret_cast<const Raw8<T>*>(p);
}
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* col, int64_t l, int64_t L, bool live) {
  Raw8<T> r;
  if (live && l + 8 <= L) {
    r = load_pack8(col + l);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = live && l + e < L ? col[l + e] : (T)0.f;
  }
  return r;
}
// Their bfloat16 parts, eight to a pack: the upper halves of x, of what its
// upper half leaves, and of what that one's leaves (each difference is exact,
// the last part as mx4.h says).  An infinity leaves nothing (infinity less
// itself would be a NaN); eight values without one, the usual case, are cut
// without looking at each.
template <typename T>
__device__ __forceinline__ void parts8(const Raw8<T>& r, i4_t (&o)[parts_of<T>()]) {
  constexpr int P = parts_of<T>();
  if constexpr (P == 1) {
    o[0] = __builtin_bit_cast(i4_t, r);
  } else {
    float v[8], top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = (float)r.v[e];
      top = fmaxf(top, fabsf(v[e]));              // (a NaN's parts hold a NaN in any case)
    }
    const bool finite = top < __builtin_inff();
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[q][e] = (int)__builtin_amdgcn_perm(__builtin_bit_cast(unsigned, v[2 * e + 1]),
                                             __builtin_bit_cast(unsigned, v[2 * e]), 0x07060302u);
      if (q + 1 < P) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v[e]) & 0xffff0000u);
      }
    }
    if (!finite) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        unsigned short x[P], y[P];
        split_bf16<P>((float)r.v[e], x);
        split_bf16<P>((float)r.v[e + 1], y);
#pragma unroll
        for (int q = 0; q < P; ++q) o[q][e / 2] = (int)((unsigned)x[q] | ((unsigned)y[q] << 16));
      }
    }
  }
}

// Position of pack p of row r in A's image.  Rows are written eight apart
// without TRANS and read one after the other, so both parts of the row's
// number take part (with r % 8 alone all 16 lanes of a write met in one bank:
// 4096 x 512 times 512 x 11008 binary32: 250 us against 169).
__device__ __forceinline__ int a_at(int r, int p) { return r * kChunkBytes + ((p ^ ((r ^ (r >> 3)) & 7)) << 4); }

// C (I x n) = op(A) B; I = m with TRANS, k without.  A tile of 64 WI x 16 NT (4 /
// WI) of C by four wavefronts of 64 x 16 NT, WI of them along i, 64 contracted
// values at a time: codes are decoded, and B is cut into its parts, on the way
// from registers to LDS, and the next chunk is loaded while the present one is
// multiplied.  Two workgroups share a compute unit, so that one converts while
// the other multiplies.  WI = 4 where there are rows for it: every column of B
// is cut up once for 256 rows of C.
template <typename T, bool TRANS, int WI, int NT>
__global__ __launch_bounds__(256, 2) void mx4_apply_kernel(ApplyArgs<T> p) {
  constexpr int P = parts_of<T>(), WJ = 4 / WI, BM = 64 * WI, BN = 16 * NT * WJ;
  constexpr int kPacks = BN * 8, kQ = (kPacks + 255) / 256;      // of B; a thread's
  constexpr int kImage = BN * kChunkBytes;
  constexpr int kA = BM / 128;                                   // a thread's 16 bytes of codes
  __shared__ __attribute__((aligned(1024))) char lds[BM * kChunkBytes + P * kImage];
  char* const la = lds;
  char* const lb = lds + BM * kChunkBytes;
  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int wi = (wv % WI) * 64, wj = (wv / WI) * 16 * NT;
  // The tiles of one column of C follow each other on a die, whose cache then
  // has their part of B.
  const int w = die_order(blockIdx.x, gridDim.x);
  const int64_t i0 = (int64_t)(w % p.ti) * BM, j0 = (int64_t)(w / p.ti) * BN;
  const int64_t I = p.rows, L = TRANS ? p.k : p.m;
  const int64_t pitch = (int64_t)p.chunks * 128, spitch = (int64_t)p.chunks * 8;
  f4_t acc[4][NT];
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < NT; ++y) acc[x][y] = f4_t{0.f, 0.f, 0.f, 0.f};
  // A with TRANS: columns i0 + 128 z + t / 2, 32 rows (one block) from l0 + 32
  // (t % 2).  Without: 8 rows from i0 + 128 z + 8 (t % 16) of the four columns
  // l0 + 4 (t / 16) ...
  // Nothing is done to what is loaded before it is staged, or the loads would be
  // waited for at once; scales are loaded as the words of four blocks.
  constexpr int kS = TRANS ? 1 : 4;
  uint4 wa[kA];
  unsigned sa[kA][kS];
  auto load_a = [&](int64_t l0) __attribute__((always_inline)) {
#pragma unroll
    for (int z = 0; z < kA; ++z) {
      if constexpr (TRANS) {
        const int64_t c = min(i0 + 128 * z + (t >> 1), p.m - 1), r = l0 + 32 * (t & 1);
        wa[z] = *reinterpret_cast<const uint4*>(p.codes + c * pitch + r / 2);
        sa[z][0] = *reinterpret_cast<const unsigned*>(p.scales + c * spitch + (l0 / 32 & ~(int64_t)3));
      } else {
        const int64_t r = min(i0 + 128 * z + 8 * (t & 15), (int64_t)p.chunks * 256 - 8);
        unsigned w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t cc = min(l0 + 4 * (t >> 4) + q, p.m - 1);
          w[q] = *reinterpret_cast<const unsigned*>(p.codes + cc * pitch + r / 2);
          sa[z][q] = *reinterpret_cast<const unsigned*>(p.scales + cc * spitch + r / 128 * 4);
        }
        wa[z] = uint4{w[0], w[1], w[2], w[3]};
      }
    }
  };
  auto stage_a = [&](int64_t l0) __attribute__((always_inline)) {
#pragma unroll
    for (int z = 0; z < kA; ++z) {
      unsigned w[4] = {wa[z].x, wa[z].y, wa[z].z, wa[z].w};
      if constexpr (TRANS) {
        const float sc = mx_scale((sa[z][0] >> (8 * ((l0 / 32 & 2) + (t & 1)))) & 255u);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          unsigned o[4];
          mx_decode8_bf16(w[q], sc, o);
          *reinterpret_cast<i4_t*>(la + a_at(128 * z + (t >> 1), 4 * (t & 1) + q)) =
              i4_t{(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
        }
      } else {
        const int64_t r0 = min(i0 + 128 * z + 8 * (t & 15), (int64_t)p.chunks * 256 - 8);
        const int shift = 8 * (int)(r0 / 32 & 3);
        unsigned o[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bool past = l0 + 4 * (t >> 4) + q >= p.m;             // zeros, scale 1
          mx_decode8_bf16(past ? 0u : w[q], mx_scale(past ? 127u : (sa[z][q] >> shift) & 255u), o[q]);
        }
        const int jg = t >> 4;                        // four columns: half a pack of a row
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const unsigned sel = (r & 1) ? 0x07060302u : 0x05040100u;
          uint2 v;
          v.x = __builtin_amdgcn_perm(o[1][r >> 1], o[0][r >> 1], sel);
          v.y = __builtin_amdgcn_perm(o[3][r >> 1], o[2][r >> 1], sel);
          *reinterpret_cast<uint2*>(la + a_at(128 * z + 8 * (t & 15) + r, jg >> 1) + 8 * (jg & 1)) = v;
        }
      }
    }
  };
  // B: values l0 + 8 (t % 8) ... of columns j0 + t / 8 + 32 q.  Whole chunks load
  // without a look at the end.
  Raw8<T> rb[kQ];
  const T* cb[kQ];
#pragma unroll
  for (int q = 0; q < kQ; ++q) cb[q] = p.B + min(j0 + (t >> 3) + 32 * q, p.n - 1) * p.ldb + 8 * (t & 7);
  auto load_b = [&](int64_t l0) __attribute__((always_inline)) {
    if (l0 + 64 <= L) {
#pragma unroll
      for (int q = 0; q < kQ; ++q) rb[q] = load_pack8(cb[q] + l0);
    } else {
#pragma unroll
      for (int q = 0; q < kQ; ++q) rb[q] = load_raw8(cb[q] - 8 * (t & 7), l0 + 8 * (t & 7), L, true);
    }
  };
  auto stage_b = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      if (kPacks % 256 != 0 && q == kQ - 1 && t + 256 * q >= kPacks) break;
      i4_t o[P];
      parts8(rb[q], o);
#pragma unroll
      for (int z = 0; z < P; ++z) *reinterpret_cast<i4_t*>(lb + z * kImage + pack_at((t >> 3) + 32 * q, t & 7)) = o[z];
    }
  };
  // This split's chunks.
  const int64_t per = ((L + 63) / 64 + p.splits - 1) / p.splits * 64;
  const int64_t first = blockIdx.y * per, last = min(L, first + per);
  load_a(first);
  load_b(first);
  for (int64_t l0 = first; l0 < last; l0 += 64) {
    stage_a(l0);
    stage_b();
    __syncthreads();
    if (l0 + 64 < last) {
      load_a(l0 + 64);
      load_b(l0 + 64);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i4_t a[4];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        a[x] = *reinterpret_cast<const i4_t*>(la + a_at(wi + 16 * x + m16, kk * 4 + g));
#pragma unroll
      for (int z = P - 1; z >= 0; --z) {            // small parts first
        i4_t b[NT];
#pragma unroll
        for (int y = 0; y < NT; ++y)
          b[y] = *reinterpret_cast<const i4_t*>(lb + z * kImage + pack_at(wj + 16 * y + m16, kk * 4 + g));
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < NT; ++y) acc[x][y] = mfma16<Kind::kBF16>(a[x], b[y], acc[x][y]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      const int64_t j = j0 + wj + 16 * y + m16;
      if (j >= p.n) continue;
      if (p.splits > 1) store4(p.part + (int64_t)blockIdx.y * p.n * I, I, i0 + wi + 16 * x + 4 * g, j, I, acc[x][y]);
      else store4(p.C, p.ldc, i0 + wi + 16 * x + 4 * g, j, I, acc[x][y]);
    }
}

// C = A^T B in tiles of 256 x 16 NT, four wavefronts of 64 x 16 NT, 128 contracted
// values at a time.  Each row of C belongs to one wavefront, so A need not pass
// through LDS: a lane's 16 bytes of codes are one block of its column, eight of
// them at a time are an operand of the matrix instruction, and the order of the
// contracted index is free as long as B's operands follow it.  LDS holds B's
// parts only (4096 x 512 transposed times 4096 x 11008 in binary32: 178 us with
// both in LDS, 162 so; 112 of them are the matrix instructions, 15 more go to
// LDS and 30 to the loads, of which two chunks under way are no faster).
template <typename T, int NT>
__global__ __launch_bounds__(256, 2) void mx4_apply_t_kernel(ApplyArgs<T> p) {
  constexpr int P = parts_of<T>(), BN = 16 * NT, kImage = BN * kChunkBytes;
  __shared__ __attribute__((aligned(1024))) char lds[P * 2 * kImage];     // [part][half of the 128 values]
  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int w = die_order(blockIdx.x, gridDim.x);
  const int64_t i0 = (int64_t)(w % p.ti) * 256 + wv * 64, j0 = (int64_t)(w / p.ti) * BN;
  const int64_t pitch = (int64_t)p.chunks * 128, spitch = (int64_t)p.chunks * 8;
  f4_t acc[4][NT];
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < NT; ++y) acc[x][y] = f4_t{0.f, 0.f, 0.f, 0.f};
  // A: block l0 / 32 + g of columns i0 + 16 x + m16.  Scales are loaded as the
  // words of four blocks: a byte would be widened, and so waited for, at once.
  uint4 wa[4];
  unsigned sa[4];
  auto load_a = [&](int64_t l0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int64_t c = min(i0 + 16 * x + m16, p.m - 1);
      wa[x] = *reinterpret_cast<const uint4*>(p.codes + c * pitch + l0 / 2 + 16 * g);
      sa[x] = *reinterpret_cast<const unsigned*>(p.scales + c * spitch + l0 / 32);
    }
  };
  // B: values l0 + 8 (t % 16) ... of columns j0 + t / 16 + 16 q.
  Raw8<T> rb[NT];
  const T* cb[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q) cb[q] = p.B + min(j0 + (t >> 4) + 16 * q, p.n - 1) * p.ldb;
  auto load_b = [&](int64_t l0) __attribute__((always_inline)) {
    if (l0 + 128 <= p.k) {
#pragma unroll
      for (int q = 0; q < NT; ++q) rb[q] = load_pack8(cb[q] + l0 + 8 * (t & 15));
    } else {
#pragma unroll
      for (int q = 0; q < NT; ++q) rb[q] = load_raw8(cb[q], l0 + 8 * (t & 15), p.k, true);
    }
  };
  const int64_t per = ((p.k + 127) / 128 + p.splits - 1) / p.splits * 128;
  const int64_t first = blockIdx.y * per, last = min(p.k, first + per);
  if (first < last) {
    load_a(first);
    load_b(first);
  }
  for (int64_t l0 = first; l0 < last; l0 += 128) {
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      i4_t o[P];
      parts8(rb[q], o);
#pragma unroll
      for (int z = 0; z < P; ++z)
        *reinterpret_cast<i4_t*>(lds + (2 * z + ((t >> 3) & 1)) * kImage + pack_at((t >> 4) + 16 * q, t & 7)) = o[z];
    }
    uint4 wc[4];
    float sc[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      wc[x] = wa[x];
      sc[x] = mx_scale((sa[x] >> (8 * g)) & 255u);
    }
    __syncthreads();
    if (l0 + 128 < last) {
      load_a(l0 + 128);
      load_b(l0 + 128);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {                   // values 32 g + 8 q ... of the chunk
      i4_t a[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        unsigned o[4];
        mx_decode8_bf16(q == 0 ? wc[x].x : q == 1 ? wc[x].y : q == 2 ? wc[x].z : wc[x].w, sc[x], o);
        a[x] = i4_t{(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
      }
#pragma unroll
      for (int z = P - 1; z >= 0; --z) {            // small parts first
        i4_t b[NT];
#pragma unroll
        for (int y = 0; y < NT; ++y)
          b[y] = *reinterpret_cast<const i4_t*>(lds + (2 * z + (g >> 1)) * kImage + pack_at(16 * y + m16, 4 * (g & 1) + q));
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < NT; ++y) acc[x][y] = mfma16<Kind::kBF16>(a[x], b[y], acc[x][y]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      const int64_t j = j0 + 16 * y + m16;
      if (j >= p.n) continue;
      if (p.splits > 1) store4(p.part + (int64_t)blockIdx.y * p.n * p.m, p.m, i0 + 16 * x + 4 * g, j, p.m, acc[x][y]);
      else store4(p.C, p.ldc, i0 + 16 * x + 4 * g, j, p.m, acc[x][y]);
    }
}

// C = A^T B for up to 16 NT columns of B: eight wavefronts take 16 columns of A
// and split its rows.  A lane's 16 bytes of codes are one block of its column;
// eight of them at a time are an operand of the matrix instruction, in which
// the order of the contracted index is free.  Bound by the latency of memory:
// all of a wavefront's loads of kFlight chunks, codes and B, are under way
// before the first is used (11008 x 4096, one column: 17 us with B loaded where
// it is used).
template <typename T, int NT>
__global__ __launch_bounds__(512) void mx4_apply_t_few_kernel(ApplyArgs<T> p) {
  constexpr int P = parts_of<T>(), kFlight = NT == 1 || (P == 1 && NT == 2) ? 2 : 1;
  __shared__ f4_t part[8 * NT * 64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int64_t i0 = (int64_t)blockIdx.x * 16;
  const int64_t row = min(i0 + m16, p.m - 1);
  const unsigned char *u = p.codes + row * p.chunks * 128 + g * 16, *su = p.scales + row * p.chunks * 8;
  f4_t acc[NT];
#pragma unroll
  for (int y = 0; y < NT; ++y) acc[y] = f4_t{0.f, 0.f, 0.f, 0.f};
  const int per = (p.chunks + 7) >> 3, c0 = wv * per, c1 = min(p.chunks, c0 + per);
  for (int c = c0; c < c1; c += kFlight) {
    uint4 a[kFlight][2];
    uint2 ka[kFlight];
    Raw8<T> r[kFlight][2][NT][4];
#pragma unroll
    for (int q = 0; q < kFlight; ++q) {
      const int64_t cc = min(c + q, c1 - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) a[q][h] = *reinterpret_cast<const uint4*>(u + cc * 128 + h * 64);
      ka[q] = *reinterpret_cast<const uint2*>(su + cc * 8);
    }
#pragma unroll
    for (int q = 0; q < kFlight; ++q) {
      // Whole chunks load without a look at the end.
      const int64_t l = (int64_t)(c + q) * 256 + g * 32;
      const bool whole = (int64_t)(c + q + 1) * 256 <= p.k;
#pragma unroll
      for (int y = 0; y < NT; ++y) {
        const int64_t j = 16 * y + m16;
        const T* col = p.B + min(j, p.n - 1) * p.ldb;
        const bool live = j < p.n && c + q < c1;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int z = 0; z < 8; ++z) r[q][h][y][e].v[z] = (T)0.f;
        if (whole) {
          if (live) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e) r[q][h][y][e] = load_pack8(col + l + 128 * h + 8 * e);
          }
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[q][h][y][e] = load_raw8(col, l + 128 * h + 8 * e, p.k, live);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < kFlight; ++q)
      if (c + q < c1) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sc = mx_scale(((h ? ka[q].y : ka[q].x) >> (8 * g)) & 255u);
          const unsigned w[4] = {a[q][h].x, a[q][h].y, a[q][h].z, a[q][h].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            unsigned o[4];
            mx_decode8_bf16(w[e], sc, o);
            const i4_t x = {(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
#pragma unroll
            for (int y = 0; y < NT; ++y) {
              i4_t b[P];
              parts8(r[q][h][y][e], b);
#pragma unroll
              for (int z = P - 1; z >= 0; --z) acc[y] = mfma16<Kind::kBF16>(x, b[z], acc[y]);
            }
          }
        }
      }
  }
  add_partials<8, NT>(part, acc, [&](int y, f4_t s) __attribute__((always_inline)) {
    const int64_t j = 16 * y + m16;
    if (j < p.n) store4(p.C, p.ldc, i0 + 4 * g, j, p.m, s);
  });
}

// C = A B for up to 16 NT columns of B: a workgroup of four wavefronts takes 128
// rows of A and splits its share of the columns.  A lane holds 8 rows, 8
// (l % 16) ..., of 8 columns, 8 (l / 16) ...: decoded and turned in registers
// that is one operand for each of the 8 rows r, of the instruction whose
// result rows are 8 m + r (their order is free).  The contraction is also
// split over workgroups, which write their sums for mx4_join_kernel, where
// there are few rows.
template <typename T, int NT>
__global__ __launch_bounds__(256) void mx4_apply_n_few_kernel(ApplyArgs<T> p) {
  constexpr int P = parts_of<T>();
  __shared__ f4_t part[4 * 8 * NT * 64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int64_t i0 = (int64_t)blockIdx.x * 128;
  const int64_t pitch = (int64_t)p.chunks * 128, spitch = (int64_t)p.chunks * 8;
  const int64_t row = i0 + 8 * m16;                     // kp is a multiple of 256
  const unsigned char *u = p.codes + row / 2, *su = p.scales + row / 32;
  // This wavefront's columns, 32 at a time.
  const int64_t groups = (p.m + 31) / 32, ways = (int64_t)p.splits * 4;
  const int64_t per = (groups + ways - 1) / ways, way = (int64_t)blockIdx.y * 4 + wv;
  const int64_t q0 = way * per, q1 = min(groups, q0 + per);
  f4_t acc[8 * NT];
#pragma unroll
  for (int y = 0; y < 8 * NT; ++y) acc[y] = f4_t{0.f, 0.f, 0.f, 0.f};
  for (int64_t q = q0; q < q1; ++q) {
    unsigned w[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t c = q * 32 + 8 * g + e, cc = min(c, p.m - 1);
      const unsigned x = *reinterpret_cast<const unsigned*>(u + cc * pitch);
      const unsigned y = su[cc * spitch];
      w[e] = c < p.m ? x : 0u;                          // past the last column: zeros, scale 1
      s[e] = c < p.m ? y : 127u;
    }
    i4_t b[NT][P];
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      const int64_t j = 16 * y + m16;
      const Raw8<T> r = load_raw8(p.B + min(j, p.n - 1) * p.ldb, q * 32 + 8 * g, p.m, j < p.n);
      parts8(r, b[y]);
    }
    unsigned o[8][4];
#pragma unroll
    for (int e = 0; e < 8; ++e) mx_decode8_bf16(w[e], mx_scale(s[e]), o[e]);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const unsigned sel = (r & 1) ? 0x07060302u : 0x05040100u;
      i4_t x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (int)__builtin_amdgcn_perm(o[2 * e + 1][r >> 1], o[2 * e][r >> 1], sel);
#pragma unroll
      for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int z = P - 1; z >= 0; --z) acc[r * NT + y] = mfma16<Kind::kBF16>(x, b[y][z], acc[r * NT + y]);
    }
  }
  add_partials<4, 8 * NT>(part, acc, [&](int ry, f4_t v) __attribute__((always_inline)) {
    const int r = ry / NT;
    const int64_t j = 16 * (ry % NT) + m16;
    if (j >= p.n) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + 8 * (4 * g + e) + r;
      if (i >= p.k) continue;
      if (p.splits > 1) p.part[((int64_t)blockIdx.y * p.n + j) * p.k + i] = v[e];
      else p.C[j * p.ldc + i] = (T)v[e];
    }
  });
}

// C = the splits' sums, added in order.
template <typename T>
__global__ __launch_bounds__(256) void mx4_join_kernel(ApplyArgs<T> p) {
  const int64_t rows = p.rows, step = p.n * rows;
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < step; w += (int64_t)gridDim.x * 256) {
    const float* q = p.part + w;
    float s = 0.f;
    for (int z0 = 0; z0 < p.splits; z0 += 8) {
      float v[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) v[z] = q[min(z0 + z, p.splits - 1) * step];
#pragma unroll
      for (int z = 0; z < 8; ++z)
        if (z0 + z < p.splits) s += v[z];
    }
    const int64_t j = w / rows;
    p.C[j * p.ldc + (w - j * rows)] = (T)s;
  }
}

// For more than 8 NT columns up to 16 NT (from one with NT = 1), if few_limit goes
// that far: else there is no such kernel, and no such call.
template <typename T, int NT>
void launch_few(ApplyArgs<T> p, int trans, hipStream_t st) {
  static_assert(few_limit(false, parts_of<T>()) <= 64 && few_limit(true, parts_of<T>()) <= 64, "columns");
  if (trans) {
    if constexpr (few_limit(true, parts_of<T>()) > 8 * NT)
      mx4_apply_t_few_kernel<T, NT><<<(unsigned)ceil_div(p.m, 16), 512, 0, st>>>(p);
  } else {
    mx4_apply_n_few_kernel<T, NT><<<dim3((unsigned)ceil_div(p.k, 128), (unsigned)p.splits), 256, 0, st>>>(p);
  }
}

template <typename T, int WI, int NT>
void launch_apply(ApplyArgs<T> p, int trans, hipStream_t st) {
  p.ti = (int)ceil_div(p.rows, 64 * WI);
  const dim3 grid((unsigned)(p.ti * ceil_div(p.n, 16 * NT * (4 / WI))), (unsigned)p.splits);
  if (!trans) {
    mx4_apply_kernel<T, false, WI, NT><<<grid, 256, 0, st>>>(p);
  } else {
    if constexpr (WI == 4) mx4_apply_t_kernel<T, NT><<<grid, 256, 0, st>>>(p);
    else mx4_apply_kernel<T, true, WI, NT><<<grid, 256, 0, st>>>(p);
  }
}

template <typename T>
rrf_status apply_typed(int trans, int64_t k, int64_t m, const void* codes, const void* scales, const void* B,
                       int64_t ldb, int64_t n, void* C, int64_t ldc, void* ws, hipStream_t st) {
  constexpr int P = parts_of<T>();
  const int64_t rows = trans ? m : k;
  ApplyArgs<T> p{(const unsigned char*)codes, (const unsigned char*)scales, k, m, (int)(mx_rows(k) / kMxPad),
                 (const T*)B, ldb, n, (T*)C, ldc, rows, 0, 1, (float*)ws};
  if (few_columns(trans, P, n)) {
    p.splits = trans ? 1 : (int)few_splits(k, m);
    if (n <= 16) launch_few<T, 1>(p, trans, st);
    else if (n <= 32) launch_few<T, 2>(p, trans, st);
    else launch_few<T, 4>(p, trans, st);
  } else {
    const ApplyChoice c = choose_apply(rows, trans ? k : m, n, P);
    p.splits = c.splits;
    switch (c.tile) {
      case 0: launch_apply<T, 4, 4>(p, trans, st); break;
      case 1: launch_apply<T, 4, 3>(p, trans, st); break;
      case 2: launch_apply<T, 2, 4>(p, trans, st); break;
      case 3: launch_apply<T, 2, 2>(p, trans, st); break;
      default: launch_apply<T, 2, 1>(p, trans, st);
    }
  }
  if (p.splits > 1)
    mx4_join_kernel<T><<<(unsigned)std::min<int64_t>(ceil_div(rows * n, 256), 4096), 256, 0, st>>>(p);
  return status_of(hipGetLastError());
}

// C <- 0 (a contraction over nothing).
template <typename T>
__global__ void mx4_zero_kernel(T* C, int64_t ldc, int64_t rows, int64_t n) {
  for (int64_t w = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; w < rows * n; w += (int64_t)gridDim.x * blockDim.x)
    C[w % rows + (w / rows) * ldc] = (T)0.f;
}

rrf_status zero(int dt, void* C, int64_t ldc, int64_t rows, int64_t n, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(rows * n, 256), 4096);
  if (dt == RRF_F32) mx4_zero_kernel<float><<<grid, 256, 0, st>>>((float*)C, ldc, rows, n);
  else mx4_zero_kernel<f16_t><<<grid, 256, 0, st>>>((f16_t*)C, ldc, rows, n);   // 0 in both 16-bit types
  return status_of(hipGetLastError());
}

bool bad_mx4(const void* codes, const void* scales) {
  return !codes || ((uintptr_t)codes & 15) || !scales || ((uintptr_t)scales & 7);
}

constexpr int64_t kMaxSide = 1 << 24;

size_t workspace_of(int dt, int trans, int64_t k, int64_t m, int64_t n) {
  if (k == 0 || m == 0 || n == 0) return 0;
  const int64_t splits = apply_splits(trans, dt == RRF_BF16 ? 1 : dt == RRF_F16 ? 2 : 3, k, m, n);
  return splits > 1 ? (size_t)(splits * (trans ? m : k) * n) * 4 : 0;
}

}  // namespace
}  // namespace ops
}  // namespace rrf

using namespace rrf::ops;
using rrf::ceil_div;

extern "C" {

rrf_status rrf_mx4_product(rrf_dtype dtype, int64_t M, int64_t N, int64_t k, const void* a_codes,
                           const void* a_scales, const void* b_codes, const void* b_scales, void* C, int64_t ldc,
                           void* hip_stream) {
  const int dt = int_bits(dtype);
  if (!valid_real(dt) || M < 0 || N < 0 || k < 0 || ldc < std::max<int64_t>(1, M)) return RRF_ERR_INVALID_ARG;
  if (M > kMaxSide || N > kMaxSide || k > kMaxSide) return RRF_ERR_SHAPE;
  if (M == 0 || N == 0) return RRF_OK;
  if (!C || ((uintptr_t)C % real_size(dt))) return RRF_ERR_INVALID_ARG;
  if (k > 0 && (bad_mx4(a_codes, a_scales) || bad_mx4(b_codes, b_scales))) return RRF_ERR_INVALID_ARG;
  if (ceil_div(M, 64) * ceil_div(N, 64) > (1ll << 31) - 1) return RRF_ERR_SHAPE;
  hipStream_t st = (hipStream_t)hip_stream;
  if (k == 0) return zero(dt, C, ldc, M, N, st);
  switch (dt) {
    case RRF_F32: return product_typed<float>(M, N, k, a_codes, a_scales, b_codes, b_scales, C, ldc, st);
    case RRF_BF16: return product_typed<bf16_t>(M, N, k, a_codes, a_scales, b_codes, b_scales, C, ldc, st);
    default: return product_typed<f16_t>(M, N, k, a_codes, a_scales, b_codes, b_scales, C, ldc, st);
  }
}

rrf_status rrf_mx4_apply_workspace(rrf_dtype dtype, int trans, int64_t k, int64_t m, int64_t n, size_t* bytes) {
  const int dt = int_bits(dtype);
  if (!bytes || !valid_real(dt) || k < 0 || m < 0 || n < 0) return RRF_ERR_INVALID_ARG;
  if (m > kMaxSide || n > kMaxSide || k > kMaxSide) return RRF_ERR_SHAPE;
  *bytes = workspace_of(dt, trans, k, m, n);
  return RRF_OK;
}

rrf_status rrf_mx4_apply(rrf_dtype dtype, int trans, int64_t k, int64_t m, const void* codes, const void* scales,
                         const void* B, int64_t ldb, int64_t n, void* C, int64_t ldc, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
  const int dt = int_bits(dtype);
  if (!valid_real(dt) || m < 0 || n < 0 || k < 0) return RRF_ERR_INVALID_ARG;
  const int64_t I = trans ? m : k, L = trans ? k : m;
  if (ldb < std::max<int64_t>(1, L) || ldc < std::max<int64_t>(1, I)) return RRF_ERR_INVALID_ARG;
  if (m > kMaxSide || n > kMaxSide || k > kMaxSide) return RRF_ERR_SHAPE;
  if (I == 0 || n == 0) return RRF_OK;
  if (!C || ((uintptr_t)C % real_size(dt))) return RRF_ERR_INVALID_ARG;
  if (ceil_div(I, 64) * ceil_div(n, 64) > (1ll << 31) - 1) return RRF_ERR_SHAPE;
  hipStream_t st = (hipStream_t)hip_stream;
  if (L == 0) return zero(dt, C, ldc, I, n, st);
  if (bad_mx4(codes, scales) || !B || ((uintptr_t)B % real_size(dt))) return RRF_ERR_INVALID_ARG;
  const size_t need = workspace_of(dt, trans, k, m, n);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return RRF_ERR_INVALID_ARG;
  switch (dt) {
    case RRF_F32: return apply_typed<float>(trans, k, m, codes, scales, B, ldb, n, C, ldc, workspace, st);
    case RRF_BF16: return apply_typed<bf16_t>(trans, k, m, codes, scales, B, ldb, n, C, ldc, workspace, st);
    default: return apply_typed<f16_t>(trans, k, m, codes, scales, B, ldb, n, C, ldc, workspace, st);
  }
}

}  // extern "C"
