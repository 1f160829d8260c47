// Orthogonalising a matrix by Newton-Schulz products, and the optimiser step
// around it (momentum before, weight decay and update after).
//
// With X_0 = G / (||G||_F + eps), X on its short side s x l (s <= l), a step
// with coefficients (a, b, c) is
//   A = X X^T,   P = a I + b A + c A^2,   X <- P X,
// which maps every singular value x to a x + b x^3 + c x^5 and leaves the
// singular vectors.  Every product is one launch of a tile product (wide.h,
// split.h).  A and P are symmetric, so only the tiles on and below the
// diagonal are formed and each is stored twice; A^2 turns into P in the
// epilogue; a product with X stores X in both orders ([l][s] is the next
// product's operand, [s][l] the next Gram product's), so that every operand is
// contiguous along the contracted index.  The last product writes the caller's
// matrix, or the updated weights, from its epilogue.
//
// Steps are taken in groups: X_{k+1} need not be formed to go on, because
//   A_{k+1} = P_k A_k P_k  and  X_{k+2} = P_{k+1} P_k X_k
// are products of the short side.  In units of s^3 a step by itself takes 3 r
// + 1 multiplications (r = l / s: Gram product r on half its tiles, A^2 1 on
// half, P X 2 r); a group of g steps 3 r + 4 g - 3.  Rounding A_k costs more
// then: an error in it grows by at most (max |a + b x^2 + c x^4|)^2 a step up
// to the next Gram product.  How many steps that allows depends on the type of
// the result (group_limit).
//
// Representation of the iterates.  Singular values stay below a bound that
// the host takes from the coefficients, so X, A and P are held in binary16
// times a power of two that puts the bound just below 2^15: 11 bits on the
// binary16 matrix rate, with no range to lose.  Every value is the sum of two
// such numbers (hi + lo, 22 bits, two planes) and a product of two of them is
// three (hi hi + hi lo + lo hi), accumulated in binary32.  That holds for bf16
// matrices too, though the result keeps 8 bits: the steps multiply small
// singular values, and with them what rounding adds there, by up to 3.4^5.  One
// plane of 11 bits was twice as fast (4096 x 11008: 2.5 ms against 5.1) and as
// exact on low rank with noise, but had two to three times the error of binary32
// steps where a twentieth of the rows or columns, or of the singular values,
// carries the matrix.
//
// Bound by the matrix instructions where the sides are large (bf16 4096 x 11008:
// 5.1 ms, 4096 x 4096 step: 3.4 ms, 1.21 PFLOP/s of 16-bit products), by LDS
// traffic of 64 x 64 tiles around 1700 (f32 3001 x 1733 step: 0.81 ms, 0.55
// PFLOP/s), by the latency of 17 launches where they are small (f32 500 x 300:
// 86 us).

#include "cost.h"
#include "split.h"
#include "store.h"
#include "wide.h"
#include "types.h"

#include <algorithm>
#include <cmath>

namespace rrf {
namespace ops {
namespace {

constexpr int kMaxSteps = 16;
constexpr int kMaxScale = 400;     // exponent of a stored matrix's scale: products of two stay in binary64
constexpr int kNormParts = 1024;   // partial sums of squares per matrix, at most
// Steps of a group from step k on at most, the growth of an error in A_k that it
// may cause, and whether it is taken though it saves no time.  Matrices that a
// twentieth of their rows, columns or singular values carries show the rounding
// of A_k most; the largest errors over 14 such and other spectra, short sides of
// 205 to 1030 (the first row: to 2000), five steps of the quintic (growth 12.3 a step):
//   groups    against 64 bits    over that of the same steps in binary32
//   2 1 1 1   4.2e-5             1.34
//   2 2 1     4.2e-5             4.7 (at 3.8e-6)
//   1 ...     6.4e-5             1.64 (every X is rounded; 1.42 at sides up to 300)
//   2 3       2.9e-4             160
// A bf16 result is rounded by 1.7e-3, an f16 one by 2.1e-4.
struct GroupLimit { int steps; double gain; bool always; };
GroupLimit group_limit(int dtype, int k, int64_t s) {
  if (dtype == RRF_BF16) return {3, 160.0, false};
  if (dtype == RRF_F16) return {2, 20.0, false};
  if (k == 0) return {2, 20.0, s > 384};
  return {1, 1.0, false};
}

// Factors of one matrix's epilogues, by group of steps (see factors_of).
struct Factors {
  float gram[kMaxSteps];                                 // acc -> stored A
  float mid[kMaxSteps];                                  // acc -> stored X, or the result
};

// What the host knows of a group of steps [first, first + count): scales of
// the stored matrices, powers of two from the bounds of their spectra.
struct Group {
  int first, count;
  double sa, sq;               // of A at its start, of the product of its P's
  double bound, gain;          // after it: of X's singular values; the largest x_k / x_0
};
struct Scales {
  int groups;
  double eps;
  Group group[kMaxSteps];
};
// And of a step: P stored = ax delta + bx A + cx A^2, and the factors of the
// products T = P A, A' = T P and Q' = P Q from accumulator to stored value.
struct Step {
  float ax, bx, cx, ft, fa, fq;
};

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }

// The caller's matrices (m x n column-major, batch of them) and the momentum.
template <typename T>
struct Source {
  const T* G; int64_t ldg, sg;
  float* M; int64_t ldm, sm;       // null: no momentum
  float mu; int nesterov;
  int64_t m, n;
};

// --- norms -------------------------------------------------------------------

// Eight consecutive rows from i on of a column at p (its first row), in
// binary32, zero past m: wide loads whatever their alignment, which the hardware
// allows (a 3001 x 1733 step's momentum pass: 40 -> 17 us).
template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t i, int64_t m, float (&v)[8]) {
  if (i + 8 <= m) {
    struct Pack { T v[8]; };
    const Pack x = *reinterpret_cast<const Pack*>(p + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f(x.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < m ? to_f(p[i + e]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, int64_t i, int64_t m, const float (&v)[8]) {
  if (i + 8 <= m) {
    struct Pack { float v[8]; };
    Pack x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v[e];
    *reinterpret_cast<Pack*>(p + i) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < m) p[i + e] = v[e];
  }
}

// part[batch][block] = sum of squares of the block's share of U, in binary64;
// with momentum, M <- mu M + G first.  A thread takes eight rows at a time,
// two groups of them in flight.
template <typename T>
__global__ __launch_bounds__(256) void ns_norm_kernel(Source<T> a, double* part) {
  const T* G = a.G + blockIdx.y * a.sg;
  float* M = a.M ? a.M + blockIdx.y * a.sm : nullptr;
  const int64_t groups = (a.m + 7) / 8, stride = (int64_t)gridDim.x * 256;
  const int64_t w0 = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t j = w0 / groups, x = w0 - j * groups;
  const int64_t dj = stride / groups, dx = stride - dj * groups;
  auto next = [&]() __attribute__((always_inline)) {
    j += dj;
    x += dx;
    if (x >= groups) { x -= groups; ++j; }
  };
  double sum = 0.0;
  while (j < a.n) {
    const int64_t j0 = j, i0 = x * 8;
    next();
    const int64_t j1 = j, i1 = x * 8;
    const bool two = j1 < a.n;
    next();
    float u[2][8] = {}, q[2][8];
    load8<T>(G + j0 * a.ldg, i0, a.m, u[0]);
    if (two) load8<T>(G + j1 * a.ldg, i1, a.m, u[1]);
    if (M) {
      load8<float>(M + j0 * a.ldm, i0, a.m, q[0]);
      if (two) load8<float>(M + j1 * a.ldm, i1, a.m, q[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float mm = a.mu * (h && !two ? 0.f : q[h][e]) + u[h][e];
          q[h][e] = mm;
          u[h][e] = a.nesterov ? u[h][e] + a.mu * mm : mm;
        }
      store8(M + j0 * a.ldm, i0, a.m, q[0]);
      if (two) store8(M + j1 * a.ldm, i1, a.m, q[1]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)u[h][e] * (double)u[h][e];
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  __shared__ double ws[4];
  if ((threadIdx.x & 63) == 0) ws[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * kNormParts + blockIdx.x] = ws[0] + ws[1] + ws[2] + ws[3];
}

// --- the first X ---------------------------------------------------------------

// Sum of a matrix's partials, in a fixed order, in every thread of the block.
__device__ __forceinline__ double total_of(const double* part, int parts, double* ws) {
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) v += part[i];
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) ws[threadIdx.x >> 6] = v;
  __syncthreads();
  return ws[0] + ws[1] + ws[2] + ws[3];
}

// Power of two that puts a norm into [2^13, 2^14); 0 for a norm of 0.
__device__ __forceinline__ int norm_exp(double norm) {
  if (!(norm > 0.0) || isinf(norm)) return 0;
  int e;
  (void)frexp(norm, &e);
  return 14 - e;
}

// The factors of one matrix.  X_k is stored times 2^x_k: the largest power
// with 2^x_k min(bound_k, gain_k nu) <= 2^15, nu = ||G|| / (||G|| + eps) (a
// matrix whose norm is far below eps stays far below the bound).
__device__ void factors_of(const Scales& sc, double norm, Factors* f) {
  const double inf = __longlong_as_double(0x7ff0000000000000ll);
  const double nu = norm / (norm + sc.eps);
  // stored X_0 / X_0; any number for a matrix of zeros, where 1 / eps^2 could
  // leave the range of the factors
  double sx = norm == 0.0 ? 1.0 : ldexp(norm + sc.eps, norm_exp(norm));
  if (!(norm < inf)) sx = inf - inf;                   // a result of NaN
  for (int k = 0; k < sc.groups; ++k) {
    const Group& q = sc.group[k];
    f->gram[k] = (float)(q.sa / (sx * sx));
    double next = 1.0;
    if (k + 1 < sc.groups) {
      double b = q.gain * nu;
      b = b < q.bound ? b : q.bound;
      int e = 0;
      if (b > 0.0) (void)frexp(b, &e);
      next = ldexp(1.0, min(15 - e, kMaxScale));
    }
    f->mid[k] = (float)(next / (sx * q.sq));
    sx = norm < inf ? next : inf - inf;
  }
}

// Eight values as hi and lo parts, stored at hi + at and lo + at.
__device__ __forceinline__ void store_parts(const float (&v)[8], f16_t* hi, f16_t* lo, int64_t at) {
  h8_t h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = (f16_t)v[e];
    l[e] = (f16_t)(v[e] - (float)h[e]);
  }
  *reinterpret_cast<h8_t*>(hi + at) = h;
  *reinterpret_cast<h8_t*>(lo + at) = l;
}

// Stored X_0 = 2^e U in both orders, zero past the matrix: a tile of 64 x 64
// values per workgroup, turned in LDS, in groups of eight values along the
// order that is read or written.  ij: [j][i], pitch ldi, rows_j rows; ji:
// [i][j], pitch ldj, rows_i rows; all four are multiples of 64.
template <typename T>
__global__ __launch_bounds__(256) void ns_load_kernel(Source<T> a, const double* part, int parts,
                                                      Scales sc, Factors* fac, f16_t* ij_hi,
                                                      f16_t* ij_lo, f16_t* ji_hi, f16_t* ji_lo,
                                                      int64_t ldi, int64_t ldj, int64_t stride) {
  __shared__ float tile[64][65];
  __shared__ double ws[4];
  const int b = blockIdx.z;
  const T* G = a.G + b * a.sg;
  const float* M = a.M ? a.M + b * a.sm : nullptr;
  const int64_t i0 = (int64_t)blockIdx.x * 64, j0 = (int64_t)blockIdx.y * 64;
  const int x = (threadIdx.x & 7) * 8, y = threadIdx.x >> 3;
  float u[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t i = i0 + x, j = j0 + y + 32 * h;
    if (j < a.n) {
      load8<T>(G + j * a.ldg, i, a.m, u[h]);
      if (M) {
        float q[8];
        load8<float>(M + j * a.ldm, i, a.m, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[h][e] = a.nesterov ? u[h][e] + a.mu * q[e] : q[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[h][e] = 0.f;
    }
  }
  const double norm = sqrt(total_of(part + (int64_t)b * kNormParts, parts, ws));
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) factors_of(sc, norm, fac + b);
  const int e2 = norm_exp(norm);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[h][e] = ldexpf(u[h][e], e2);
      tile[y + 32 * h][x + e] = u[h][e];
    }
    store_parts(u[h], ij_hi, ij_lo, b * stride + (j0 + y + 32 * h) * ldi + i0 + x);
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[h][e] = tile[x + e][y + 32 * h];
    store_parts(u[h], ji_hi, ji_lo, b * stride + (i0 + y + 32 * h) * ldj + j0 + x);
  }
}

// --- products --------------------------------------------------------------------

// hi + lo of four values.  hi must be the same number in both places: left to
// itself the compiler rounds a product v = x y to hi and takes fma(x, y, -hi')
// with a hi' rounded from the exact product, which differs from hi by a whole
// unit in one of 2^12 values; so v is fixed as a binary32 number first.
__device__ __forceinline__ void split4(float (&v)[4], h4_t& hi, h4_t& lo) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    asm volatile("" : "+v"(v[r]));
    hi[r] = (f16_t)v[r];
    lo[r] = (f16_t)(v[r] - (float)hi[r]);
  }
}

// The 4 x 4 values of four neighbouring lanes turned: lane s of a quad gives
// values 0..3 and gets value s of the four lanes.
__device__ __forceinline__ h4_t turn4(h4_t v, int lane) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  const bool high = lane & 2;
  // pairs (0, 1) and (2, 3) between lanes s and s ^ 2 ...
  const unsigned mine = high ? w.y : w.x;
  const unsigned got = (unsigned)__builtin_amdgcn_mov_dpp((int)(high ? w.x : w.y), 0x4e, 0xf, 0xf, true);
  const unsigned p0 = high ? got : mine, p1 = high ? mine : got;
  // ... and single values between s and s ^ 1
  const unsigned n0 = (unsigned)__builtin_amdgcn_mov_dpp((int)p0, 0xb1, 0xf, 0xf, true);
  const unsigned n1 = (unsigned)__builtin_amdgcn_mov_dpp((int)p1, 0xb1, 0xf, 0xf, true);
  const unsigned sel = (lane & 1) ? 0x03020706u : 0x05040100u;
  uint2 o;
  o.x = __builtin_amdgcn_perm(n0, p0, sel);
  o.y = __builtin_amdgcn_perm(n1, p1, sel);
  return __builtin_bit_cast(h4_t, o);
}

// What a product's result becomes.
enum class Role {
  kGram,      // A, both triangles
  kGramPart,  // a split's share of X X^T, in binary32, on the tiles of one triangle
  kPoly,      // P from A^2 and A, both triangles
  kSym,       // a product of two polynomials of A, both triangles
  kMid,       // the next X, in both orders
  kLast       // the caller's matrix
};
constexpr bool on_triangle(Role r) { return r != Role::kMid && r != Role::kLast; }

struct ProductArgs {
  Operands op;
  int64_t su, sv;              // batch strides in bytes
  int ti, tj;                  // tiles along i and j (a triangle: ti = tj)
  int group;
  const Factors* fac;
  float factor;                // kSym
  // stored results [j][i] (pitch ld) and turned [i][j] (pitch ldt), in values
  f16_t *hi, *lo, *thi, *tlo;
  int64_t ld, ldt, sd, sdt;
  int rows_i, rows_j;          // extent of the stored result, multiples of 64
  float* part;                 // kGramPart: [batch][split][j][i], pitch ld
  int splits;
  // kPoly
  const f16_t *ahi, *alo;
  float ax, bx, cx;
  // kLast: the caller's matrix
  void* O; int64_t ldo, so;
  void* W; int64_t ldw, sw;
  float keep, rate;            // W <- keep W - rate O
  int m, n;
};

// Four values of a stored result at (i .. i + 3, j), its parts in both orders.
__device__ __forceinline__ void store_both(const ProductArgs& p, int b, int i, int j, float (&v)[4], bool turned,
                                           int lane) {
  h4_t hi, lo;
  split4(v, hi, lo);
  const int64_t at = b * p.sd + j * p.ld + i;
  *reinterpret_cast<h4_t*>(p.hi + at) = hi;
  *reinterpret_cast<h4_t*>(p.lo + at) = lo;
  if (turned) {
    const int64_t tat = b * p.sdt + (int64_t)(i + (lane & 3)) * p.ldt + (j & ~3);
    *reinterpret_cast<h4_t*>(p.thi + tat) = turn4(hi, lane);
    *reinterpret_cast<h4_t*>(p.tlo + tat) = turn4(lo, lane);
  }
}

// One lane's share of a 16 x 16 tile of the product, rows i .. i + 3 of column
// j (in range): what is stored for it, before its rounding.
template <Role ROLE>
__device__ __forceinline__ f4_t value(const ProductArgs& p, int b, int i, int j, f4_t acc, float factor) {
  if constexpr (ROLE == Role::kPoly) {
    const int64_t at = b * p.sd + j * p.ld + i;
    const h4_t ah = *reinterpret_cast<const h4_t*>(p.ahi + at), al = *reinterpret_cast<const h4_t*>(p.alo + at);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      acc[r] = p.bx * ((float)ah[r] + (float)al[r]) + p.cx * acc[r] + (i + r == j ? p.ax : 0.f);
  } else if constexpr (ROLE != Role::kGramPart) {
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] *= factor;
  }
  return acc;
}

// The end of a small tile's 16 x 16 part, stored as the lanes hold it.
template <typename T, Role ROLE>
__device__ __forceinline__ void finish(const ProductArgs& p, int b, int split, int i, int j, f4_t acc,
                                       bool turned, float factor, int lane) {
  // Stored extents are multiples of 64: a 16 x 16 part is in or out as a whole.
  if (i >= p.rows_i || j >= p.rows_j) return;
  acc = value<ROLE>(p, b, i, j, acc, factor);
  if constexpr (ROLE == Role::kLast) {
    if (i >= p.m || j >= p.n) return;
    T* out = p.W ? (T*)p.W + b * p.sw + i + j * p.ldw : (T*)p.O + b * p.so + i + j * p.ldo;
    Run<T, 4> o = {};
    if (p.W) o = read_run<T, 4>(out, i, p.m);
#pragma unroll
    for (int r = 0; r < 4; ++r) o.v[r] = (T)(p.W ? p.keep * to_f(o.v[r]) - p.rate * acc[r] : acc[r]);
    write_run<T, 4>(out, i, p.m, o);
  } else if constexpr (ROLE == Role::kGramPart) {
    *reinterpret_cast<f4_t*>(p.part + ((int64_t)(b * p.splits + split) * p.rows_j + j) * p.ld + i) = acc;
  } else {
    float v[4] = {acc[0], acc[1], acc[2], acc[3]};
    store_both(p, b, i, j, v, turned, lane);
  }
}

// The end of a wavefront's 16 TS x 16 TS part of a large tile, whose corner is
// (iw, jw), in strips through LDS (store.h; Q X of 4096 x 11008 with one plane
// each: 421 -> 388 us).
template <typename T, Role ROLE, int TS>
__device__ __forceinline__ void finish_tile(const ProductArgs& p, int b, int split, int iw, int jw, f4_t (&acc)[TS][TS],
                                            bool turned, float factor, int lane, char* buf) {
  const int g = lane >> 4, m16 = lane & 15;
#pragma unroll
  for (int y = 0; y < TS; ++y)
#pragma unroll
    for (int x = 0; x < TS; ++x) {
      const int i = iw + 16 * x + 4 * g, j = jw + 16 * y + m16;
      if (i < p.rows_i && j < p.rows_j) acc[x][y] = value<ROLE>(p, b, i, j, acc[x][y], factor);
    }
  if constexpr (ROLE == Role::kGramPart) {
    float* part = p.part + (int64_t)(b * p.splits + split) * p.rows_j * p.ld;
#pragma unroll
    for (int y = 0; y < TS; ++y)
#pragma unroll
      for (int x = 0; x < TS; ++x) {
        const int i = iw + 16 * x + 4 * g, j = jw + 16 * y + m16;
        if (i < p.rows_i && j < p.rows_j) *reinterpret_cast<f4_t*>(part + j * p.ld + i) = acc[x][y];
      }
  } else if constexpr (ROLE == Role::kLast) {
    if (p.W)
      store_tile<T, TS, true>(acc, (T*)p.W + b * p.sw, p.ldw, iw, jw, p.m, p.n, lane, buf,
                              [&](float old, float o) __attribute__((always_inline)) { return p.keep * old - p.rate * o; });
    else
      store_tile<T, TS, false>(acc, (T*)p.O + b * p.so, p.ldo, iw, jw, p.m, p.n, lane, buf,
                               [](float, float o) __attribute__((always_inline)) { return o; });
  } else {
    constexpr int kPitch = 32 * TS + 16, kRow = 2 * TS, kRuns = 16 * kRow / 64;
    // Strip z (of 16 rows) in buf + part goes to rows j0 ... from column i0 on.
    auto leave = [&](char* from, f16_t* to, int64_t ld, int i0, int j0, int rows_i, int rows_j) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < kRuns; ++q) {
        const int k = q * 64 + lane, i = i0 + k % kRow * 8, j = j0 + k / kRow;
        const i4_t v = *reinterpret_cast<const i4_t*>(from + k / kRow * kPitch + k % kRow * 16);
        if (i < rows_i && j < rows_j) *reinterpret_cast<i4_t*>(to + j * ld + i) = v;
      }
    };
    auto strips = [&](bool turn, f16_t* hi, f16_t* lo, int64_t ld, int i0, int j0, int rows_i, int rows_j) __attribute__((always_inline)) {
#pragma unroll
      for (int z = 0; z < TS; ++z) {
#pragma unroll
        for (int e = 0; e < TS; ++e) {
          const f4_t a = turn ? acc[z][e] : acc[e][z];
          float v[4] = {a[0], a[1], a[2], a[3]};
          h4_t h, l;
          split4(v, h, l);
          char* at = turn ? buf + (4 * g + (lane & 3)) * kPitch + (16 * e + (m16 & 12)) * 2
                          : buf + m16 * kPitch + (16 * e + 4 * g) * 2;
          *reinterpret_cast<h4_t*>(at) = turn ? turn4(h, lane) : h;
          *reinterpret_cast<h4_t*>(at + 16 * kPitch) = turn ? turn4(l, lane) : l;
        }
        wave_lds();
        leave(buf, hi, ld, i0, j0 + 16 * z, rows_i, rows_j);
        leave(buf + 16 * kPitch, lo, ld, i0, j0 + 16 * z, rows_i, rows_j);
        wave_lds();
      }
    };
    strips(false, p.hi + b * p.sd, p.lo + b * p.sd, p.ld, iw, jw, p.rows_i, p.rows_j);
    if (turned) strips(true, p.thi + b * p.sdt, p.tlo + b * p.sdt, p.ldt, jw, iw, p.rows_j, p.rows_i);
  }
}

// Tile (bi, bj), bi <= bj, number w of the triangle.
__device__ __forceinline__ void triangle_tile(int w, int& bi, int& bj) {
  bj = (int)((sqrtf(8.f * w + 1.f) - 1.f) * 0.5f);
  while ((bj + 1) * (bj + 2) / 2 <= w) ++bj;
  while (bj * (bj + 1) / 2 > w) --bj;
  bi = w - bj * (bj + 1) / 2;
}

// Tile (bi, bj), bi <= bj < n, number w of the triangle in bands of H tiles
// along i: a band's corner, then its columns.  A die's tiles (32, or 64 where
// two workgroups share a unit) then share 12 to 16 operand rows of tiles, not
// 24 (A^2 of 1733: 45 -> 42 us; with one plane each, Gram product of 4096 x
// 11008: 175 -> 166).  With less than 64 tiles there is nothing to gain.
template <int H>
__device__ __forceinline__ void band_triangle_tile(int w, int n, int& bi, int& bj) {
  int i0 = 0, h = min(H, n);
  for (;;) {
    const int tiles = h * (h + 1) / 2 + h * (n - i0 - h);
    if (w < tiles) break;
    w -= tiles;
    i0 += h;
    h = min(H, n - i0);
  }
  const int corner = h * (h + 1) / 2;
  if (w < corner) {
    triangle_tile(w, bi, bj);
    bi += i0;
    bj += i0;
  } else {
    bi = i0 + (w - corner) % h;
    bj = i0 + h + (w - corner) / h;
  }
}

// TS = 0: the split tile of 32 x 32; else the wide tile of 32 TS with S stages.
template <typename T, Role ROLE, int TS, int S>
__global__ __launch_bounds__(256) void ns_product_kernel(ProductArgs p) {
  const int b = blockIdx.z, split = blockIdx.y;
  int bi, bj;
  const bool ordered = TS > 0 && gridDim.x >= 64;
  const int w = ordered ? die_order(blockIdx.x, gridDim.x) : blockIdx.x;
  if (on_triangle(ROLE)) {
    if (ordered) band_triangle_tile<TS >= 6 ? 6 : 8>(w, p.ti, bi, bj);
    else triangle_tile(w, bi, bj);
  } else if (ordered) {
    band_tile(w, p.ti, p.tj, bi, bj);
  } else {
    bi = w % p.ti;
    bj = w / p.ti;
  }
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const bool turned = ROLE == Role::kMid || bi != bj;
  const float factor = ROLE == Role::kSym ? p.factor : ROLE == Role::kGram ? p.fac[b].gram[p.group] : p.fac[b].mid[p.group];
  int64_t first = 0;             // byte of a row to start at, chunks from there
  int nk = p.op.nk;
  if (ROLE == Role::kGramPart) {
    // this split's chunks of a row
    const int per = (p.op.nk + p.splits - 1) / p.splits, k0 = split * per;
    nk = min(per, p.op.nk - k0);
    first = (int64_t)k0 * kChunkBytes;
  }
  if constexpr (TS == 0) {
    typedef SplitTile<2, 2> ST;
    __shared__ __attribute__((aligned(1024))) char lds[ST::kLds];
    const int i0 = bi * ST::BM, j0 = bj * ST::BN;
    ST::run(p.op, nk, b * p.su + first, b * p.sv + first, i0, j0, lds, [&](int x, int y, f4_t v) __attribute__((always_inline)) {
      finish<T, ROLE>(p, b, split, i0 + 16 * x + 4 * g, j0 + 16 * y + m16, v, turned, factor, lane);
    });
  } else {
    constexpr int size = 32 * TS, kShare = 16 * (64 * TS + 32);      // LDS of a wavefront in finish_tile
    f4_t acc[TS][TS];
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int iw = bi * size + (wv & 1) * 16 * TS, jw = bj * size + (wv >> 1) * 16 * TS;
    typedef WideTile<TS, S> WT;
    static_assert(4 * kShare <= WT::kLds, "LDS");
    __shared__ __attribute__((aligned(1024))) char lds[WT::kLds];
    WT::run(p.op, 2 * nk, b * p.su + first, b * p.sv + first, bi * size, bj * size, lds, acc);
    finish_tile<T, ROLE, TS>(p, b, split, iw, jw, acc, turned, factor, lane, lds + wv * kShare);
  }
}

// A from the splits' shares, added in order: a 32 x 32 block (bi <= bj) of the
// triangle per workgroup, which is as fine as the smallest tiles that the
// shares were formed by; a wavefront takes 16 x 16 of it, eight splits' values
// in flight.
__global__ __launch_bounds__(256) void ns_join_kernel(ProductArgs p) {
  int bi, bj;
  triangle_tile(blockIdx.x, bi, bj);
  const int b = blockIdx.z, lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15, wv = threadIdx.x >> 6;
  const int i = bi * 32 + 16 * (wv & 1) + 4 * g, j = bj * 32 + 16 * (wv >> 1) + m16;
  const float factor = p.fac[b].gram[p.group];
  const float* q = p.part + ((int64_t)b * p.splits * p.rows_j + j) * p.ld + i;
  const int64_t step = (int64_t)p.rows_j * p.ld;
  f4_t s = {0.f, 0.f, 0.f, 0.f};
  for (int z0 = 0; z0 < p.splits; z0 += 8) {
    f4_t v[8];
#pragma unroll
    for (int z = 0; z < 8; ++z) v[z] = *reinterpret_cast<const f4_t*>(q + min(z0 + z, p.splits - 1) * step);
#pragma unroll
    for (int z = 0; z < 8; ++z)
      if (z0 + z < p.splits) s += v[z];
  }
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = s[r] * factor;
  store_both(p, b, i, j, v, bi != bj, lane);
}

// --- host ------------------------------------------------------------------------

struct Layout {
  int64_t s, l, sp, lp;        // short and long side, padded to whole chunks
  size_t part, fac, xl[2], xs[2][2], sq[5][2], total;      // byte offsets
  size_t share[2];             // of the Gram product of the X in xs[0], xs[1]
};

Layout layout_of(int dtype, int64_t m, int64_t n, int64_t batch) {
  Layout y{};
  y.s = std::min(m, n);
  y.l = std::max(m, n);
  y.sp = round_up(y.s, 64);
  y.lp = round_up(y.l, 64);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = (size_t)round_up((int64_t)(at + bytes), 256);
    return o;
  };
  const size_t x = (size_t)(y.sp * y.lp * batch) * 2, q = (size_t)(y.sp * y.sp * batch) * 2;
  y.part = take((size_t)batch * kNormParts * 8);
  y.fac = take((size_t)batch * sizeof(Factors));
  for (int h = 0; h < 2; ++h) {
    y.xl[h] = take(x);
    for (int z = 0; z < 5; ++z) y.sq[z][h] = take(q);
  }
  for (int z = 0; z < 2; ++z)
    for (int h = 0; h < 2; ++h) y.xs[z][h] = take(x);
  // A call on bf16 matrices needs less room than one on f32 or f16 ones: the
  // shares lie where the next X will be, not in a place of their own.
  const int64_t splits = gram_splits(y.sp, y.lp);
  const size_t share = splits > 1 ? (size_t)(y.sp * y.sp * batch * splits) * 4 : 0;
  for (int z = 0; z < 2; ++z) y.share[z] = y.xs[z ^ 1][0];
  if (dtype != RRF_BF16 && share > 0) y.share[0] = y.share[1] = take(share);
  y.total = at;
  return y;
}

// Largest power of two that keeps x times it below 2^15, and the product for
// x of 1.02 times what the bounds say (the spectrum's bound is of the exact
// matrices, and an entry is below it).
double scale_of(double x) {
  int e;
  (void)std::frexp(1.02 * x, &e);
  return std::ldexp(1.0, std::min(15 - e, kMaxScale));
}

// The groups of the steps and all scales, for matrices of sides s and l.
// Bounds of the singular values come from the coefficients: X_0's lie in
// [0, 1], and the largest |x p(x)| and |p(x)| are taken over a fine grid, with
// a margin for what lies between its points and for rounding.  False if a
// bound leaves the range that binary16 times a power of two can hold.
bool scales_of(int dtype, const double* coeffs, int steps, double eps, const Layout& y, int64_t batch, Scales* sc,
               Step* step) {
  double top[kMaxSteps + 1], pm[kMaxSteps];      // bounds of X_k's singular values and of |p_k|
  top[0] = 1.0;
  for (int k = 0; k < steps; ++k) {
    const double a = coeffs[3 * k], b = coeffs[3 * k + 1], c = coeffs[3 * k + 2];
    double xm = 0.0, qm = 0.0;
    for (int i = 0; i <= 4096; ++i) {
      const double x = top[k] * i / 4096.0, q = a + x * x * (b + c * x * x);
      qm = std::max(qm, std::fabs(q));
      xm = std::max(xm, std::fabs(x * q));
    }
    top[k + 1] = 1.02 * xm;
    pm[k] = 1.02 * qm;
    if (!(xm > 0.0) || !(top[k + 1] < 1e4) || !(pm[k] < 1e4)) return false;
  }
  // Time of a group's products with X, and of one of the short side.
  double long_time = 0.0, short_time = 0.0;
  if (batch > 0 && y.s > 0) {
    long_time = choose_tile(y.sp, y.sp, true, batch, y.lp / 64, gram_splits(y.sp, y.lp)).time +
                choose_tile(y.sp, y.lp, false, batch, y.sp / 64, 1).time;
    short_time = choose_tile(y.sp, y.sp, true, batch, y.sp / 64, 1).time;
  }
  sc->eps = eps;
  sc->groups = 0;
  double gain = 1.0;
  for (int k = 0; k < steps;) {
    // The number of steps with the least time a step, within the limits.
    int count = 1;
    double growth = 1.0, least = long_time + short_time, product = pm[k];
    const GroupLimit limit = group_limit(dtype, k, y.s);
    for (int g = 2; g <= limit.steps && k + g <= steps; ++g) {
      growth *= pm[k + g - 2] * pm[k + g - 2];
      product *= pm[k + g - 1];
      const double work = (long_time + (4 * g - 3) * short_time) / g;
      if (growth > limit.gain || product > 1e4) break;
      if (work < least || limit.always) { least = work; count = g; }
    }
    Group& q = sc->group[sc->groups++];
    q.first = k;
    q.count = count;
    q.sa = scale_of(top[k] * top[k]);
    double sq = 1.0;
    product = 1.0;
    for (int j = k; j < k + count; ++j) {
      const double sa = scale_of(top[j] * top[j]), sp = scale_of(pm[j]);
      Step& t = step[j];
      t.ax = (float)(coeffs[3 * j] * sp);
      t.bx = (float)(coeffs[3 * j + 1] * sp / sa);
      t.cx = (float)(coeffs[3 * j + 2] * sp / (sa * sa));
      const double st = scale_of(pm[j] * top[j] * top[j]);
      t.ft = (float)(st / (sp * sa));
      t.fa = (float)(scale_of(top[j + 1] * top[j + 1]) / (st * sp));
      product *= pm[j];
      const double sn = j == k ? sp : scale_of(product);
      t.fq = (float)(sn / (sp * sq));
      sq = sn;
    }
    gain *= product;
    q.sq = sq;
    q.bound = top[k + count];
    q.gain = gain;
    k += count;
  }
  return true;
}

template <typename T>
struct Call {
  Source<T> src;
  int64_t batch;
  T* O; int64_t ldo, so;
  T* W; int64_t ldw, sw;
  float keep, rate;
};

template <typename T, Role ROLE, int TS, int S>
hipError_t launch_tiles(ProductArgs p, int64_t batch, hipStream_t st) {
  constexpr int size = TS == 0 ? 32 : 32 * TS;
  p.ti = (int)ceil_div(p.op.rows_u, size);
  p.tj = (int)ceil_div(p.op.rows_v, size);
  const int64_t tiles = on_triangle(ROLE) ? (int64_t)p.ti * (p.ti + 1) / 2 : (int64_t)p.ti * p.tj;
  const unsigned splits = ROLE == Role::kGramPart ? p.splits : 1;
  const dim3 grid((unsigned)tiles, splits, (unsigned)batch);
  ns_product_kernel<T, ROLE, TS, S><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

// T: the caller's type, for its matrix (kLast); what is not the caller's does
// not depend on it.
template <typename T, Role ROLE>
hipError_t launch_product(const ProductArgs& p, int tile, int64_t batch, hipStream_t st) {
  switch (tile) {
    case 0: return launch_tiles<T, ROLE, 0, 0>(p, batch, st);
    case 1: return launch_tiles<T, ROLE, 2, 4>(p, batch, st);
    case 2: {
      const bool deep = one_a_unit(p.op.rows_u, p.op.rows_v, on_triangle(ROLE), batch,
                                   ROLE == Role::kGramPart ? p.splits : 1);
      return deep ? launch_tiles<T, ROLE, 4, 4>(p, batch, st) : launch_tiles<T, ROLE, 4, 2>(p, batch, st);
    }
    case 3: return launch_tiles<T, ROLE, 6, 3>(p, batch, st);
    default: return launch_tiles<T, ROLE, 8, 2>(p, batch, st);
  }
}

template <typename T>
hipError_t iterate(const Call<T>& c, const Scales& sc, const Step* step, const Layout& y, char* ws, hipStream_t st) {
  const int64_t m = c.src.m, n = c.src.n;
  const bool wide_m = m <= n;      // the contiguous index is the short one
  double* part = (double*)(ws + y.part);
  Factors* fac = (Factors*)(ws + y.fac);
  auto plane = [&](size_t o) { return (f16_t*)(ws + o); };
  const int64_t sx = y.sp * y.lp, sq_stride = y.sp * y.sp;
  hipError_t e;
  // About four groups of eight rows a thread, as many as the device holds at once.
  const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, 2048 / c.batch),
                    std::min<int64_t>(kNormParts, ceil_div(ceil_div(m, 8) * n, 1024))));
  ns_norm_kernel<T><<<dim3(parts, (unsigned)c.batch), 256, 0, st>>>(c.src, part);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  {
    f16_t *xs_hi = plane(y.xs[0][0]), *xs_lo = plane(y.xs[0][1]);
    f16_t *xl_hi = plane(y.xl[0]), *xl_lo = plane(y.xl[1]);
    const int64_t ip = round_up(m, 64), jp = round_up(n, 64);
    const dim3 grid((unsigned)(ip / 64), (unsigned)(jp / 64), (unsigned)c.batch);
    const bool sw = !wide_m;      // ij is then the long side's order
    ns_load_kernel<T><<<grid, 256, 0, st>>>(c.src, part, parts, sc, fac, sw ? xl_hi : xs_hi, sw ? xl_lo : xs_lo,
                                 sw ? xs_hi : xl_hi, sw ? xs_lo : xl_lo, ip, jp, sx);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  auto operands = [&](f16_t* uh, f16_t* ul, f16_t* vh, f16_t* vl, int64_t ru, int64_t rv, int64_t kp) {
    Operands o{};
    o.u = (const char*)uh; o.ul = (const char*)ul;
    o.v = (const char*)vh; o.vl = (const char*)vl;
    o.rows_u = (int)ru; o.rows_v = (int)rv;
    o.ldu = o.ldv = kp * 2;
    o.nk = (int)(kp / 64);
    return o;
  };
  struct Square { f16_t *hi, *lo; };
  Square sq[5];
  for (int z = 0; z < 5; ++z) sq[z] = Square{plane(y.sq[z][0]), plane(y.sq[z][1])};
  const Square A = sq[0], B = sq[1], P = sq[2];
  // A product of short-side matrices, both triangles stored.
  auto square = [&](const Square& u, const Square& v, const Square& out) {
    ProductArgs q{};
    q.fac = fac;
    q.op = operands(u.hi, u.lo, v.hi, v.lo, y.sp, y.sp, y.sp);
    q.su = q.sv = sq_stride * 2;
    q.hi = q.thi = out.hi; q.lo = q.tlo = out.lo;
    q.ld = q.ldt = y.sp; q.sd = q.sdt = sq_stride;
    q.rows_i = q.rows_j = (int)y.sp;
    return q;
  };
  int cur = 0;
  for (int gr = 0; gr < sc.groups; ++gr) {
    const Group& grp = sc.group[gr];
    f16_t *xl = plane(y.xl[0]), *xll = plane(y.xl[1]);
    f16_t *X = plane(y.xs[cur][0]), *Xl = plane(y.xs[cur][1]);
    Square Q = sq[3], R = sq[4];       // the product of the group's P's, and the next one's place
    {
      ProductArgs q = square(A, A, A);
      q.group = gr;
      q.op = operands(xl, xll, xl, xll, y.sp, y.sp, y.lp);
      q.su = q.sv = sx * 2;
      const Choice t = choose_tile(y.sp, y.sp, true, c.batch, q.op.nk, gram_splits(y.sp, y.lp));
      if (t.splits > 1) {
        q.splits = t.splits;
        q.part = (float*)(ws + y.share[cur]);
        if ((e = launch_product<float, Role::kGramPart>(q, t.tile, c.batch, st)) != hipSuccess) return e;
        const int64_t blocks = y.sp / 32;
        ns_join_kernel<<<dim3((unsigned)(blocks * (blocks + 1) / 2), 1, (unsigned)c.batch), 256, 0, st>>>(q);
        e = hipGetLastError();
      } else {
        e = launch_product<float, Role::kGram>(q, t.tile, c.batch, st);
      }
      if (e != hipSuccess) return e;
    }
    for (int k = 0; k < grp.count; ++k) {
      const Step& t = step[grp.first + k];
      const Square& out = k == 0 ? Q : P;
      ProductArgs q = square(A, A, out);
      const int tile = choose_tile(y.sp, y.sp, true, c.batch, q.op.nk, 1).tile;
      q.ahi = A.hi; q.alo = A.lo;
      q.ax = t.ax; q.bx = t.bx; q.cx = t.cx;
      if ((e = launch_product<float, Role::kPoly>(q, tile, c.batch, st)) != hipSuccess) return e;
      if (k + 1 < grp.count) {
        q = square(out, A, B);
        q.factor = t.ft;
        if ((e = launch_product<float, Role::kSym>(q, tile, c.batch, st)) != hipSuccess) return e;
        q = square(B, out, A);
        q.factor = t.fa;
        if ((e = launch_product<float, Role::kSym>(q, tile, c.batch, st)) != hipSuccess) return e;
      }
      if (k > 0) {
        q = square(P, Q, R);
        q.factor = t.fq;
        if ((e = launch_product<float, Role::kSym>(q, tile, c.batch, st)) != hipSuccess) return e;
        std::swap(Q, R);
      }
    }
    ProductArgs q{};
    q.group = gr;
    q.fac = fac;
    q.rows_i = (int)(wide_m || gr + 1 < sc.groups ? y.sp : y.lp);
    q.rows_j = (int)(wide_m || gr + 1 < sc.groups ? y.lp : y.sp);
    if (gr + 1 < sc.groups) {
      q.op = operands(Q.hi, Q.lo, X, Xl, y.sp, y.lp, y.sp);
      q.su = sq_stride * 2; q.sv = sx * 2;
      q.hi = plane(y.xs[cur ^ 1][0]); q.lo = plane(y.xs[cur ^ 1][1]);
      q.thi = xl; q.tlo = xll;
      q.ld = y.sp; q.ldt = y.lp; q.sd = q.sdt = sx;
      e = launch_product<float, Role::kMid>(
          q, choose_tile(y.sp, y.lp, false, c.batch, q.op.nk, 1).tile, c.batch, st);
      if (e != hipSuccess) return e;
      cur ^= 1;
    } else {
      // Rows i of the result are the caller's contiguous index.
      if (wide_m) {
        q.op = operands(Q.hi, Q.lo, X, Xl, y.sp, y.lp, y.sp);
        q.su = sq_stride * 2; q.sv = sx * 2;
      } else {
        q.op = operands(X, Xl, Q.hi, Q.lo, y.lp, y.sp, y.sp);
        q.su = sx * 2; q.sv = sq_stride * 2;
      }
      q.O = c.O; q.ldo = c.ldo; q.so = c.so;
      q.W = c.W; q.ldw = c.ldw; q.sw = c.sw;
      q.keep = c.keep; q.rate = c.rate;
      q.m = (int)m; q.n = (int)n;
      e = launch_product<T, Role::kLast>(
          q, choose_tile(y.sp, y.lp, false, c.batch, q.op.nk, 1).tile, c.batch, st);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

// The steps of a call.
struct Schedule {
  Scales scales;
  Step step[kMaxSteps];
};

// What every call checks: sizes, coefficients, workspace.
rrf_status check_common(int dtype, int64_t m, int64_t n, int64_t batch, const double* coeffs, int64_t steps,
                        double eps, const void* ws, size_t bytes, Schedule* sc, Layout* y) {
  if (!valid_real(dtype) || m < 0 || n < 0 || batch < 0) return RRF_ERR_INVALID_ARG;
  if (!coeffs || steps < 1 || steps > kMaxSteps || !(eps > 0.0) || !std::isfinite(eps))
    return RRF_ERR_INVALID_ARG;
  for (int64_t i = 0; i < 3 * steps; ++i)
    if (!std::isfinite(coeffs[i])) return RRF_ERR_INVALID_ARG;
  if (m > (1 << 20) || n > (1 << 20) || std::min(m, n) > 65536 || batch > 65535) return RRF_ERR_SHAPE;
  *y = layout_of(dtype, m, n, batch);
  if (!scales_of(dtype, coeffs, (int)steps, eps, *y, batch, &sc->scales, sc->step)) return RRF_ERR_INVALID_ARG;
  if (m == 0 || n == 0 || batch == 0) return RRF_OK;
  if (!ws || ((uintptr_t)ws & 255) || bytes < y->total) return RRF_ERR_INVALID_ARG;
  return RRF_OK;
}

bool bad_matrix(const void* p, int64_t ld, int64_t stride, int64_t m, int64_t n, int64_t batch, int size) {
  return !p || ((uintptr_t)p % size) || ld < std::max<int64_t>(1, m) ||
         (batch > 1 && stride < 0);
}

template <typename T>
rrf_status ortho_typed(int64_t m, int64_t n, int64_t batch, const void* G, int64_t ldg, int64_t sg, void* O,
                       int64_t ldo, int64_t so, const Schedule& sc, const Layout& y, void* ws, void* stream) {
  Call<T> c{};
  c.src = Source<T>{(const T*)G, ldg, sg, nullptr, 0, 0, 0.f, 0, m, n};
  c.batch = batch;
  c.O = (T*)O; c.ldo = ldo; c.so = so;
  return status_of(iterate<T>(c, sc.scales, sc.step, y, (char*)ws, (hipStream_t)stream));
}

template <typename T>
rrf_status muon_typed(int64_t m, int64_t n, int64_t batch, void* W, int64_t ldw, int64_t sw, float* M,
                      int64_t ldm, int64_t sm, const void* G, int64_t ldg, int64_t sg, float mu, int nesterov,
                      float keep, float rate, const Schedule& sc, const Layout& y, void* ws, void* stream) {
  Call<T> c{};
  c.src = Source<T>{(const T*)G, ldg, sg, M, ldm, sm, mu, nesterov, m, n};
  c.batch = batch;
  c.W = (T*)W; c.ldw = ldw; c.sw = sw;
  c.keep = keep; c.rate = rate;
  return status_of(iterate<T>(c, sc.scales, sc.step, y, (char*)ws, (hipStream_t)stream));
}

}  // namespace
}  // namespace ops
}  // namespace rrf

using namespace rrf::ops;

extern "C" {

rrf_status rrf_orthogonalize_workspace(rrf_dtype dtype, int64_t m, int64_t n, int64_t batch, int,
                                       size_t* bytes) {
  const int dt = int_bits(dtype);
  if (!bytes || !valid_real(dt) || m < 0 || n < 0 || batch < 0) return RRF_ERR_INVALID_ARG;
  if (m > (1 << 20) || n > (1 << 20) || std::min(m, n) > 65536 || batch > 65535) return RRF_ERR_SHAPE;
  *bytes = (m == 0 || n == 0 || batch == 0) ? 0 : layout_of(dt, m, n, batch).total;
  return RRF_OK;
}

rrf_status rrf_orthogonalize(rrf_dtype dtype, int64_t m, int64_t n, int64_t batch, const void* G, int64_t ldg,
                             int64_t stride_g, void* O, int64_t ldo, int64_t stride_o, const double* coeffs,
                             int64_t steps, double eps, void* workspace, size_t workspace_bytes,
                             void* hip_stream) {
  const int dt = int_bits(dtype);
  Schedule sc;
  Layout y;
  const rrf_status s = check_common(dt, m, n, batch, coeffs, steps, eps, workspace, workspace_bytes, &sc, &y);
  if (s != RRF_OK || m == 0 || n == 0 || batch == 0) return s;
  const int size = real_size(dt);
  if (bad_matrix(G, ldg, stride_g, m, n, batch, size) || bad_matrix(O, ldo, stride_o, m, n, batch, size) ||
      (batch > 1 && stride_o < ldo * (n - 1) + m))
    return RRF_ERR_INVALID_ARG;
  switch (dt) {
    case RRF_F32:
      return ortho_typed<float>(m, n, batch, G, ldg, stride_g, O, ldo, stride_o, sc, y, workspace, hip_stream);
    case RRF_BF16:
      return ortho_typed<bf16_t>(m, n, batch, G, ldg, stride_g, O, ldo, stride_o, sc, y, workspace, hip_stream);
    default:
      return ortho_typed<f16_t>(m, n, batch, G, ldg, stride_g, O, ldo, stride_o, sc, y, workspace, hip_stream);
  }
}

rrf_status rrf_muon_step(rrf_dtype dtype, int64_t m, int64_t n, int64_t batch, void* W, int64_t ldw,
                         int64_t stride_w, float* M, int64_t ldm, int64_t stride_m, const void* G, int64_t ldg,
                         int64_t stride_g, double lr, double momentum, int nesterov, double weight_decay,
                         double scale, const double* coeffs, int64_t steps, double eps, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
  const int dt = int_bits(dtype);
  Schedule sc;
  Layout y;
  if (!std::isfinite(lr) || !std::isfinite(momentum) || !std::isfinite(weight_decay) || !std::isfinite(scale))
    return RRF_ERR_INVALID_ARG;
  const rrf_status s = check_common(dt, m, n, batch, coeffs, steps, eps, workspace, workspace_bytes, &sc, &y);
  if (s != RRF_OK || m == 0 || n == 0 || batch == 0) return s;
  const int size = real_size(dt);
  if (bad_matrix(G, ldg, stride_g, m, n, batch, size) || bad_matrix(W, ldw, stride_w, m, n, batch, size) ||
      bad_matrix(M, ldm, stride_m, m, n, batch, 4) ||
      (batch > 1 && (stride_w < ldw * (n - 1) + m || stride_m < ldm * (n - 1) + m)))
    return RRF_ERR_INVALID_ARG;
  const float mu = (float)momentum, keep = (float)(1.0 - lr * weight_decay), rate = (float)(lr * scale);
  switch (dt) {
    case RRF_F32:
      return muon_typed<float>(m, n, batch, W, ldw, stride_w, M, ldm, stride_m, G, ldg, stride_g, mu, nesterov,
                               keep, rate, sc, y, workspace, hip_stream);
    case RRF_BF16:
      return muon_typed<bf16_t>(m, n, batch, W, ldw, stride_w, M, ldm, stride_m, G, ldg, stride_g, mu, nesterov,
                                keep, rate, sc, y, workspace, hip_stream);
    default:
      return muon_typed<f16_t>(m, n, batch, W, ldw, stride_w, M, ldm, stride_m, G, ldg, stride_g, mu, nesterov,
                               keep, rate, sc, y, workspace, hip_stream);
  }
}

}  // extern "C"
