// A tile of the product (tile.h) of operands of two planes, u = u_hi + u_lo and v
// = v_hi + v_lo: D = u_hi v_hi + u_hi v_lo + u_lo v_hi, its parts overlapped by
// hand (ring.h).
//
// A stage of the ring holds 32 values of a row, of both planes of both
// operands, so that a loaded operand serves all the products it is part of:
// four images for three products, instead of six when the three are summed up
// one after the other (4096 x 4096 x 4096: 323 us against 364).  Rows are of
// 64 bytes; pack p of row r lies at p ^ ((r / 2) % 4), which spreads the 16
// lanes that read one pack column over all banks.
//
// Phase one multiplies hi by hi and reads the low parts; at its end every
// operand of the stage is in registers and its place in the ring is free.
// Phase two multiplies lo by hi, then hi by lo, and there reads the next
// stage's high parts, each into registers whose last use has gone by.
#pragma once

#include "ring.h"

namespace rrf {
namespace ops {

template <int T, int S>
struct WideTile {
  static constexpr int BM = 32 * T, BN = 32 * T, kThreads = 256;
  static constexpr int kRow = 64;
  static constexpr int kImage = BM * kRow;      // a plane of an operand
  static constexpr int kStage = 4 * kImage;     // u_hi, v_hi, u_lo, v_lo
  static constexpr int kLds = S * kStage;
  static constexpr int kLoads = 2 * T;          // a thread and stage
  static_assert(S >= 2 && (S - 1) * kLoads < 64 && T % 2 == 0, "ring");

  static __device__ __forceinline__ int at_pack(int r, int p) { return r * kRow + ((p ^ ((r >> 1) & 3)) << 4); }

  static __device__ __forceinline__ void run(const Operands& op, int nk, int64_t batch_u, int64_t batch_v, int i0,
                                             int j0, char* lds, f4_t (&acc)[T][T]) {
    const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wi = (wv & 1) * 16 * T, wj = (wv >> 1) * 16 * T;
    const int g = lane >> 4, m16 = lane & 15;
    const int r16 = lane >> 2, pk = (lane & 3) ^ ((r16 >> 1) & 3);
    // A load covers 16 rows of an image; a wavefront has T / 2 of each image's
    // 2 T, the low planes' at the same offsets as the high ones'.
    int ou[T / 2], ov[T / 2];
#pragma unroll
    for (int q = 0; q < T / 2; ++q) {
      const int r = (wv * (T / 2) + q) * 16 + r16;
      ou[q] = (int)((int64_t)(min(i0 + r, op.rows_u - 1) - i0) * op.ldu + pk * 16);
      ov[q] = (int)((int64_t)(min(j0 + r, op.rows_v - 1) - j0) * op.ldv + pk * 16);
    }
    const int64_t bu = batch_u + (int64_t)i0 * op.ldu, bv = batch_v + (int64_t)j0 * op.ldv;
    const rsrc_t ruh = rsrc_of(op.u + bu), rul = rsrc_of(op.ul + bu);
    const rsrc_t rvh = rsrc_of(op.v + bv), rvl = rsrc_of(op.vl + bv);
#pragma unroll
    for (int a = 0; a < T; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] = f4_t{0.f, 0.f, 0.f, 0.f};
    const int total = nk;
    int k = 0, so = 0, slot = 0;              // of the next load
    // Past the last stage the first one is loaded again, and not used.
    auto advance = [&]() __attribute__((always_inline)) {
      so += kRow;
      slot = slot == (S - 1) * kStage ? 0 : slot + kStage;
      if (++k == total) { k = 0; so = 0; }
    };
    auto load1 = [&](int q) __attribute__((always_inline)) {
      const int image = q & 3, x = q >> 2;
      __attribute__((address_space(3))) char* l =
          (__attribute__((address_space(3))) char*)(lds + slot + image * kImage + (wv * (T / 2) + x) * 1024);
      const rsrc_t r = image == 0 ? ruh : image == 1 ? rvh : image == 2 ? rul : rvl;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)l, 16,
                                               (image & 1) ? ov[x] : ou[x], so, 0, 0);
    };
    const int lu = at_pack(wi + m16, g), lv = kImage + at_pack(wj + m16, g);
    i4_t uh[T], ul[T], vh[T], vl[T];
    auto read_u = [&](int at, int x) __attribute__((always_inline)) {
      return *reinterpret_cast<const i4_t*>(lds + at + lu + x * (16 * kRow));
    };
    auto read_v = [&](int at, int x) __attribute__((always_inline)) {
      return *reinterpret_cast<const i4_t*>(lds + at + lv + x * (16 * kRow));
    };
    auto barrier = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    // Half a row of D's tiles: T / 2 matrix instructions.
    auto mul = [&](const i4_t& u, i4_t (&v)[T], int x, int half) __attribute__((always_inline)) {
#pragma unroll
      for (int y = 0; y < T / 2; ++y) mfma_acc(acc[x][half * (T / 2) + y], u, v[half * (T / 2) + y]);
    };
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int q = 0; q < kLoads; ++q) load1(q);
      advance();
    }
    wait_mem<(S - 1) * kLoads>();
    barrier();
#pragma unroll
    for (int x = 0; x < T; ++x) vh[x] = read_v(0, x);
#pragma unroll
    for (int x = 0; x < T; ++x) uh[x] = read_u(0, x);
    int at = 0;
    for (int c = 0; c < total; ++c) {
#pragma unroll
      for (int q = 0; q < 2 * T; ++q) {
        const int x = q >> 1;
        if (q < T) ul[q] = read_u(at + 2 * kImage, q);
        else vl[q - T] = read_v(at + 2 * kImage, q - T);
        mul(uh[x], vh, x, q & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_mem<(S - 2) * kLoads>();
      barrier();
      at = at == (S - 1) * kStage ? 0 : at + kStage;
#pragma unroll
      for (int q = 0; q < 2 * T; ++q) {
        const int x = q >> 1;
        if ((q & 1) == 0) load1(x);
        mul(ul[x], vh, x, q & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int q = 0; q < 2 * T; ++q) {
        const int x = q >> 1;
        if ((q & 1) == 0) load1(T + x);
        if (q < T) vh[q] = read_v(at, q);
        mul(uh[x], vl, x, q & 1);
        if (q & 1) uh[x] = read_u(at, x);
        __builtin_amdgcn_sched_barrier(0);
      }
      advance();
    }
    wait_mem<0>();
    asm volatile("s_nop 15\n s_nop 15" ::: "memory");
    barrier();
  }
};

}  // namespace ops
}  // namespace rrf
