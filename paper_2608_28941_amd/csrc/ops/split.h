// A tile of the product (tile.h) for small results: a workgroup of four wavefronts
// forms a 16 T x 16 T tile of D, every wavefront the whole of it from every
// fourth chunk, with a ring of R chunks of its own in LDS.
//
// A small product is bound by latency.  Wavefronts that share chunks wait for
// each other at a barrier for every one of them; here none waits for another
// until the four partial tiles are added, in a fixed order, and the first R
// chunks of all four are under way at once.  (512 x 512 x 512 with one plane
// each: 3.4 us with 32 x 32 tiles, T = 2, R = 2, against 4.9 with 64 x 64 tiles
// from a shared ring, which 64 x 64 tiles here do not beat.)
#pragma once

#include "ring.h"

namespace rrf {
namespace ops {

template <int T, int R>
struct SplitTile {
  static constexpr int BM = 16 * T, BN = 16 * T, kThreads = 256;
  static constexpr int kStage = (BM + BN) * kChunkBytes;
  static constexpr int kLoads = kStage / 1024;                 // a lane and chunk
  static constexpr int kPartial = T * T * 1024;                // a wavefront's tile in binary32
  static constexpr int kLds = 4 * (R * kStage > kPartial ? R * kStage : kPartial);
  static_assert(R * kLoads < 64, "loads in flight");

  // emit(x, y, value): 16 x 16 tile (x, y) of D, once, by one of the wavefronts.
  template <typename EMIT>
  static __device__ __forceinline__ void run(const Operands& op, int nk, int64_t batch_u, int64_t batch_v, int i0,
                                             int j0, char* lds, EMIT emit) {
    const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    const int g = lane >> 4, m16 = lane & 15;
    const int r8 = lane >> 3, pk = (lane & 7) ^ r8;
    constexpr int LU = BM / 8;        // loads of U's rows, then of V's
    int off[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int r = (q % LU) * 8 + r8;
      off[q] = q < LU ? (int)((int64_t)(min(i0 + r, op.rows_u - 1) - i0) * op.ldu + pk * 16)
                      : (int)((int64_t)(min(j0 + r, op.rows_v - 1) - j0) * op.ldv + pk * 16);
    }
    const int64_t bu = batch_u + (int64_t)i0 * op.ldu, bv = batch_v + (int64_t)j0 * op.ldv;
    f4_t acc[T][T];
#pragma unroll
    for (int a = 0; a < T; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] = f4_t{0.f, 0.f, 0.f, 0.f};
    const int total = 3 * nk;
    const int mine = (total - wv + 3) >> 2;      // chunks wv, wv + 4, ...
    char* ring = lds + wv * (R * kStage);
    int issued = 0, slot = 0;
    auto issue = [&]() __attribute__((always_inline)) {
      const int c = wv + 4 * issued, seg = c / nk, k = c - seg * nk;
      const rsrc_t ru = rsrc_of((seg == 1 ? op.ul : op.u) + bu), rv = rsrc_of((seg == 2 ? op.vl : op.v) + bv);
      char* l = ring + slot * kStage;
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        const rsrc_t r = q < LU ? ru : rv;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(l + q * 1024), 16,
                                                 off[q], k * kChunkBytes, 0, 0);
      }
      ++issued;
      slot = slot == R - 1 ? 0 : slot + 1;
    };
    for (int s = 0; s < R && s < mine; ++s) issue();
    int at = 0;
    for (int c = 0; c < mine; ++c) {
      // Chunk c's loads are the oldest; from the last R on, all are waited for.
      if (issued - c == R) wait_mem<(R - 1) * kLoads>();
      else wait_mem<0>();
      __builtin_amdgcn_sched_barrier(0);
      const char* l = ring + at * kStage;
      i4_t a[2][T], b[2][T];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int x = 0; x < T; ++x) {
          a[kk][x] = *reinterpret_cast<const i4_t*>(l + pack_at(16 * x + m16, kk * 4 + g));
          b[kk][x] = *reinterpret_cast<const i4_t*>(l + BM * kChunkBytes + pack_at(16 * x + m16, kk * 4 + g));
        }
      // The place is free once the operands are in registers.
      __builtin_amdgcn_s_waitcnt(0xc07f);     // LDS only
      __builtin_amdgcn_sched_barrier(0);
      if (issued < mine) issue();
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int x = 0; x < T; ++x)
#pragma unroll
          for (int y = 0; y < T; ++y) acc[x][y] = mfma16<Kind::kF16>(a[kk][x], b[kk][y], acc[x][y]);
      at = at == R - 1 ? 0 : at + 1;
    }
    __syncthreads();
    f4_t* part = reinterpret_cast<f4_t*>(lds);
#pragma unroll
    for (int x = 0; x < T; ++x)
#pragma unroll
      for (int y = 0; y < T; ++y) part[(wv * T * T + x * T + y) * 64 + lane] = acc[x][y];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < T * T / 4; ++q) {
      const int z = wv * (T * T / 4) + q;
      f4_t s = part[z * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) s += part[(w * T * T + z) * 64 + lane];
      emit(z / T, z % T, s);
    }
  }
};

}  // namespace ops
}  // namespace rrf
