// A tile of the product (tile.h) of operands of 4 bits with a scale for 32 values,
// on the scaled matrix instruction, its parts overlapped by hand (ring.h).
//
// A chunk of a row is 128 bytes (256 values), a lane's 16-byte pack is
// one block of 32 values, and its scale is one byte.  The scales of four chunks,
// 32 bytes a row, are loaded into LDS at a time, one group of four ahead: rows
// are far apart in memory, and a load that takes 4 bytes of each of 64 rows
// costs as much as one that takes whole lines.  From LDS a lane reads its row's
// 16 bytes of two chunks at once and keeps byte g of each of the four words,
// for the four half chunks.  (11008 x 2048, K = 4096: 105 us with a chunk's
// scales loaded by words and read by bytes.)
#pragma once

#include <type_traits>

#include "ring.h"

namespace rrf {
namespace ops {

// With byte B of either lane's scales.
template <int B>
__device__ __forceinline__ void mfma_mx4(f4_t& c, i4_t a, i4_t b, int sa, int sb) {
  if constexpr (B == 0)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else if constexpr (B == 1)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else if constexpr (B == 2)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}

struct Mx4Operands {
  const char *u, *su, *v, *sv;      // codes and scales
  int nk;                           // chunks of a row
  int rows_u, rows_v;
};

template <int T, int S>
struct Mx4Tile {
  static constexpr int BM = 32 * T, BN = 32 * T, kThreads = 256;
  static constexpr int kStage = (BM + BN) * kChunkBytes;
  static constexpr int kScales = (BM + BN) * 32;    // of four chunks
  static constexpr int kLds = S * kStage + 2 * kScales;
  static constexpr int kLoads = 2 * T;              // of codes, a thread and chunk
  // The scales of group q + 1 are loaded in the second half of chunk 4 q and
  // first read in that of chunk 4 q + 3: the wait before, which leaves the
  // loads of S - 2 chunks under way, covers them for S <= 4.
  static_assert(S >= 2 && S <= 4 && (S - 2) * kLoads < 64 && T % 2 == 0, "ring");

  static __device__ __forceinline__ void run(const Mx4Operands& op, int i0, int j0, char* lds,
                                             f4_t (&acc)[T][T]) {
    const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wi = (wv & 1) * 16 * T, wj = (wv >> 1) * 16 * T;
    const int g = lane >> 4, m16 = lane & 15;
    const int r8 = lane >> 3, pk = (lane & 7) ^ r8;
    const int64_t pitch = (int64_t)op.nk * kChunkBytes, spitch = (int64_t)op.nk * 8;
    int ou[T], ov[T];
#pragma unroll
    for (int q = 0; q < T; ++q) {
      const int r = wv * 8 * T + q * 8 + r8;
      ou[q] = (int)((min(i0 + r, op.rows_u - 1) - i0) * pitch + pk * 16);
      ov[q] = (int)((min(j0 + r, op.rows_v - 1) - j0) * pitch + pk * 16);
    }
    // Scales: 32 rows a load, both their 16-byte halves ([half][row] in LDS);
    // loads 0 .. T - 1 are U's, the others V's; a wavefront has T / 2 of them.
    int os[T / 2];
#pragma unroll
    for (int q = 0; q < T / 2; ++q) {
      const int z = wv * (T / 2) + q, r = (z % T) * 32 + (lane & 31);
      os[q] = (int)((z < T ? min(i0 + r, op.rows_u - 1) - i0 : min(j0 + r, op.rows_v - 1) - j0) * spitch) +
              16 * (lane >> 5);
    }
    const rsrc_t ru = rsrc_of(op.u + i0 * pitch), rv = rsrc_of(op.v + j0 * pitch);
    // The last row's last group may end past the matrix: those bytes read as 0.
    // The group is part of the lane's offset for that, as an instruction's scalar
    // offset need not count in the comparison with the buffer's size.
    const rsrc_t rsu = rsrc_of(op.su + i0 * spitch, min(BM, op.rows_u - i0) * spitch);
    const rsrc_t rsv = rsrc_of(op.sv + j0 * spitch, min(BN, op.rows_v - j0) * spitch);
#pragma unroll
    for (int a = 0; a < T; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] = f4_t{0.f, 0.f, 0.f, 0.f};
    int k = 0, slot = 0;                      // of the next load
    // Past the last chunk the first one is loaded again, and not used.
    auto advance = [&]() __attribute__((always_inline)) {
      slot = slot == (S - 1) * kStage ? 0 : slot + kStage;
      if (++k == op.nk) k = 0;
    };
    typedef __attribute__((address_space(3))) void* lds_ptr;
    auto load1 = [&](int q) __attribute__((always_inline)) {
      char* l = lds + slot + wv * (1024 * T) + (q >> 1) * 1024;
      if (q & 1)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_ptr)(l + BM * kChunkBytes), 16, ov[q >> 1],
                                                 k * kChunkBytes, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ru, (lds_ptr)l, 16, ou[q >> 1], k * kChunkBytes, 0, 0);
    };
    auto load_scales = [&](int group) __attribute__((always_inline)) {
      if (4 * group >= op.nk) return;
#pragma unroll
      for (int q = 0; q < T / 2; ++q) {
        const int z = wv * (T / 2) + q;
        char* l = lds + S * kStage + (group & 1) * kScales + z * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(z < T ? rsu : rsv, (lds_ptr)l, 16, os[q] + group * 32, 0, 0, 0);
      }
    };
    int lu[2], lv[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      lu[kk] = pack_at(wi + m16, kk * 4 + g);
      lv[kk] = BM * kChunkBytes + pack_at(wj + m16, kk * 4 + g);
    }
    // This lane's rows' scales: rows wi + 16 x + m16 lie in block (wi + 16 x) /
    // 32 at row 16 (x % 2) + m16 (wi and wj are multiples of 32).
    const int lsu = S * kStage + wi * 32 + m16 * 16, lsv = S * kStage + (BM + wj) * 32 + m16 * 16;
    const unsigned take = (unsigned)((4 + g) << 8 | g);
    i4_t f0[2 * T], f1[2 * T];      // V's, then U's operands of a half chunk
    int s[2 * T], sn[2 * T];        // and their scales, four half chunks', of this pair and the next
    auto fetch1 = [&](int at, int kk, int q, i4_t (&f)[2 * T]) __attribute__((always_inline)) {
      f[q] = *reinterpret_cast<const i4_t*>(lds + at + (q < T ? lv[kk] : lu[kk]) + (q % T) * 2048);
    };
    // The scales of chunks c and c + 1 (c even): as read, and byte g of each word.
    auto fetch_scale = [&](int c, int q) __attribute__((always_inline)) {
      const int x = q % T, part = ((c >> 2) & 1) * kScales + ((c >> 1) & 1) * 512;
      return *reinterpret_cast<const i4_t*>(lds + part + (q < T ? lsv : lsu) + (x >> 1) * 1024 + (x & 1) * 256);
    };
    auto own_bytes = [&](i4_t w) __attribute__((always_inline)) {
      const unsigned p0 = __builtin_amdgcn_perm((unsigned)w[1], (unsigned)w[0], take),
                     p1 = __builtin_amdgcn_perm((unsigned)w[3], (unsigned)w[2], take);
      return (int)__builtin_amdgcn_perm(p1, p0, 0x05040100u);
    };
    auto mul = [&](auto byte, int q, int part, i4_t (&f)[2 * T]) __attribute__((always_inline)) {
      constexpr int N = T / 2;
      const int x = q >> 1, y0 = (q & 1) * N;
#pragma unroll
      for (int y = part ? N / 2 : 0; y < (part ? N : N / 2); ++y)
        mfma_mx4<decltype(byte)::value>(acc[x][y0 + y], f[T + x], f[y0 + y], s[T + x], s[y0 + y]);
    };
    auto barrier = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    load_scales(0);
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int q = 0; q < kLoads; ++q) load1(q);
      advance();
    }
    wait_mem<(S - 1) * kLoads < 64 ? (S - 1) * kLoads : 63>();
    barrier();
#pragma unroll
    for (int q = 0; q < 2 * T; ++q) {
      fetch1(0, 0, q, f0);
      s[q] = own_bytes(fetch_scale(0, q));
    }
    int at = 0;
    // Chunk c, the first (odd = 0) or second of its pair.
    auto chunk = [&](auto odd, int c) __attribute__((always_inline)) {
      constexpr int O = decltype(odd)::value;
#pragma unroll
      for (int q = 0; q < 2 * T; ++q) {
        fetch1(at, 1, q, f1);
        mul(std::integral_constant<int, 2 * O>(), q, 0, f0);
        mul(std::integral_constant<int, 2 * O>(), q, 1, f0);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_mem<(S - 2) * kLoads>();
      barrier();
      at = at == (S - 1) * kStage ? 0 : at + kStage;
      if (O == 0 && (c & 2) == 0) load_scales((c >> 2) + 1);
      i4_t raw[3];
#pragma unroll
      for (int q = 0; q < 2 * T; ++q) {
        fetch1(at, 0, q, f0);
        if (O == 1) {               // taken apart three steps later, when it has arrived
          if (q >= 3) sn[q - 3] = own_bytes(raw[q % 3]);
          raw[q % 3] = fetch_scale(c + 1, q);
        }
        mul(std::integral_constant<int, 2 * O + 1>(), q, 0, f1);
        __builtin_amdgcn_sched_barrier(0);
        load1(q);
        mul(std::integral_constant<int, 2 * O + 1>(), q, 1, f1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (O == 1) {
#pragma unroll
        for (int q = 2 * T - 3; q < 2 * T; ++q) sn[q] = own_bytes(raw[q % 3]);
#pragma unroll
        for (int q = 0; q < 2 * T; ++q) s[q] = sn[q];
      }
      advance();
    };
    int c = 0;
    for (; c + 1 < op.nk; c += 2) {
      chunk(std::integral_constant<int, 0>(), c);
      chunk(std::integral_constant<int, 1>(), c + 1);
    }
    if (c < op.nk) chunk(std::integral_constant<int, 0>(), c);
    wait_mem<0>();
    asm volatile("s_nop 15\n s_nop 15" ::: "memory");
    barrier();
  }
};

}  // namespace ops
}  // namespace rrf
