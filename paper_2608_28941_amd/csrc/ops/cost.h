// Which tiles, and how many splits of the contraction, a product is formed by:
// what takes the least time by a fitted cost of its launch.  Host code only.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace rrf {
namespace ops {

inline int64_t blocks(int64_t n, int64_t size) { return (n + size - 1) / size; }

// What a launch takes, in ns, with tiles of a size: for a chunk of a row with one
// workgroup on the device, with 256 and with 512 of them (0: no more than 256
// fit), and apart from the chunks.
struct TileCost { int size; double alone, busy256, busy512, fixed; };

inline double tile_time(const TileCost& c, int64_t tiles, int64_t chunks) {
  const int64_t cap = c.busy512 > 0 ? 512 : 256;
  auto round = [&](int64_t busy) {
    const double chunk = busy <= 256 ? c.alone + (c.busy256 - c.alone) * busy / 256.0
                                     : c.busy256 + (c.busy512 - c.busy256) * (busy - 256) / 256.0;
    return chunk * chunks + c.fixed;
  };
  const int64_t rest = tiles % cap;
  return (tiles / cap) * round(cap) + (rest ? round(rest) : 0.0);
}

// --- products of the orthogonalised steps ---------------------------------------------

constexpr int kMaxSplits = 16;     // of the Gram product's long side

// Splits of the Gram product that the workspace allows: their shares take no
// more room than the two planes of X.
inline int64_t gram_splits(int64_t sp, int64_t lp) {
  return sp == 0 ? 1 : std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, lp / sp));
}

// Costs of the launches, chunks of 64 values.  A fit to the measured times of the
// five sizes at sides from 64 to 11008 and batches of 1 to 16 (within 15 % of
// them on average).
constexpr TileCost kOrthoTiles[5] = {{32, 200, 500, 560, 3100}, {64, 330, 940, 1310, 5600},
                                     {128, 890, 1530, 3150, 11000}, {192, 1610, 2790, 0, 15100},
                                     {256, 3250, 4180, 0, 25600}};

// The tile size of a product (index into kOrthoTiles), and for Gram products the
// number of splits of the contraction, with the least time by that model.
struct Choice { int tile, splits; double time; };
inline Choice choose_tile(int64_t rows_i, int64_t rows_j, bool triangle, int64_t batch, int64_t nk,
                          int64_t max_splits) {
  Choice best{0, 1, 1e300};
  for (int q = 0; q < 5; ++q) {
    const TileCost& c = kOrthoTiles[q];
    const int64_t ti = blocks(rows_i, c.size), tj = blocks(rows_j, c.size);
    const int64_t tiles = batch * (triangle ? ti * (ti + 1) / 2 : ti * tj);
    for (int64_t z = 1; z <= max_splits; ++z) {
      const int64_t per = blocks(nk, z);
      if (z > 1 && (z - 1) * per >= nk) continue;      // a split without chunks
      // joining is a launch, reads z values of 4 bytes a place and writes one, at 4 TB/s
      const double join = z == 1 ? 0.0 : 4000.0 + 4.0 * (z + 1) * batch * rows_i * rows_j / 2 / 4000.0;
      const double cost = tile_time(c, tiles * z, per) + join;
      if (cost < best.time) best = Choice{q, (int)z, cost};
    }
  }
  return best;
}

// Whether a product's 128 x 128 tiles leave a compute unit one workgroup only: then
// the ring is deeper (1792 x 1792 x 5376: 60 -> 40 us), and two workgroups share a
// unit where there are more.
inline bool one_a_unit(int64_t rows_i, int64_t rows_j, bool triangle, int64_t batch, int64_t splits) {
  const int64_t ti = blocks(rows_i, 128), tj = blocks(rows_j, 128);
  return batch * splits * (triangle ? ti * (ti + 1) / 2 : ti * tj) <= 256;
}

// --- both operands in 4 bits ---------------------------------------------------------

// Costs of the tiles' launches, chunks of 256 values; a fit to the times of 15
// sizes from 1024 x 1024 to 11008 x 8192 (K = 512 to 11008).  The size it chooses
// takes at most 2 % more than the best one there: 4096^3 43 us with 256 (58 with
// 128), 11008 x 2048 with K = 4096 67 with 128 (70 with 256), 1024 x 1024 9.2
// with 64 (12.8 with 128), 6000 x 6000 99 with 192 (102 and 105).
constexpr TileCost kProductTiles[4] = {{64, 380, 385, 440, 3050}, {128, 460, 730, 1200, 5400},
                                       {192, 790, 1250, 0, 7500}, {256, 1200, 1940, 0, 10700}};

// The tile size (index into kProductTiles) of C (M x N), nk chunks.
inline int choose_product(int64_t M, int64_t N, int64_t nk) {
  int best = 0;
  double least = 1e300;
  for (int q = 0; q < 4; ++q) {
    const int64_t tiles = blocks(M, kProductTiles[q].size) * blocks(N, kProductTiles[q].size);
    const double time = tile_time(kProductTiles[q], tiles, nk);
    if (time < least) { least = time; best = q; }
  }
  return best;
}

// --- a 4-bit matrix times real columns -----------------------------------------------

// Columns of B up to which it takes the kernels for few of them: A^T B with
// several parts would convert all of B again for every 16 columns of A.
constexpr int64_t few_limit(bool trans, int parts) { return trans && parts > 1 ? 32 : 64; }
inline bool few_columns(int trans, int parts, int64_t n) { return n <= few_limit(trans, parts); }

// Splits of the contraction of C = A B with few columns: about two workgroups
// to a compute unit, at least 128 columns of A each.
inline int64_t few_splits(int64_t k, int64_t m) {
  return std::max<int64_t>(1, std::min(blocks(512, blocks(k, 128)), m / 128));
}

// Tiles of the kernel for many columns, the workgroups of them that the device
// holds, and what a launch takes in ns: for a chunk of 64 contracted values with
// one workgroup, with 256 and with all of them busy, and apart from the chunks;
// for one part of B and for three (between them for two).  A fit to the measured
// times of 34 shapes with 1 to 16 splits (within 11 % of them on average; the
// choice takes 4 % more than the best one).
struct ApplyTile { int wi, nt, cap; double one[4], three[4]; };
constexpr ApplyTile kApplyTiles[5] = {{4, 4, 512, {920, 1220, 1340, 3900}, {1380, 2110, 2820, 5300}},
                                      {4, 3, 512, {870, 1110, 1220, 3500}, {1260, 2090, 2090, 3600}},
                                      {2, 4, 512, {950, 1210, 1230, 4200}, {1740, 2280, 2860, 6100}},
                                      {2, 2, 768, {680, 920, 1090, 3700}, {1050, 1350, 2310, 3700}},
                                      {2, 1, 1024, {540, 750, 1080, 2700}, {660, 920, 1650, 2600}}};
constexpr int kMaxApplySplits = 16;

// The tile and the number of splits of C (rows x n) with a contraction over L
// that take the least time by that model.
struct ApplyChoice { int tile, splits; };
inline ApplyChoice choose_apply(int64_t rows, int64_t L, int64_t n, int parts) {
  ApplyChoice best{0, 1};
  double least = 1e300;
  const int64_t chunks = blocks(L, 64);
  for (int q = 0; q < 5; ++q) {
    const ApplyTile& t = kApplyTiles[q];
    double c[4];
    for (int i = 0; i < 4; ++i) c[i] = parts == 1 ? t.one[i] : parts == 3 ? t.three[i] : 0.5 * (t.one[i] + t.three[i]);
    const int64_t tiles = blocks(rows, 64 * t.wi) * blocks(n, 16 * t.nt * (4 / t.wi));
    for (int z = 1; z <= kMaxApplySplits; ++z) {
      const int64_t per = blocks(chunks, z), w = tiles * z;
      if (z > 1 && ((z - 1) * per >= chunks || w > 1024)) continue;
      auto round = [&](int64_t busy) {
        const double chunk = busy <= 256 ? c[0] + (c[1] - c[0]) * busy / 256.0
                                         : c[1] + (c[2] - c[1]) * (busy - 256) / (t.cap - 256.0);
        return chunk * per + c[3];
      };
      // joining: a launch, and the sums written, read and added up
      const double join = z == 1 ? 0.0 : 6000.0 + 4.0 * (z + 1) * rows * n / 4500.0;
      const double time = (w / t.cap) * round(t.cap) + (w % t.cap ? round(w % t.cap) : 0.0) + join;
      if (time < least) { least = time; best = ApplyChoice{q, z}; }
    }
  }
  return best;
}

inline int64_t apply_splits(int trans, int parts, int64_t k, int64_t m, int64_t n) {
  if (few_columns(trans, parts, n)) return trans ? 1 : few_splits(k, m);
  return choose_apply(trans ? m : k, trans ? k : m, n, parts).splits;
}

}  // namespace ops
}  // namespace rrf
