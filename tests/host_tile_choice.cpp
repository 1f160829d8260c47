// Which tiles the host chooses (csrc/ops/cost.h), for the shapes on stdin:
//   ortho S L BATCH        short and long side: the Gram product's tile, splits and
//                          whether its 128 x 128 tiles have the deep ring, the
//                          short products' tile and ring, X's tile and ring
//   product M N K          of two 4-bit matrices: the tile, -1 without one
//   apply TRANS K M N P    P parts of a real value: the tile (-1 without one) and
//                          the splits

#include "cost.h"

#include <iostream>
#include <string>

using namespace rrf::ops;

int main() {
  std::string what;
  while (std::cin >> what) {
    if (what == "ortho") {
      int64_t s, l, batch;
      std::cin >> s >> l >> batch;
      s = blocks(s, 64) * 64;
      l = blocks(l, 64) * 64;
      const Choice g = choose_tile(s, s, true, batch, l / 64, gram_splits(s, l));
      const Choice q = choose_tile(s, s, true, batch, s / 64, 1), x = choose_tile(s, l, false, batch, s / 64, 1);
      std::cout << g.tile << ' ' << g.splits << ' ' << one_a_unit(s, s, true, batch, g.splits) << ' ' << q.tile << ' '
                << one_a_unit(s, s, true, batch, 1) << ' ' << x.tile << ' ' << one_a_unit(s, l, false, batch, 1) << '\n';
    } else if (what == "product") {
      int64_t M, N, k;
      std::cin >> M >> N >> k;
      std::cout << (N <= 64 ? -1 : choose_product(M, N, blocks(k, 256))) << '\n';
    } else {
      int64_t trans, k, m, n, parts;
      std::cin >> trans >> k >> m >> n >> parts;
      const bool few = few_columns((int)trans, (int)parts, n);
      std::cout << (few ? -1 : choose_apply(trans ? m : k, trans ? k : m, n, (int)parts).tile) << ' '
                << apply_splits((int)trans, (int)parts, k, m, n) << '\n';
    }
  }
}
