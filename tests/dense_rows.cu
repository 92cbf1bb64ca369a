// For each line "D G pieces wide" of the standard input, how often the features of a
// row of D are taken by its group of G threads: the least and the most, and
// how many features outside the row are. pieces: of a thread, or 0 where a loop
// goes over a row of any length four pieces at a time.
#include <algorithm>
#include <cstdio>
#include <vector>

#include "sjd_dense_rows.cuh"

using namespace sjd_dense_ops;

template <bool W>
void count(int D, int G, int pieces) {
  std::vector<int> taken(D, 0);
  int outside = 0;
  const int all = pieces ? pieces : pieces_of(D, G), loop = pieces ? pieces : (all + 3) / 4 * 4;
  for (int lane = 0; lane < G; ++lane) {
    const Place at = place_of<W>(lane, G, all);
    for (int i = 0; i < loop; ++i) {
      for (int j = 0; j < 8; ++j) {
        if (!is_mine<W>(i, all) || !is_there<W>(i, j, at, D)) continue;
        const int e = feature<W>(i, j, at);
        if (e >= 0 && e < D) ++taken[e];
        else ++outside;
      }
    }
  }
  std::printf("%d %d %d\n", *std::min_element(taken.begin(), taken.end()), *std::max_element(taken.begin(), taken.end()), outside);
}

int main() {
  int D, G, pieces, wide;
  while (std::scanf("%d %d %d %d", &D, &G, &pieces, &wide) == 4) wide ? count<true>(D, G, pieces) : count<false>(D, G, pieces);
}
