// csrc/ortho_tiles.h over random layouts: every tile of a symmetric product is
// launched once, whole or in pieces that take its sum in order and are joined
// once; the pieces stay within the workspace that is documented.  Prints the
// layouts with and without pieces, and those that the limit kept from cutting
// further.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <tuple>

#include "ortho_tiles.h"

using namespace edit;

namespace {

void check(bool ok, const char* what) {
  if (ok) return;
  std::printf("%s\n", what);
  std::exit(1);
}

using Key = std::tuple<int32_t, int32_t, int32_t>;

}  // namespace

int main() {
  std::mt19937_64 gen(7);
  auto uniform = [&](int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(gen); };
  int whole = 0, cut = 0, limited = 0;
  for (int round = 0; round < 6000; ++round) {
    const int side = uniform(0, 1) ? 128 : 64;
    const int num_cu = uniform(0, 3) ? 256 : static_cast<int>(uniform(1, 1024));
    std::vector<std::vector<OrthoTile>> of_matrix(uniform(1, 6));
    std::vector<int> order(of_matrix.size());
    size_t tiles_in = 0;
    for (size_t m = 0; m < of_matrix.size(); ++m) {
      order[m] = static_cast<int>(m);
      const int32_t n = static_cast<int32_t>(uniform(1, uniform(0, 4) ? 24 : 60));
      const int32_t slabs = static_cast<int32_t>(uniform(1, uniform(0, 2) ? 100 : 4000));
      for (int32_t a = 0; a < n; ++a)
        for (int32_t b = 0; b <= a; ++b) of_matrix[m].push_back({static_cast<int32_t>(m), a, b, -1, 0, slabs});
      tiles_in += of_matrix[m].size();
    }
    std::shuffle(order.begin(), order.end(), gen);
    std::vector<OrthoTile> tiles, join;
    const int count = cut_tiles(of_matrix, order, side, num_cu, &tiles, &join);
    check(int64_t(count) * side * side * 4 <= kPieceBytes, "more unfinished sums than documented");
    limited += int64_t(count + 64) * side * side * 4 > kPieceBytes;
    std::map<Key, int32_t> wholes;
    std::vector<OrthoTile> piece(count, OrthoTile{-1, 0, 0, 0, 0, 0});
    for (const OrthoTile& t : tiles) {
      if (t.mat < 0) continue;
      const int32_t end = of_matrix[t.mat][0].end;
      if (t.slot < 0) {
        check(t.begin == 0 && t.end == end, "a whole tile's sum");
        check(++wholes[{t.mat, t.m, t.n}] == 1, "a tile twice");
      } else {
        check(t.slot < count && piece[t.slot].mat < 0, "a piece's place");
        check(0 <= t.begin && t.begin < t.end && t.end <= end, "a piece's sum");
        piece[t.slot] = t;
      }
    }
    int next = 0;
    for (const OrthoTile& j : join) {
      check(j.begin == next && j.end > j.begin + 1 && j.end <= count, "the pieces of a joined tile");
      next = j.end;
      int32_t at = 0;
      for (int k = j.begin; k < j.end; ++k) {
        const OrthoTile& t = piece[k];
        check(t.mat == j.mat && t.m == j.m && t.n == j.n && t.begin == at, "a piece out of order");
        at = t.end;
      }
      check(at == of_matrix[j.mat][0].end, "a sum that ends early");
      check(++wholes[{j.mat, j.m, j.n}] == 1, "a tile whole and in pieces");
    }
    check(next == count, "a piece that is joined nowhere");
    check(wholes.size() == tiles_in, "a tile that is missing");
    check(join.empty() == (count == 0), "pieces without a join");
    (count ? cut : whole) += 1;
  }
  std::printf("%d %d %d\n", whole, cut, limited);
  return 0;
}
