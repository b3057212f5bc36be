// Which tiles a product of the orthogonalised updates launches, and in which
// order (host code without HIP).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <functional>
#include <queue>
#include <vector>

namespace edit {

// Tile (m, n) of a matrix: of its rows and columns (load), of C's p and q (products); mat = -1: none.
struct OrthoTile {
  int32_t mat, m, n;
  int32_t slot;        // update: of x_part;  gram, square: of `pieces` (-1: a whole sum)
  int32_t begin, end;  // products: slabs of the sum;  join: pieces
};

constexpr int kXcds = 8;  // workgroups go to the XCDs in turn
constexpr int kOrthoLargeSide = 128;

inline int64_t tiles_ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The tiles of all matrices, so that the workgroups of an XCD (every eighth)
// take neighbouring ones of a matrix, whose operands they share in its L2;
// matrices with the longest sums first, so that short ones fill the end.
// What a matrix has beyond a multiple of eight is not evened out over the
// matrices: seven of 36 tiles come out as 28 and 35 a list.
inline std::vector<OrthoTile> spread_tiles(const std::vector<std::vector<OrthoTile>>& of_matrix,
                                           const std::vector<int>& order) {
  std::vector<OrthoTile> list[kXcds];
  int turn = 0;  // matrices of few tiles start on different XCDs
  for (int m : order) {
    const std::vector<OrthoTile>& t = of_matrix[m];
    const size_t n = t.size();
    for (int x = 0; x < kXcds; ++x) {
      std::vector<OrthoTile>& to = list[(x + turn) % kXcds];
      to.insert(to.end(), t.begin() + n * x / kXcds, t.begin() + n * (x + 1) / kXcds);
    }
    turn = (turn + static_cast<int>(n % kXcds)) % kXcds;
  }
  size_t longest = 0;
  for (const auto& l : list) longest = std::max(longest, l.size());
  std::vector<OrthoTile> out;
  for (size_t i = 0; i < longest; ++i)
    for (const auto& l : list) out.push_back(i < l.size() ? l[i] : OrthoTile{-1, 0, 0, 0, 0, 0});
  while (!out.empty() && out.back().mat < 0) out.pop_back();
  return out;
}

// Tiles of the symmetric products that would run on when most CUs are done are
// cut into pieces of the sum, of some kPieceSlabs slabs at least, where that is
// expected to save what a tile or piece by itself costs (kTileSlabs), the join
// pass (kCutGain) and the pieces' way through memory (cut_tiles()).  Whole calls, us
// without and with: one 4096 x 11008 matrix (528 tiles where 512 run at a time;
// the last 16 in pieces) 3490 and 3240.  Where it does not save that: one 1024 x
// 1024 matrix with FULL (136 tiles of 32 slabs where 1024 run at a time) 197
// whole and 214 in four pieces each; a 1B layer's outer step with FULL, the gram
// product's last 232 of 952 cut, 6624 and 6728.
constexpr int64_t kPieceSlabs = 10, kTileSlabs = 4, kCutGain = 20;
// The workspace holds this much of unfinished sums at most; tiles beyond stay
// whole.  Of 80,000 random layouts for 256 CUs none asks for more (177 MB; one
// 4096 x 11008 matrix for 18 with FAST and 35 with FULL, a 1B layer for none).
constexpr int64_t kPieceBytes = int64_t(192) << 20;
inline int tiles_per_cu(int side) { return side == kOrthoLargeSide ? 2 : 4; }  // that run side by side

// A symmetric product's tiles (whole sums, in `order` of the matrices) for
// `slots` that run at a time: `tiles` is what to launch, `join` the tiles that
// are left in pieces.  Each tile goes to the slot that is free first; one that
// would end behind an even share of all work is cut into pieces that fill what
// the share leaves.  Returns the number of pieces.
inline int cut_tiles(const std::vector<std::vector<OrthoTile>>& of_matrix, const std::vector<int>& order, int side,
                     int num_cu, std::vector<OrthoTile>* tiles, std::vector<OrthoTile>* join) {
  using Ends = std::priority_queue<int64_t, std::vector<int64_t>, std::greater<int64_t>>;
  int64_t work = 0;
  for (const auto& l : of_matrix)
    for (const OrthoTile& t : l) work += t.end + kTileSlabs;
  const int slots = tiles_per_cu(side) * num_cu;
  const int64_t share = tiles_ceil_div(work, slots);
  std::vector<std::vector<OrthoTile>> lists = of_matrix, pieces(of_matrix.size());
  int64_t last_whole = 0, last_cut = 0;
  int count = 0;
  const int64_t most = kPieceBytes / (4 * side * side);
  Ends whole(std::greater<int64_t>(), std::vector<int64_t>(slots, 0)), parts = whole;
  auto run = [](Ends& ends, int64_t slabs, int64_t* last) {
    const int64_t end = ends.top() + slabs + kTileSlabs;
    ends.pop();
    ends.push(end);
    *last = std::max(*last, end);
  };
  for (int m : order) {
    lists[m].clear();
    for (const OrthoTile& t : of_matrix[m]) {
      run(whole, t.end, &last_whole);
      const int64_t room = std::max(kPieceSlabs, share - parts.top() - kTileSlabs);
      const int32_t n = t.end <= room + kPieceSlabs ? 1 : static_cast<int32_t>(tiles_ceil_div(t.end, room));
      if (n == 1 || count + n > most) {
        run(parts, t.end, &last_cut);
        lists[m].push_back(t);
        continue;
      }
      join->push_back({t.mat, t.m, t.n, 0, count, count + n});
      for (int32_t k = 0; k < n; ++k) {
        const int32_t begin = static_cast<int32_t>(static_cast<int64_t>(t.end) * k / n);
        const int32_t end = static_cast<int32_t>(static_cast<int64_t>(t.end) * (k + 1) / n);
        pieces[m].push_back({t.mat, t.m, t.n, count++, begin, end});
        run(parts, end - begin, &last_cut);
      }
    }
  }
  if (last_whole - last_cut < kCutGain + count / (side == kOrthoLargeSide ? 16 : 64)) {
    join->clear();
    *tiles = spread_tiles(of_matrix, order);
    return 0;
  }
  std::vector<int> all = order;
  for (int m : order) {  // a matrix's pieces behind all whole tiles
    all.push_back(static_cast<int>(lists.size()));
    lists.push_back(pieces[m]);
  }
  *tiles = spread_tiles(lists, all);
  return count;
}

}  // namespace edit
