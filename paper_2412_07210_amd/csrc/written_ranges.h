// The buffers of one call, by kind: what the call writes has to overlap nothing
// else of them; what it only reads may.  Host code only; used by edit_adamw_*.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <vector>

namespace edit {

enum Overlap { kOverlapNone = 0, kOverlapWritten = 1, kOverlapRead = 2 };

// N kinds of buffers, each listed in the call's order.
template <int N>
class WrittenRanges {
 public:
  // Room for `count` buffers of each kind, so that a call allocates nothing.
  void reserve(size_t count) {
    for (Kind& k : kind_) k.ranges.reserve(count);
    written_.reserve(N * count);
    read_.reserve(N * count);
  }
  void clear() {
    for (Kind& k : kind_) k.ranges.clear(), k.lo = UINTPTR_MAX, k.hi = 0, k.ascending = true;
  }
  // [lo, hi), not empty
  void add(int kind, uintptr_t lo, uintptr_t hi) {
    Kind& k = kind_[kind];
    k.ascending = k.ascending && lo >= k.hi;
    k.lo = std::min(k.lo, lo), k.hi = std::max(k.hi, hi);
    k.ranges.push_back({lo, hi});
  }
  // Whether written buffers meet each other, or read ones; `writes`: a bit for
  // each kind that is written.
  Overlap find(unsigned writes) {
    // Mostly every kind lies in a stretch of its own, in order: nothing to sort.
    bool clear = true;
    for (int i = 0; i < N; ++i) {
      const Kind& a = kind_[i];
      clear = clear && (a.ascending || !(writes >> i & 1));
      for (int j = 0; j < i; ++j)
        if ((writes >> i | writes >> j) & 1) clear = clear && (a.hi <= kind_[j].lo || kind_[j].hi <= a.lo);
    }
    if (clear) return kOverlapNone;
    written_.clear();
    read_.clear();
    for (int i = 0; i < N; ++i) {
      std::vector<Range>& to = writes >> i & 1 ? written_ : read_;
      to.insert(to.end(), kind_[i].ranges.begin(), kind_[i].ranges.end());
    }
    std::sort(written_.begin(), written_.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    for (size_t i = 1; i < written_.size(); ++i)
      if (written_[i].lo < written_[i - 1].hi) return kOverlapWritten;
    // written ranges are disjoint, so ascending at both ends
    for (const Range& r : read_) {
      const auto it = std::upper_bound(written_.begin(), written_.end(), r.lo,
                                       [](uintptr_t lo, const Range& w) { return lo < w.hi; });
      if (it != written_.end() && it->lo < r.hi) return kOverlapRead;
    }
    return kOverlapNone;
  }
  // Whether [lo, hi) meets a written buffer.  For the few buffers that lie anywhere,
  // a number of the call, say: added above, they would have all of it sorted.
  bool written_at(unsigned writes, uintptr_t lo, uintptr_t hi) const {
    for (int i = 0; i < N; ++i) {
      const Kind& a = kind_[i];
      if (!(writes >> i & 1) || a.hi <= lo || hi <= a.lo) continue;
      for (const Range& r : a.ranges)
        if (r.lo < hi && lo < r.hi) return true;
    }
    return false;
  }

 private:
  struct Range {
    uintptr_t lo, hi;
  };
  struct Kind {
    std::vector<Range> ranges;
    uintptr_t lo = UINTPTR_MAX, hi = 0;  // around all of them
    bool ascending = true;               // and disjoint
  };
  Kind kind_[N];
  std::vector<Range> written_, read_;
};

}  // namespace edit
