// Drives WrittenRanges beside a comparison of every pair, over lists in order
// and out of it, of kinds apart and mixed.  Prints how often it found none, a
// written buffer met by a written one, and by a read one; how often a stretch
// met no written buffer, and one.
#include <cstdio>
#include <random>
#include <vector>

#include "written_ranges.h"

struct One {
  int kind;
  uintptr_t lo, hi;
};

int main() {
  constexpr int N = 6;
  std::mt19937 gen(7);
  long found[3] = {0, 0, 0}, hit[2] = {0, 0};
  edit::WrittenRanges<N> set;
  set.reserve(64);
  for (int round = 0; round < 300000; ++round) {
    set.clear();
    std::vector<One> list;
    const unsigned writes = gen() % (1u << N);
    const bool apart = gen() % 2, ascending = gen() % 2;  // as a program's buffers mostly lie
    const uintptr_t span = 10 + gen() % 2000;
    const int count = gen() % 8;
    for (int k = 0; k < N; ++k) {
      uintptr_t at = apart ? 4000 * k : 0;
      for (int i = 0; i < count; ++i) {
        if (gen() % 8 == 0) continue;  // an empty tensor, or one without a gradient
        const uintptr_t size = 1 + gen() % 30;
        const uintptr_t lo = ascending ? at + gen() % 3 - (i && gen() % 64 == 0) : (apart ? 4000 * k : 0) + gen() % span;
        list.push_back({k, lo, lo + size});
        set.add(k, lo, lo + size);
        at = lo + size;
      }
    }
    bool written = false, read = false;
    for (size_t i = 0; i < list.size(); ++i)
      for (size_t j = 0; j < i; ++j) {
        const One &a = list[i], &b = list[j];
        if (!(a.lo < b.hi && b.lo < a.hi)) continue;
        const int w = (writes >> a.kind & 1) + (writes >> b.kind & 1);
        written = written || w == 2;
        read = read || w == 1;
      }
    const edit::Overlap want = written ? edit::kOverlapWritten : read ? edit::kOverlapRead : edit::kOverlapNone;
    if (set.find(writes) != want) {
      std::printf("round %d: %d, not %d\n", round, set.find(writes), want);
      return 1;
    }
    ++found[want];
    const uintptr_t lo = gen() % (apart ? 4000 * N : span), hi = lo + 1 + gen() % 10;
    bool met = false;
    for (const One& a : list) met = met || ((writes >> a.kind & 1) && a.lo < hi && lo < a.hi);
    if (set.written_at(writes, lo, hi) != met) {
      std::printf("round %d: [%lu, %lu) %d\n", round, static_cast<unsigned long>(lo), static_cast<unsigned long>(hi), met);
      return 1;
    }
    ++hit[met];
  }
  std::printf("%ld %ld %ld %ld %ld\n", found[0], found[1], found[2], hit[0], hit[1]);
  return 0;
}
