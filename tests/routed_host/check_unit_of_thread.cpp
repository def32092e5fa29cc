// Host check of unit_of_thread (csrc/common.h), the row and unit of a thread of the
// adapters' last launch: over launches from one thread to nearly 2^32, the first and last
// units, those about 2^31, row ends and random ones are named as 64-bit division has
// them, each thread past the last is refused.  Exits 1 on any mismatch.
#include <cstdio>
#include <cstdint>
#include "common.h"
using namespace cnnlib;
int main() {
  uint64_t bad = 0, n = 0;
  uint32_t seed = 99;
  // rows of `per` units: 352 rows of 25e6 features, 351 of 4 (2^31 / 351) and more
  const int sizes[][2] = {{1, 1},          {3, 7},          {333, 385},      {512, 1024},  {352, 6250000},
                          {351, 6118192},  {351, 6118194},  {352, 12000000}, {1, 1 << 28}, {16, 1 << 27},
                          {15, 286331135}, {255, 16843007}, {512, 8388607}};
  for (const auto& s : sizes) {
    const int64_t all = (int64_t)s[0] * s[1], threads = (all + 255) / 256 * 256;
    if (threads > kMostThreads) return printf("no such launch\n"), 1;
    auto look = [&](int64_t i) {
      if (i < 0 || i >= threads) return;
      int row = -1, unit = -1;
      const bool there = unit_of_thread((uint32_t)(i / 256), (uint32_t)(i % 256), s[0], s[1], &row, &unit);
      ++n;
      if (there != (i < all) || (there && (row != i / s[1] || unit != i % s[1]))) ++bad;
    };
    for (int64_t d = -300; d <= 300; ++d)
      for (int64_t at : {(int64_t)0, all, threads, (int64_t)1 << 31, (int64_t)s[1], all - s[1], all / 2}) look(at + d);
    for (int k = 0; k < 100000; ++k) {
      seed = seed * 1664525u + 1013904223u;
      look((int64_t)((unsigned __int128)seed * (uint64_t)threads >> 32));
    }
  }
  printf("checked %llu bad %llu\n", (unsigned long long)n, (unsigned long long)bad);
  return bad != 0;
}
