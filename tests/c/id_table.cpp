// The table that counts a column's ids, a slice of them at a time (csrc/id_table.h):
// however many slices there are, the slices stay even and every id of one finds a
// place close to its own.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "id_table.h"

using namespace kbc;

namespace {

int failures = 0;

// Columns of `ids` ids 0, step, 2 step, ..: the slices' sizes, and in some of them the
// farthest that an id lands from its place.
void column(int64_t ids, uint32_t step) {
  const uint32_t slices = (uint32_t)((ids + kSlice - 1) / kSlice);
  std::vector<int> size(slices);
  constexpr int kSampled = 64;
  std::vector<std::vector<uint32_t>> sampled(kSampled);
  for (int64_t i = 0; i < ids; ++i) {
    const uint32_t h = id_hash((uint32_t)i * step);
    const int s = id_slice(h, slices);
    if (s < 0 || s >= (int)slices) {
      std::printf("slice %d of %u\n", s, slices);
      ++failures;
      return;
    }
    ++size[s];
    const int k = (int)((int64_t)s * kSampled / slices);
    if (s == (int)((int64_t)slices * k / kSampled)) sampled[k].push_back(h);
  }
  int most = 0, farthest = 0, lost = 0;
  for (int n : size) most = n > most ? n : most;
  for (const auto &hashes : sampled) {
    std::vector<bool> taken(kTable);
    for (uint32_t h : hashes) {
      int probe = 0, at = id_place(h);
      while (probe < kProbes && taken[at]) {
        ++probe;
        at = (at + 1) % kTable;
      }
      if (probe == kProbes)
        ++lost;
      else
        taken[at] = true;
      farthest = probe > farthest ? probe : farthest;
    }
  }
  std::printf("%lld ids, step %u: %u slices of at most %d ids, farthest %d, lost %d\n",
              (long long)ids, step, slices, most, farthest, lost);
  // 1024 ids a slice: 1400 is 11 times sqrt(1024) more.  At half of the places taken the
  // longest of the runs that such a slice leaves is below 100 with room.
  if (most > 1400 || farthest > 100 || lost) {
    std::printf("  too uneven\n");
    ++failures;
  }
}

}  // namespace

int main() {
  for (int64_t slices : {2, 3, 17, 64, 333, 500, 1000, 1024, 2048, 4000, 16000, 65536})
    for (uint32_t step : {1u, 2u, 3u, 7u, 64u, 100u, 255u, 2048u, 4096u, 65536u}) {
      const int64_t ids = slices * kSlice;
      if ((uint64_t)ids * step <= (uint64_t)INT32_MAX) column(ids, step);
    }
  if (failures) {
    std::printf("%d checks failed\n", failures);
    return 1;
  }
  std::printf("the table holds\n");
  return 0;
}
