// id_table.h -- where constrain.hip's table of a column's ids keeps each of them
// (internal to libkbchain; plain C++, also compiled for the host by the tests).
#pragma once

#include <cstdint>

namespace kbc {

constexpr int kTableThreads = 512;
constexpr int kTable = kTableThreads * 4;  // places
constexpr int kSlice = kTable / 2;         // ids of a slice, on average
constexpr int kProbes = 256;               // places that an id is looked for in

// Two multiplications by an odd number (2^32 over the golden ratio), a shift between
// them: one to one, so different ids have different hashes.
constexpr uint32_t id_hash(uint32_t id) {
  uint32_t h = id * 0x9E3779B9u;
  h = (h ^ h >> 15) * 0x9E3779B9u;
  return h;
}
// The place is the hash's lower bits, the slice its upper ones, so that up to 2^21
// slices leave the places within one as spread as they are: columns of up to 67 million
// neighbouring or evenly spaced ids have theirs within 50 places of their own.  (With
// the slice from bit 19 down, whose bits meet the place's from 1024 slices on, half of the ids
// of 4 million found no place.)
constexpr int id_place(uint32_t hash) { return (int)(hash % kTable); }
constexpr int id_slice(uint32_t hash, uint32_t slices) {
  return (int)((uint64_t)hash * slices >> 32);
}

}  // namespace kbc
