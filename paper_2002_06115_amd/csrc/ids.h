// ids.h -- what the operators on lists of ids share (internal to libkbchain).
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "kbchain.h"

namespace kbc {

constexpr int kThreads = 256;
constexpr int kWave = 64;

// The ids and offsets of a call, int32 or int64.
struct Ints {
  const void *p;
  int bytes;
};
__device__ __forceinline__ int64_t load_int(const Ints &a, int64_t i) {
  return a.bytes == 8 ? static_cast<const int64_t *>(a.p)[i]
                      : (int64_t)static_cast<const int32_t *>(a.p)[i];
}

// How tokens are grouped into bags: bag g holds tokens [begin(g), begin(g + 1)).
struct Bags {
  int64_t n;       // 0: every token is an output row of its own
  Ints offsets;    // null: n bags of `each` tokens
  int64_t each;
  int64_t tokens;
};
__device__ __forceinline__ int64_t bag_begin(const Bags &b, int64_t g) {
  if (!b.offsets.p) return g * b.each;
  const int64_t o = load_int(b.offsets, g);
  return o < 0 ? 0 : o > b.tokens ? b.tokens : o;  // never a token past the last
}
// The bag of token t, -1 where it is in none.
__device__ __forceinline__ int64_t bag_of(const Bags &b, int64_t t) {
  if (!b.offsets.p) return t / b.each;
  int64_t lo = 0, hi = b.n + 1;  // offsets [0, lo) are <= t, [hi, n] are > t
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (bag_begin(b, mid) <= t)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo >= 1 && lo <= b.n ? lo - 1 : -1;
}

// The same by L neighbouring lanes for a token of theirs, L + 1 parts a step.
template <int L>
__device__ __forceinline__ int64_t bag_of_lanes(const Bags &b, int64_t t, int lane) {
  if (!b.offsets.p) return t / b.each;
  int64_t lo = 0, hi = b.n + 1;
  while (lo < hi) {
    const int64_t step = (hi - lo + L) / (L + 1);
    const int64_t at = lo + step * (lane + 1) - 1;  // the last of the lane's part
    const bool below = at < hi && bag_begin(b, at) <= t;
    const unsigned long long mask = __ballot(below) >> (threadIdx.x % kWave / L * L) & ((1ull << L) - 1);
    const int parts = __popcll(mask);  // that end at or before t
    const int64_t from = lo + parts * step;
    if (parts < L && hi > from + step - 1) hi = from + step - 1;
    lo = from;
  }
  return lo >= 1 && lo <= b.n ? lo - 1 : -1;
}

// -- host side ----------------------------------------------------------------------

inline Bags bags_of(int64_t bags, const void *offsets, int32_t id_bytes, int64_t tokens) {
  return {bags, {offsets, id_bytes}, bags > 0 ? tokens / bags : 1, tokens};
}

// A grid's threads fit 32 bits.
constexpr int64_t kMostBlocks = (int64_t(1) << 32) / kThreads - 1;
// Every index into rows, ids and bags fits an int, and so do places in a list.
constexpr int64_t kMostTokens = int64_t(1) << 30;
constexpr int64_t kMostRows = (int64_t)INT32_MAX - 1;

inline int64_t size_of(kbc_type t) { return t == KBC_F32 ? 4 : 2; }
inline bool bad_type(kbc_type t) { return t != KBC_F32 && t != KBC_BF16 && t != KBC_F16; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline kbc_status launched() { return hipGetLastError() == hipSuccess ? KBC_OK : KBC_EHIP; }

}  // namespace kbc
