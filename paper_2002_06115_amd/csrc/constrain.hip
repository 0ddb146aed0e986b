// constrain.hip -- penalties for what a column has had, biases and masks on logits
// (kbchain.h: kbc_constrain, kbc_constrain_backward).
//
// Element (i, beta) of an [n][b] array, c the number of times i is in column
// beta's history:
//     v = z;  c > 0:  v = v > 0 ? v / repeat : v * repeat,
//                     v -= presence + frequency * c
//     v += bias;  not allowed:  v = fill
// and the gradient:  not allowed: 0, else dz = dout * (c > 0 ? (z > 0 ? 1 / repeat :
// repeat) : 1), dbias = dout.
//
// One pass over the arrays in the order they lie in, 4 elements a lane, writes every
// element as if no history were, bound by the bytes it moves; then the few elements
// of the history are written again, by the threads that count them.  (A dense array
// of counts would be read and written as a whole for them.)  Where array and history
// are small each workgroup counts for its own elements first, and one launch is all.
// Otherwise a short column's ids are compared with each other, a block of them in LDS
// at a time, where an id that occurs twice is written twice with the same value, and
// a long column's are counted in a table in LDS.  A shared bias' gradient is summed row
// by row, in double, in a fixed order, by the lanes that write the row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "id_table.h"
#include "ids.h"
#include "kbchain.h"

namespace {

using namespace kbc;

typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned char uchar4_any __attribute__((ext_vector_type(4), aligned(1)));
template <class T>
using vec4_any = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));

enum Allowed { kAll, kBytes, kBits };

struct Args {
  int64_t n;
  int32_t b;
  uint32_t magic;  // ceil(2^32 / b), for b <= kMostTile
  const void *z;   // logits (forward), or null
  const float *dout;
  const float *bias;
  int32_t bias_each;
  const void *allowed;
  int32_t allowed_kind, allowed_each;
  float fill;
  void *out;       // float (forward), dz of the logits' type (backward)
  float *dbias;
};

__device__ __forceinline__ bool is_allowed(const Args &a, int64_t i, int32_t col) {
  if (a.allowed_kind == kAll) return true;
  if (a.allowed_kind == kBytes)
    return static_cast<const uint8_t *>(a.allowed)[a.allowed_each ? i * a.b + col : i] != 0;
  const uint32_t *w = static_cast<const uint32_t *>(a.allowed);
  return w[a.allowed_each ? (i >> 5) * a.b + col : i >> 5] >> (i & 31) & 1;
}
__device__ __forceinline__ float bias_of(const Args &a, int64_t i, int32_t col) {
  return a.bias ? a.bias[a.bias_each ? i * a.b + col : i] : 0.0f;
}

// M <= 4 neighbours of the arrays: the place, row and column of the first.
struct Four {
  int64_t f, i;
  int32_t col;
  int m;
};
__device__ __forceinline__ bool one_row(const Args &a, const Four &p) {
  return p.m == 4 && p.col <= a.b - 4;  // (b may be 2^31 - 1)
}
// idx(row, column) of each of the four, the first's again where there are less.
template <class F>
__device__ __forceinline__ void places(const Args &a, const Four &p, F idx, int64_t (&at)[4]) {
  int64_t i = p.i;
  int32_t col = p.col;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    at[e] = e < p.m ? idx(i, col) : idx(p.i, p.col);
    if (++col == a.b) {
      col = 0;
      ++i;
    }
  }
}
// Bit e: whether the e-th of them is allowed.
__device__ __forceinline__ unsigned allowed4(const Args &a, const Four &p) {
  if (a.allowed_kind == kAll) return 15;
  if (a.allowed_kind == kBytes) {
    const uint8_t *w = static_cast<const uint8_t *>(a.allowed);
    if (!a.allowed_each && one_row(a, p)) return w[p.i] ? 15 : 0;
    uchar4_any t;
    if (a.allowed_each && p.m == 4) {
      t = *reinterpret_cast<const uchar4_any *>(w + p.f);
    } else {
      int64_t at[4];
      places(a, p, [&](int64_t i, int32_t col) { return a.allowed_each ? i * a.b + col : i; }, at);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = w[at[e]];
    }
    return (t[0] ? 1 : 0) | (t[1] ? 2 : 0) | (t[2] ? 4 : 0) | (t[3] ? 8 : 0);
  }
  const uint32_t *w = static_cast<const uint32_t *>(a.allowed);
  if (one_row(a, p)) {
    const int bit = (int)(p.i & 31);
    if (!a.allowed_each) return w[p.i >> 5] >> bit & 1 ? 15 : 0;
    const vec4_any<uint32_t> t =
        *reinterpret_cast<const vec4_any<uint32_t> *>(w + (p.i >> 5) * a.b + p.col);
    return (t[0] >> bit & 1) | (t[1] >> bit & 1) << 1 | (t[2] >> bit & 1) << 2 |
           (t[3] >> bit & 1) << 3;
  }
  int64_t at[4], row[4];
  places(a, p, [&](int64_t i, int32_t col) { return a.allowed_each ? (i >> 5) * a.b + col : i >> 5; },
         at);
  places(a, p, [&](int64_t i, int32_t) { return i; }, row);
  uint32_t t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = w[at[e]];
  unsigned ok = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) ok |= (t[e] >> (row[e] & 31) & 1) << e;
  return ok;
}
__device__ __forceinline__ void bias4(const Args &a, const Four &p, float (&v)[4]) {
  if (!a.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = 0.0f;
  } else if (a.bias_each && p.m == 4) {
    const float4_any t = *reinterpret_cast<const float4_any *>(a.bias + p.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e];
  } else if (!a.bias_each && one_row(a, p)) {
    const float t = a.bias[p.i];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t;
  } else {
    int64_t at[4];
    places(a, p, [&](int64_t i, int32_t col) { return a.bias_each ? i * a.b + col : i; }, at);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a.bias[at[e]];
  }
}
// The first m <= 4 values at p (zeros for the others), and the way back.
template <class T>
__device__ __forceinline__ vec4_any<T> load4(const T *p, int m) {
  vec4_any<T> v;
  if (m == 4) {
    v = *reinterpret_cast<const vec4_any<T> *>(p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < m ? p[e] : (T)0.0f;
  }
  return v;
}
template <class T>
__device__ __forceinline__ void store4(T *p, int m, const float (&y)[4]) {
  if (m == 4) {
    vec4_any<T> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (T)y[e];
    __builtin_nontemporal_store(v, reinterpret_cast<vec4_any<T> *>(p));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < m) p[e] = (T)y[e];
  }
}

struct Penalties {
  Ints ids;
  Bags columns;
  const float *repeat, *presence, *frequency;  // [b], or null:
  float repeat_all, presence_all, frequency_all;
};

// The row that entry t names, -1 for padding.
__device__ __forceinline__ int row_of(const Penalties &p, int64_t n, int64_t t) {
  const int64_t id = load_int(p.ids, t);
  return id >= 0 && id < n ? (int)id : -1;
}

// An element of the history, in double: the logit, and the slope of the logit.
__device__ __forceinline__ float penalised(const Penalties &p, int32_t col, float logit, int count,
                                           float bias) {
  const double z = (double)logit, repeat = p.repeat ? p.repeat[col] : p.repeat_all;
  double v = z > 0.0 ? z / repeat : z * repeat;
  v -= p.presence ? p.presence[col] : p.presence_all;
  v -= (double)(p.frequency ? p.frequency[col] : p.frequency_all) * count;
  return (float)(v + (double)bias);
}
__device__ __forceinline__ float scaled(const Penalties &p, int32_t col, float logit, float dout) {
  const double g = (double)dout, repeat = p.repeat ? p.repeat[col] : p.repeat_all;
  return (float)(logit > 0.0f ? g / repeat : g * repeat);
}

// A few ids over a small array: every workgroup counts those of its own elements,
// size of them from `first` on, in LDS.
constexpr int kFewTile = kThreads * 4;
constexpr int kFewColumns = 1024;
__device__ void count_few(const Args &a, const Penalties &p, int64_t first, int size, int *counts,
                          int *begins) {
  for (int i = threadIdx.x; i < size; i += kThreads) counts[i] = 0;
  if (p.columns.offsets.p)
    for (int c = threadIdx.x; c <= a.b; c += kThreads) begins[c] = (int)bag_begin(p.columns, c);
  __syncthreads();
  for (int t = threadIdx.x; t < (int)p.columns.tokens; t += kThreads) {
    const int id = row_of(p, a.n, t);
    int col;
    if (!p.columns.offsets.p) {
      col = t / (int)p.columns.each;
    } else {
      int lo = 0, hi = a.b + 1;  // begins [0, lo) are <= t, [hi, b] are > t
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (begins[mid] <= t)
          lo = mid + 1;
        else
          hi = mid;
      }
      col = lo - 1;
    }
    const int64_t f = (int64_t)id * a.b + col - first;
    if (id >= 0 && col >= 0 && col < a.b && f >= 0 && f < size) atomicAdd(&counts[f], 1);
  }
  __syncthreads();
}

// -- every element, as if no history were, or with that of a few ids -----------------------

// Vectors of 4 elements of a thread, and elements of a workgroup: DEPTH 1 where an
// array is small and latency counts, 4 where it is large.
template <int DEPTH>
constexpr int kTile = kThreads * 4 * DEPTH;
constexpr int kMostTile = kTile<4>;

// BACKWARD: dz (and a bias' own gradient, one an element) from dout.  FEW: with the
// history (DEPTH 1).
template <class T, bool BACKWARD, int DEPTH, bool FEW>
__global__ __launch_bounds__(kThreads) void dense_kernel(Args a, Penalties h) {
  static_assert(!FEW || kTile<DEPTH> == kFewTile, "a count for each element");
  using In = std::conditional_t<BACKWARD, float, T>;
  using Out = std::conditional_t<BACKWARD, T, float>;
  const In *in = BACKWARD ? reinterpret_cast<const In *>(a.dout) : static_cast<const In *>(a.z);
  Out *out = static_cast<Out *>(a.out);
  const int64_t first = (int64_t)blockIdx.x * kTile<DEPTH>, size = a.n * a.b;
  const int64_t row0 = first / a.b;
  const uint32_t rest = (uint32_t)(first - row0 * a.b);
  vec4_any<In> v[DEPTH];
  Four p[DEPTH];
#pragma unroll
  for (int k = 0; k < DEPTH; ++k) {
    const uint32_t local = (uint32_t)(k * kThreads + (int)threadIdx.x) * 4;
    // The row and column of the first of the four: exact, as the dividend is
    // below 2 b where b is above kMostTile, and below 2 kMostTile where it is not.
    const uint32_t x = rest + local;
    const uint32_t q = a.b > kMostTile ? (uint32_t)(x >= (uint32_t)a.b)
                       : a.b == 1      ? x
                                       : __umulhi(x, a.magic);
    p[k] = {first + local, row0 + q, (int32_t)(x - q * (uint32_t)a.b),
            (int)max((int64_t)0, min((int64_t)4, size - first - local))};
    v[k] = load4<In>(in + p[k].f, p[k].m);
  }
  __shared__ int counts[FEW ? kFewTile : 1], begins[FEW ? kFewColumns + 1 : 1];
  if constexpr (FEW) count_few(a, h, first, kFewTile, counts, begins);
#pragma unroll
  for (int k = 0; k < DEPTH; ++k) {
    if (p[k].m == 0) break;
    const unsigned ok = allowed4(a, p[k]);
    float y[4], bias[4];
    if constexpr (BACKWARD) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = ok >> e & 1 ? (float)v[k][e] : 0.0f;
      if (a.dbias) store4<float>(a.dbias + p[k].f, p[k].m, y);
    } else {
      bias4(a, p[k], bias);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = ok >> e & 1 ? (float)v[k][e] + bias[e] : a.fill;
    }
    if constexpr (FEW) {
      int32_t col = p[k].col;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e < p[k].m && (ok >> e & 1)) {
          const int count = counts[threadIdx.x * 4 + e];
          if (count > 0) {
            if constexpr (BACKWARD)
              y[e] = scaled(h, col, (float)static_cast<const T *>(a.z)[p[k].f + e], y[e]);
            else
              y[e] = penalised(h, col, (float)v[k][e], count, bias[e]);
          }
        }
        if (++col == a.b) col = 0;
      }
    }
    store4<Out>(out + p[k].f, p[k].m, y);
  }
}

// The backward pass with a shared bias: G lanes a row, which they also sum.  (Four
// rows of a group in flight took as long for 64 million elements, and 16.8 us for
// 14.8 for 4 million, with the history's launch.)
template <class T, int G, bool FEW>
__global__ __launch_bounds__(kThreads) void row_kernel(Args a, Penalties h) {
  constexpr int GPB = kThreads / G;
  __shared__ int counts[FEW ? kFewTile : 1], begins[FEW ? kFewColumns + 1 : 1];
  if constexpr (FEW)  // (b is at most 4 G)
    count_few(a, h, (int64_t)blockIdx.x * GPB * a.b, GPB * a.b, counts, begins);
  const int lane = threadIdx.x % G;
  const int64_t i = (int64_t)blockIdx.x * GPB + threadIdx.x / G;
  if (i >= a.n) return;  // whole groups; their shuffles stay inside the group
  double sum = 0.0;
  for (int64_t c = lane * 4; c < a.b; c += G * 4) {
    const Four p = {i * a.b + c, i, (int32_t)c, (int)min((int64_t)4, a.b - c)};
    const vec4_any<float> v = load4<float>(a.dout + p.f, p.m);
    const unsigned ok = allowed4(a, p);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = ok >> e & 1 ? v[e] : 0.0f;  // (those past the row are zeros)
      sum += (double)y[e];
      if constexpr (FEW)
        if (e < p.m && (ok >> e & 1) && counts[(int)(threadIdx.x / G) * a.b + (int)c + e] > 0)
          y[e] = scaled(h, (int32_t)c + e, (float)static_cast<const T *>(a.z)[p.f + e], y[e]);
    }
    store4<T>(static_cast<T *>(a.out) + p.f, p.m, y);
  }
#pragma unroll
  for (int m = 1; m < G; m <<= 1) sum += __shfl_xor(sum, m);
  if (lane == 0) a.dbias[i] = (float)sum;
}

// -- the elements of the history --------------------------------------------------------

// Lanes that share an entry's count: 15200 ids of 8 columns take 14 us with 16 lanes,
// 17 with 8, 27 with 4.  Where nothing is counted they only find the entry's column: 16
// / 8 lanes take, with the dense launch, 8.3 / 8.6 us for 93 columns of 3 ids, 56 / 38 for
// 128 of 4000, 49 / 35 for 20000 of 16.  4 lanes against 1: 7.6 and 8.7 us for 93 columns
// of 3 ids, 6.2 and 7.5 for 500 of 16, 5.5 and 6.0 for 8 of 2000, but from about 100,000 ids
// on 1 lane is ahead, 9.4 and 8.7 for 128 of 1000, 27 and 22 for 128 of 4000, 36 and 30 for
// 20000 of 16 (gradient 38.5 and 34.6): the histories of a model's columns are the shorter.
constexpr int kCountLanes = 16;
constexpr int kFindLanes = 4;
constexpr int kBlockIds = 2048;                      // ids in LDS at a time
constexpr int kCompare = 4;                          // quads of them in flight

template <class T, bool BACKWARD, int LANES>
__global__ __launch_bounds__(kThreads) void history_kernel(Args a, Penalties p, int64_t from,
                                                           int64_t longest) {
  constexpr int kEntries = kThreads / LANES;  // of a workgroup, those of the launch from `from` on
  __shared__ int4 lds[kBlockIds / 4];
  __shared__ int64_t range[2];
  int *ids = reinterpret_cast<int *>(lds);
  const int lane = threadIdx.x % LANES;
  const int64_t t0 = from + (int64_t)blockIdx.x * kEntries, t = t0 + threadIdx.x / LANES;
  const int64_t total = p.columns.tokens;
  const int64_t col = t < total ? bag_of_lanes<LANES>(p.columns, t, lane) : -1;
  int id = -1;
  int64_t begin = t, end = t + 1;  // the ids of the entry's column
  if (col >= 0) {
    const int64_t b0 = bag_begin(p.columns, col), b1 = bag_begin(p.columns, col + 1);
    if (b1 - b0 <= longest) {  // else table_kernel's
      id = row_of(p, a.n, t);
      begin = b0;
      end = b1;
    }
  }
  const bool valid = id >= 0;  // the same for the lanes of an entry
  const bool counts = !BACKWARD && (p.frequency || p.frequency_all != 0.0f);
  int count = 0;
  if (counts) {  // uniform
    // The ids of every column that the workgroup's entries are of.
    if (threadIdx.x == 0) range[0] = begin;
    if (lane == 0 && t == min(t0 + kEntries, total) - 1) range[1] = end;
    __syncthreads();
    const int64_t r1 = min(range[1], total);
    // The next block is on its way while one is compared.
    int next[kBlockIds / kThreads];
    auto fetch = [&](int64_t r0) {
#pragma unroll
      for (int u = 0; u < kBlockIds / kThreads; ++u)
        next[u] = row_of(p, a.n, min(r0 + u * kThreads + threadIdx.x, r1 - 1));
    };
    if (range[0] < r1) fetch(range[0]);
    for (int64_t r0 = range[0]; r0 < r1; r0 += kBlockIds) {
      __syncthreads();  // the block before has been read
#pragma unroll
      for (int u = 0; u < kBlockIds / kThreads; ++u) ids[u * kThreads + threadIdx.x] = next[u];
      __syncthreads();
      if (r0 + kBlockIds < r1) fetch(r0 + kBlockIds);
      if (valid) {
        const int lo = (int)max((int64_t)0, begin - r0);
        const int hi = (int)min((int64_t)kBlockIds, end - r0);
        // Whole quads of the column, kCompare in flight, then its ends one by one.
        const int q0 = (lo + 3) / 4, q1 = hi / 4;
        int q = q0 + lane;
        for (; q + (kCompare - 1) * LANES < q1; q += kCompare * LANES) {
          int4 x[kCompare];
#pragma unroll
          for (int u = 0; u < kCompare; ++u) x[u] = lds[q + u * LANES];
#pragma unroll
          for (int u = 0; u < kCompare; ++u)
            count += (x[u].x == id) + (x[u].y == id) + (x[u].z == id) + (x[u].w == id);
        }
        for (; q < q1; q += LANES) {
          const int4 x = lds[q];
          count += (x.x == id) + (x.y == id) + (x.z == id) + (x.w == id);
        }
        const int head = lo + lane, tail = max(q1, q0) * 4 + lane;
        if (head < min(q0 * 4, hi)) count += ids[head] == id;
        if (tail < hi) count += ids[tail] == id;
      }
    }
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) count += __shfl_xor(count, m);
  }
  if (!valid || lane != 0) return;
  const int64_t f = (int64_t)id * a.b + col;
  const bool ok = is_allowed(a, id, (int32_t)col);
  const float z = (float)static_cast<const T *>(a.z)[f];
  if constexpr (BACKWARD)
    static_cast<T *>(a.out)[f] = (T)(ok ? scaled(p, (int32_t)col, z, a.dout[f]) : 0.0f);
  else
    static_cast<float *>(a.out)[f] =
        ok ? penalised(p, (int32_t)col, z, count, bias_of(a, id, (int32_t)col)) : a.fill;
}

// Few columns are shared by workgroups that take a slice each: up to this many
// workgroups, and a column up to one for every 512 ids of all columns together, not of its
// own, as it may hold most of them.  (8 columns of 1900 ids, by the 256 / 512 / 1024 ids of
// all columns 9.0 / 8.3 / 8.6 us, by 512 of its own 9.4; the same of uneven lengths 11.4 / 11.1
// / 11.5 and 23; one column of 16000 16.1 / 17.9 / 24.4, of 100000 51 / 51 / 63.)
constexpr int64_t kTableBlocks = 512;
constexpr int64_t kShare = 512;

// The forward pass where columns have many ids: a workgroup puts a column's ids
// into a table in LDS and counts them there, a slice of the ids at a time (by hash,
// at most about half as many as the table holds), then each place of the table writes
// its element.  Where an id finds no place, as ids chosen for it can bring about, the
// slice is taken again by ranges of the id, an eighth as wide each time, until the
// table holds them; at the latest a range has a place for each of its ids.
// (1024 threads and 4096 places: 128 columns of 4000 ids 35 us for 29, 1024 of 64 30 for
// 24, one of 16000 19 for 19.)
//
// Ragged columns differ: one may have nearly all of the ids.  Those of more than
// `longest` ids are shared by the first `sharing` workgroups, kShare ids of the list to
// each of them in turn; of the others each takes a part of one column.  (SHARING: there are
// such; without, 20,000 columns of 64 ids take 120 us for 129.)
template <class T, bool SHARING>
__global__ __launch_bounds__(kTableThreads) void table_kernel(Args a, Penalties p, int parts,
                                                              int sharing, int64_t longest) {
  __shared__ int4 keys4[kTableThreads], counts4[kTableThreads];
  __shared__ int full;  // the last turn in which an id found no place
  int *keys = reinterpret_cast<int *>(keys4), *counts = reinterpret_cast<int *>(counts4);
  int32_t col = 0;  // the column at hand, its ids and their slices
  int64_t begin = 0, end = 0;
  int slices = 0;
  // What an element is made of, and its place once its ids are counted.
  struct Element {
    float z, bias;
    bool ok;
  };
  auto element = [&](int id) {
    return Element{(float)static_cast<const T *>(a.z)[(int64_t)id * a.b + col], bias_of(a, id, col),
                   is_allowed(a, id, col)};
  };
  auto write = [&](int id, int count, const Element &e) {
    static_cast<float *>(a.out)[(int64_t)id * a.b + col] =
        e.ok ? penalised(p, col, e.z, count, e.bias) : a.fill;
  };
  if (threadIdx.x == 0) full = 0;
  int turn = 0;
  // The ids of [lo, lo + width) in the slice; false where the table cannot hold them.
  auto count_range = [&](int slice, int lo, uint32_t width) {
    const bool own_places = width <= (uint32_t)kTable;
    ++turn;
    // (A thread clears the places that it read the last time.)
    keys4[threadIdx.x] = {-1, -1, -1, -1};
    counts4[threadIdx.x] = {0, 0, 0, 0};
    __syncthreads();
    for (int64_t r = begin; r < end; r += kTable) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t t = r + u * kTableThreads + threadIdx.x;
        id[u] = row_of(p, a.n, min(t, end - 1));
        if (t >= end) id[u] = -1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if ((uint32_t)id[u] - (uint32_t)lo >= width) continue;  // padding, too
        const uint32_t hash = id_hash((uint32_t)id[u]);
        if (id_slice(hash, (uint32_t)slices) != slice) continue;
        int at = own_places ? id[u] - lo : id_place(hash), probe = 0;
        for (; probe < kProbes; ++probe, at = (at + 1) % kTable) {
          int key = keys[at];
          if (key == -1) key = atomicCAS(&keys[at], -1, id[u]);
          if (key == -1 || key == id[u]) break;
        }
        if (probe < kProbes)
          atomicAdd(&counts[at], 1);
        else
          full = turn;
      }
    }
    __syncthreads();
    if (full == turn) return false;  // the same for the whole workgroup
    const int4 k = keys4[threadIdx.x], c = counts4[threadIdx.x];
    const int id[4] = {k.x, k.y, k.z, k.w}, count[4] = {c.x, c.y, c.z, c.w};
    Element e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) e[u] = element(max(id[u], 0));  // all four on their way
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (id[u] >= 0) write(id[u], count[u], e[u]);
    return true;
  };
  // Slices part, part + of, .. of the column at hand.
  auto take = [&](int part, int of) {
    slices = max(of, (int)((end - begin + kSlice - 1) / kSlice));
    for (int slice = part; slice < slices; slice += of) {
      // 2^bits ranges (at most 8 n / kTable, so the products fit).
      for (int64_t r = 0, bits = 0; r >> bits == 0;) {
        const int64_t lo = a.n * r >> bits, hi = a.n * (r + 1) >> bits;
        if (count_range(slice, (int)lo, (uint32_t)(hi - lo))) {
          ++r;
        } else {  // what is left, in narrower ranges
          bits += 3;
          r <<= 3;
        }
      }
    }
  };
  const int own = (int)blockIdx.x - (SHARING ? sharing : 0);
  if (own >= 0) {
    col = own / parts;
    begin = bag_begin(p.columns, col);
    end = bag_begin(p.columns, col + 1);
    if (end > begin && (!SHARING || end - begin <= longest)) take(own % parts, parts);
    return;
  }
  if constexpr (SHARING) {
    // A column of more than `longest` ids has one of every longest-th of the list; the
    // first of them finds it.
    __shared__ int32_t found[kTableThreads];
    __shared__ unsigned long long any[kTableThreads / kWave];
    const int64_t total = p.columns.tokens;
    for (int64_t base = 0; base * longest < total; base += kTableThreads) {
      const int64_t t = (base + threadIdx.x) * longest;
      int64_t c = t < total ? bag_of(p.columns, t) : -1;
      if (c >= 0) {
        const int64_t b0 = bag_begin(p.columns, c), b1 = bag_begin(p.columns, c + 1);
        if (b1 - b0 <= longest || t - longest >= b0) c = -1;
      }
      const unsigned long long mask = __ballot(c >= 0);
      __syncthreads();  // the last ones have been read
      found[threadIdx.x] = (int32_t)c;
      if (threadIdx.x % kWave == 0) any[threadIdx.x / kWave] = mask;
      __syncthreads();
      for (int w = 0; w < kTableThreads / kWave; ++w)
        for (unsigned long long m = any[w]; m; m &= m - 1) {  // uniform
          col = found[w * kWave + __builtin_ctzll(m)];
          begin = bag_begin(p.columns, col);
          end = bag_begin(p.columns, col + 1);
          const int shares = (int)min((int64_t)sharing, (end - begin + kShare - 1) / kShare);
          const int first = (int)(begin / kShare % sharing);
          const int mine = ((int)blockIdx.x - first + sharing) % sharing;
          if (mine < shares) take(mine, shares);
        }
    }
  }
}

// -- how a call is launched ----------------------------------------------------------------

// Elements from which workgroups take 4 vectors a thread: 64 million take 81 us with
// four and 90 with one; 4 million of 43000 rows of 93 columns, with the history's
// launch, 15.8 and 12.9.
constexpr int64_t kSmall = 1 << 22;

template <class F>
void with_type(kbc_type type, F f) {
  switch (type) {
    case KBC_F32: f(float{}); break;
    case KBC_BF16: f(__bf16{}); break;
    case KBC_F16: f(_Float16{}); break;
  }
}

bool bad_limits(int64_t n, int32_t b, kbc_type type, const kbc_limits *l) {
  if (n < 1 || n > kMostRows || b < 1 || bad_type(type) || !l) return true;
  if (ceil_div(n * b, kMostTile) > kMostBlocks) return true;
  if (l->entries < 0 || l->entries > kMostTokens) return true;
  if (l->entries > 0) {
    if (!l->history || (l->id_bytes != 4 && l->id_bytes != 8)) return true;
    if (!l->offsets && l->entries % b != 0) return true;
  }
  auto bad = [](float x) { return !std::isfinite(x); };
  return bad(l->repeat_all) || bad(l->presence_all) || bad(l->frequency_all) ||
         (!l->repeat && !(l->repeat_all > 0.0f));
}

Args args_for(int64_t n, int32_t b, const kbc_limits *l) {
  Args a{};
  a.n = n;
  a.b = b;
  a.magic = (uint32_t)((((uint64_t)1 << 32) + b - 1) / b);
  a.bias = l->bias;
  a.bias_each = l->bias_each;
  a.allowed = l->allowed;
  a.allowed_kind = !l->allowed ? kAll : l->allowed_bits ? kBits : kBytes;
  a.allowed_each = l->allowed_each;
  return a;
}
Penalties penalties_for(int32_t b, const kbc_limits *l) {
  return {{l->history, l->id_bytes}, bags_of(b, l->offsets, l->id_bytes, l->entries),
          l->repeat, l->presence, l->frequency, l->repeat_all, l->presence_all, l->frequency_all};
}

// Ids of a column, on average, from which table_kernel counts them.  With the dense
// launch, compared and by table, us: 32 columns of 128 ids 9.6 and 9.6, of 512 11.3 and
// 10.7, 8 of 1900 13.4 and 9.7, 1 of 16000 34 and 19, of 100000 755 and 52, 128 of 1000 37
// and 17, of 4000 196 and 29, 1024 of 64 29 and 24; but 93 of 32 9.7 and 9.8, 20000 of 64
// 240 and 117, of 16 70 and 109.
constexpr int64_t kLongColumn = 64;
// Ragged columns' lengths are on the device.  Lists of more ids than kSkewed, where
// one column may hold them all, have their columns of more than kLongest ids shared by
// up to kTableBlocks workgroups (20,000 columns, one of which has 1.2 million ids, 1.7 ms;
// with the launch, and nothing to share, 20,000 of 16 85 us for 77, of 64 140 for 128).
constexpr int64_t kSkewed = 16384;
constexpr int64_t kLongest = 4096;
// What is counted is read once for every kSlice ids of a column: 2^20 ids of one take
// 0.9 ms, 2^22 13.5, so 2^26 seconds, and 2^30 would take a quarter of an hour.
constexpr int64_t kMostCounted = int64_t(1) << 26;

bool counts_ids(const kbc_limits *l) {
  return l->entries > 0 && (l->frequency || l->frequency_all != 0.0f);
}

template <class T, bool BACKWARD>
void launch_history(const Args &a, const Penalties &h, hipStream_t s) {
  const int64_t total = h.columns.tokens;
  const bool counts = !BACKWARD && (h.frequency || h.frequency_all != 0.0f);
  const bool skewed = counts && h.columns.offsets.p && total > kSkewed;
  const int64_t longest = skewed ? kLongest : INT64_MAX;
  const int sharing = skewed ? (int)std::min(kTableBlocks, ceil_div(total, kShare)) : 0;
  const bool by_table = counts && total / a.b >= kLongColumn && a.b <= kMostBlocks / 4;
  auto go = [&](auto kernel, int lanes) {  // as many ids at a time as a grid holds
    const int64_t per_block = kThreads / lanes, most = kMostBlocks * per_block;
    for (int64_t from = 0; from < total; from += most)
      hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(std::min(most, total - from), per_block)),
                         dim3(kThreads), 0, s, a, h, from, longest);
  };
  if (!counts)
    go(history_kernel<T, BACKWARD, kFindLanes>, kFindLanes);
  else if (!by_table)
    go(history_kernel<T, BACKWARD, kCountLanes>, kCountLanes);
  if constexpr (!BACKWARD)
    if (by_table || skewed) {
      const int64_t parts = std::clamp<int64_t>(kTableBlocks / a.b, 1, ceil_div(total, kShare));
      const int64_t blocks = sharing + (by_table ? a.b * parts : 0);
      const auto kernel = skewed ? table_kernel<T, true> : table_kernel<T, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kTableThreads), 0, s, a, h, (int)parts,
                         sharing, longest);
    }
}

// Few ids over a small array, which every workgroup then reads: at most 1024, and 2^28
// for ids times elements.  One launch against two, forward us: 256 ids over 18 x 128
// 3.5 and 5.7, 700 over 32000 x 1 4.0 and 7.4, 279 over 8000 x 93 3.9 and 6.1, 4 over a
// million x 4 6.7 and 7.6; 1000 over 1000 x 1000 9.4 and 9.1, 279 over 43000 x 93 11.7 and
// 10.5 (not taken).  Taken, and a loss, are up to 64 ids over more elements than kSmall: one
// vector a thread costs more there than a launch, 4 ids over 16 million x 4 83 and 76, 8
// over 4 million x 8 44 and 41, the gradients alike.
bool few_ids(const Args &a, const kbc_limits *l) {
  return l->entries <= 1024 && a.b <= kFewColumns &&
         a.n * a.b <= (int64_t(1) << 28) / l->entries;
}

// history: with the ids' penalties (forward), or slopes (backward).
template <class T, bool BACKWARD>
void launch_dense(const Args &a, bool history, const kbc_limits *l, hipStream_t s) {
  const int64_t size = a.n * a.b;
  const Penalties h = penalties_for(a.b, l);
  auto go = [&](auto kernel, int tile) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(size, tile)), dim3(kThreads), 0, s, a, h);
  };
  if (history && few_ids(a, l)) return go(dense_kernel<T, BACKWARD, 1, true>, kTile<1>);
  if (size < kSmall)
    go(dense_kernel<T, BACKWARD, 1, false>, kTile<1>);
  else
    go(dense_kernel<T, BACKWARD, 4, false>, kTile<4>);
  if (history) launch_history<T, BACKWARD>(a, h, s);
}

// Lanes of a row in row_kernel: 4 elements each, or 4 at a time.
int row_lanes(int32_t b) {
  int lanes = 2;
  while (lanes * 4 < b && lanes < kWave) lanes <<= 1;
  return lanes;
}

template <class T, bool FEW>
void launch_rows(const Args &a, const Penalties &h, hipStream_t s) {
  const int lanes = row_lanes(a.b);
  const dim3 grid((unsigned)ceil_div(a.n, kThreads / lanes));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, h); };
  switch (lanes) {
    case 2: go(row_kernel<T, 2, FEW>); break;
    case 4: go(row_kernel<T, 4, FEW>); break;
    case 8: go(row_kernel<T, 8, FEW>); break;
    case 16: go(row_kernel<T, 16, FEW>); break;
    case 32: go(row_kernel<T, 32, FEW>); break;
    default: go(row_kernel<T, 64, FEW>); break;
  }
}
template <class T>
void launch_rows(const Args &a, bool history, const kbc_limits *l, hipStream_t s) {
  const Penalties h = penalties_for(a.b, l);
  if (history && few_ids(a, l) && a.b <= 4 * kWave) return launch_rows<T, true>(a, h, s);
  launch_rows<T, false>(a, h, s);
  if (history) launch_history<T, true>(a, h, s);
}

}  // namespace

extern "C" {

kbc_status kbc_constrain(int64_t n, int32_t b, const void *z, kbc_type type, const kbc_limits *l,
                         float fill, float *out, void *stream) {
  if (bad_limits(n, b, type, l) || !z || !out) return KBC_EINVAL;
  if (counts_ids(l) && (l->offsets ? l->entries : l->entries / b) > kMostCounted) return KBC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Args a = args_for(n, b, l);
  a.z = z;
  a.fill = fill;
  a.out = out;
  const bool penalised = l->entries > 0 && (l->repeat || l->presence || l->frequency ||
                                            l->repeat_all != 1.0f || l->presence_all != 0.0f ||
                                            l->frequency_all != 0.0f);
  with_type(type, [&](auto t) {
    using T = decltype(t);
    launch_dense<T, false>(a, penalised, l, s);
  });
  return launched();
}

kbc_status kbc_constrain_backward(int64_t n, int32_t b, const void *z, kbc_type type,
                                  const kbc_limits *l, const float *dout, void *dz, float *dbias,
                                  void *stream) {
  if (bad_limits(n, b, type, l) || !dout || !dz) return KBC_EINVAL;
  const bool scaled = l->entries > 0 && (l->repeat || l->repeat_all != 1.0f);
  if (scaled && !z) return KBC_EINVAL;
  const bool shared = dbias && !l->bias_each;
  if (shared && ceil_div(n, kThreads / row_lanes(b)) > kMostBlocks) return KBC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Args a = args_for(n, b, l);
  a.z = z;
  a.dout = dout;
  a.out = dz;
  a.dbias = dbias;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    if (shared)
      launch_rows<T>(a, scaled, l, s);
    else
      launch_dense<T, true>(a, scaled, l, s);
  });
  return launched();
}

}  // extern "C"
