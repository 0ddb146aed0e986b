// embed.hip -- embedding lookup with scaling, plain and pooled, and its gradient
// by sorted tokens (kbchain.h: kbc_embed, kbc_embed_pool, kbc_embed_backward).
//
//     out[t] = scale * table[ids[t]]                                (plain)
//     out[g] = scale (/ tokens of g) * sum over t in g of table[ids[t]]   (pooled)
//     dtable[v] = sum over t with ids[t] == v of scale (/ tokens of g(t)) *
//                 dout[t or g(t)]
//
// All of it moves rows: a lane group of LPG lanes reads a row of dim values 16
// bytes a lane (a row whose width is not a multiple of that ends in a lane that
// takes its last 16 bytes again), several rows in flight.  A pooled sum over few
// tokens is one workgroup a bag.  The gradient, and pooled sums over many
// tokens, are one segmented sum: a list of (row of the output, row read), sorted
// by the first, is cut into equal chunks, one a workgroup, and those into runs, one
// a lane group, that are walked in order.  A row that lies inside its run is written
// at once, one inside its chunk after the groups have met in LDS, and one that
// crosses chunks leaves one partial sum per chunk, added in order by the next launch.
// So the work is spread evenly however often a word occurs, nothing is atomic,
// and two calls give the same bits.  Sums are taken in double (see Slot); an output is
// rounded to float and, in a 16-bit type, from there to the type.
//
// The list is sorted by the tokens' ids, stably.  Up to kRankTokens tokens, each
// token's place is counted: the number of tokens with a smaller id, or the same
// and before it, against all ids in LDS, in one launch over the whole chip.
// More take a radix sort, up to 9 bits a pass, three launches each, which also clear
// the output by shares, as they leave the memory idle.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "ids.h"
#include "kbchain.h"

namespace {

using namespace kbc;

constexpr int kWaves = kThreads / kWave;

// -- rows of a type ---------------------------------------------------------------

// Neighbouring values of a row, wherever the row begins: 16 bytes of them.
template <class T, int VEC>
using vec_any = T __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

template <class T, int VEC>
__device__ __forceinline__ void load_vals(const T *p, T (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = *p;
  } else {
    const vec_any<T, VEC> t = *reinterpret_cast<const vec_any<T, VEC> *>(p);
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = t[k];
  }
}

// x rounded to float, and from there to T.  The compiler would otherwise make one
// conversion of the two, 40 instructions long.
template <class T>
__device__ __forceinline__ T round_to(double x) {
  float f = (float)x;
  if constexpr (sizeof(T) == 2) asm("" : "+v"(f));
  return (T)f;
}

// Output rows are written once and not read again by these kernels.
template <class T, int VEC>
__device__ __forceinline__ void store_vals(T *p, const T (&v)[VEC]) {
  if constexpr (VEC == 1) {
    *p = v[0];
  } else {
    vec_any<T, VEC> t;
#pragma unroll
    for (int k = 0; k < VEC; ++k) t[k] = v[k];
    __builtin_nontemporal_store(t, reinterpret_cast<vec_any<T, VEC> *>(p));
  }
}

// -- plain lookup -------------------------------------------------------------------

struct LookupArgs {
  Ints ids;
  int64_t tokens, rows;
  int32_t dim;
  const void *table;
  int64_t stride;
  float scale;
  void *out;
};

// Rows of one lane group in flight.
constexpr int kLookupRows = 4;

template <class T, int VEC, int LPG>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a) {
  constexpr int GPB = kThreads / LPG;
  const int lane = threadIdx.x % LPG;
  const int64_t t0 = ((int64_t)blockIdx.x * GPB + threadIdx.x / LPG) * kLookupRows;
  const T *table = static_cast<const T *>(a.table);
  T *out = static_cast<T *>(a.out);
  int64_t id[kLookupRows];
#pragma unroll
  for (int k = 0; k < kLookupRows; ++k) {
    id[k] = t0 + k < a.tokens ? load_int(a.ids, t0 + k) : -1;
    if (id[k] >= a.rows) id[k] = -1;
  }
  for (int c0 = lane * VEC; c0 < a.dim; c0 += LPG * VEC) {
    const int c = min(c0, a.dim - VEC);
    T v[kLookupRows][VEC];
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k)
      if (id[k] >= 0) load_vals<T, VEC>(table + id[k] * a.stride + c, v[k]);
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
      if (t0 + k >= a.tokens) break;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[k][i] = id[k] >= 0 ? (T)((float)v[k][i] * a.scale) : (T)0.0f;
      store_vals<T, VEC>(out + (t0 + k) * a.dim + c, v[k]);
    }
  }
}

// -- pooled lookup, a workgroup per bag ---------------------------------------------

struct PoolArgs {
  Ints ids;
  Bags bags;
  int64_t rows;
  int32_t dim, mean;
  const void *table;
  int64_t stride;
  float scale;
  void *out;
};

constexpr int kPoolRows = 4;

template <class T, int VEC, int LPG>
__global__ __launch_bounds__(kThreads) void pool_kernel(PoolArgs a) {
  constexpr int GPB = kThreads / LPG;
  __shared__ double part[GPB][LPG * VEC];
  __shared__ int counts[GPB];
  const int lane = threadIdx.x % LPG, grp = threadIdx.x / LPG;
  const int64_t g = blockIdx.x;
  const int c0 = blockIdx.y * (LPG * VEC) + lane * VEC;
  const bool active = c0 < a.dim;
  const int c = active ? min(c0, a.dim - VEC) : 0;
  const int64_t begin = bag_begin(a.bags, g), end = bag_begin(a.bags, g + 1);
  const T *table = static_cast<const T *>(a.table);
  double acc[VEC];
  int count = 0;
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc[i] = 0.0;
  for (int64_t t0 = begin + grp; t0 < end; t0 += GPB * kPoolRows) {
    int64_t id[kPoolRows];
    T v[kPoolRows][VEC];
#pragma unroll
    for (int k = 0; k < kPoolRows; ++k) {
      id[k] = t0 + k * GPB < end ? load_int(a.ids, t0 + k * GPB) : -1;
      if (id[k] >= a.rows) id[k] = -1;
    }
#pragma unroll
    for (int k = 0; k < kPoolRows; ++k)
      if (id[k] >= 0) load_vals<T, VEC>(table + id[k] * a.stride + c, v[k]);
#pragma unroll
    for (int k = 0; k < kPoolRows; ++k)
      if (id[k] >= 0) {
        ++count;
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += (double)(float)v[k][i];
      }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) part[grp][lane * VEC + i] = acc[i];
  if (lane == 0) counts[grp] = count;
  __syncthreads();
  if (grp != 0 || !active) return;
  for (int k = 1; k < GPB; ++k) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] += part[k][lane * VEC + i];
    count += counts[k];
  }
  const double w = (double)a.scale / (a.mean && count > 0 ? (double)count : 1.0);
  T y[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) y[i] = round_to<T>(acc[i] * w);
  store_vals<T, VEC>(static_cast<T *>(a.out) + g * a.dim + c, y);
}

// -- the list of a segmented sum ------------------------------------------------------
//
// Entries (row of the output, row read): for the gradient (id, token or bag),
// for a pooled sum (bag, id).  An entry whose second field is -1 adds nothing, one
// whose first is the number of output rows is of no row.

// The weights of a mean's bags: few tokens' in one launch, a wave or a workgroup a bag;
// else in three, as a bag may hold any share of the tokens: counts cleared, tokens
// counted (whole numbers added in any order), weights made of them.
enum Weigh { kNone, kAtOnce, kClearCounts, kCountTokens, kWeighBags };

struct ListArgs {
  Ints ids;
  Bags bags;
  int64_t tokens, rows;
  int32_t mean;
  int32_t weigh;    // with mean: which step of the bags' weights the launch takes
  int32_t count_per;  // tokens that a thread counts
  int32_t *counts;  // tokens of each bag
  double *weights;  // 1 / those (0: none)
  void *fill;       // output rows to clear
  int64_t fill_bytes;
  int2 *entries;
  // workgroups of a launch: list_wgs make the list, then weight_wgs, then those of a
  // share of the fill, from its piece first_fill on
  uint32_t list_wgs, weight_wgs, first_fill;
};

// Token t's key in the gradient's list: its id, or `rows` where it names none.
__device__ __forceinline__ int key_of(const ListArgs &a, int64_t t) {
  const int64_t id = load_int(a.ids, t);
  return id < 0 || id >= a.rows ? (int)a.rows : (int)id;
}
__device__ __forceinline__ int2 grad_entry(const ListArgs &a, int key, int64_t t) {
  const int64_t src = a.bags.n ? bag_of(a.bags, t) : t;
  return make_int2(key, (int)src);
}

// 1 / tokens of four bags, a wave each; a long one by the whole workgroup.
constexpr int64_t kLongBag = 4096;
constexpr int kCountLoads = 8;  // in flight
__device__ __forceinline__ int count_ids(const ListArgs &a, int64_t begin, int64_t end, int lane,
                                         int lanes) {
  int n = 0;
  for (int64_t t = begin + lane; t < end; t += lanes * kCountLoads) {
    int64_t id[kCountLoads];
#pragma unroll
    for (int u = 0; u < kCountLoads; ++u) id[u] = load_int(a.ids, min(t + u * lanes, end - 1));
#pragma unroll
    for (int u = 0; u < kCountLoads; ++u)
      n += t + u * lanes < end && id[u] >= 0 && id[u] < a.rows;
  }
  for (int m = 1; m < kWave; m <<= 1) n += __shfl_xor(n, m);
  return n;
}
__device__ void bag_weights(const ListArgs &a, int64_t block) {
  __shared__ int counts[kWaves];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  for (int k = 0; k < kWaves; ++k) {
    const int64_t g = block * kWaves + k;
    if (g >= a.bags.n) break;
    const int64_t begin = bag_begin(a.bags, g), end = bag_begin(a.bags, g + 1);
    if (end - begin < kLongBag) {  // the same for the whole workgroup
      if (k != wave) continue;
      const int n = count_ids(a, begin, end, lane, kWave);
      if (lane == 0) a.weights[g] = n > 0 ? 1.0 / (double)n : 0.0;
    } else {
      const int n = count_ids(a, begin, end, threadIdx.x, kThreads);
      __syncthreads();
      if (lane == 0) counts[wave] = n;
      __syncthreads();
      if (threadIdx.x == 0) {
        int all = 0;
        for (int w = 0; w < kWaves; ++w) all += counts[w];
        a.weights[g] = all > 0 ? 1.0 / (double)all : 0.0;
      }
    }
  }
}

// Counts the tokens of a block of kThreads * count_per for their bags: one bag's, as in
// a long bag, with one addition, others with one for each bag and wave.  (Additions
// to one count take 12 ns each, one a wave 49 us for a bag of 262144.)
__device__ void count_tokens(const ListArgs &a, int64_t block) {
  __shared__ int counts[kWaves];
  const int64_t first = block * kThreads * a.count_per;
  const int64_t end = min(a.tokens, first + (int64_t)kThreads * a.count_per);
  const int64_t g = bag_of(a.bags, first);  // the same for the whole workgroup, as what follows
  if (g >= 0 && bag_begin(a.bags, g + 1) >= end) {
    const int n = count_ids(a, first, end, threadIdx.x, kThreads);
    if (threadIdx.x % kWave == 0) counts[threadIdx.x / kWave] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      int all = 0;
      for (int w = 0; w < kWaves; ++w) all += counts[w];
      if (all) atomicAdd(&a.counts[g], all);
    }
    return;
  }
  const int lane = threadIdx.x % kWave;
  for (int64_t t0 = first + threadIdx.x - lane; t0 < end; t0 += kThreads) {  // a wave's tokens
    const int64_t t = min(t0 + lane, end - 1), id = load_int(a.ids, t);
    const bool valid = t0 + lane < end && id >= 0 && id < a.rows;
    const int own = (int)bag_of(a.bags, t);  // (bags are below 2^31)
    // A bag's tokens are neighbours: the first lane of them adds all.
    const int before = __shfl_up(own, 1);
    const bool begins = lane == 0 || own != before;
    const unsigned long long behind = __ballot(begins) >> lane >> 1;
    const int n = behind ? 1 + __builtin_ctzll(behind) : kWave - lane;
    const unsigned long long mine = __ballot(valid) >> lane & (n < kWave ? (1ull << n) - 1 : ~0ull);
    if (begins && own >= 0 && mine) atomicAdd(&a.counts[own], __popcll(mine));
  }
}
__device__ __forceinline__ void weigh(const ListArgs &a, int64_t block) {
  if (a.weigh == kAtOnce) return bag_weights(a, block);
  if (a.weigh == kCountTokens) return count_tokens(a, block);
  const int64_t g = block * kThreads + threadIdx.x;
  if (g >= a.bags.n) return;
  if (a.weigh == kClearCounts)
    a.counts[g] = 0;
  else
    a.weights[g] = a.counts[g] > 0 ? 1.0 / (double)a.counts[g] : 0.0;
}

// 64 KB of zeros from each workgroup.
typedef unsigned int fill_vec __attribute__((ext_vector_type(4), aligned(2)));
constexpr int64_t kFillBytes = 16 * kThreads * 16;
__device__ __forceinline__ void clear(const ListArgs &a, int64_t block) {
  char *p = static_cast<char *>(a.fill);
  const int64_t end = min(a.fill_bytes, (block + 1) * kFillBytes);
  for (int64_t i = block * kFillBytes + (int64_t)threadIdx.x * 16; i < end; i += kThreads * 16) {
    if (i + 16 <= end) {
      const fill_vec zero = {0, 0, 0, 0};
      __builtin_nontemporal_store(zero, reinterpret_cast<fill_vec *>(p + i));
    } else {
      for (int64_t j = i; j < end; j += 2) *reinterpret_cast<uint16_t *>(p + j) = 0;
    }
  }
}

// What the workgroups past list_wgs of a launch do.
__device__ __forceinline__ bool other_work(const ListArgs &a) {
  if (blockIdx.x < a.list_wgs) return false;
  const uint32_t k = blockIdx.x - a.list_wgs;
  if (k < a.weight_wgs)
    weigh(a, k);
  else
    clear(a, (int64_t)a.first_fill + (k - a.weight_wgs));
  return true;
}

__global__ __launch_bounds__(kThreads) void prepare_kernel(ListArgs a) { (void)other_work(a); }

// A pooled sum's list, which is in order as it is.
__global__ __launch_bounds__(kThreads) void pool_list_kernel(ListArgs a) {
  if (other_work(a)) return;
  const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (t >= a.tokens) return;
  const int64_t g = bag_of(a.bags, t), id = load_int(a.ids, t);
  // A token before the first bag or behind the last one is of no row: bags.n.
  a.entries[t] = make_int2(g < 0 ? (int)a.bags.n : (int)g,
                           id < 0 || id >= a.rows ? -1 : (int)id);
}

// -- the gradient's list, few tokens: places counted ----------------------------------

// (16389 tokens: gradient 111 us counted, 94 sorted.)
constexpr int64_t kRankTokens = 8192;
constexpr int kRankLanes = 8;                          // lanes that share a token's count
constexpr int kRankDepth = 4;                          // quads of keys in flight
constexpr int kRankLoads = 8;                          // ids in flight on their way to LDS
constexpr int kRankPer = kThreads / kRankLanes;        // tokens of a workgroup

__global__ __launch_bounds__(kThreads) void rank_kernel(ListArgs a) {
  if (other_work(a)) return;
  extern __shared__ int4 rank_lds[];
  int *keys = reinterpret_cast<int *>(rank_lds);
  const int n = (int)a.tokens, quads = (n + 3) / 4;
  for (int t0 = threadIdx.x; t0 < quads * 4; t0 += kThreads * kRankLoads) {
    int k[kRankLoads];
#pragma unroll
    for (int u = 0; u < kRankLoads; ++u) k[u] = key_of(a, min(t0 + u * kThreads, n - 1));
#pragma unroll
    for (int u = 0; u < kRankLoads; ++u) {
      const int t = t0 + u * kThreads;
      if (t < quads * 4) keys[t] = t < n ? k[u] : INT32_MAX;
    }
  }
  const int lane = threadIdx.x % kRankLanes;
  const int t = blockIdx.x * kRankPer + threadIdx.x / kRankLanes;
  // Searched for while the keys are on their way.
  const int src = a.bags.n ? (int)bag_of_lanes<kRankLanes>(a.bags, min(t, n - 1), lane) : t;
  __syncthreads();
  const int key = keys[min(t, n - 1)];
  // Four keys at a time, kRankDepth times: all up to the token's own four count that
  // are not larger, all behind that are smaller; those four one by one.
  int place = 0;
  const int own = t / 4;
  auto count = [&](int from, int to, int bar) {
    int q = from + lane;
    for (; q + (kRankDepth - 1) * kRankLanes < to; q += kRankDepth * kRankLanes) {
      int4 k[kRankDepth];
#pragma unroll
      for (int u = 0; u < kRankDepth; ++u) k[u] = rank_lds[q + u * kRankLanes];
#pragma unroll
      for (int u = 0; u < kRankDepth; ++u)
        place += (k[u].x <= bar) + (k[u].y <= bar) + (k[u].z <= bar) + (k[u].w <= bar);
    }
    for (; q < to; q += kRankLanes) {
      const int4 k = rank_lds[q];
      place += (k.x <= bar) + (k.y <= bar) + (k.z <= bar) + (k.w <= bar);
    }
  };
  count(0, min(own, quads), key);
  count(own, quads, key - 1);  // (keys are not negative)
  if (lane == own % kRankLanes)
    for (int j = own * 4; j < t && j < n; ++j) place += keys[j] == key;
#pragma unroll
  for (int m = 1; m < kRankLanes; m <<= 1) place += __shfl_xor(place, m);
  if (lane == 0 && t < n) a.entries[place] = make_int2(key, src);
}

// -- the gradient's list, many tokens: radix sort -------------------------------------

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
// Entries of a thread: 2, which keeps a workgroup's steps few (262144 tokens on 512
// workgroups 142 us for the whole gradient, with 8 on 128 154; 16389 tokens 82
// against 95); 8 for long lists, whose counts would be many.
constexpr int64_t kLongList = 1 << 20;
template <int ITEMS>
constexpr int kTile = kThreads * ITEMS;
int64_t tiles_of(int64_t tokens) {
  const int64_t tile = tokens < kLongList ? kTile<2> : kTile<8>;
  return (tokens + tile - 1) / tile;
}

struct RadixArgs {
  ListArgs list;
  const int2 *in;    // null: the tokens themselves
  int2 *out;
  int32_t shift, bits;
  uint32_t tiles;
  uint32_t *counts;  // [digit][tile]; after the scan, entries of the digit in the tiles before
  uint32_t *totals;  // [digit]
};

__device__ __forceinline__ int radix_key(const RadixArgs &a, int64_t i) {
  return a.in ? a.in[i].x : key_of(a.list, i);
}

template <int ITEMS>
__global__ __launch_bounds__(kThreads) void radix_count_kernel(RadixArgs a) {
  if (other_work(a.list)) return;
  __shared__ uint32_t count[kDigits];
  const int digits = 1 << a.bits;
  for (int i = threadIdx.x; i < digits; i += kThreads) count[i] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kTile<ITEMS>;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int64_t i = base + k * kThreads + threadIdx.x;
    if (i < a.list.tokens) atomicAdd(&count[(radix_key(a, i) >> a.shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += kThreads)
    a.counts[(int64_t)i * a.tiles + blockIdx.x] = count[i];
}

// The sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ uint32_t scan_threads(uint32_t v, uint32_t *lds, uint32_t *all) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t x = v;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const uint32_t y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  __syncthreads();  // earlier readers of lds are done
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += lds[w];
    sum += lds[w];
  }
  *all = sum;
  return before + x - v;
}

// One workgroup per digit: its counts become the entries in the tiles before.
__global__ __launch_bounds__(kThreads) void radix_scan_kernel(RadixArgs a) {
  if (other_work(a.list)) return;
  __shared__ uint32_t lds[kWaves];
  uint32_t *c = a.counts + (int64_t)blockIdx.x * a.tiles;
  uint32_t sum = 0;
  for (uint32_t i0 = 0; i0 < a.tiles; i0 += kThreads) {
    const uint32_t i = i0 + threadIdx.x;
    const uint32_t v = i < a.tiles ? c[i] : 0;
    uint32_t all;
    const uint32_t before = scan_threads(v, lds, &all);
    if (i < a.tiles) c[i] = sum + before;
    sum += all;
  }
  if (threadIdx.x == 0) a.totals[blockIdx.x] = sum;
}

// Each wave places 64 ITEMS consecutive entries, 64 at a time in order: lanes of one
// digit find each other by ballots, and the wave's own counter of the digit
// gives the place of the first of them.
template <int ITEMS>
__global__ __launch_bounds__(kThreads) void radix_place_kernel(RadixArgs a) {
  if (other_work(a.list)) return;
  // Lanes of a wave read what others of it wrote: volatile keeps every access.
  __shared__ volatile uint32_t count[kWaves][kDigits];
  __shared__ uint32_t base[kDigits];
  __shared__ uint32_t lds[kWaves];
  const int digits = 1 << a.bits;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t first = (int64_t)blockIdx.x * kTile<ITEMS> + wave * (ITEMS * kWave);
  int2 e[ITEMS];
  int digit[ITEMS];
  uint32_t place[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int64_t i = first + k * kWave + lane;
    digit[k] = -1;
    if (i < a.list.tokens) {
      e[k] = a.in ? a.in[i] : grad_entry(a.list, key_of(a.list, i), i);
      digit[k] = (e[k].x >> a.shift) & (digits - 1);
    }
  }
  for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) count[i / kDigits][i % kDigits] = 0;
  {  // where each digit's entries begin
    constexpr int kPer = kDigits / kThreads;
    uint32_t v[kPer], before[kPer], sum = 0, all;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = threadIdx.x * kPer + k;
      v[k] = i < digits ? a.totals[i] : 0;
      before[k] = i < digits ? a.counts[(int64_t)i * a.tiles + blockIdx.x] : 0;
      sum += v[k];
    }
    uint32_t at = scan_threads(sum, lds, &all);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = threadIdx.x * kPer + k;
      base[i] = at + before[k];
      at += v[k];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const bool valid = digit[k] >= 0;
    unsigned long long same = __ballot(valid);
    for (int bit = 0; bit < a.bits; ++bit) {
      const bool set = valid && (digit[k] >> bit & 1);
      const unsigned long long m = __ballot(set);
      same &= set ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    const uint32_t before = valid ? count[wave][digit[k]] : 0;
    place[k] = before + rank;
    __builtin_amdgcn_wave_barrier();
    if (valid && rank == 0) count[wave][digit[k]] = before + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITEMS; ++k)
    if (digit[k] >= 0) {
      uint32_t at = base[digit[k]] + place[k];
      for (int w = 0; w < wave; ++w) at += count[w][digit[k]];
      a.out[at] = e[k];
    }
}

// -- the segmented sum ------------------------------------------------------------------

struct SumArgs {
  const int2 *entries;
  int64_t n;
  int32_t run;    // entries of a lane group
  int32_t chunk;  // of a workgroup
  const void *src;
  int64_t src_stride;
  int32_t dim;
  const double *src_weights;  // of the rows read, or null
  const int32_t *out_counts;  // terms of the rows written, whose mean it is, or null
  double scale;
  void *out;
  int64_t out_rows;
  void *slots;  // Slot<type> [chunk][2][dim]: the sum of the chunk's first row, if it began
                // before the chunk, and of its last one, if it began in it and goes on
};
// Partial sums of a row: double, and float where the row is rounded to float16 in the
// end, 2^-24 of them against its 2^-12 (half the bytes, a tenth of all that the sum over
// 262144 tokens of 512 values moves).  Sums of 2^30 float16 values are far from a float's
// end, but those of a few bfloat16 values may pass it, where the scale or the mean, or
// other terms, bring the row back.
template <class T>
using Slot = std::conditional_t<std::is_same_v<T, _Float16>, float, double>;

constexpr int kSumRows = 8;  // of a lane group in flight

template <class T, int VEC>
__device__ __forceinline__ void write_row(const SumArgs &a, int key, int c,
                                          const double (&acc)[VEC]) {
  if (key < 0 || key >= a.out_rows) return;
  // (A row of no terms is zero.)
  const double w = a.out_counts ? a.scale / (double)max(a.out_counts[key], 1) : a.scale;
  T y[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) y[i] = round_to<T>(acc[i] * w);
  store_vals<T, VEC>(static_cast<T *>(a.out) + (int64_t)key * a.dim + c, y);
}

template <class T, int VEC, int LPG>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a) {
  constexpr int GPB = kThreads / LPG;
  // Of each lane group: the sum of its first row, if that began before its entries,
  // and whether it goes on behind them.
  __shared__ Slot<T> head[GPB][LPG * VEC];
  __shared__ int goes_on[GPB];
  const int lane = threadIdx.x % LPG, grp = threadIdx.x / LPG;
  const int c0 = blockIdx.y * (LPG * VEC) + lane * VEC;
  const int64_t p0 = (int64_t)blockIdx.x * a.chunk + (int64_t)grp * a.run;
  const int64_t p1 = min(a.n, p0 + a.run);
  const bool active = c0 < a.dim;
  const int c = active ? min(c0, a.dim - VEC) : 0;
  const T *src = static_cast<const T *>(a.src);
  double acc[VEC];
  int key = -1;
  bool late = false;  // the group's first row began before its entries
  bool open = false;  // its last row began in them and goes on: acc is its sum so far
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < VEC; ++i) head[grp][lane * VEC + i] = (Slot<T>)acc[i];
  };
  if (active && p0 < a.n) {
    key = a.entries[p0].x;
    late = p0 > 0 && a.entries[p0 - 1].x == key;
    bool began = !late;  // the current row began in these entries
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0;
    int2 next[kSumRows];  // the entries of the next rows are read while these arrive
#pragma unroll
    for (int k = 0; k < kSumRows; ++k) next[k] = a.entries[min(p0 + k, p1 - 1)];
    for (int64_t p = p0; p < p1; p += kSumRows) {
      int2 e[kSumRows];
      T v[kSumRows][VEC];
      double w[kSumRows];
#pragma unroll
      for (int k = 0; k < kSumRows; ++k) e[k] = next[k];
#pragma unroll
      for (int k = 0; k < kSumRows; ++k) {
        const int r = max(e[k].y, 0);
        load_vals<T, VEC>(src + (int64_t)r * a.src_stride + c, v[k]);
        w[k] = a.src_weights ? a.src_weights[r] : 1.0;
      }
#pragma unroll
      for (int k = 0; k < kSumRows; ++k) next[k] = a.entries[min(p + kSumRows + k, p1 - 1)];
#pragma unroll
      for (int k = 0; k < kSumRows; ++k) {
        if (p + k >= p1) break;
        if (e[k].x != key) {
          if (began)
            write_row<T, VEC>(a, key, c, acc);
          else
            put();
          began = true;
          key = e[k].x;
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[i] = 0.0;
        }
        if (e[k].y >= 0) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[i] += (double)(float)v[k][i] * w[k];
        }
      }
    }
    const bool more = p1 < a.n && a.entries[p1].x == key;
    if (!began)
      put();
    else if (more)
      open = true;
    else
      write_row<T, VEC>(a, key, c, acc);
    if (late) goes_on[grp] = !began && more;
  }
  __syncthreads();
  // Rows that go on in the workgroup's next groups: the group where one began adds
  // theirs in order; what crosses the workgroup's ends goes to its slots.
  auto add_heads = [&](int k) {  // of groups k on; whether the row goes on behind all
    for (; k < GPB; ++k) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) acc[i] += (double)head[k][lane * VEC + i];
      if (!goes_on[k]) return false;
    }
    return true;
  };
  auto slot = [&](int which) {
    Slot<T> *s = static_cast<Slot<T> *>(a.slots) + ((int64_t)blockIdx.x * 2 + which) * a.dim + c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[i] = (Slot<T>)acc[i];
  };
  if (open) {
    if (add_heads(grp + 1))
      slot(1);
    else
      write_row<T, VEC>(a, key, c, acc);
  }
  if (grp == 0 && late) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0;
    (void)add_heads(0);
    slot(0);
  }
}

// Rows that cross chunks: the wave of the chunk where the row began adds its partial
// sums in the chunks' order, VEC columns a lane; those of a row of more than
// kJoinAlone chunks are shared by the workgroup's waves, every kWaves-th each, and
// the waves' sums are added in order.
constexpr int kJoinAlone = 24;
constexpr int kJoinDepth = 8;  // partial sums in flight

// The sum of chunks k0, k0 + step, .. last of the row that began in chunk q.
template <class S, int VEC>
__device__ __forceinline__ void add_slots(const SumArgs &a, int c, int64_t q, int64_t k0,
                                          int64_t last, int step, double (&acc)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc[i] = 0.0;
  for (int64_t k = k0; k <= last; k += step * kJoinDepth) {
    S v[kJoinDepth][VEC];
#pragma unroll
    for (int u = 0; u < kJoinDepth; ++u) {
      const int64_t m = min(k + u * step, last);
      load_vals<S, VEC>(static_cast<const S *>(a.slots) + (m * 2 + (m == q ? 1 : 0)) * a.dim + c, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kJoinDepth; ++u)
      if (k + u * step <= last) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += (double)v[u][i];
      }
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(kThreads) void join_kernel(SumArgs a, int64_t chunks) {
  __shared__ double part[kWaves][kWave * VEC];
  __shared__ int64_t first[kWaves], end[kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c0 = blockIdx.y * (kWave * VEC) + lane * VEC;
  const bool active = c0 < a.dim;
  const int c = active ? min(c0, a.dim - VEC) : 0;
  const int64_t q = (int64_t)blockIdx.x * kWaves + wave;
  const int64_t p0 = q * a.chunk, p1 = p0 + a.chunk;
  bool mine = q < chunks && p1 < a.n;  // uniform in the wave, as all that follows from it
  int key = 0;
  if (mine) {
    key = a.entries[p1].x;
    const int before = p0 > 0 ? a.entries[p0 - 1].x : -1;
    mine = a.entries[p1 - 1].x == key && key < a.out_rows && before != key;
  }
  int64_t last = q;  // chunks q + 1 .. last begin in the row
  while (mine) {
    const int64_t at = (last + 1 + lane) * a.chunk;
    const unsigned long long in = __ballot(at < a.n && a.entries[min(at, a.n - 1)].x == key);
    if (in != ~0ull) {
      last += __builtin_ctzll(~in);
      break;
    }
    last += kWave;
  }
  double acc[VEC];
  const bool alone = mine && last - q < kJoinAlone;
  if (alone && active) {
    add_slots<Slot<T>, VEC>(a, c, q, q, last, 1, acc);
    write_row<T, VEC>(a, key, c, acc);
  }
  if (lane == 0) {
    first[wave] = mine && !alone ? q : -1;
    end[wave] = last;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    const int64_t q0 = first[w];  // the same for the whole workgroup
    if (q0 < 0) continue;
    add_slots<Slot<T>, VEC>(a, c, q0, q0 + wave, end[w], kWaves, acc);
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[wave][lane * VEC + i] = acc[i];
    __syncthreads();
    if (wave == w && active) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        acc[i] = part[0][lane * VEC + i];
        for (int k = 1; k < kWaves; ++k) acc[i] += part[k][lane * VEC + i];
      }
      write_row<T, VEC>(a, key, c, acc);
    }
    __syncthreads();
  }
}

// -- how a call is launched ----------------------------------------------------------------

int lanes_for(int32_t dim, int vec) {
  const int lanes = (dim + vec - 1) / vec;
  int lpg = 1;
  while (lpg < lanes && lpg < kWave) lpg <<= 1;
  return lpg;
}

// f(T{}, vec, lanes) for the type and width of a call's rows, as constants.
template <class T, class F>
void with_lanes(int32_t dim, F f) {
  constexpr int V = kVec<T>;
  const bool wide = dim >= V;
  const int lpg = lanes_for(dim, wide ? V : 1);
  auto go = [&](auto lanes) {
    if (wide)
      f(T{}, std::integral_constant<int, V>{}, lanes);
    else
      f(T{}, std::integral_constant<int, 1>{}, lanes);
  };
  switch (lpg) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    case 8: go(std::integral_constant<int, 8>{}); break;
    case 16: go(std::integral_constant<int, 16>{}); break;
    case 32: go(std::integral_constant<int, 32>{}); break;
    default: go(std::integral_constant<int, 64>{}); break;
  }
}
template <class F>
void with_rows(kbc_type type, int32_t dim, F f) {
  switch (type) {
    case KBC_F32: with_lanes<float>(dim, f); break;
    case KBC_BF16: with_lanes<__bf16>(dim, f); break;
    case KBC_F16: with_lanes<_Float16>(dim, f); break;
  }
}

// Entries of a lane group: about 2048 waves' worth of groups over the list, at least
// kSumRows entries each.  More waves leave more partial sums, fewer leave CUs idle.
// The gradient, with 1024 / 2048 / 4096 / 8192 waves, us:
//   bfloat16  16,389 tokens of 1001 values   70 / 66 / 66 / 67
//   float16   262,144 of 512                102 / 102 / 103 / 111
//   float32   262,144 of 128, of 512         68 / 62 / 62 / 66, 141 / 141 / 147 / 154
//   float32   30,000 of 300                  42 / 41 / 45 / 45
//   float32   a million of 3                 76 / 76 / 79 / 82
// and 100,000 of 8 or 64, 30,000 of 64 the same with all.
int32_t run_for(int64_t tokens, int lpg) {
  int32_t run = kSumRows;
  while (run < 128 && tokens * lpg > (int64_t)run * 2048 * kWave) run *= 2;
  return run;
}
int32_t chunk_for(int64_t tokens, int lpg) { return run_for(tokens, lpg) * (kThreads / lpg); }

// Where a call's scratch holds what.
size_t padded(int64_t bytes) { return (size_t)ceil_div(bytes, 256) * 256; }
struct Scratch {
  size_t entries, sorted, counts, totals, bag_counts, weights, slots, bytes;
};
Scratch scratch_for(int64_t tokens, int64_t bags, int32_t dim, bool sorted, bool mean, int lpg) {
  Scratch s = {};
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += padded(bytes);
    return here;
  };
  s.entries = take(tokens * 8);
  if (sorted && tokens > kRankTokens) {
    s.sorted = take(tokens * 8);
    s.counts = take(kDigits * tiles_of(tokens) * 4);
    s.totals = take(kDigits * 4);
  }
  if (mean) {
    s.bag_counts = take(bags * 4);
    s.weights = take(bags * 8);
  }
  const int64_t chunks = ceil_div(tokens, chunk_for(tokens, lpg));
  if (chunks > 1) s.slots = take(chunks * 2 * dim * 8);  // (half of it with float16)
  s.bytes = at;
  return s;
}
int group_lanes(kbc_type type, int32_t dim) {
  const int v = type == KBC_F32 ? 4 : 8;
  return lanes_for(dim, dim >= v ? v : 1);
}

// A pooled sum takes a workgroup per bag where no bag can be long: bags of one, small
// length (512 of 32 rows of 512 bfloat16 values 6 us, as a segmented mean 17; 2048 of
// 128 rows of 256 22 and 41; 128 of 512 rows of 128 floats 19 and 20; 512 of 512 rows of
// 512 bfloat16 68 and 55), or few tokens in all (one bag of 256 / 1024 / 4096 rows of
// 128 floats 8 / 24 / 87 us, as a segmented mean 10 / 13 / 15; 128 bags of 11 5 and 12).
bool pools_directly(int64_t tokens, int64_t bags, bool ragged) {
  if (bags > kMostBlocks) return false;
  const int64_t mean = tokens / bags;
  return ragged ? tokens <= 512 || (tokens <= 4096 && mean <= 64) : mean <= 512;
}

void launch_sum(kbc_type type, const SumArgs &a, hipStream_t s) {
  const int64_t chunks = ceil_div(a.n, a.chunk);
  with_rows(type, a.dim, [&](auto t, auto vec, auto lanes) {
    using T = decltype(t);
    constexpr int V = decltype(vec)::value, L = decltype(lanes)::value;
    const dim3 grid((unsigned)chunks, (unsigned)ceil_div(a.dim, L * V));
    hipLaunchKernelGGL((sum_kernel<T, V, L>), grid, dim3(kThreads), 0, s, a);
  });
  if (chunks <= 1) return;
  auto join = [&](auto t) {
    using T = decltype(t);
    const unsigned wgs = (unsigned)ceil_div(chunks, kWaves);
    if (a.dim >= 2)
      hipLaunchKernelGGL((join_kernel<T, 2>), dim3(wgs, (unsigned)ceil_div(a.dim, kWave * 2)),
                         dim3(kThreads), 0, s, a, chunks);
    else
      hipLaunchKernelGGL((join_kernel<T, 1>), dim3(wgs), dim3(kThreads), 0, s, a, chunks);
  };
  switch (type) {
    case KBC_F32: join(float{}); break;
    case KBC_BF16: join(__bf16{}); break;
    case KBC_F16: join(_Float16{}); break;
  }
}

// The grid of launch k of `launches` that make a list: with a mean each takes the
// step `weigh` of the bags' weights, and each clears a share of the output.
dim3 list_grid(ListArgs *a, int64_t list_wgs, int k, int launches, Weigh weigh) {
  const int64_t pieces = ceil_div(a->fill_bytes, kFillBytes);
  const int64_t from = pieces * k / launches, to = pieces * (k + 1) / launches;
  a->weigh = a->mean ? weigh : kNone;
  a->count_per = a->mean && a->tokens / a->bags.n >= kLongBag ? 8 : 1;
  a->list_wgs = (uint32_t)list_wgs;
  a->weight_wgs = (uint32_t)(a->weigh == kNone          ? 0
                             : a->weigh == kAtOnce      ? ceil_div(a->bags.n, kWaves)
                             : a->weigh == kCountTokens ? ceil_div(a->tokens, kThreads * a->count_per)
                                                        : ceil_div(a->bags.n, kThreads));
  a->first_fill = (uint32_t)from;
  return dim3((unsigned)(list_wgs + a->weight_wgs + to - from));
}

// Whether the workgroups that weigh bags fit a grid beside the others.
bool too_many_bags(int64_t bags, int32_t mean) {
  return mean && bags >= int64_t(1) << 25;
}
bool bad_sizes(int64_t tokens, int64_t bags, int64_t rows, int32_t dim, int32_t id_bytes) {
  return tokens < 0 || tokens > kMostTokens || bags < 0 || bags > kMostRows || rows < 1 ||
         rows > kMostRows || dim < 1 || dim > 65536 || (id_bytes != 4 && id_bytes != 8);
}
bool bad_scratch(const Scratch &need, const void *scratch, size_t bytes) {
  return need.bytes > 0 &&
         (!scratch || bytes < need.bytes || reinterpret_cast<uintptr_t>(scratch) % 16 != 0);
}

}  // namespace

extern "C" {

kbc_status kbc_embed(int64_t tokens, const void *ids, int32_t id_bytes, int64_t rows, int32_t dim,
                     const void *table, int64_t stride, kbc_type type, float scale, void *out,
                     void *stream) {
  if (bad_sizes(tokens, 0, rows, dim, id_bytes) || bad_type(type) || !table || stride < dim)
    return KBC_EINVAL;
  if (tokens == 0) return KBC_OK;
  if (!ids || !out) return KBC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_rows(type, dim, [&](auto t, auto vec, auto lanes) {
    using T = decltype(t);
    constexpr int V = decltype(vec)::value, L = decltype(lanes)::value;
    constexpr int64_t kPerBlock = kThreads / L * kLookupRows;
    // As many tokens at a time as a grid holds.
    for (int64_t from = 0; from < tokens; from += kMostBlocks * kPerBlock) {
      const int64_t n = std::min(kMostBlocks * kPerBlock, tokens - from);
      const LookupArgs a{{static_cast<const char *>(ids) + from * id_bytes, id_bytes},
                         n, rows, dim, table, stride, scale, static_cast<T *>(out) + from * dim};
      hipLaunchKernelGGL((lookup_kernel<T, V, L>), dim3((unsigned)ceil_div(n, kPerBlock)),
                         dim3(kThreads), 0, s, a);
    }
  });
  return launched();
}

size_t kbc_embed_pool_scratch_size(int64_t tokens, int64_t bags, int32_t ragged, int32_t dim,
                                   kbc_type type, int32_t mean) {
  if (bad_sizes(tokens, bags, 1, dim, 4) || bad_type(type) || bags < 1 ||
      pools_directly(tokens, bags, ragged != 0))
    return 0;
  return scratch_for(tokens, bags, dim, false, mean != 0, group_lanes(type, dim)).bytes;
}

kbc_status kbc_embed_pool(int64_t tokens, const void *ids, int32_t id_bytes, int64_t bags,
                          const void *offsets, int64_t rows, int32_t dim, const void *table,
                          int64_t stride, kbc_type type, float scale, int32_t mean, void *out,
                          void *scratch, size_t bytes, void *stream) {
  if (bad_sizes(tokens, bags, rows, dim, id_bytes) || bad_type(type) || !table || stride < dim ||
      (!offsets && bags > 0 && tokens % bags != 0))
    return KBC_EINVAL;
  if (bags == 0) return KBC_OK;
  if ((tokens > 0 && !ids) || !out) return KBC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Bags of = bags_of(bags, offsets, id_bytes, tokens);
  if (pools_directly(tokens, bags, offsets != nullptr)) {
    const PoolArgs a{{ids, id_bytes}, of, rows, dim, mean, table, stride, scale, out};
    with_rows(type, dim, [&](auto t, auto vec, auto lanes) {
      using T = decltype(t);
      constexpr int V = decltype(vec)::value, L = decltype(lanes)::value;
      const dim3 grid((unsigned)bags, (unsigned)ceil_div(dim, L * V));
      hipLaunchKernelGGL((pool_kernel<T, V, L>), grid, dim3(kThreads), 0, s, a);
    });
    return launched();
  }
  const int lpg = group_lanes(type, dim);
  const Scratch at = scratch_for(tokens, bags, dim, false, mean != 0, lpg);
  if (too_many_bags(bags, mean)) return KBC_EINVAL;
  if (bad_scratch(at, scratch, bytes)) return KBC_EINVAL;
  char *w = static_cast<char *>(scratch);
  ListArgs l{{ids, id_bytes}, of, tokens, rows, mean, kNone, 1,
             reinterpret_cast<int32_t *>(w + at.bag_counts), nullptr, out,
             bags * dim * size_of(type), reinterpret_cast<int2 *>(w + at.entries), 0, 0, 0};
  if (mean || tokens == 0) {  // counts cleared with the output, then counted beside the list
    const dim3 grid = list_grid(&l, 0, 0, 1, kClearCounts);
    hipLaunchKernelGGL(prepare_kernel, grid, dim3(kThreads), 0, s, l);
    l.fill_bytes = 0;
  }
  if (tokens == 0) return launched();
  const dim3 grid = list_grid(&l, ceil_div(tokens, kThreads), 0, 1, kCountTokens);
  hipLaunchKernelGGL(pool_list_kernel, grid, dim3(kThreads), 0, s, l);
  const SumArgs a{l.entries, tokens, run_for(tokens, lpg), chunk_for(tokens, lpg), table, stride,
                  dim, nullptr, mean ? l.counts : nullptr, scale, out, bags, w + at.slots};
  launch_sum(type, a, s);
  return launched();
}

size_t kbc_embed_backward_scratch_size(int64_t tokens, int64_t bags, int32_t dim, kbc_type type,
                                       int32_t mean) {
  if (bad_sizes(tokens, bags, 1, dim, 4) || bad_type(type)) return 0;
  return scratch_for(tokens, bags, dim, true, mean != 0 && bags > 0, group_lanes(type, dim)).bytes;
}

kbc_status kbc_embed_backward(int64_t tokens, const void *ids, int32_t id_bytes, int64_t bags,
                              const void *offsets, int64_t rows, int32_t dim, const void *dout,
                              kbc_type type, float scale, int32_t mean, void *dtable,
                              void *scratch, size_t bytes, void *stream) {
  if (bad_sizes(tokens, bags, rows, dim, id_bytes) || bad_type(type) || !dtable ||
      (!offsets && bags > 0 && tokens % bags != 0))
    return KBC_EINVAL;
  if (tokens > 0 && (!ids || !dout)) return KBC_EINVAL;
  const int lpg = group_lanes(type, dim);
  mean = mean && bags > 0;
  if (too_many_bags(bags, mean)) return KBC_EINVAL;
  const Scratch at = scratch_for(tokens, bags, dim, true, mean != 0, lpg);
  if (bad_scratch(at, scratch, bytes)) return KBC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char *w = static_cast<char *>(scratch);
  ListArgs l{{ids, id_bytes}, bags_of(bags, offsets, id_bytes, tokens), tokens, rows, mean, kNone, 1,
             reinterpret_cast<int32_t *>(w + at.bag_counts),
             reinterpret_cast<double *>(w + at.weights), dtable, rows * dim * size_of(type),
             reinterpret_cast<int2 *>(w + at.entries), 0, 0, 0};
  if (tokens <= kRankTokens) {
    const dim3 grid = list_grid(&l, ceil_div(tokens, kRankPer), 0, 1, kAtOnce);
    hipLaunchKernelGGL(rank_kernel, grid, dim3(kThreads), (size_t)ceil_div(tokens, 4) * 16, s, l);
  } else {
    int bits = 1;
    while ((rows >> bits) != 0) ++bits;  // keys are 0 .. rows
    const int passes = (int)ceil_div(bits, kDigitBits);
    RadixArgs r{l, nullptr, nullptr, 0, 0, (uint32_t)tiles_of(tokens),
                reinterpret_cast<uint32_t *>(w + at.counts),
                reinterpret_cast<uint32_t *>(w + at.totals)};
    int2 *to[2] = {l.entries, reinterpret_cast<int2 *>(w + at.sorted)};
    for (int p = 0; p < passes; ++p) {
      r.bits = (bits - r.shift + (passes - p) - 1) / (passes - p);
      r.out = to[(passes - 1 - p) % 2];  // the last pass writes the entries
      const Weigh steps[3] = {kClearCounts, kCountTokens, kWeighBags};
      auto grid = [&](int64_t wgs, int k) {
        return list_grid(&r.list, wgs, p * 3 + k, passes * 3, p == 0 ? steps[k] : kNone);
      };
      const dim3 count = grid(r.tiles, 0);
      const bool long_list = tokens >= kLongList;
      hipLaunchKernelGGL(long_list ? radix_count_kernel<8> : radix_count_kernel<2>, count,
                         dim3(kThreads), 0, s, r);
      const dim3 scan = grid(int64_t(1) << r.bits, 1);
      hipLaunchKernelGGL(radix_scan_kernel, scan, dim3(kThreads), 0, s, r);
      const dim3 place = grid(r.tiles, 2);
      hipLaunchKernelGGL(long_list ? radix_place_kernel<8> : radix_place_kernel<2>, place,
                         dim3(kThreads), 0, s, r);
      r.in = r.out;
      r.shift += r.bits;
    }
  }
  if (tokens > 0) {
    const SumArgs a{l.entries, tokens, run_for(tokens, lpg), chunk_for(tokens, lpg), dout, dim, dim,
                    mean ? l.weights : nullptr, nullptr, scale, dtable, rows, w + at.slots};
    launch_sum(type, a, s);
  }
  return launched();
}

}  // extern "C"
