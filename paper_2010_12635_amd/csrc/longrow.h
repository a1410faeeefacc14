// Rows of class scores too long for a lane group: a workgroup of NT threads
// takes a row and reads it once from memory and then, a few passes more, from
// its die's L2 (one row a compute unit: 32 rows share 4 MiB).  Against keeping
// the row in registers (8 vectors a thread, unrolled passes that spill): top 64
// of 2048 rows of 50001 bf16 classes, of 1024 threads, 122 us when that was tried
// (72 now) and 221.
#pragma once

#include "sorted.h"

namespace gcn {

// Thread t has the vectors t, t + NT, ..., or, with RANGES, wave w the `span`
// groups of 64 consecutive vectors from w span on (a lane a vector of each), so
// that the waves' classes are in the waves' order.
template <typename T, int NT_, bool RANGES = false>
struct LongRow {
  typedef T Elem;
  static constexpr int VE = Vec<T>::N;
  static constexpr int NT = NT_;
  const T* __restrict__ z;
  int C, span;

  __device__ __forceinline__ LongRow(const T* row, int classes)
      : z(row), C(classes), span((classes + NT * VE - 1) / (NT * VE)) {}
  __device__ __forceinline__ int first_class(int v) const {
    if constexpr (RANGES) return (((int)(threadIdx.x >> 6) * span + v) * 64 + (int)(threadIdx.x & 63)) * VE;
    else return (v * NT + (int)threadIdx.x) * VE;
  }
  // f(scores of a vector, its first class) for the vectors of the thread, four
  // loads in flight (eight: 73 us instead of 72 for the case above, 48 instead of
  // 35 for rows of 4001 fp32 classes).  Every lane takes part in each call; past the row's end it
  // gets scores of -inf.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int v = 0; v < span; v += 4) {
      uint4 raw[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) raw[q] = load_row(z, v + q < span ? first_class(v + q) : C, C, -INFINITY);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (v + q >= span) break;
        float x[VE];
        unpack<T>(raw[q], x);
        f(x, first_class(v + q));
      }
    }
  }
};

// Sum into shared memory: whole numbers, whose sums know no order.
__device__ __forceinline__ void lds_add(uint64_t* at, uint64_t v) {
  __hip_atomic_fetch_add(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// A score's item with 64 bits, whatever its type.
__device__ __forceinline__ Item64 score_item(float v, int c) { return item64(score_key(v), (uint32_t)c); }

// Lists at least the first K items of the row's order (all of them if there
// are fewer), K <= 256:
//   1. Every thread finds the largest of its scores.
//   2. In each wave the r-th largest of these, r = ceil(K / waves), is a score
//      that r classes of the wave reach; the smallest over the waves, b, is one
//      that at least K classes of the row reach.  (Only waves whose lanes all
//      hold scores are asked.)
//   3. The classes that reach b are listed in shared memory: for scores in no
//      particular order a few times K.  Where they are too many (rows sorted by
//      class, many equal scores), b is raised by bisection between what K
//      items reach and what fewer do, until the list holds them.
constexpr int TOP_LIST = 1024;

template <int NT>
struct TopList {
  float b[NT / 64];
  int n[NT / 64];
  int count;
  double item[TOP_LIST];
};

// Returns the number of items listed; mx: this thread's largest score; bad:
// whether it saw NaN or +inf.
template <typename Row, int NT = Row::NT>
__device__ __forceinline__ int list_top(const Row r, int K, TopList<NT>& sh, float& mx, bool& bad) {
  constexpr int VE = Row::VE;
  constexpr int NW = NT / 64;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if (t == 0) sh.count = 0;
  bad = false;
  mx = -INFINITY;
  r.each([&](const float (&v)[VE], int) {
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      bad |= !(v[i] < INFINITY);
      mx = fmaxf(mx, v[i]);                              // NaN is passed over
    }
  });
  const int full = r.C / (64 * VE) < NW ? r.C / (64 * VE) : NW;   // at least 1: shorter rows have a lane group
  const int rounds = (K + full - 1) / full;
  float left = mx, b = -INFINITY;
  if (rounds <= 64) {
    for (int i = 0; i < rounds; ++i) {
      b = group_max<64>(left);
      const uint64_t who = __ballot(left == b);
      if (lane == __ffsll((unsigned long long)who) - 1) left = -INFINITY;
    }
  }
  if (lane == 0) sh.b[wave] = b;
  __syncthreads();
  b = sh.b[0];
  for (int i = 1; i < full; ++i) b = fminf(b, sh.b[i]);
  auto list = [&](double from) {
    r.each([&](const float (&v)[VE], int c0) {
      float most = v[0];
#pragma unroll
      for (int i = 1; i < VE; ++i) most = fmaxf(most, v[i]);
      if (!(most >= b)) return;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        if (!(v[i] >= b && v[i] > -INFINITY)) continue;
        const Item64 e = score_item(v[i], c0 + i);
        if (e.v < from) continue;
        const int at = atomicAdd(&sh.count, 1);
        if (at < TOP_LIST) sh.item[at] = e.v;
      }
    });
  };
  list(0.0);
  __syncthreads();
  int cnt = sh.count;
  if (cnt > TOP_LIST) {
    // items from lo on are K at least and, at the end, TOP_LIST at most
    uint64_t lo = b > -INFINITY ? (uint64_t)__double_as_longlong(score_item(b, 0x3fffffff).v) : 0;
    uint64_t hi = (uint64_t)__double_as_longlong(item64(0xffffffffu, 0).v);
    while (cnt > TOP_LIST) {
      const uint64_t mid = lo + (hi - lo) / 2 + 1;
      const double m = __longlong_as_double((long long)mid);
      int n = 0;
      r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (v[i] >= b && v[i] > -INFINITY) n += score_item(v[i], c0 + i).v >= m ? 1 : 0;
      });
      n = block_reduce<NW>(n, sh.n, AddF());
      if (n >= K) { lo = mid; cnt = n; }
      else hi = mid - 1;
    }
    if (t == 0) sh.count = 0;
    __syncthreads();
    list(__longlong_as_double((long long)lo));
    __syncthreads();
    cnt = sh.count;
  }
  return cnt;
}

// f(place, item) for the first K of the cnt listed items: an item's place is
// the number of items above it, counted by several threads where the list is
// short.
template <int NT, typename F>
__device__ __forceinline__ void rank_list(const TopList<NT>& sh, int cnt, int K, F f) {
  int per = 1;
  while (per < 64 && 2 * per * cnt <= NT) per *= 2;
  const int sub = threadIdx.x % per;
  for (int i = threadIdx.x / per; i < cnt; i += NT / per) {
    const double e = sh.item[i];
    int above = 0;
    for (int j = sub; j < cnt; j += per) above += sh.item[j] > e ? 1 : 0;
    for (int m = 1; m < per; m <<= 1) above += __shfl_xor(above, m);
    if (sub == 0 && above < K) f(above, e);
  }
}

}  // namespace gcn
