// Scores of a row as sortable items, one number each: the score's key above,
// the complement of the class below, so that a larger item comes earlier in
// the row's order and no two items are equal.  16-bit scores of rows of at most
// 65536 classes fit 32 bits; others take 64 bits held as a positive double,
// whose order is that of its bits and whose maximum and minimum are one
// instruction.  Absent classes (-inf, or past the row's end) are items below
// every score's.
#pragma once

#include "common.h"
#include "lanes.h"
#include "rows.h"

namespace gcn {

struct Item32 { uint32_t v; };
struct Item64 { double v; };

__device__ __forceinline__ Item32 item_max(Item32 a, Item32 b) { return {a.v > b.v ? a.v : b.v}; }
__device__ __forceinline__ Item32 item_min(Item32 a, Item32 b) { return {a.v < b.v ? a.v : b.v}; }
// No item is NaN, so the plain instruction is meant: fmax() would quiet its
// operands first, an instruction each.
__device__ __forceinline__ Item64 item_max(Item64 a, Item64 b) {
  Item64 r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r.v) : "v"(a.v), "v"(b.v));
  return r;
}
__device__ __forceinline__ Item64 item_min(Item64 a, Item64 b) {
  Item64 r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r.v) : "v"(a.v), "v"(b.v));
  return r;
}
__device__ __forceinline__ bool item_above(Item32 a, Item32 b) { return a.v > b.v; }
__device__ __forceinline__ bool item_above(Item64 a, Item64 b) { return a.v > b.v; }
__device__ __forceinline__ Item32 item_pick(bool c, Item32 a, Item32 b) { return {c ? a.v : b.v}; }
__device__ __forceinline__ Item64 item_pick(bool c, Item64 a, Item64 b) { return {c ? a.v : b.v}; }

// The lane whose number differs in the bits of M (M < 64).
template <int M>
__device__ __forceinline__ int lane_xor(int v) {
  if constexpr (M == 1) return dpp_i<DPP_XOR1>(v);
  else if constexpr (M == 2) return dpp_i<DPP_XOR2>(v);
  else if constexpr (M == 3) return dpp_i<0x1B>(v);                 // quad_perm [3, 2, 1, 0]
  else if constexpr (M == 7) return dpp_i<DPP_HALF_MIRROR>(v);
  else if constexpr (M == 15) return dpp_i<DPP_MIRROR>(v);
  else if constexpr (M == 4) return dpp_i<0x1B>(dpp_i<DPP_HALF_MIRROR>(v));
  else if constexpr (M == 8) return dpp_i<DPP_HALF_MIRROR>(dpp_i<DPP_MIRROR>(v));
  else return __shfl_xor(v, M);
}
template <int M>
__device__ __forceinline__ Item32 lane_xor(Item32 a) { return {(uint32_t)lane_xor<M>((int)a.v)}; }
template <int M>
__device__ __forceinline__ Item64 lane_xor(Item64 a) {
  return {__hiloint2double(lane_xor<M>(__double2hiint(a.v)), lane_xor<M>(__double2loint(a.v)))};
}

// Items of 16-bit scores: keys of 16 bits, in the score's own bit patterns.
template <typename T> struct ItemOf;
template <> struct ItemOf<float> { typedef Item64 type; };
template <> struct ItemOf<f16> { typedef Item32 type; };
template <> struct ItemOf<bf16> { typedef Item32 type; };

// 64 bits: the key in bits 30 to 61, so that the number is positive and
// finite, the class's complement below it.
__device__ __forceinline__ Item64 item64(uint32_t key, uint32_t c) {
  return {__longlong_as_double((long long)(((uint64_t)key << 30) | (0x3fffffffu - c)))};
}
__device__ __forceinline__ uint32_t item_key(Item64 a) {
  return (uint32_t)((uint64_t)__double_as_longlong(a.v) >> 30);
}
__device__ __forceinline__ int32_t item_class(Item64 a) {
  return (int32_t)(0x3fffffffu - ((uint32_t)__double2loint(a.v) & 0x3fffffffu));
}
__device__ __forceinline__ int32_t item_class(Item32 a) { return (int32_t)(0xffffu - (a.v & 0xffffu)); }

// The bits of -inf among the 16-bit patterns, complemented: its key.
template <typename T> __device__ __forceinline__ uint32_t key16_neg_inf();
template <> __device__ __forceinline__ uint32_t key16_neg_inf<f16>() { return 0x03ffu; }
template <> __device__ __forceinline__ uint32_t key16_neg_inf<bf16>() { return 0x007fu; }

// Whether an item stands for a score (not absent).
template <typename T>
__device__ __forceinline__ bool item_present(Item32 a) { return a.v >> 16 > key16_neg_inf<T>(); }
template <typename T>
__device__ __forceinline__ bool item_present(Item64 a) { return item_key(a) > KEY_NEG_INF; }

// The score of an item.
template <typename T>
__device__ __forceinline__ T item_score(Item32 a) {
  const uint32_t k = a.v >> 16;
  const uint16_t b = (uint16_t)(k & 0x8000u ? k ^ 0x8000u : ~k);
  T r;
  __builtin_memcpy(&r, &b, 2);
  return r;
}
template <typename T>
__device__ __forceinline__ T item_score(Item64 a) { return from_f32<T>(key_score(item_key(a))); }

template <typename T> __device__ __forceinline__ uint32_t bits_neg_inf();
template <> __device__ __forceinline__ uint32_t bits_neg_inf<f16>() { return 0xfc00u; }
template <> __device__ __forceinline__ uint32_t bits_neg_inf<bf16>() { return 0xff80u; }

// -0 as +0, both halves of a word.
__device__ __forceinline__ uint32_t plus_zero(f16, uint32_t w) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  f16x2 h;
  __builtin_memcpy(&h, &w, 4);
  h += (f16x2)(_Float16)0;
  __builtin_memcpy(&w, &h, 4);
  return w;
}
__device__ __forceinline__ uint32_t plus_zero(bf16, uint32_t w) {
  w = (w & 0xffffu) == 0x8000u ? w & 0xffff0000u : w;
  return w >> 16 == 0x8000u ? w & 0xffffu : w;
}
// The items of 16 bytes of scores from class c0 on.  NaN takes its place by its
// bits, above +inf or below -inf, where items_regular() sees it.
template <typename T>
__device__ __forceinline__ void order_items(uint4 raw, int c0, Item32* p) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const uint32_t x = plus_zero(T(), w[h]);
    const uint32_t s = (x >> 15) & 0x00010001u;
    const uint32_t k = x ^ (((s << 15) - s) | 0x80008000u);
    p[2 * h].v = k << 16 | (0xffffu - (uint32_t)(c0 + 2 * h));
    p[2 * h + 1].v = (k & 0xffff0000u) | (0xffffu - (uint32_t)(c0 + 2 * h + 1));
  }
}
template <typename T>
__device__ __forceinline__ void order_items(uint4 raw, int c0, Item64* p) {
  float z[4];
  unpack<float>(raw, z);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = item64(score_key(z[i]), (uint32_t)(c0 + i));
}
// The items of 16 bytes of scores from class c0 on; NaN is absent.
template <typename T>
__device__ __forceinline__ void make_items(uint4 raw, int c0, Item32 (&a)[8]) {
  uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  float v[8];
  unpack<T>(raw, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int sh = 16 * (i & 1);
    if (v[i] != v[i]) w[i / 2] = (w[i / 2] & ~(0xffffu << sh)) | bits_neg_inf<T>() << sh;
  }
  order_items<T>(make_uint4(w[0], w[1], w[2], w[3]), c0, a);
}
template <typename T>
__device__ __forceinline__ void make_items(uint4 raw, int c0, Item64 (&a)[4]) {
  float z[4];
  unpack<float>(raw, z);
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = item64(z[i] != z[i] ? KEY_NEG_INF : score_key(z[i]), (uint32_t)(c0 + i));
}
// Whether the row with these largest and smallest items holds neither NaN nor
// +inf.
template <typename T> __device__ __forceinline__ bool items_regular(Item32 most, Item32 least) {
  const uint32_t inf = 0xffffu - key16_neg_inf<T>();
  return most.v >> 16 < inf && least.v >> 16 >= key16_neg_inf<T>();
}
template <typename T> __device__ __forceinline__ bool items_regular(Item64 most, Item64 least) {
  return item_key(most) < 0xff800000u && item_key(least) >= KEY_NEG_INF;
}

// Sorting networks on registers, largest first.
template <typename I>
__device__ __forceinline__ void order2(I& a, I& b) {
  const I hi = item_max(a, b);
  b = item_min(a, b);
  a = hi;
}
// A sequence that falls and rises (or any rotation of one) into order.
template <int N, typename I>
__device__ __forceinline__ void merge_bitonic(I* a) {
#pragma unroll
  for (int d = N / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & d)) order2(a[i], a[i + d]);
}
// Batcher's odd-even merge sort.
template <int N, typename I>
__device__ __forceinline__ void sort_items(I* a) {
#pragma unroll
  for (int p = 1; p < N; p <<= 1)
#pragma unroll
    for (int k = p; k > 0; k >>= 1)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order2(a[i + j], a[i + j + k]);
}

// The largest item of a lane group.
template <int LPR, int M = 1, typename I>
__device__ __forceinline__ I group_max_item(I a) {
  if constexpr (M < LPR) return group_max_item<LPR, 2 * M>(item_max(a, lane_xor<M>(a)));
  else return a;
}
template <int LPR, int M = 1>
__device__ __forceinline__ int group_max_int(int a) {
  if constexpr (M < LPR) {
    const int o = lane_xor<M>(a);
    return group_max_int<LPR, 2 * M>(a > o ? a : o);
  } else {
    return a;
  }
}

template <int LPR, int M = 1, typename I>
__device__ __forceinline__ I group_min_item(I a) {
  if constexpr (M < LPR) return group_min_item<LPR, 2 * M>(item_min(a, lane_xor<M>(a)));
  else return a;
}

// The larger of two items in the front lane, the smaller in the other: for 32
// bits the median of both and the largest or smallest number.
__device__ __forceinline__ Item32 item_side(bool front, Item32 a, Item32 o) {
  const uint32_t end = front ? 0xffffffffu : 0u;
  uint32_t r;
  asm("v_med3_u32 %0, %1, %2, %3" : "=v"(r) : "v"(a.v), "v"(o.v), "v"(end));
  return {r};
}
__device__ __forceinline__ Item64 item_side(bool front, Item64 a, Item64 o) {
  return item_pick(front, item_max(a, o), item_min(a, o));
}

// The LPR * N items of a lane group, N a lane, into order over the whole
// group: lane li then holds items li N .. li N + N - 1 of the order.  Merge
// sort whose first step of each merge pairs an item with its mirror image, so
// that every comparison puts the larger item in front.
template <int LPR, int N, int W, typename I>
__device__ __forceinline__ void group_merge_steps(I (&a)[N], int li) {
  // lanes W apart, then closer ones
  const bool front = (li & W) == 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const I o = lane_xor<W>(a[i]);
    a[i] = item_side(front, a[i], o);
  }
  if constexpr (W > 1) group_merge_steps<LPR, N, W / 2>(a, li);
}
template <int LPR, int N, int W, typename I>
__device__ __forceinline__ void group_merge_levels(I (&a)[N], int li) {
  if constexpr (W <= LPR) {
    const bool front = (li & (W / 2)) == 0;
    I o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = lane_xor<W - 1>(a[N - 1 - i]);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = item_side(front, a[i], o[i]);
    if constexpr (W > 2) group_merge_steps<LPR, N, W / 4>(a, li);
    merge_bitonic<N>(a);
    group_merge_levels<LPR, N, 2 * W>(a, li);
  }
}
template <int LPR, int N, typename I>
__device__ __forceinline__ void group_sort(I (&a)[N], int li) {
  sort_items<N>(a);
  group_merge_levels<LPR, N, 2>(a, li);
}

}  // namespace gcn
