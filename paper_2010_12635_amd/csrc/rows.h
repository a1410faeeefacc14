// Rows of class scores taken by a whole workgroup (or one wave): the order of
// the scores, and reductions over NW waves.
#pragma once

#include "common.h"

namespace gcn {

// Long rows take a workgroup each (or several): a launch takes as many rows as
// fill 2^18 workgroups, whatever their threads (HIP launches less than 2^32
// threads), and the next one goes on at row0.  launch(p, rows) launches.
constexpr int64_t LAUNCH_WORKGROUPS = 1 << 18;
template <typename P, typename F>
hipError_t launch_long_rows(P p, int64_t workgroups_a_row, F launch) {
  const int64_t most = LAUNCH_WORKGROUPS / workgroups_a_row > 0 ? LAUNCH_WORKGROUPS / workgroups_a_row : 1;
  for (p.row0 = 0; p.row0 < p.n; p.row0 += most) {
    const hipError_t e = launch(p, p.n - p.row0 < most ? p.n - p.row0 : most);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// A score as an unsigned key of the same order: a larger score has a larger
// key, equal scores (-0 and +0 among them) equal keys.  NaN has no place in
// the order and is dealt with before.
__device__ __forceinline__ uint32_t score_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);           // -0 + 0 = +0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t KEY_NEG_INF = 0x007fffffu;            // score_key(-inf)

// Reductions over a wave, every lane ending with the result, in a fixed order:
// within rows of 16 lanes by DPP moves, then over the four rows' results (a
// move costs a few cycles, an exchange through shared memory's crossbar a
// hundred).
template <int CTRL, typename V>
__device__ __forceinline__ V dpp_move(V v) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "whole registers");
  constexpr int N = sizeof(V) / 4;
  int w[N];
  __builtin_memcpy(w, &v, sizeof(V));
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = __builtin_amdgcn_update_dpp(0, w[i], CTRL, 0xF, 0xF, true);
  __builtin_memcpy(&v, w, sizeof(V));
  return v;
}
template <typename V>
__device__ __forceinline__ V from_lane(V v, int lane) {
  constexpr int N = sizeof(V) / 4;
  int w[N];
  __builtin_memcpy(w, &v, sizeof(V));
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = __builtin_amdgcn_readlane(w[i], lane);
  __builtin_memcpy(&v, w, sizeof(V));
  return v;
}
template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F f) {
  v = f(v, dpp_move<0xB1>(v));                           // lanes differing in bit 0, then bit 1
  v = f(v, dpp_move<0x4E>(v));
  v = f(v, dpp_move<0x141>(v));                          // halves of 8 and rows of 16, mirrored
  v = f(v, dpp_move<0x140>(v));
  return f(f(from_lane(v, 0), from_lane(v, 16)), f(from_lane(v, 32), from_lane(v, 48)));
}

// The same over the NW waves of a workgroup.  sh: NW elements of shared memory,
// free again when the call returns.
template <int NW, typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* sh, F f) {
  v = wave_reduce(v, f);
  if constexpr (NW == 1) return v;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  V r = sh[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) r = f(r, sh[i]);
  __syncthreads();
  return r;
}
struct AddF { template <typename V> __device__ V operator()(V a, V b) const { return a + b; } };
struct MaxF { template <typename V> __device__ V operator()(V a, V b) const { return a > b ? a : b; } };
struct MinF { template <typename V> __device__ V operator()(V a, V b) const { return a < b ? a : b; } };

// Sum over the lanes up to the lane itself (before it: 0 for lane 0).
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  const int lane = threadIdx.x & 63, in_row = lane & 15;
  V o = dpp_move<0x111>(v);                              // row_shr by 1, 2, 4, 8
  v += in_row >= 1 ? o : V(0);
  o = dpp_move<0x112>(v);
  v += in_row >= 2 ? o : V(0);
  o = dpp_move<0x114>(v);
  v += in_row >= 4 ? o : V(0);
  o = dpp_move<0x118>(v);
  v += in_row >= 8 ? o : V(0);
  const V a = from_lane(v, 15), b = a + from_lane(v, 31), c = b + from_lane(v, 47);
  return lane < 16 ? v : v + (lane < 32 ? a : lane < 48 ? b : c);
}
template <typename V>
__device__ __forceinline__ V wave_before(V upto) {
  const V o = __shfl_up(upto, 1);
  return (threadIdx.x & 63) == 0 ? V(0) : o;
}

}  // namespace gcn
