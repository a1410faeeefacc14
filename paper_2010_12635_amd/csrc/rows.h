// Rows of class scores taken by a whole workgroup (or one wave): the order of
// the scores, and reductions over NW waves.
#pragma once

#include "common.h"

namespace gcn {

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

// Reductions over the NW waves of a workgroup, every thread ending with the
// result, in a fixed order.  sh: NW elements of shared memory, free again
// when the call returns.
template <int NW, typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* sh, F f) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v = f(v, __shfl_xor(v, m));
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

// Inclusive sum over the lanes below and the lane itself.
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const V o = __shfl_up(v, m);
    if (lane >= m) v += o;
  }
  return v;
}

}  // namespace gcn
