// The K largest scores of every row with their classes, in falling order, the
// lower class first among equals.
//
// One workgroup takes a row.  Round j finds the largest (key, class) pair that
// comes after the one round j - 1 found, so no list is kept and rows of any
// length and any number of equal scores are right.
#include "internal.h"
#include "rows.h"

namespace gcn {

namespace {

// score key above, complement of the class below: the larger pair comes first
__device__ __forceinline__ uint64_t pair_of(uint32_t key, int64_t c) {
  return ((uint64_t)key << 32) | (uint32_t)~(uint32_t)c;
}

template <typename T>
__global__ __launch_bounds__(256) void top_rounds_kernel(TopParams p) {
  __shared__ uint64_t sh[4];
  const int64_t row = blockIdx.x;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  T* __restrict__ vals = reinterpret_cast<T*>(p.values) + row * p.ld_top;
  int32_t* __restrict__ ids = p.classes + row * p.ld_top;
  bool bad = false;
  uint64_t last = ~0ull;
  for (int64_t j = 0; j < p.K; ++j) {
    uint64_t best = 0;
    for (int64_t c = threadIdx.x; c < p.C; c += 256) {
      const float v = to_f32<T>(z[c]);
      if (!(v < INFINITY)) bad = true;
      if (!(v > -INFINITY)) continue;                    // -inf and NaN are no candidates
      const uint64_t q = pair_of(score_key(v), c);
      if (q < last && q > best) best = q;
    }
    best = block_reduce<4>(best, sh, MaxF());
    if (threadIdx.x == 0) {
      vals[j] = from_f32<T>(best ? key_score((uint32_t)(best >> 32)) : -INFINITY);
      ids[j] = best ? (int32_t)~(uint32_t)best : -1;
    }
    last = best;
  }
  if (bad) raise_flag(p.flag);
}

}  // namespace

size_t top_workspace_bytes(int prec, int64_t n, int64_t C, int64_t K) { return 256; }

hipError_t top_launch(int prec, const TopParams& p, void* ws, hipStream_t s) {
  const dim3 grid((unsigned)p.n);
  switch (prec) {
    case 0: hipLaunchKernelGGL((top_rounds_kernel<float>), grid, dim3(256), 0, s, p); break;
    case 1: hipLaunchKernelGGL((top_rounds_kernel<f16>), grid, dim3(256), 0, s, p); break;
    case 2: hipLaunchKernelGGL((top_rounds_kernel<bf16>), grid, dim3(256), 0, s, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace gcn
