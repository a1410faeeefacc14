// The layer's product from rows and weights in 8 bits (gcn_transform_q8):
// S_ij = h_scale[i] w_scale[j] sum_k Hq_ik Wq_jk, the sums exact in 32-bit
// integers.
//
// The matrix instruction multiplies signed bytes.  ReLU rows have codes 0 ..
// 255: their top bit flipped, a code u is the signed byte u - 128, and
// sum u w = sum (u - 128) w + 128 sum w, with the sums of the weights' columns
// laid out beside the weights.  All three stay below 2^31 up to 65536 columns
// (255 * 127 * 65536 = 2.12e9).
#include "internal.h"
#include "nt_tile.h"
#include "q8.h"

#include <algorithm>

namespace gcn {

namespace {

// A scale as mantissa and exponent: a sum times both mantissas, shifted by both
// exponents at the end, so that a product of scales below or above the fp32
// range does no harm where the result is inside it.
struct Scale { float m; int e; };
__device__ __forceinline__ Scale split(float s) { return Scale{__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }

template <typename T>
__global__ __launch_bounds__(256) void product_tile_kernel(ProductQ8Params p) {
  __shared__ __align__(16) uint8_t lds[16384];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col0 = (int64_t)blockIdx.y * NT_B;
  const NtOperands o{p.Hq, p.ld_q, p.n, p.Wq, p.ld_wq, p.N, p.K};
  // codes past the contracted columns count as 0 and turn into -128: the
  // weights are 0 there
  bool bad = false;
  for (int64_t row0 = (int64_t)blockIdx.x * NT_B; row0 < p.n; row0 += (int64_t)gridDim.x * NT_B) {
    i32x4 acc[2][2];
    nt_tile<int8_t>(o, row0, col0, lds, acc, p.relu ? 0x80808080u : 0u);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t r = row0 + (wave >> 1) * 32 + j * 16 + (lane & 15);
      if (r >= p.n) continue;
      const Scale sr = split(p.h_scale[r]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t c = col0 + (wave & 1) * 32 + i * 16 + (lane >> 4) * 4;
        if (c >= p.N) continue;
        float z[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int64_t cv = min(c + v, p.N - 1);
          const Scale sc = split(p.w_scale[cv]);
          const int sum = acc[i][j][v] + (p.relu ? p.w_sum[cv] * 128 : 0);
          z[v] = c + v < p.N ? __builtin_amdgcn_ldexpf((float)sum * (sr.m * sc.m), sr.e + sc.e) : 0.f;
        }
        bad |= store4<T>(static_cast<T*>(p.S) + r * p.ld_s + c, z);
      }
    }
  }
  if (bad) raise_flag(p.flag);
}

template <typename T>
hipError_t product_t(const ProductQ8Params& p, hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>((p.n + NT_B - 1) / NT_B, 1 << 16), (unsigned)((p.N + NT_B - 1) / NT_B));
  hipLaunchKernelGGL((product_tile_kernel<T>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t product_q8_launch(int prec, const ProductQ8Params& p, hipStream_t s) {
  switch (prec) {
    case 0: return product_t<float>(p, s);
    case 1: return product_t<f16>(p, s);
    case 2: return product_t<bf16>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace gcn
