// Backward pass of S = H W from H in 8 bits (gcn_transform_bwd_q8):
//   dW = H~^T G, dZ = (G W^T) * [Hq > 0] / (1 - p), db = column sums of dZ.
// The general way, for any widths: the weight gradient's kernel with codes
// turned into numbers as they come in (wgrad.hip), and a tiled product for dZ.
#include "internal.h"
#include "lanes.h"
#include "nt_tile.h"
#include "q8.h"

#include <algorithm>

namespace gcn {

namespace {

// dZ of 64 rows x 64 columns at a time; a workgroup walks the row blocks
// blockIdx.x, blockIdx.x + gridDim.x, .. and writes the column sums of what it
// computed, before rounding, as a row of colsum ([gridDim.x][M]).
template <typename T>
__global__ __launch_bounds__(256) void dz_tile_kernel(BwdQ8Params p, float* colsum) {
  __shared__ __align__(16) uint8_t lds[16384];
  __shared__ float part[2][NT_B];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col0 = (int64_t)blockIdx.y * NT_B;
  const NtOperands o{static_cast<const uint8_t*>(p.G), p.ldg * (int64_t)sizeof(T), p.n,
                     static_cast<const uint8_t*>(p.W), p.ldw * (int64_t)sizeof(T), p.M, p.N * (int64_t)sizeof(T)};
  float sum[2][4] = {};
  bool bad = false;
  for (int64_t row0 = (int64_t)blockIdx.x * NT_B; row0 < p.n; row0 += (int64_t)gridDim.x * NT_B) {
    f32x4 acc[2][2];
    nt_tile<T>(o, row0, col0, lds, acc);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t r = row0 + (wave >> 1) * 32 + j * 16 + (lane & 15);
      if (r >= p.n) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t c = col0 + (wave & 1) * 32 + i * 16 + (lane >> 4) * 4;
        if (c >= p.M) continue;
        uint32_t q = 0xffffffffu;
        if (p.relu) q = *reinterpret_cast<const uint32_t*>(p.Hq + r * p.ld_q + c);
        float z[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          z[v] = c + v < p.M && ((q >> (8 * v)) & 0xffu) ? acc[i][j][v] * p.keep : 0.f;
          sum[i][v] += z[v];
        }
        bad |= store4<T>(static_cast<T*>(p.dZ) + r * p.ldz + c, z);
      }
    }
  }
  if (bad) raise_flag(p.flag);
  if (!colsum) return;
  // the 16 lanes that share columns, then the two waves along the rows
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float t = group_sum<16>(sum[i][v]);
      if ((lane & 15) == 0) part[wave >> 1][(wave & 1) * 32 + i * 16 + (lane >> 4) * 4 + v] = t;
    }
  __syncthreads();
  if (threadIdx.x < NT_B && col0 + threadIdx.x < p.M)
    colsum[(int64_t)blockIdx.x * p.M + col0 + threadIdx.x] = part[0][threadIdx.x] + part[1][threadIdx.x];
}

// Row blocks walked at once: enough workgroups to fill the chip a few times.
int64_t dz_blocks(int64_t n, int64_t M) {
  const int64_t cols = (M + NT_B - 1) / NT_B;
  return std::min((n + NT_B - 1) / NT_B, std::max<int64_t>(8, 4096 / cols));
}

template <typename T>
hipError_t dz_t(const BwdQ8Params& p, float* colsum, hipStream_t s) {
  const dim3 grid((unsigned)dz_blocks(p.n, p.M), (unsigned)((p.M + NT_B - 1) / NT_B));
  hipLaunchKernelGGL((dz_tile_kernel<T>), grid, dim3(256), 0, s, p, colsum);
  return hipGetLastError();
}

int64_t pad64(int64_t x) { return (x + 63) / 64 * 64; }

}  // namespace

int64_t bwd_q8_floats(int prec, int64_t n, int64_t M, int64_t N) {
  return pad64((int64_t)wgrad_splits(prec, n, M, N) * M * N) + pad64(dz_blocks(n, M) * M);
}

hipError_t bwd_q8_launch(int prec, const BwdQ8Params& p, const Epilogue& dw, const Epilogue* db, float* ws,
                         hipStream_t s) {
  const int splits = wgrad_splits(prec, p.n, p.M, p.N);
  float* cs = ws + pad64((int64_t)splits * p.M * p.N);
  hipError_t e = wgrad_q8_launch(prec, p.Hq, p.ld_q, p.scale, p.kind, p.G, p.ldg, p.n, p.M, p.N, splits, ws, s);
  if (e != hipSuccess) return e;
  const RedJob jw = make_job(ws, splits, p.M, p.N, dw);
  if (!p.dZ) return reduce_partials2(prec, jw, nullptr, s);
  float* colsum = db ? cs : nullptr;
  switch (prec) {
    case 0: e = dz_t<float>(p, colsum, s); break;
    case 1: e = dz_t<f16>(p, colsum, s); break;
    case 2: e = dz_t<bf16>(p, colsum, s); break;
    default: e = hipErrorInvalidValue;
  }
  if (e != hipSuccess) return e;
  if (!db) return reduce_partials2(prec, jw, nullptr, s);
  const RedJob jb = make_job(cs, (int)dz_blocks(p.n, p.M), 1, p.M, *db);
  return reduce_partials2(prec, jw, &jb, s);
}

}  // namespace gcn
