// Backward pass of S = H W from H in 8 bits (gcn_transform_bwd_q8):
//   dW = H~^T G, dZ = (G W^T) * [Hq > 0] / (1 - p), db = column sums of dZ.
//
// Both products read G and both need the codes, so up to 128 columns of G one
// kernel makes all three from one pass over them (n (f_in + (f_in + f_out) s)
// bytes; bound by HBM in 16 bits, by the matrix instructions in fp32):
//  * A workgroup walks tiles of 64 rows.  Codes and G come straight from memory
//    into LDS, a tile ahead.  Each wave owns 32 columns of H for good: 32 rows
//    of W in registers for dZ, a 32 x f_out block of dW in accumulators.  The
//    waves share G and nothing else.
//  * dZ: W's rows are the matrix instruction's first operand and G's the second,
//    both contiguous along f_out as they lie.  W's rows are dealt to the two 16-row
//    operands so that a lane ends with eight consecutive columns of a row of dZ.
//  * dW contracts over rows, so both operands have to be turned: gfx950's
//    transposing LDS reads do it on the way (ds_read_b64_tr_b8 for the codes,
//    _tr_b16 for G; fp32 takes G element by element, its operands hold one row a
//    lane).  Codes are turned into numbers after the turn, by the one wave that
//    multiplies them.
//  * 16-byte pieces of a row in LDS change places with its row number, so that
//    no read of 16 rows at the same column meets a bank twice.
// Wider G goes the general way: the weight gradient's kernel with codes turned
// into numbers as they come in (wgrad.hip), and a tiled product for dZ.
#include "internal.h"
#include "lanes.h"
#include "nt_tile.h"
#include "q8.h"
#include "xpose.h"

#include <algorithm>

namespace gcn {

namespace {

constexpr int TV = 64;            // rows of a tile

// Where 16-byte piece c of row v of a tile with C pieces a row lies in its row:
// piece c ^ swz(v).  Reads of one column over 16 rows, and of two pieces over
// rows 0 .. 3 and 8 .. 11 (or 4 .. 7 and 12 .. 15) then use every bank once.
template <int C>
__device__ __forceinline__ int swz(int v) {
  const int b0 = v & 1, b1 = (v >> 1) & 1, b2 = (v >> 2) & 1, b3 = (v >> 3) & 1;
  if (C >= 16) return b3 << 3 | b1 << 2 | b0 << 1 | b2;
  if (C == 8) return b3 << 2 | b1 << 1 | b2;
  if (C == 4) return b3 << 1 | b2;
  if (C == 2) return b3;
  return 0;
}
template <int C>
__device__ __forceinline__ int piece_at(int v, int c) { return (v * C + (c ^ swz<C>(v))) * 16; }

// 1 KiB from memory into LDS: lane l's 16 bytes at its own address go to lds +
// 16 l.  Counted by vmcnt; no register is written.  As asm, because the compiler
// otherwise waits for it before any LDS read.
__device__ __forceinline__ void to_lds_1k(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds) : "memory", "m0");
}
typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Eight rows of one column, for a matrix instruction that contracts over rows:
// lane l holds rows 8 (l / 16) .. + 7 of column l % 16.
template <typename T> struct Turned { uint4 v; };
template <> struct Turned<float> { float v[8]; };

template <typename T>
__device__ __forceinline__ f32x4 turned_mfma(const Turned<T>& a, const Turned<T>& b, f32x4 c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
  } else {
    return NtMfma<T>::run(a.v, b.v, c);
  }
}

template <typename T, int NB, int WM>
__global__ __launch_bounds__(64 * WM) void bwd_q8_kernel(BwdQ8Params p, int64_t tiles, float* partials, float* colsum) {
  constexpr int VE = Vec<T>::N, FB = 32 * WM;              // columns of H a workgroup takes
  constexpr int CC = FB / 16, GC = NB * (int)sizeof(T) / 16;   // 16-byte pieces of a row of codes, of G
  constexpr int CB = TV * FB, GB = TV * GC * 16, STAGE = CB + GB;
  constexpr int KS = (GC + 3) / 4;                         // steps of 64 bytes along f_out
  constexpr int NT = NB / 16;
  constexpr int STORES = TV / 16 * (int)(8 * sizeof(T) / 16);   // stores of dZ a wave issues for a tile
  __shared__ __align__(1024) uint8_t lds[2 * STAGE];
  __shared__ __align__(16) float scales[2][TV];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t m0 = (int64_t)blockIdx.y * FB;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)lds;

  // this wave's 1 KiB pieces of tile t into a stage; rows past the last one are
  // copies of it (their scale is 0), pieces past the widths copies of the first
  auto issue = [&](int64_t t, int st) {
#pragma unroll
    for (int q = 0; q < (STAGE / 1024 + WM - 1) / WM; ++q) {
      const int pc = q * WM + wave;
      if (pc >= STAGE / 1024) break;
      const void* src;
      if (pc < CB / 1024) {
        const int at = pc * 64 + lane, row = at / CC;
        const int64_t r = min(t * TV + row, p.n - 1), c = m0 + (((at % CC) ^ swz<CC>(row)) * 16);
        src = p.Hq + r * p.ld_q + (c < p.M ? c : 0);
      } else {
        const int at = (pc - CB / 1024) * 64 + lane, row = at / GC;
        const int64_t r = min(t * TV + row, p.n - 1), c = ((at % GC) ^ swz<GC>(row)) * VE;
        src = static_cast<const T*>(p.G) + r * p.ldg + (c < p.N ? c : 0);
      }
      to_lds_1k(src, lds0 + st * STAGE + pc * 1024);
    }
  };
  auto scale_of = [&](int64_t t) { return t * TV + tid < p.n ? p.scale[t * TV + tid] : 0.f; };   // tid < TV

  // 32 rows of W: operand i's row m is column m0 + 32 wave + 8 (m / 4) + 4 i + m % 4 of H
  const int64_t f0 = m0 + wave * 32;
  uint4 w[2][KS];
  int live[KS];                                            // columns of G in this lane's pieces
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int64_t left = p.N - (ks * 4 + lg) * VE;
    live[ks] = left <= 0 ? 0 : left >= VE ? VE : (int)left;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t f = min(f0 + 8 * (l16 >> 2) + 4 * i + (l16 & 3), p.M - 1);
      w[i][ks] = make_uint4(0, 0, 0, 0);
      if (p.dZ && live[ks]) w[i][ks] = keep_first<T>(ldg16(static_cast<const T*>(p.W) + f * p.ldw + (ks * 4 + lg) * VE), live[ks]);
    }
  }
  const bool ragged = p.N < NB;
  const uint32_t flip = p.kind == Q8_SIGNED ? 0x80808080u : 0u;
  const float zero = p.kind == Q8_SIGNED ? -128.f : 0.f;

  f32x4 acc[2][NT];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float sum[8] = {};
  bool bad = false;

  // stores of this wave behind the loads waited for: all STORES of the tile
  // before where every column of the wave is stored
  const bool counted = p.dZ && f0 + 32 <= p.M;
  int64_t t = blockIdx.x;
  if (tid < TV) scales[0][tid] = scale_of(t);              // the launch has no more workgroups than tiles
  issue(t, 0);
  bool first = true;
  for (int st = 0; t < tiles; t += gridDim.x, st ^= 1) {
    if (counted && !first) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(STORES) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    first = false;
    const int64_t tn = t + gridDim.x;
    float next_scale = 0.f;
    if (tn < tiles) {
      if (tid < TV) next_scale = scale_of(tn);
      issue(tn, st ^ 1);
    }
    const uint8_t* cod = lds + st * STAGE;
    const uint8_t* g = cod + CB;

    if (p.dZ) {
#pragma unroll
      for (int vt = 0; vt < TV / 16; ++vt) {
        const int v = vt * 16 + l16;
        f32x4 z[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint4 b = make_uint4(0, 0, 0, 0);
          if (GC >= 4 || lg < GC) b = *reinterpret_cast<const uint4*>(g + piece_at<GC>(v, ks * 4 + lg));
          if (ragged) b = keep_first<T>(b, live[ks]);
#pragma unroll
          for (int i = 0; i < 2; ++i) z[i] = NtMfma<T>::run(w[i][ks], b, z[i]);
        }
        uint2 q = make_uint2(~0u, ~0u);
        if (p.relu) q = *reinterpret_cast<const uint2*>(cod + piece_at<CC>(v, wave * 2 + (lg >> 1)) + 8 * (lg & 1));
        const int64_t r = t * TV + v, c = f0 + 8 * lg;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t code = ((e < 4 ? q.x : q.y) >> (8 * (e & 3))) & 0xffu;
          x[e] = code && c + e < p.M ? z[e >> 2][e & 3] * p.keep : 0.f;
        }
        if (r < p.n && c < p.M) {
          T* dst = static_cast<T*>(p.dZ) + r * p.ldz + c;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += x[e];
          if constexpr (sizeof(T) == 4) {
            stg16(dst, pack<float>(x));
            stg16(dst + 4, pack<float>(x + 4));
          } else {
            stg16(dst, pack<T>(x));
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) bad |= !finite_f32(to_f32<T>(from_f32<T>(x[e])));
        }
      }
    }

#pragma unroll
    for (int ks = 0; ks < TV / 32; ++ks) {
      const int v0 = ks * 32 + lg * 8;
      float sc[8];
      *reinterpret_cast<float4*>(sc) = *reinterpret_cast<const float4*>(&scales[st][v0]);
      *reinterpret_cast<float4*>(sc + 4) = *reinterpret_cast<const float4*>(&scales[st][v0 + 4]);
      Turned<T> a[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int v = v0 + (l16 >> 1);
        const i32x2 q = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) i32x2*)(cod + piece_at<CC>(v, wave * 2 + i) + 8 * (l16 & 1)));
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t b = (((uint32_t)q[e >> 2] ^ flip) >> (8 * (e & 3))) & 0xffu;
          x[e] = fmaf((float)b, sc[e], zero * sc[e]);      // exact: (b - 128) * scale has 24 bits
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int e = 0; e < 8; ++e) a[i].v[e] = x[e];
        } else {
          a[i].v = pack<T>(x);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        Turned<T> b;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            b.v[e] = *reinterpret_cast<const float*>(g + piece_at<GC>(v0 + e, j * 4 + (l16 >> 2)) + 4 * (l16 & 3));
        } else {
          s16x4 h[2];
#pragma unroll
          for (int e = 0; e < 2; ++e)
            h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(g + piece_at<GC>(v0 + 4 * e + (l16 >> 2), j * 2 + ((l16 & 3) >> 1)) +
                                                           8 * (l16 & 1)));
          __builtin_memcpy(&b.v, h, 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[i][j] = turned_mfma<T>(a[i], b, acc[i][j]);
      }
    }
    if (tid < TV) scales[st ^ 1][tid] = next_scale;
  }
  if (bad) raise_flag(p.flag);

  // rows 4 (lane / 16) + v, column lane % 16 of each 16 x 16 block
  float* out = partials + (int64_t)blockIdx.x * p.M * p.N;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int64_t m = f0 + i * 16 + lg * 4 + v, n = j * 16 + l16;
        if (m < p.M && n < p.N) out[m * p.N + n] = acc[i][j][v];
      }
  if (!colsum) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float s = group_sum<16>(sum[e]);
    if (l16 == 0 && f0 + 8 * lg + e < p.M) colsum[(int64_t)blockIdx.x * p.M + f0 + 8 * lg + e] = s;
  }
}

constexpr int64_t FUSED_MAX_N = 128;

// Workgroups along the rows, each with its own partial sums.
int64_t fused_splits(int64_t n, int64_t M) {
  const int64_t fb = M <= 32 ? 32 : M <= 64 ? 64 : 128, blocks = (M + fb - 1) / fb;
  return std::min((n + TV - 1) / TV, std::max<int64_t>(32, 1024 / blocks));
}

template <typename T, int NB>
hipError_t fused_nb(const BwdQ8Params& p, float* partials, float* colsum, hipStream_t s) {
  const int64_t tiles = (p.n + TV - 1) / TV;
  const int wm = p.M <= 32 ? 1 : p.M <= 64 ? 2 : 4;
  const dim3 grid((unsigned)fused_splits(p.n, p.M), (unsigned)((p.M + 32 * wm - 1) / (32 * wm)));
  switch (wm) {
    case 1: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, 1>), grid, dim3(64), 0, s, p, tiles, partials, colsum); break;
    case 2: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, 2>), grid, dim3(128), 0, s, p, tiles, partials, colsum); break;
    default: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, 4>), grid, dim3(256), 0, s, p, tiles, partials, colsum);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t fused_t(const BwdQ8Params& p, float* partials, float* colsum, hipStream_t s) {
  if (p.N <= 16) return fused_nb<T, 16>(p, partials, colsum, s);
  if (p.N <= 32) return fused_nb<T, 32>(p, partials, colsum, s);
  if (p.N <= 64) return fused_nb<T, 64>(p, partials, colsum, s);
  return fused_nb<T, 128>(p, partials, colsum, s);
}

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
  if (N <= FUSED_MAX_N) return pad64(fused_splits(n, M) * M * N) + pad64(fused_splits(n, M) * M);
  return pad64((int64_t)wgrad_splits(prec, n, M, N) * M * N) + pad64(dz_blocks(n, M) * M);
}

hipError_t bwd_q8_launch(int prec, const BwdQ8Params& p, const Epilogue& dw, const Epilogue* db, float* ws,
                         hipStream_t s) {
  const bool fused = p.N <= FUSED_MAX_N;
  const int splits = fused ? (int)fused_splits(p.n, p.M) : wgrad_splits(prec, p.n, p.M, p.N);
  const int sums = fused ? splits : (int)dz_blocks(p.n, p.M);
  float* cs = ws + pad64((int64_t)splits * p.M * p.N);
  float* colsum = db ? cs : nullptr;
  hipError_t e = hipErrorInvalidValue;
  if (fused) {
    switch (prec) {
      case 0: e = fused_t<float>(p, ws, colsum, s); break;
      case 1: e = fused_t<f16>(p, ws, colsum, s); break;
      case 2: e = fused_t<bf16>(p, ws, colsum, s); break;
    }
  } else {
    e = wgrad_q8_launch(prec, p.Hq, p.ld_q, p.scale, p.kind, p.G, p.ldg, p.n, p.M, p.N, splits, ws, s);
    if (e == hipSuccess && p.dZ) {
      switch (prec) {
        case 0: e = dz_t<float>(p, colsum, s); break;
        case 1: e = dz_t<f16>(p, colsum, s); break;
        case 2: e = dz_t<bf16>(p, colsum, s); break;
      }
    }
  }
  if (e != hipSuccess) return e;
  const RedJob jw = make_job(ws, splits, p.M, p.N, dw);
  if (!db) return reduce_partials2(prec, jw, nullptr, s);
  const RedJob jb = make_job(cs, sums, 1, p.M, *db);
  return reduce_partials2(prec, jw, &jb, s);
}

}  // namespace gcn
