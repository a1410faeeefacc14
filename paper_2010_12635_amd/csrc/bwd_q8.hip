// Backward pass of S = H W from H in 8 bits (gcn_transform_bwd_q8):
//   dW = H~^T G, dZ = (G W^T) * [Hq > 0] / (1 - p), db = column sums of dZ.
//
// Both products read G and both need the codes, so up to 256 columns of G (128 in
// fp32) one kernel makes all three from one pass over them (n (f_in + (f_in +
// f_out) s) bytes; bound by HBM in 16 bits, 2^21 rows, 128 <- 64 fp16 212 us (5.1
// TB/s); by instructions in fp32, whose matrix and vector ones do not overlap,
// 131072 rows, 256 <- 64 98 us (0.57 of the matrix rate)):
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
// Wider G takes two: a product for dZ, and for dW the same kernel with 256
// columns of G a workgroup (16 bits) or the weight gradient's kernel with codes
// turned into numbers as they come in (wgrad.hip).
#include "internal.h"
#include "lanes.h"
#include "nt_tile.h"
#include "q8.h"
#include "xpose.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

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

// 1 KiB from memory into LDS: lane l's 16 bytes at base + off go to lds + 16 l.
// Counted by vmcnt; no register is written.  As asm, because the compiler
// otherwise waits for it before any LDS read.
__device__ __forceinline__ void to_lds_1k(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
// An address that all lanes share, for the scalar registers.
__device__ __forceinline__ const void* uniform(const void* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const void*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 |
                                       (uint32_t)__builtin_amdgcn_readfirstlane((int)a));
}
// The same for 4 bytes a lane.
__device__ __forceinline__ void to_lds_256(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Eight rows of one column, for a matrix instruction that contracts over rows:
// lane l holds rows 8 (l / 16) .. + 7 of column l % 16.
template <typename T> struct Turned { uint4 v; };
template <> struct Turned<float> { float v[8]; };

template <typename T, int FI, int NT>
__device__ __forceinline__ void turned_mfma(const Turned<T> (&a)[FI], const Turned<T>& b, f32x4 (&acc)[FI][NT], int j) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < FI; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i].v[e], b.v[e], acc[i][j], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < FI; ++i) acc[i][j] = NtMfma<T>::run(a[i].v, b.v, acc[i][j]);
  }
}

// The smallest size that rounds to infinity in T: its largest number and half a
// step, a tie that goes to the even side.
template <typename T> __device__ __forceinline__ float overflow_at() { return __builtin_inff(); }
template <> __device__ __forceinline__ float overflow_at<f16>() { return 65520.f; }
template <> __device__ __forceinline__ float overflow_at<bf16>() { return __uint_as_float(0x7f7f8000u); }

// E = 4 or 8 consecutive elements of a row, rounded to T, in 8- or 16-byte
// stores.
template <typename T, int E>
__device__ __forceinline__ void store_cols(T* dst, const float (&x)[E]) {
  typedef T V __attribute__((ext_vector_type(E)));
  V v;
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = from_f32<T>(x[i]);
  if constexpr (E * sizeof(T) == 32) {
    const uint4* h = reinterpret_cast<const uint4*>(&v);
    stg16(dst, h[0]);
    stg16(dst + 4, h[1]);
  } else {
    *reinterpret_cast<V*>(dst) = v;
  }
}

template <typename T, int NB, int WM, int FI>
__global__ __launch_bounds__(64 * WM) __attribute__((amdgpu_waves_per_eu(2))) void bwd_q8_kernel(BwdQ8Params p, int64_t tiles, float* partials, int64_t stride, int sums) {
  constexpr int VE = Vec<T>::N, FW = 16 * FI, FB = FW * WM;  // columns of H a wave and a workgroup take
  constexpr int XE = 4 * FI;                               // columns of a row of dZ a lane ends with
  constexpr int CC = FB / 16, GC = NB * (int)sizeof(T) / 16;   // 16-byte pieces of a row of codes, of G
  constexpr int CB = TV * FB, GB = TV * GC * 16, STAGE = CB + GB;
  constexpr int KS = (GC + 3) / 4;                         // steps of 64 bytes along f_out
  constexpr int NT = NB / 16;
  constexpr int STORES = TV / 16 * (XE * sizeof(T) > 16 ? 2 : 1);   // stores of dZ a wave issues for a tile
  __shared__ __align__(1024) uint8_t lds[2 * STAGE];
  __shared__ __align__(16) float scales[2][TV];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t m0 = (int64_t)blockIdx.y * FB;
  // columns of G this workgroup takes: all of them where there is dZ
  const int64_t n0 = (int64_t)blockIdx.z * NB;
  const int N = (int)min(p.N - n0, (int64_t)NB);
  const T* const G = static_cast<const T*>(p.G) + n0;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)lds;
  const uint32_t scales0 = (uint32_t)(uintptr_t)(lds_byte*)scales;
  const int64_t step = gridDim.x;

  // A wave's 1 KiB pieces of a tile, by wave 0 its scales: where a lane's 16 bytes
  // of piece pc lie from the tile's first row on.  Rows past `last` are copies of
  // it, pieces past the widths of the first.  The places stay the same from tile
  // to tile and are kept up to 128 columns of G and six pieces a wave (2^21 rows,
  // 128 <- 64 fp16 220 -> 208 us); of these, fp32 with 128 columns of both spills 68
  // bytes a lane.
  constexpr int PIECES = STAGE / 1024, PPW = (PIECES + WM - 1) / WM;
  constexpr bool KEEP = PPW <= 6 && NB <= 128;
  auto place = [&](int pc, int last) -> uint32_t {
    if (pc < CB / 1024) {
      const int at = pc * 64 + lane, row = at / CC;
      const int64_t c = m0 + (((at % CC) ^ swz<CC>(row)) * 16);
      return (uint32_t)min(row, last) * (uint32_t)p.ld_q + (uint32_t)(c < p.M ? c : 0);
    }
    const int at = (pc - CB / 1024) * 64 + lane, row = at / GC, c = ((at % GC) ^ swz<GC>(row)) * VE;
    return ((uint32_t)min(row, last) * (uint32_t)p.ldg + (uint32_t)(c < N ? c : 0)) * (uint32_t)sizeof(T);
  };
  uint32_t off[KEEP ? PPW : 1];
  auto place_all = [&](int last) {
    if constexpr (KEEP) {
#pragma unroll
      for (int j = 0; j < PPW; ++j) off[j] = place(j * WM + wave, last);
    }
  };
  auto issue = [&](int64_t t, int st) {
    const int64_t r0 = t * TV;
    const int last = (int)min(p.n - 1 - r0, (int64_t)TV - 1);
    const uint8_t* codes = p.Hq + r0 * p.ld_q;
    const T* grad = G + r0 * p.ldg;
    auto one = [&](int pc, uint32_t at) {
      to_lds_1k(uniform(pc < CB / 1024 ? (const void*)codes : (const void*)grad), at,
                __builtin_amdgcn_readfirstlane(lds0 + st * STAGE + pc * 1024));
    };
    if constexpr (KEEP) {
      if (last < TV - 1) place_all(last);                  // the last tile, the last of its workgroup
#pragma unroll
      for (int j = 0; j < PPW; ++j)
        if (PIECES % WM == 0 || j * WM + wave < PIECES) one(j * WM + wave, off[j]);
    } else {
#pragma unroll 1
      for (int pc = wave; pc < PIECES; pc += WM) one(pc, place(pc, last));
    }
    if (wave == 0)
      to_lds_256(uniform(p.scale + r0), (uint32_t)min(lane, last) * 4, __builtin_amdgcn_readfirstlane(scales0 + st * (TV * 4)));
  };

  // rows of W: operand i's row m is column f0 + XE (m / 4) + 4 i + m % 4 of H
  const int64_t f0 = m0 + wave * FW;
  uint4 w[FI][KS];
  int live[KS];                                            // columns of G in this lane's pieces
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int left = N - (ks * 4 + lg) * VE;
    live[ks] = left <= 0 ? 0 : left >= VE ? VE : left;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int64_t f = min(f0 + XE * (l16 >> 2) + 4 * i + (l16 & 3), p.M - 1);
      w[i][ks] = make_uint4(0, 0, 0, 0);
      if (p.dZ && live[ks]) w[i][ks] = keep_first<T>(ldg16(static_cast<const T*>(p.W) + f * p.ldw + (ks * 4 + lg) * VE), live[ks]);
    }
  }
  const bool ragged = N < NB;
  const bool with_sign = p.kind == Q8_SIGNED;

  f32x4 acc[FI][NT];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // this lane's columns of dZ, within the workgroup's and of all, and those of
  // them that are columns of H, a byte each
  const int cc = wave * FW + XE * lg;
  const int64_t c = m0 + cc;
  uint32_t cols[FI];
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const int64_t left = p.M - c - 4 * i;
    cols[i] = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
  }
  const uint32_t dz_off = (uint32_t)l16 * (uint32_t)p.ldz + (uint32_t)c;
  const uint32_t every = p.relu ? 0u : ~0u;                // no mask: every code counts
  float sum[XE] = {}, most = 0.f;                          // sums, and the largest size of any element

  // stores of this wave behind the loads waited for: all STORES of the tile
  // before where every column of the wave is stored
  const bool counted = p.dZ && f0 + FW <= p.M;
  const bool mine = c < p.M;                               // some of this lane's columns are
  int64_t t = blockIdx.x;
  place_all(TV - 1);
  issue(t, 0);                                             // the launch has no more workgroups than tiles
  bool first = true;
  auto tile = [&](auto stage) {
    const int st = stage;
    constexpr int HALVES = sizeof(T) == 4 && NB >= 128 ? 1 : 2;   // of a tile at once for dW, registers allowing
    if (counted && !first) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(STORES) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    first = false;
    if (t + step < tiles) issue(t + step, st ^ 1);
    const int rows = (int)min(p.n - t * TV, (int64_t)TV);
    if (rows < TV) {                                       // rows past the last one: of scale 0
      if (tid < TV && tid >= rows) scales[st][tid] = 0.f;
      __syncthreads();
    }
    const uint8_t* cod = lds + st * STAGE;
    const uint8_t* g = cod + CB;

    if (p.dZ) {
#pragma unroll 1
      for (int vt = 0; vt < TV / 16; ++vt) {
        const int v = vt * 16 + l16;
        f32x4 z[FI];
#pragma unroll
        for (int i = 0; i < FI; ++i) z[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        uint4 gv[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          gv[ks] = make_uint4(0, 0, 0, 0);
          if (GC >= 4 || lg < GC) gv[ks] = *reinterpret_cast<const uint4*>(g + piece_at<GC>(v, ks * 4 + lg));
        }
        uint32_t q[FI];
#pragma unroll
        for (int i = 0; i < FI; ++i)
          q[i] = *reinterpret_cast<const uint32_t*>(cod + piece_at<CC>(v, cc >> 4) + (cc & 15) + 4 * i);
        if (ragged) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) gv[ks] = keep_first<T>(gv[ks], live[ks]);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 b = gv[ks];
          if constexpr (sizeof(T) == 4) {                  // in turn: each sum waits for its last addition
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int i = 0; i < FI; ++i)
                z[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((&w[i][ks].x)[e]),
                                                            __uint_as_float((&b.x)[e]), z[i], 0, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < FI; ++i) z[i] = NtMfma<T>::run(w[i][ks], b, z[i]);
          }
        }
        float x[XE];
#pragma unroll
        for (int i = 0; i < FI; ++i) {
          uint32_t k = (q[i] | every) & cols[i];
          k |= (k & 0x7f7f7f7fu) + 0x7f7f7f7fu;            // the top bit of every byte that is not 0
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = z[i][e] * p.keep;
            x[4 * i + e] = __uint_as_float(__float_as_uint(y) & (uint32_t)((int32_t)(k << (24 - 8 * e)) >> 31));
          }
        }
        if (v < rows && mine) {
#pragma unroll
          for (int e = 0; e < XE; ++e) {
            sum[e] += x[e];
            most = fmaxf(most, fabsf(x[e]));
          }
          store_cols<T, XE>(static_cast<T*>(p.dZ) + (t * TV + vt * 16) * p.ldz + dz_off, x);
        }
      }
    }

#pragma unroll HALVES
    for (int ks = 0; ks < TV / 32; ++ks) {
      const int v0 = ks * 32 + lg * 8;
      float sc[8];
      *reinterpret_cast<float4*>(sc) = *reinterpret_cast<const float4*>(&scales[st][v0]);
      *reinterpret_cast<float4*>(sc + 4) = *reinterpret_cast<const float4*>(&scales[st][v0 + 4]);
      Turned<T> a[FI];
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        const int v = v0 + (l16 >> 1);
        const i32x2 q = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) i32x2*)(cod + piece_at<CC>(v, wave * FI + i) + 8 * (l16 & 1)));
        float x[8];
        if (with_sign) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = (float)((int32_t)((uint32_t)q[e >> 2] << (24 - 8 * (e & 3))) >> 24) * sc[e];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = (float)(((uint32_t)q[e >> 2] >> (8 * (e & 3))) & 0xffu) * sc[e];
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
        turned_mfma<T, FI, NT>(a, b, acc, j);
      }
    }
    t += step;
  };
  if constexpr (NB <= 128) {                               // the stages in turn, each with its own code
    while (true) {
      tile(std::integral_constant<int, 0>());
      if (t >= tiles) break;
      tile(std::integral_constant<int, 1>());
      if (t >= tiles) break;
    }
  } else {                                                 // registers: twice the code spills
    for (int st = 0; t < tiles; st ^= 1) tile(st);
  }
  // an element that T cannot hold, or a NaN, which ends in its column's sum
  bool bad = most >= overflow_at<T>();
#pragma unroll
  for (int e = 0; e < XE; ++e) bad |= sum[e] != sum[e];
  if (bad) raise_flag(p.flag);

  // rows 4 (lane / 16) + v, column lane % 16 of each 16 x 16 block
  float* out = partials + (int64_t)blockIdx.x * stride;
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int64_t m = f0 + i * 16 + lg * 4 + v;
        const int n = j * 16 + l16;
        if (m < p.M && n < N) out[m * p.N + n0 + n] = acc[i][j][v];
      }
  if (!sums) return;
#pragma unroll
  for (int e = 0; e < XE; ++e) {
    const float s = group_sum<16>(sum[e]);
    if (l16 == 0 && f0 + XE * lg + e < p.M) out[p.M * p.N + f0 + XE * lg + e] = s;
  }
}

// The workgroups' partial sums (`splits` rows of `stride` floats: dW, then db)
// added in a fixed order: 64 outputs a workgroup, sixteen groups of rows each
// added in order, then the groups in order.  The workgroups behind the sums
// clear the padding of dW and db.
__global__ __launch_bounds__(256) void sum_partials_kernel(const float* __restrict__ partials, int64_t splits,
                                                           int64_t stride, int64_t M, int64_t N, float* dW, int64_t ldw,
                                                           float* db, int64_t blocks, int32_t* flag) {
  const int64_t dw_len = M * N, len = dw_len + (db ? M : 0), db_len = (M + 7) / 8 * 8;
  if ((int64_t)blockIdx.x >= blocks) {
    const int64_t at = ((int64_t)blockIdx.x - blocks) * 256 + threadIdx.x, pad = ldw - N;
    if (at < M * pad) dW[at / pad * ldw + N + at % pad] = 0.f;
    else if (db && at - M * pad < db_len - M) db[M + at - M * pad] = 0.f;
    return;
  }
  __shared__ __align__(16) float part[16][64];
  const int c = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const int64_t base = (int64_t)blockIdx.x * 64, per = (splits + 15) / 16;
  const int64_t s0 = min(grp * per, splits), s1 = min(s0 + per, splits);
  const float* src = partials + base + 4 * c;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  int64_t s = s0;
  for (; s + 8 <= s1; s += 8) {
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const float4*>(src + (s + i) * stride);
#pragma unroll
    for (int i = 0; i < 8; ++i) { a.x += v[i].x; a.y += v[i].y; a.z += v[i].z; a.w += v[i].w; }
  }
  for (; s < s1; ++s) {
    const float4 v = *reinterpret_cast<const float4*>(src + s * stride);
    a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
  }
  *reinterpret_cast<float4*>(&part[grp][4 * c]) = a;
  __syncthreads();
  const int64_t at = base + threadIdx.x;
  if (threadIdx.x >= 64 || at >= len) return;
  float z = part[0][threadIdx.x];
#pragma unroll
  for (int i = 1; i < 16; ++i) z += part[i][threadIdx.x];
  if (at < dw_len) dW[at / N * ldw + at % N] = z;
  else db[at - dw_len] = z;
  if (!finite_f32(z)) raise_flag(flag);
}

int64_t pad64(int64_t x) { return (x + 63) / 64 * 64; }
int64_t partial_stride(int64_t M, int64_t N) { return pad64(M * N + M); }

hipError_t sum_partials(const float* partials, int64_t splits, const BwdQ8Params& p, const Epilogue& dw,
                        const Epilogue* db, hipStream_t s) {
  const int64_t len = p.M * p.N + (db ? p.M : 0), blocks = (len + 63) / 64;
  const int64_t pad = p.M * (dw.ldo - p.N) + (db ? 7 : 0);
  hipLaunchKernelGGL(sum_partials_kernel, dim3((unsigned)(blocks + (pad + 255) / 256)), dim3(256), 0, s, partials, splits,
                     partial_stride(p.M, p.N), p.M, p.N, static_cast<float*>(dw.out), dw.ldo,
                     db ? static_cast<float*>(db->out) : nullptr, blocks, p.flag);
  return hipGetLastError();
}

// fp32 stops at 128: 256 columns would take half as many accumulators again as a
// wave has registers.
int64_t fused_max_n(int prec) { return prec == 0 ? 128 : 256; }

int64_t fused_columns(int64_t M) { return M <= 32 ? 32 : M <= 64 ? 64 : 128; }

// Workgroups along the rows, each with its own partial sums: two of four waves a
// compute unit, or fewer where a tile more for each costs less than another row
// of partial sums to write and read back.  With a tile at 1 us and partial sums
// at 4 TB/s both ways, tiles / w + w 8 M N / 4e6 is least at w = sqrt(5e5 tiles /
// (M N)).  Measured (us; 256, 512, 768, 1024 workgroups in all, before tiles were
// placed ahead): 2^21 rows, 128 <- 64 fp16 277, 220, 224, 229; 32768 rows, 2048
// <- 16 fp16 66, 54, 54, 59; 16384 rows, 500 <- 64 bf16 13.4 with 64 along the
// rows, 20 with 192 (the rule's 63: 12.9).  The rule does not count rounds: with 16
// columns a wave, 128 columns of H are eight waves and one workgroup a compute
// unit (82 KB of LDS), and 2^18 rows, 256 <- 256 get 352 of them, a round of 256 and
// a third of another; the 63 of 16384 rows walk 256 tiles, four or five each.
int64_t fused_splits(int prec, int64_t n, int64_t M, int64_t N) {
  const int64_t fb = fused_columns(M), nb = fused_max_n(prec), tiles = (n + TV - 1) / TV;
  const int64_t blocks = (M + fb - 1) / fb * ((N + nb - 1) / nb), held = 512 * (128 / fb) / blocks;
  const int64_t cheap = (int64_t)std::sqrt(5e5 * (double)tiles / ((double)M * (double)N));
  return std::min({tiles, std::max<int64_t>(1, held), std::max<int64_t>(1, cheap)});
}

// 32 columns of H a wave, or 16 (FI = 1) where 32 would leave registers for one
// wave a SIMD only.
template <typename T, int NB, int FI = NB * sizeof(T) >= 512 ? 1 : 2>
hipError_t fused_nb(int prec, const BwdQ8Params& p, float* partials, int64_t stride, int sums, hipStream_t s) {
  constexpr int W1 = 2 / FI;
  const int64_t tiles = (p.n + TV - 1) / TV;
  const int fb = (int)fused_columns(p.M);
  const dim3 grid((unsigned)fused_splits(prec, p.n, p.M, p.N), (unsigned)((p.M + fb - 1) / fb),
                  (unsigned)((p.N + NB - 1) / NB));
  const dim3 block(64 * W1 * fb / 32);
  switch (fb) {
    case 32: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, W1, FI>), grid, block, 0, s, p, tiles, partials, stride, sums); break;
    case 64: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, 2 * W1, FI>), grid, block, 0, s, p, tiles, partials, stride, sums); break;
    default: hipLaunchKernelGGL((bwd_q8_kernel<T, NB, 4 * W1, FI>), grid, block, 0, s, p, tiles, partials, stride, sums);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t fused_t(int prec, const BwdQ8Params& p, float* partials, int64_t stride, int sums, hipStream_t s) {
  if (p.N <= 16) return fused_nb<T, 16>(prec, p, partials, stride, sums, s);
  if (p.N <= 32) return fused_nb<T, 32>(prec, p, partials, stride, sums, s);
  if (p.N <= 64) return fused_nb<T, 64>(prec, p, partials, stride, sums, s);
  if constexpr (sizeof(T) == 2) {
    if (p.N > 128) return fused_nb<T, 256>(prec, p, partials, stride, sums, s);
    // 16 columns a wave, twice the waves, where there is one workgroup a compute
    // unit (us; 32, 16 columns): 262144 rows, 256 <- 100 fp16 76, 89; 65536 rows 40,
    // 45 (282 workgroups); 131072 rows, 128 <- 128 34.6, 33.4 (250); 65536 rows, 128
    // <- 100 27, 25 (200).
    const int64_t fb = fused_columns(p.M), wgs = fused_splits(prec, p.n, p.M, p.N) * ((p.M + fb - 1) / fb);
    if (wgs <= 256) return fused_nb<T, 128, 1>(prec, p, partials, stride, sums, s);
  }
  return fused_nb<T, 128>(prec, p, partials, stride, sums, s);
}

hipError_t fused(int prec, const BwdQ8Params& p, float* partials, int64_t stride, int sums, hipStream_t s) {
  switch (prec) {
    case 0: return fused_t<float>(prec, p, partials, stride, sums, s);
    case 1: return fused_t<f16>(prec, p, partials, stride, sums, s);
    case 2: return fused_t<bf16>(prec, p, partials, stride, sums, s);
  }
  return hipErrorInvalidValue;
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

// dZ by the row-streaming product with the codes as its mask, which keeps W in
// LDS, from 1024 rows on and where 16 rows of W fit; else in tiles (both
// products and db, us; streamed, tiles: 131072 rows, 300 <- 512 fp16 268, 326,
// 256 <- 200 fp32 339, 373; 32768 rows, 1000 <- 300 bf16 167, 172; 1528 rows, 589
// <- 181 fp32 33, 34).
bool stream_dz(int prec, int64_t n, int64_t N) { return n >= 1024 && tsgemm_supported(prec, N); }

}  // namespace

int64_t bwd_q8_floats(int prec, int64_t n, int64_t M, int64_t N) {
  const int64_t splits = std::max<int64_t>(wgrad_splits(prec, n, M, N), fused_splits(prec, n, M, N));   // either, by the strides
  const int64_t general = pad64(splits * M * N) + pad64(std::max<int64_t>(dz_blocks(n, M), tsgemm_colsum_rows_max()) * M);
  return N <= fused_max_n(prec) ? std::max(general, fused_splits(prec, n, M, N) * partial_stride(M, N)) : general;
}

hipError_t bwd_q8_launch(int prec, const BwdQ8Params& p, const Epilogue& dw, const Epilogue* db, float* ws,
                         hipStream_t s) {
  hipError_t e;
  // a tile's addresses are 32-bit offsets from its first row
  const int64_t es = prec == 0 ? 4 : 2;
  const bool near = TV * std::max({p.ld_q, p.ldg * es, p.dZ ? p.ldz * es : 0}) < (int64_t)1 << 31;
  if (p.N <= fused_max_n(prec) && near) {
    e = fused(prec, p, ws, partial_stride(p.M, p.N), db != nullptr, s);
    return e != hipSuccess ? e : sum_partials(ws, fused_splits(prec, p.n, p.M, p.N), p, dw, db, s);
  }
  // dW alone (us; one kernel, wgrad): 131072 rows, 300 <- 512 fp16 124, 188; 32768
  // rows, 1000 <- 300 bf16 88, 107; fp32, at 128 columns a workgroup: 131072 rows,
  // 256 <- 200 200, 170; 1528 rows, 589 <- 181 28, 21.
  const bool one = near && prec != 0;
  const int splits = one ? (int)fused_splits(prec, p.n, p.M, p.N) : wgrad_splits(prec, p.n, p.M, p.N);
  float* cs = ws + pad64((int64_t)splits * p.M * p.N);
  if (one) {
    BwdQ8Params w = p;
    w.dZ = nullptr;
    e = fused(prec, w, ws, p.M * p.N, 0, s);
  } else {
    e = wgrad_q8_launch(prec, p.Hq, p.ld_q, p.scale, p.kind, p.G, p.ldg, p.n, p.M, p.N, splits, ws, s);
  }
  int rows = (int)dz_blocks(p.n, p.M);                     // of partial column sums
  if (e == hipSuccess && p.dZ) {
    float* colsum = db ? cs : nullptr;
    if (stream_dz(prec, p.n, p.N)) {
      Epilogue ez{};
      ez.out = p.dZ; ez.ldo = p.ldz; ez.rows = p.n; ez.cols = p.M; ez.mode = EPI_QMASK; ez.flag = p.flag;
      ez.relu = p.relu; ez.keep_scale = p.keep; ez.hmask = p.Hq; ez.ldh = p.ld_q;
      e = tsgemm_launch(prec, p.G, p.ldg, p.W, p.ldw, true, p.n, p.M, p.N, ez, s, colsum, &rows);
    } else {
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
  const RedJob jb = make_job(cs, rows, 1, p.M, *db);
  return reduce_partials2(prec, jw, &jb, s);
}

}  // namespace gcn
