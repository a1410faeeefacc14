// Reductions over lane groups and tests of packed values, shared by the
// kernels that work on rows of class scores.
#pragma once

#include "common.h"

namespace gcn {

// Reductions over a lane group of LPR lanes (aligned, a power of two),
// every lane ending with the result: lanes exchange values through DPP
// moves inside rows of 16 lanes (quad permutations, then the half-row and
// row mirrors, each pairing a lane with one of the other half once the
// halves agree), across rows through lane shuffles.
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true);
}
constexpr int DPP_XOR1 = 0xB1;         // quad_perm [1, 0, 3, 2]
constexpr int DPP_XOR2 = 0x4E;         // quad_perm [2, 3, 0, 1]
constexpr int DPP_HALF_MIRROR = 0x141; // lane i <-> 7 - i of each 8
constexpr int DPP_MIRROR = 0x140;      // lane i <-> 15 - i of each 16

template <int LPR>
__device__ __forceinline__ float group_sum(float v) {
  if (LPR >= 2) v += dpp_f<DPP_XOR1>(v);
  if (LPR >= 4) v += dpp_f<DPP_XOR2>(v);
  if (LPR >= 8) v += dpp_f<DPP_HALF_MIRROR>(v);
  if (LPR >= 16) v += dpp_f<DPP_MIRROR>(v);
  if (LPR >= 32) v += __shfl_xor(v, 16);
  if (LPR >= 64) v += __shfl_xor(v, 32);
  return v;
}

template <int LPR>
__device__ __forceinline__ float group_max(float v) {
  if (LPR >= 2) v = fmaxf(v, dpp_f<DPP_XOR1>(v));
  if (LPR >= 4) v = fmaxf(v, dpp_f<DPP_XOR2>(v));
  if (LPR >= 8) v = fmaxf(v, dpp_f<DPP_HALF_MIRROR>(v));
  if (LPR >= 16) v = fmaxf(v, dpp_f<DPP_MIRROR>(v));
  if (LPR >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  if (LPR >= 64) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

// Sum over the lanes of the group before this one (li: the lane's place in it),
// 0 for the first: never the difference of a sum and this lane's own share,
// which would lose what is small beside it.
template <int M>
__device__ __forceinline__ float lane_before(float v) {
  return dpp_f<0x110 + M>(v);                            // row_shr, M < 16: within rows of 16
}
template <int M>
__device__ __forceinline__ double lane_before(double v) { return __shfl_up(v, M); }
template <int LPR, int M, typename W>
__device__ __forceinline__ W group_scan_steps(W v, int li) {
  if constexpr (M < LPR) {
    W o;
    if constexpr (LPR > 16) o = __shfl_up(v, M);         // groups of several rows of 16 lanes
    else o = lane_before<M>(v);
    v += li >= M ? o : W(0);
    return group_scan_steps<LPR, 2 * M>(v, li);
  } else {
    return v;
  }
}
template <int LPR, typename W>
__device__ __forceinline__ W group_sum_before(W v, int li) {
  if constexpr (LPR == 1) return W(0);
  const W upto = group_scan_steps<LPR, 1>(v, li);
  W o;
  if constexpr (LPR > 16) o = __shfl_up(upto, 1);
  else o = lane_before<1>(upto);
  return li >= 1 ? o : W(0);
}

template <int LPR>
__device__ __forceinline__ double group_sum(double v) {
#pragma unroll
  for (int m = 1; m < LPR; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
template <int LPR>
__device__ __forceinline__ int group_sum(int v) {
  if (LPR >= 2) v += dpp_i<DPP_XOR1>(v);
  if (LPR >= 4) v += dpp_i<DPP_XOR2>(v);
  if (LPR >= 8) v += dpp_i<DPP_HALF_MIRROR>(v);
  if (LPR >= 16) v += dpp_i<DPP_MIRROR>(v);
  if (LPR >= 32) v += __shfl_xor(v, 16);
  if (LPR >= 64) v += __shfl_xor(v, 32);
  return v;
}

// Whether any lane of the group holds true.
template <int LPR>
__device__ __forceinline__ bool group_any(bool v) {
  constexpr uint64_t GROUP = LPR == 64 ? ~0ull : (1ull << (LPR & 63)) - 1;
  const int first = (threadIdx.x & 63) / LPR * LPR;
  return (__ballot(v) >> first & GROUP) != 0;
}

// Orders the shared-memory accesses of a wave's lanes: what any lane wrote
// before is seen by every lane after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// (maximum, lowest index among the maxima) over the group
__device__ __forceinline__ void argmax_step(float& mx, int& am, float om, int oa) {
  const bool take = om > mx || (om == mx && oa < am);
  mx = take ? om : mx;
  am = take ? oa : am;
}
template <int LPR>
__device__ __forceinline__ void group_argmax(float& mx, int& am) {
  if (LPR >= 2) argmax_step(mx, am, dpp_f<DPP_XOR1>(mx), dpp_i<DPP_XOR1>(am));
  if (LPR >= 4) argmax_step(mx, am, dpp_f<DPP_XOR2>(mx), dpp_i<DPP_XOR2>(am));
  if (LPR >= 8) argmax_step(mx, am, dpp_f<DPP_HALF_MIRROR>(mx), dpp_i<DPP_HALF_MIRROR>(am));
  if (LPR >= 16) argmax_step(mx, am, dpp_f<DPP_MIRROR>(mx), dpp_i<DPP_MIRROR>(am));
  if (LPR >= 32) argmax_step(mx, am, __shfl_xor(mx, 16), __shfl_xor(am, 16));
  if (LPR >= 64) argmax_step(mx, am, __shfl_xor(mx, 32), __shfl_xor(am, 32));
}

template <typename T> __device__ __forceinline__ float max_finite();
template <> __device__ __forceinline__ float max_finite<float>() { return 3.40282347e38f; }
template <> __device__ __forceinline__ float max_finite<f16>() { return 65504.f; }
template <> __device__ __forceinline__ float max_finite<bf16>() { return 3.38953139e38f; }

// Any non-finite element among the VE packed values (exponent field all ones).
template <typename T> __device__ __forceinline__ bool packed_nonfinite(uint4 o);
template <> __device__ __forceinline__ bool packed_nonfinite<float>(uint4 o) {
  const uint32_t e = 0x7f800000u;
  return (o.x & e) == e || (o.y & e) == e || (o.z & e) == e || (o.w & e) == e;
}
// Both halves of a word at once: one is not finite if adding a one at its
// exponent's lowest bit carries into its (cleared) sign bit.
template <uint32_t E, uint32_t ONE>
__device__ __forceinline__ bool half_words_nonfinite(uint4 o) {
  constexpr uint32_t EE = E | E << 16, ONES = ONE | ONE << 16;
  const uint32_t c = (((o.x & EE) + ONES) | ((o.y & EE) + ONES)) | (((o.z & EE) + ONES) | ((o.w & EE) + ONES));
  return (c & 0x80008000u) != 0;
}
template <> __device__ __forceinline__ bool packed_nonfinite<f16>(uint4 o) {
  return half_words_nonfinite<0x7c00u, 0x0400u>(o);
}
template <> __device__ __forceinline__ bool packed_nonfinite<bf16>(uint4 o) {
  return half_words_nonfinite<0x7f80u, 0x0080u>(o);
}

// The vector with the elements from nv < VE on replaced by `fill`: what lies
// behind a row's end takes no part and needs no test later.
template <typename T>
__device__ __forceinline__ uint4 fill_tail(uint4 raw, int nv, float fill) {
  float v[Vec<T>::N];
  unpack<T>(raw, v);
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) v[i] = i < nv ? v[i] : fill;
  return pack<T>(v);                                 // the others as they were: exact
}
template <typename T>
__device__ __forceinline__ uint4 load_row(const T* row, int c0, int C, float fill) {
  uint4 raw = ldg16(row + (c0 < C ? c0 : 0));
  if (C - c0 < Vec<T>::N) raw = fill_tail<T>(raw, C - c0, fill);
  return raw;
}
}  // namespace gcn
