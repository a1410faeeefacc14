// Rows in 8 bits (format in gcn.h): scales, codes and what they stand for.
#pragma once

#include "common.h"

namespace gcn {

enum Q8Kind : int { Q8_SIGNED = 0, Q8_RELU = 1 };
template <int KIND> constexpr float q8_levels() { return KIND == Q8_RELU ? 255.f : 127.f; }

// The scale of a row whose largest value is a >= 0: a / levels cut off after 16
// significant bits, 2^-126 at the least.  The quotient is taken in fp32 and may
// miss the cut by one unit of the 16th bit; levels * c is exact (24 bits), so
// the right one is the largest c with levels * c <= a.
template <int KIND>
__device__ __forceinline__ float q8_scale(float a) {
  constexpr float L = q8_levels<KIND>();
  uint32_t c = __float_as_uint(a * (1.f / L)) & 0xffffff00u;
  if (c < 0x00800000u) c = 0x00800000u;                     // 2^-126: the smallest normal number
  if (c > 0x00800000u && L * __uint_as_float(c) > a) c -= 0x100u;
  else if (L * __uint_as_float(c + 0x100u) <= a) c += 0x100u;
  return __uint_as_float(c);
}

// h / s rounded to the nearest whole number, ties to even, from inv = about
// 1 / s.  The product h * inv may fall on the wrong side of a border: the
// remainder h - q s is exact (q s has 24 bits, and the difference is a multiple
// of s 2^-24 below s), so it decides.
__device__ __forceinline__ float q8_round(float h, float s, float inv) {
  float q = rintf(h * inv);
  const float r = fmaf(-q, s, h), d = fabsf(r) + fabsf(r);
  // past the border, or on it beside an odd number: one step towards h
  const bool odd = ((int)q & 1) != 0;
  if (d > s || (d == s && odd)) q += r > 0.f ? 1.f : -1.f;
  return q;
}

// The code of h as a whole number in fp32.
template <int KIND>
__device__ __forceinline__ float q8_code(float h, float s, float inv) {
  const float q = q8_round(h, s, inv);
  if (KIND == Q8_SIGNED) return q;
  return h > 0.f ? fmaxf(q, 1.f) : 0.f;
}

// The four codes of a dword as numbers.
template <int KIND>
__device__ __forceinline__ void q8_unpack4(uint32_t w, float (&q)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    q[i] = KIND == Q8_RELU ? (float)((w >> (8 * i)) & 0xffu) : (float)((int32_t)(w << (24 - 8 * i)) >> 24);
}

}  // namespace gcn
