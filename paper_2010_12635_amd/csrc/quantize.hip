// Rows in 8 bits: codes and scales of activations and weights, and back.
// The format's definition is in gcn.h.
#include "internal.h"
#include "lanes.h"
#include "q8.h"
#include "rows.h"

#include <algorithm>

namespace gcn {

namespace {

// Eight consecutive elements of a row, at column c0, as numbers; those past
// f count as 0.  ld % 8 == 0, so the whole group lies in the row.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ at, int64_t c0, int64_t f, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    unpack<float>(ldg16_nt(at), x);
    unpack<float>(ldg16_nt(at + 4), x + 4);
  } else {
    unpack<T>(ldg16_nt(at), x);
  }
  if (c0 + 8 > f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c0 + i < f ? x[i] : 0.f;
  }
}

// What the scale is taken from, as an integer that orders like it: the bits of
// the largest value (of |h|, or of h where that is positive), and from TOP_NAN on
// if any value is not finite.
constexpr int TOP_NAN = 0x7f800000;
template <int KIND>
__device__ __forceinline__ int top_of(const float (&x)[8]) {
  int most = 0, size = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int b = __float_as_int(x[i]);
    size = max(size, b & 0x7fffffff);
    if (KIND == Q8_RELU) most = max(most, b);
  }
  return KIND == Q8_SIGNED || size >= TOP_NAN ? size : most;
}

// Eight codes.  h * inv is rounded to a whole number by adding 1.5 2^23, whose
// low byte is then the code; inv is off by less than 2^-22 of itself, the product
// by less than 2^-14, so only a lane with a product that near to half takes the
// exact way (one row in sixteen of 512 values has one).
template <int KIND>
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float s, float inv) {
  constexpr float WHOLE = 12582912.f;                      // 1.5 2^23
  uint32_t q[8];
  float off = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float h = KIND == Q8_RELU ? fmaxf(x[i], 0.f) : x[i];
    float r = fmaf(h, inv, WHOLE);
    off = fmaxf(off, fabsf(fmaf(h, inv, WHOLE - r)));
    if (KIND == Q8_RELU) r = fmaxf(r, h > 0.f ? WHOLE + 1.f : WHOLE);
    q[i] = __float_as_uint(r);
  }
  if (off > 0.5f - 0x1p-13f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = (uint32_t)(int)q8_code<KIND>(x[i], s, inv);
  }
  auto bytes = [](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t b3) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b3, b2, 0x0c0c0400u), __builtin_amdgcn_perm(b1, b0, 0x0c0c0400u),
                                 0x05040100u);
  };
  return make_uint2(bytes(q[0], q[1], q[2], q[3]), bytes(q[4], q[5], q[6], q[7]));
}

struct QuantParams {
  int64_t n, f, ld, ld_q, row0;
  const void* H;
  uint8_t* Hq;
  float* scale;
  int32_t* flag;
};

template <int LPR>
__device__ __forceinline__ int group_max_i(int v) {
  if (LPR >= 2) v = max(v, dpp_i<DPP_XOR1>(v));
  if (LPR >= 4) v = max(v, dpp_i<DPP_XOR2>(v));
  if (LPR >= 8) v = max(v, dpp_i<DPP_HALF_MIRROR>(v));
  if (LPR >= 16) v = max(v, dpp_i<DPP_MIRROR>(v));
  if (LPR >= 32) v = max(v, __shfl_xor(v, 16));
  if (LPR >= 64) v = max(v, __shfl_xor(v, 32));
  return v;
}

// Rows of up to 8 LPR elements: LPR lanes a row, eight elements a lane, ROWS
// rows' loads on their way at a time.  Bound by HBM, n f (s + 1) bytes: 2^21 x 128
// fp16 163 us (4.9 TB/s), 16384 x 500 bf16 11.
constexpr int ROWS = 4;
template <typename T, int KIND, int LPR>
__global__ __launch_bounds__(256) void quantize_kernel(QuantParams p) {
  const int li = threadIdx.x % LPR;
  const int64_t rows = 256 / LPR, step = (int64_t)gridDim.x * rows;
  const int64_t c0 = (int64_t)li * 8;
  const bool here = c0 < p.f;
  const T* H = reinterpret_cast<const T*>(p.H) + (here ? c0 : 0);
  bool bad = false;
  for (int64_t r0 = (int64_t)blockIdx.x * rows + threadIdx.x / LPR; r0 < p.n; r0 += ROWS * step) {
    float x[ROWS][8];
#pragma unroll
    for (int k = 0; k < ROWS; ++k)                         // past the last row: it again, not stored
      load8<T>(H + min(r0 + k * step, p.n - 1) * p.ld, here ? c0 : 0, p.f, x[k]);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t r = r0 + k * step;
      const int top = group_max_i<LPR>(top_of<KIND>(x[k]));
      const bool fin = top < TOP_NAN;
      const float s = q8_scale<KIND>(__int_as_float(fin ? top : 0)), inv = __builtin_amdgcn_rcpf(s);
      const uint2 w = codes8<KIND>(x[k], s, inv);
      if (r < p.n) {
        if (here) *reinterpret_cast<uint2*>(p.Hq + r * p.ld_q + c0) = fin ? w : make_uint2(0, 0);
        if (li == 0) p.scale[r] = fin ? s : __int_as_float(0x7fc00000);
        bad |= !fin;
      }
    }
  }
  if (bad) raise_flag(p.flag);
}

// Longer rows, a workgroup each: read once for the scale, again (from the caches)
// for the codes.  All 256 threads run for as many as the row's eighths need: 2^18
// x 600 fp16 276 us, of them 175 of vector instructions (93 at a copy's rate), 2^15
// x 4096 fp16 106 (79), fp32 212 (132), 16384 x 1433 fp16 27 (14).
template <typename T, int KIND>
__global__ __launch_bounds__(256) void quantize_long_kernel(QuantParams p) {
  __shared__ int sh[4];
  const int64_t r = p.row0 + blockIdx.x;
  const T* row = reinterpret_cast<const T*>(p.H) + r * p.ld;
  int top = 0;
  for (int64_t c0 = (int64_t)threadIdx.x * 8; c0 < p.f; c0 += 2048) {
    float x[8];
    load8<T>(row + c0, c0, p.f, x);
    top = max(top, top_of<KIND>(x));
  }
  top = block_reduce<4>(top, sh, MaxF());
  const bool fin = top < TOP_NAN;
  const float s = q8_scale<KIND>(__int_as_float(fin ? top : 0)), inv = __builtin_amdgcn_rcpf(s);
  for (int64_t c0 = (int64_t)threadIdx.x * 8; c0 < p.f; c0 += 2048) {
    float x[8];
    load8<T>(row + c0, c0, p.f, x);
    const uint2 w = codes8<KIND>(x, s, inv);
    *reinterpret_cast<uint2*>(p.Hq + r * p.ld_q + c0) = fin ? w : make_uint2(0, 0);
  }
  if (threadIdx.x == 0) {
    p.scale[r] = fin ? s : __int_as_float(0x7fc00000);
    if (!fin) raise_flag(p.flag);
  }
}

unsigned few(int64_t blocks) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(blocks, 8192)); }

template <typename T, int KIND>
hipError_t quantize_t(const QuantParams& p, hipStream_t s) {
  const int64_t u = (p.f + 7) / 8;
#define GCN_Q(LPR)                                                                                             \
  if (u <= LPR) {                                                                                              \
    hipLaunchKernelGGL((quantize_kernel<T, KIND, LPR>), dim3(few((p.n * LPR + 256 * ROWS - 1) / (256 * ROWS))), dim3(256), 0, s, p); \
    return hipGetLastError();                                                                                  \
  }
  GCN_Q(1) GCN_Q(2) GCN_Q(4) GCN_Q(8) GCN_Q(16) GCN_Q(32) GCN_Q(64)
#undef GCN_Q
  return launch_long_rows(p, 1, [&](const QuantParams& q, int64_t rows) {
    hipLaunchKernelGGL((quantize_long_kernel<T, KIND>), dim3((unsigned)rows), dim3(256), 0, s, q);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t quantize_k(int kind, const QuantParams& p, hipStream_t s) {
  return kind == Q8_RELU ? quantize_t<T, Q8_RELU>(p, s) : quantize_t<T, Q8_SIGNED>(p, s);
}

// Eight elements a thread.  Bound by HBM: 2^21 x 128 fp16 165 us (4.9 TB/s), 2^15 x
// 4096 74 (5.5); fp32, four fifths of it writes, 2^15 x 4096 181 (3.7).
template <typename T, int KIND>
__global__ __launch_bounds__(256) void dequantize_kernel(int64_t n, int64_t f, const uint8_t* __restrict__ Hq,
                                                         int64_t ld_q, const float* __restrict__ scale,
                                                         T* __restrict__ H, int64_t ld, int32_t* flag) {
  const int64_t upr = (f + 7) >> 3, total = n * upr;
  bool bad = false;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / upr, c0 = (i - r * upr) << 3;
    const uint2 w = *reinterpret_cast<const uint2*>(Hq + r * ld_q + c0);
    const float s = scale[r];
    float q[2][4], x[8];
    q8_unpack4<KIND>(w.x, q[0]);
    q8_unpack4<KIND>(w.y, q[1]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = c0 + k < f ? to_f32<T>(from_f32<T>(q[k >> 2][k & 3] * s)) : 0.f;
      bad |= !finite_f32(x[k]);
    }
    T* dst = H + r * ld + c0;
    if constexpr (sizeof(T) == 4) {
      stg16(dst, pack<float>(x));
      stg16(dst + 4, pack<float>(x + 4));
    } else {
      stg16(dst, pack<T>(x));
    }
  }
  if (bad) raise_flag(flag);
}

template <typename T>
hipError_t dequantize_t(int64_t n, int64_t f, int kind, const void* Hq, int64_t ld_q, const float* scale, void* H,
                        int64_t ld, int32_t* flag, hipStream_t s) {
  const dim3 grid(few((n * ((f + 7) / 8) + 255) / 256));
  auto k = kind == Q8_RELU ? dequantize_kernel<T, Q8_RELU> : dequantize_kernel<T, Q8_SIGNED>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, n, f, static_cast<const uint8_t*>(Hq), ld_q, scale, static_cast<T*>(H),
                     ld, flag);
  return hipGetLastError();
}

// Weights: a workgroup takes 16 columns of W (16 threads along them, 16 along
// the rows), finds their scales in one pass and turns blocks of 256 rows round
// through LDS in a second one, which finds them in L2.  Once for all products with
// the weights, so it is kept simple; bound by the waits of each workgroup for its
// own rows, 16 at a time: 500 x 64 bf16 12 us, 2048 x 2048 97, 2048 x 16 fp16 43,
// 65536 x 16 1326.
template <typename T>
__global__ __launch_bounds__(256) void quantize_weights_kernel(int64_t f_in, int64_t f_out, const T* __restrict__ W,
                                                               int64_t ld_w, uint8_t* __restrict__ Wq, int64_t ld_wq,
                                                               float* __restrict__ scale, int32_t* __restrict__ sum,
                                                               int32_t* flag) {
  __shared__ int tops[16][17];
  __shared__ __align__(16) uint8_t codes[16][256 + 16];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t j = (int64_t)blockIdx.x * 16 + c, jc = j < f_out ? j : f_out - 1;
  int top = 0;
  for (int64_t k = r; k < f_in; k += 16) {
    const int b = __float_as_int(to_f32<T>(W[k * ld_w + jc])) & 0x7fffffff;
    top = max(top, b);
  }
  tops[r][c] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, tops[i][c]);
  const bool fin = top < TOP_NAN;
  const float s = q8_scale<Q8_SIGNED>(__int_as_float(fin ? top : 0)), inv = __builtin_amdgcn_rcpf(s);
  const int64_t f16 = (f_in + 15) / 16 * 16;               // written with zeros up to here; ld_wq % 16 == 0
  int total = 0;
  for (int64_t k0 = 0; k0 < f16; k0 += 256) {
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int64_t k = k0 + i * 16 + r;
      int q = 0;
      if (k < f_in && fin) q = (int)q8_round(to_f32<T>(W[k * ld_w + jc]), s, inv);
      total += q;
      codes[c][i * 16 + r] = (uint8_t)q;
    }
    __syncthreads();
    // thread t stores 16 codes of column t / 16
    const int64_t jo = (int64_t)blockIdx.x * 16 + r, ko = k0 + c * 16;
    if (jo < f_out && ko < f16)
      stg16(Wq + jo * ld_wq + ko, *reinterpret_cast<const uint4*>(&codes[r][c * 16]));
    __syncthreads();
  }
  tops[r][c] = total;
  __syncthreads();
  if (r == 0 && j < f_out) {
    int t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += tops[i][c];
    sum[j] = t;
    scale[j] = fin ? s : __int_as_float(0x7fc00000);
    if (!fin) raise_flag(flag);
  }
}

template <typename T>
hipError_t quantize_weights_t(int64_t f_in, int64_t f_out, const void* W, int64_t ld_w, void* Wq, int64_t ld_wq,
                              float* scale, int32_t* sum, int32_t* flag, hipStream_t s) {
  hipLaunchKernelGGL((quantize_weights_kernel<T>), dim3((unsigned)((f_out + 15) / 16)), dim3(256), 0, s, f_in, f_out,
                     static_cast<const T*>(W), ld_w, static_cast<uint8_t*>(Wq), ld_wq, scale, sum, flag);
  return hipGetLastError();
}

}  // namespace

hipError_t quantize_launch(int prec, int kind, int64_t n, int64_t f, const void* H, int64_t ld, void* Hq, int64_t ld_q,
                           float* scale, int32_t* flag, hipStream_t s) {
  QuantParams p{n, f, ld, ld_q, 0, H, static_cast<uint8_t*>(Hq), scale, flag};
  switch (prec) {
    case 0: return quantize_k<float>(kind, p, s);
    case 1: return quantize_k<f16>(kind, p, s);
    case 2: return quantize_k<bf16>(kind, p, s);
  }
  return hipErrorInvalidValue;
}

hipError_t dequantize_launch(int prec, int kind, int64_t n, int64_t f, const void* Hq, int64_t ld_q, const float* scale,
                             void* H, int64_t ld, int32_t* flag, hipStream_t s) {
  switch (prec) {
    case 0: return dequantize_t<float>(n, f, kind, Hq, ld_q, scale, H, ld, flag, s);
    case 1: return dequantize_t<f16>(n, f, kind, Hq, ld_q, scale, H, ld, flag, s);
    case 2: return dequantize_t<bf16>(n, f, kind, Hq, ld_q, scale, H, ld, flag, s);
  }
  return hipErrorInvalidValue;
}

hipError_t quantize_weights_launch(int prec, int64_t f_in, int64_t f_out, const void* W, int64_t ld_w, void* Wq,
                                   int64_t ld_wq, float* scale, int32_t* sum, int32_t* flag, hipStream_t s) {
  switch (prec) {
    case 0: return quantize_weights_t<float>(f_in, f_out, W, ld_w, Wq, ld_wq, scale, sum, flag, s);
    case 1: return quantize_weights_t<f16>(f_in, f_out, W, ld_w, Wq, ld_wq, scale, sum, flag, s);
    case 2: return quantize_weights_t<bf16>(f_in, f_out, W, ld_w, Wq, ld_wq, scale, sum, flag, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace gcn
