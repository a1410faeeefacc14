// Products C = A B^T of two row-major operands whose rows are contracted (both
// contiguous along k): the matrix instructions of each storage type and a plain
// tiled loop for any sizes.
//
// The instructions are given B's rows as their first operand and A's as their
// second, so that a lane ends with four consecutive columns of one row of C.
#pragma once

#include "common.h"

namespace gcn {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// One step of 64 bytes along k: 16 rows of B (lane l: row l % 16, bytes
// 16 (l / 16) ..) times 16 rows of A.  D: column 4 (lane / 16) + v, row lane % 16.
template <typename T> struct NtMfma;
template <> struct NtMfma<int8_t> {
  typedef i32x4 Acc;
  static constexpr int BYTES = 1;
  static __device__ __forceinline__ Acc run(uint4 b, uint4 a, Acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), c, 0, 0, 0);
  }
};
template <> struct NtMfma<f16> {
  typedef f32x4 Acc;
  static constexpr int BYTES = 2;
  static __device__ __forceinline__ Acc run(uint4 b, uint4 a, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
  }
};
template <> struct NtMfma<bf16> {
  typedef f32x4 Acc;
  static constexpr int BYTES = 2;
  static __device__ __forceinline__ Acc run(uint4 b, uint4 a, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
  }
};
template <> struct NtMfma<float> {
  typedef f32x4 Acc;
  static constexpr int BYTES = 4;
  static __device__ __forceinline__ Acc run(uint4 b, uint4 a, Acc c) {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.x), __uint_as_float(a.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.y), __uint_as_float(a.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.z), __uint_as_float(a.z), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.w), __uint_as_float(a.w), c, 0, 0, 0);
    return c;
  }
};

// The first nb bytes of a vector, the others 0.
__device__ __forceinline__ uint4 keep_bytes(uint4 x, int nb) {
  auto m = [&](int w) -> uint32_t {
    const int left = nb - 4 * w;
    return left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1;
  };
  return make_uint4(x.x & m(0), x.y & m(1), x.z & m(2), x.w & m(3));
}

// Four consecutive elements of a row, rounded to T; true if one is not finite.
template <typename T>
__device__ __forceinline__ bool store4(T* dst, const float (&z)[4]) {
  typedef T V4 __attribute__((ext_vector_type(4)));
  V4 v;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = from_f32<T>(z[i]);
    bad |= !finite_f32(to_f32<T>(v[i]));
  }
  *reinterpret_cast<V4*>(dst) = v;
  return bad;
}

constexpr int NT_B = 64;          // rows and columns of a workgroup's tile
struct NtOperands {
  const uint8_t* A; int64_t lda, n;     // lda, ldb in bytes (multiples of 16)
  const uint8_t* B; int64_t ldb, N;
  int64_t kbytes;                       // bytes contracted of each row; what follows is ignored
};

// The 64 x 64 tile at (row0, col0) by 2 x 2 waves; acc[i][j]: columns col0 + 32
// (wave % 2) + 16 i .., rows row0 + 32 (wave / 2) + 16 j ... lds: 16 KB.  Rows
// and columns outside the operands hold copies of their last ones.
template <typename T>
__device__ __forceinline__ void nt_tile(const NtOperands& p, int64_t row0, int64_t col0, uint8_t* lds,
                                        typename NtMfma<T>::Acc (&acc)[2][2]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int piece_row = (tid >> 6) * 16 + (tid & 15), off = ((tid >> 4) & 3) * 16;
  const uint8_t* a = p.A + min(row0 + piece_row, p.n - 1) * p.lda;
  const uint8_t* b = p.B + min(col0 + piece_row, p.N - 1) * p.ldb;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = typename NtMfma<T>::Acc{0, 0, 0, 0};
  auto load = [&](const uint8_t* row, int64_t k) {
    const int64_t at = k + off, left = p.kbytes - at;
    const uint4 v = ldg16(row + (left > 0 ? at : 0));
    return keep_bytes(v, left >= 16 ? 16 : left > 0 ? (int)left : 0);
  };
  uint4 va = load(a, 0), vb = load(b, 0);
  int st = 0;
  for (int64_t k = 0; k < p.kbytes; k += 64, st ^= 8192) {
    *reinterpret_cast<uint4*>(lds + st + tid * 16) = va;
    *reinterpret_cast<uint4*>(lds + st + 4096 + tid * 16) = vb;
    __syncthreads();
    if (k + 64 < p.kbytes) {
      va = load(a, k + 64);
      vb = load(b, k + 64);
    }
    uint4 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *reinterpret_cast<const uint4*>(lds + st + ((wave >> 1) * 2 + i) * 1024 + lane * 16);
      fb[i] = *reinterpret_cast<const uint4*>(lds + st + 4096 + ((wave & 1) * 2 + i) * 1024 + lane * 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = NtMfma<T>::run(fb[i], fa[j], acc[i][j]);
  }
  __syncthreads();      // the buffers are free again
}

}  // namespace gcn
