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

// A result is (sum * a) * row scale * b for a column's scale a b: b is 1 but for
// scales above 2^96, where it is 2^32, so that no product on the way leaves the
// fp32 range where the result is inside it: a sum has at most 31 bits, and
// scales are 2^-126 or more.
struct Factors { float a, b; };
__device__ __forceinline__ Factors factors(float s) {
  const bool large = s > 0x1p96f;
  return Factors{large ? s * 0x1p-32f : s, large ? 0x1p32f : 1.f};
}

// Columns are dealt to 16-column operands in pairs (16-bit results) or one by
// one (fp32), so that a lane ends with 16 bytes of a row: operand i of a group's
// FI, row m holds column XE (m / 4) + 4 i + m % 4 of the group's 16 FI.
template <typename T> struct Deal {
  static constexpr int FI = sizeof(T) == 2 ? 2 : 1, XE = 4 * FI;
  static __device__ __forceinline__ int column(int tile, int m) {
    return tile / FI * (16 * FI) + XE * (m >> 2) + 4 * (tile % FI) + (m & 3);
  }
};

// The smallest size that T rounds to infinity.
template <typename T> __device__ __forceinline__ float too_large() { return __builtin_inff(); }
template <> __device__ __forceinline__ float too_large<f16>() { return 65520.f; }
template <> __device__ __forceinline__ float too_large<bf16>() { return __uint_as_float(0x7f7f8000u); }

// A wave's 16 rows of 16 NT results on their way out.  They pass through LDS, in
// 16-byte parts whose places change with the row (for the banks), so that each
// store covers whole lines of them: stored as the matrix instructions leave them,
// neighbouring lanes in different rows, 2^21 x 128 by 128 took 180 us instead of
// 152 (fp32 348 instead of 254).
template <typename T, int NT>
struct ResultRows {
  static constexpr int XE = Deal<T>::XE, PARTS = NT * (int)sizeof(T), BYTES = 16 * PARTS * 16;
  uint8_t* stage;
  int lane;
  float most = 0.f;                                        // the largest size of any result
  // Lanes read what others of their wave wrote, and then write over it.
  static __device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  __device__ __forceinline__ ResultRows(uint8_t* s, int l) : stage(s), lane(l) {}
  // Group q's XE columns of this lane's row, of which `left` are columns of S;
  // the others are padding: 0.
  __device__ __forceinline__ void put(int q, float (&z)[XE], int left, int strip = 0) {
    if (left < XE) {
#pragma unroll
      for (int e = 0; e < XE; ++e) z[e] = e < left ? z[e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < XE; ++e) most = fmaxf(most, fabsf(z[e]));
    const int row = lane & 15;
    stg16(stage + strip * BYTES + (row * PARTS + ((q * 4 + (lane >> 4)) ^ (row & (PARTS - 1)))) * 16, pack<T>(z));
  }
  // The rows from row0 on, 16 a strip; those past the last one are copies of it.
  template <int STRIPS = 1>
  __device__ __forceinline__ void store(const ProductQ8Params& p, int64_t row0, int64_t col0) {
    constexpr int RPS = 64 / PARTS;                        // rows of a store
    const int row = lane / PARTS, part = lane % PARTS;
    const int64_t c = col0 + part * Vec<T>::N;
    const bool all = row0 + 16 * STRIPS <= p.n, here = c < p.N;
    T* dst = static_cast<T*>(p.S) + (all ? row0 + row : 0) * p.ld_s + c;
    lanes_meet();
#pragma unroll
    for (int k = 0; k < 16 * STRIPS / RPS; ++k) {
      const int rk = row + k * RPS;
      const uint4 v = ldg16(stage + (rk * PARTS + (part ^ (rk & 15 & (PARTS - 1)))) * 16);   // row & 15 of its strip
      T* at = all ? dst + k * RPS * p.ld_s : dst + min(row0 + rk, p.n - 1) * p.ld_s;
      if (here) stg16(at, v);
    }
    lanes_meet();
  }
};

// 16-column operands whose results leave together in the kernel below: a line of
// 128 bytes of each row.
template <typename T, int NT>
constexpr int ROW_NT = NT * sizeof(T) < 8 ? NT : 8 / (int)sizeof(T);

// Many rows, weights that fit LDS.  A workgroup keeps 16 NT columns of the
// weights in LDS in the order the matrix instructions take them, with zeros
// behind the last k, and their factors and first sums (128 times the columns'
// sums for ReLU codes) beside them; its waves walk 16 rows at a time, whose codes
// come straight into the second operand, GK steps of 64 bytes ahead.  Nothing is
// shared after the weights.  Bound by HBM, n (f_in + s f_out) bytes: 2^21 x 128 by
// 128 152 us in fp16 (5.3 TB/s), 254 in fp32.
template <typename T, int NT, int GK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void product_rows_kernel(ProductQ8Params p, int groups) {
  typedef Deal<T> D;
  constexpr int BN = 16 * NT;
  extern __shared__ __align__(16) uint8_t lds[];           // groups * GK * NT pieces of 1 KiB, then 3 BN words
  float* fa = reinterpret_cast<float*>(lds + (int64_t)groups * GK * NT * 1024);
  float* fb = fa + BN;
  int* first = reinterpret_cast<int*>(fb + BN);
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t col0 = (int64_t)blockIdx.y * BN;
  const uint32_t flip = p.relu ? 0x80808080u : 0u;
  bool bad = false, large = false;
  for (int pc = wave; pc < groups * GK * NT; pc += 4) {
    const int64_t c = col0 + D::column(pc % NT, l16), at = (int64_t)(pc / NT) * 64 + lg * 16, left = p.K - at;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (c < p.N && left > 0) v = keep_bytes(ldg16(p.Wq + c * p.ld_wq + at), left >= 16 ? 16 : (int)left);
    *reinterpret_cast<uint4*>(lds + pc * 1024 + lane * 16) = v;
  }
  if (threadIdx.x < BN) {
    const int64_t c = col0 + threadIdx.x;
    const float s = c < p.N ? p.w_scale[c] : 0.f;
    const Factors f = factors(s);
    fa[threadIdx.x] = f.a;
    fb[threadIdx.x] = f.b;
    first[threadIdx.x] = c < p.N && p.relu ? p.w_sum[c] * 128 : 0;
    bad |= !finite_f32(s);
    large = f.b != 1.f;
  }
  large = __syncthreads_or(large);

  const int64_t tiles = (p.n + 15) / 16, step = (int64_t)gridDim.x * 4;
  int64_t t = (int64_t)blockIdx.x * 4 + wave;
  uint4 a[2][GK];
  float rs[2];
  auto load = [&](uint4 (&x)[GK], float& s, int64_t tile, int g) {
    const int64_t r = min(tile * 16 + l16, p.n - 1);       // past the last row: read, not used
    const uint8_t* row = p.Hq + r * p.ld_q;
#pragma unroll
    for (int k = 0; k < GK; ++k) {
      const int64_t at = ((int64_t)g * GK + k) * 64 + lg * 16;
      x[k] = ldg16_nt(row + (at < p.K ? at : 0));          // past the last k the weights are 0
    }
    s = p.h_scale[r];
  };
  i32x4 acc[NT];
  auto clear = [&]() {                                     // 4 consecutive columns a tile and lane
#pragma unroll
    for (int i = 0; i < NT; ++i)
      acc[i] = *reinterpret_cast<const i32x4*>(first + i / D::FI * (16 * D::FI) + D::XE * lg + 4 * (i % D::FI));
  };
  auto multiply = [&](const uint4 (&x)[GK], int g) {
#pragma unroll
    for (int k = 0; k < GK; ++k) {
      const uint4 f = make_uint4(x[k].x ^ flip, x[k].y ^ flip, x[k].z ^ flip, x[k].w ^ flip);
      const uint8_t* w = lds + (int64_t)(g * GK + k) * NT * 1024 + lane * 16;
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i] = NtMfma<int8_t>::run(*reinterpret_cast<const uint4*>(w + i * 1024), f, acc[i]);
    }
  };
  typedef ResultRows<T, ROW_NT<T, NT>> Out;
  Out out(reinterpret_cast<uint8_t*>(first + BN) + wave * Out::BYTES, lane);
  const int left = (int)min(p.N - col0 - D::XE * lg, (int64_t)BN);
  auto finish = [&](int64_t tile, float s) {               // lanes past the last row hold it again
    bad |= !finite_f32(s);
#pragma unroll
    for (int q = 0; q < NT / D::FI; ++q) {
      constexpr int GROUPS = ROW_NT<T, NT> / D::FI;        // that go out together
      const int c = q * 16 * D::FI + D::XE * lg;
      float z[D::XE];
#pragma unroll
      for (int e = 0; e < D::XE; ++e) z[e] = ((float)acc[q * D::FI + e / 4][e % 4] * fa[c + e]) * s;
      if (large) {
#pragma unroll
        for (int e = 0; e < D::XE; ++e) z[e] *= fb[c + e];
      }
      out.put(q % GROUPS, z, left - q * 16 * D::FI);
      if ((q + 1) % GROUPS == 0) out.store(p, tile * 16, col0 + (q + 1 - GROUPS) * 16 * D::FI);
    }
  };
  // the (tile, group) pairs in order, the next pair's codes on their way while
  // one is multiplied
  int g = 0, ga = 0;
  int64_t ta = t;
  auto ahead = [&](int i) {
    load(a[i], rs[i], ta, ga);
    if (++ga == groups) { ga = 0; ta += step; }
  };
  ahead(0);
  clear();
  while (t < tiles) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (t >= tiles) break;
      ahead(1 - i);
      multiply(a[i], g);
      if (++g == groups) {
        finish(t, rs[i]);
        clear();
        g = 0;
        t += step;
      }
    }
  }
  if (bad || out.most >= too_large<T>()) raise_flag(p.flag);
}

// Few rows: the weights are all there is to read.  A workgroup takes 16 FI
// columns and up to 16 RT rows; its eight waves split k (steps of 64 bytes in
// turn), and the sums meet in LDS, exact in any order.  One row by 2048 x 2048:
// 5.4 us (4.2 MB; in 64 x 64 tiles without the split 13).
constexpr int FEW_WAVES = 8;
template <typename T, int RT>
__global__ __launch_bounds__(64 * FEW_WAVES) void product_few_kernel(ProductQ8Params p) {
  typedef Deal<T> D;
  __shared__ int part[FEW_WAVES][D::FI * RT * 256];
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t col0 = (int64_t)blockIdx.x * 16 * D::FI, row0 = (int64_t)blockIdx.y * 16 * RT;
  const uint32_t flip = p.relu ? 0x80808080u : 0u;
  i32x4 acc[D::FI][RT];
#pragma unroll
  for (int i = 0; i < D::FI; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll 2
  for (int64_t k = (int64_t)wave * 64; k < p.K; k += 64 * FEW_WAVES) {
    const int64_t at = k + lg * 16, left = p.K - at, in = left > 0 ? at : 0;
    const int nb = left >= 16 ? 16 : left > 0 ? (int)left : 0;
    uint4 b[D::FI], a[RT];
#pragma unroll
    for (int i = 0; i < D::FI; ++i) b[i] = ldg16(p.Wq + min(col0 + D::column(i, l16), p.N - 1) * p.ld_wq + in);
#pragma unroll
    for (int j = 0; j < RT; ++j) a[j] = ldg16(p.Hq + min(row0 + j * 16 + l16, p.n - 1) * p.ld_q + in);
#pragma unroll
    for (int i = 0; i < D::FI; ++i) b[i] = keep_bytes(b[i], nb);
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      a[j] = make_uint4(a[j].x ^ flip, a[j].y ^ flip, a[j].z ^ flip, a[j].w ^ flip);
#pragma unroll
      for (int i = 0; i < D::FI; ++i) acc[i][j] = NtMfma<int8_t>::run(b[i], a[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < D::FI; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) *reinterpret_cast<i32x4*>(&part[wave][(j * D::FI + i) * 256 + lane * 4]) = acc[i][j];
  __syncthreads();
  if (wave >= RT) return;                                  // wave j finishes rows 16 j ..
  const int64_t r = row0 + wave * 16 + l16, c = col0 + D::XE * lg;
  if (r >= p.n || c >= p.N) return;
  int sum[D::XE] = {};
#pragma unroll
  for (int s = 0; s < FEW_WAVES; ++s)
#pragma unroll
    for (int i = 0; i < D::FI; ++i) {
      const i32x4 v = *reinterpret_cast<const i32x4*>(&part[s][(wave * D::FI + i) * 256 + lane * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[4 * i + e] += v[e];
    }
  const float s = p.h_scale[r];
  bool bad = !finite_f32(s);
  float most = 0.f, z[D::XE];
#pragma unroll
  for (int e = 0; e < D::XE; ++e) {
    const int64_t ce = min(c + e, p.N - 1);
    const float sc = p.w_scale[ce];
    const Factors f = factors(sc);
    bad |= !finite_f32(sc);
    z[e] = ((float)(sum[e] + (p.relu ? p.w_sum[ce] * 128 : 0)) * f.a) * s * f.b;
  }
#pragma unroll
  for (int e = 0; e < D::XE; ++e) {
    z[e] = c + e < p.N ? z[e] : 0.f;                       // padding
    most = fmaxf(most, fabsf(z[e]));
  }
  stg16(static_cast<T*>(p.S) + r * p.ld_s + c, pack<T>(z));
  if (bad || most >= too_large<T>()) raise_flag(p.flag);
}

// Many rows and wide weights: bound by the matrix cores.  A workgroup takes 32 TM
// rows x 32 TN columns, a wave (2 x 2 of them) 16 TM x 16 TN in accumulators;
// steps of 64 bytes of k lie in LDS in the order of the operands, S steps in a
// ring that loads straight from memory fill.  While a step is multiplied out of
// registers, the next one's operands are read from LDS into others and the step
// S ahead is requested, so neither latency is waited for.  One wave a SIMD with
// all its registers.  k past the last whole step is multiplied first, from
// masked loads: the sums are whole numbers, their order is free.
__device__ __forceinline__ void to_lds_1k(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds) : "memory", "m0");
}
constexpr int MM_STAGES = 4;
constexpr int64_t MM_MIN_STEPS = 8;

template <typename T, int TM, int TN>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, TM == 8 ? 1 : 2)))
void product_mm_kernel(ProductQ8Params p, int64_t tiles, int64_t per_xcd) {
  typedef Deal<T> D;
  constexpr int S = MM_STAGES, NP = 2 * (TM + TN), LPW = NP / 4;
  static_assert(LPW <= TM && TN <= TM && TN % D::FI == 0, "requests and operands spread over the TM operand rows");
  __shared__ __align__(1024) uint8_t ring[S * NP * 1024];
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // consecutive tiles, which share rows, on the same die
  const int64_t u = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (u >= tiles) return;
  const int64_t cb = (p.N + 32 * TN - 1) / (32 * TN);
  const int64_t row0 = u / cb * (32 * TM), col0 = u % cb * (32 * TN);
  const uint32_t ring0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;
  const uint32_t flip = p.relu ? 0x80808080u : 0u;
  // rows and columns past the last ones are copies of them, not stored
  auto row_of = [&](int piece, int m) { return p.Hq + min(row0 + piece * 16 + m, p.n - 1) * p.ld_q; };
  auto col_of = [&](int piece, int m) { return p.Wq + min(col0 + D::column(piece, m), p.N - 1) * p.ld_wq; };
  // a 1 KiB piece is 16 rows of 64 bytes, four neighbouring lanes to a row so that
  // their loads join; 16-byte part c of row m lies at c ^ (m / 4), so that 16 rows'
  // parts lie in different banks
  const int part = (lane & 3) ^ (lane >> 4);
  const uint8_t* src[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int pc = wave * LPW + j;
    src[j] = (pc < 2 * TM ? row_of(pc, lane >> 2) : col_of(pc - 2 * TM, lane >> 2)) + part * 16;
  }
  i32x4 acc[TM][TN];                                       // [rows][columns]
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  struct Fr { uint4 a[TM], b[TN]; };
  auto turn = [&](uint4 v) { return make_uint4(v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip); };
  const int nc = (int)(p.K / 64);
  if (p.K % 64) {                                          // the rest of k
    const int64_t at = (int64_t)nc * 64, left = p.K - at - lg * 16;
    const int nb = left >= 16 ? 16 : left > 0 ? (int)left : 0;
    const int64_t in = nb ? at + lg * 16 : 0;              // a row's first bytes where none are left
    Fr f;
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = turn(ldg16(row_of((wave >> 1) * TM + i, l16) + in));
#pragma unroll
    for (int j = 0; j < TN; ++j) f.b[j] = keep_bytes(ldg16(col_of((wave & 1) * TN + j, l16) + in), nb);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = NtMfma<int8_t>::run(f.b[j], f.a[i], acc[i][j]);
  }
  const int at = l16 * 64 + (lg ^ (l16 >> 2)) * 16;
  const uint8_t* afrag = ring + (wave >> 1) * TM * 1024 + at;
  const uint8_t* bfrag = ring + (2 * TM + (wave & 1) * TN) * 1024 + at;
  auto issue = [&](int j, int c, int stage) {              // past the last step: in bounds, not used
    const int cc = c < nc ? c : nc - 1;
    to_lds_1k(src[j] + cc * 64, ring0 + stage * (NP * 1024) + (wave * LPW + j) * 1024);
  };
  auto read_a = [&](Fr& f, int i, int stage) {
    f.a[i] = *reinterpret_cast<const uint4*>(afrag + stage * (NP * 1024) + i * 1024);
  };
  auto read_b = [&](Fr& f, int j, int stage) {
    f.b[j] = *reinterpret_cast<const uint4*>(bfrag + stage * (NP * 1024) + j * 1024);
  };
#define MM_FENCE() __builtin_amdgcn_sched_barrier(0)
  // every wave's requests but those of the newest `steps` steps have landed, and
  // every wave holds what it read from LDS so far
#define MM_LANDED(steps)                                                                     \
  do {                                                                                       \
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((steps) * LPW) : "memory");          \
    __builtin_amdgcn_s_barrier();                                                            \
    asm volatile("" ::: "memory");                                                           \
    MM_FENCE();                                                                              \
  } while (0)
  // step c is in F; step c + 1 (stage s1) goes to G, step c + S into the stage s0
  // that step c was read from.  Requests and LDS reads are issued one by one
  // between matrix instructions, whose 16 cycles hide them (32768 x 2048 by 2048
  // x 2048 159 us; before each row's eight instead, 165; with the codes' top bits
  // turned over where they are read, which waits for LDS, 204).
  auto step = [&](const Fr& F, Fr& G, int c, int s0, int s1) {
    MM_LANDED(S - 2);
    uint4 fa = turn(F.a[0]);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      uint4 after = fa;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        acc[i][j] = NtMfma<int8_t>::run(F.b[j], fa, acc[i][j]);
        if (j == 0 && i < LPW) issue(i, c + S, s0);
        if (j == 1) read_a(G, i, s1);
        if (j == 2 % TN && i < TN) read_b(G, i, s1);
        if (j == TN - 1 && i + 1 < TM) after = turn(F.a[i + 1]);
        MM_FENCE();
      }
      fa = after;
    }
  };
#pragma unroll
  for (int d = 0; d < S; ++d)
#pragma unroll
    for (int j = 0; j < LPW; ++j) issue(j, d, d);
  MM_LANDED(S - 1);
  Fr f0, f1;
  auto next = [](int s) { return s + 1 < S ? s + 1 : 0; };
  // an odd step is done first, so that nothing follows the loop, which runs at
  // least once (the launch sees to eight steps)
  int c = 0, s0 = 0;
  if (nc & 1) {
#pragma unroll
    for (int i = 0; i < TM; ++i) read_a(f1, i, 0);
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(f1, j, 0);
    step(f1, f0, 0, 0, 1);
    c = 1;
    s0 = 1;
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i) read_a(f0, i, 0);
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(f0, j, 0);
  }
  do {
    const int s1 = next(s0), s2 = next(s1);
    step(f0, f1, c, s0, s1);
    step(f1, f0, c + 1, s1, s2);
    s0 = s2;
    c += 2;
  } while (c < nc);
  MM_LANDED(0);                                            // the ring is free, no request is left
#undef MM_FENCE
#undef MM_LANDED

  constexpr int BN = 32 * TN;
  float* fa = reinterpret_cast<float*>(ring);
  float* fb = fa + BN;
  int* first = reinterpret_cast<int*>(fb + BN);
  bool bad = false, large = false;
  if (threadIdx.x < BN) {
    const int64_t c = min(col0 + threadIdx.x, p.N - 1);
    const float s = p.w_scale[c];
    const Factors f = factors(s);
    fa[threadIdx.x] = f.a;
    fb[threadIdx.x] = f.b;
    first[threadIdx.x] = p.relu ? p.w_sum[c] * 128 : 0;
    bad |= !finite_f32(s);
    large = f.b != 1.f;
  }
  float rs[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    rs[i] = p.h_scale[min(row0 + ((wave >> 1) * TM + i) * 16 + l16, p.n - 1)];
    bad |= !finite_f32(rs[i]);
  }
  large = __syncthreads_or(large);
  const int c0 = (wave & 1) * 16 * TN;                     // the wave's columns within the tile
  const int left = (int)min(p.N - col0 - c0 - D::XE * lg, (int64_t)BN);
  float most = 0.f;
  auto results = [&](int i, int q, float (&z)[D::XE]) {
    const int c = c0 + q * 16 * D::FI + D::XE * lg;
#pragma unroll
    for (int e = 0; e < D::XE; ++e) z[e] = ((float)(acc[i][q * D::FI + e / 4][e % 4] + first[c + e]) * fa[c + e]) * rs[i];
    if (large) {
#pragma unroll
      for (int e = 0; e < D::XE; ++e) z[e] *= fb[c + e];
    }
  };
  if constexpr (sizeof(T) == 4) {                          // 2^15 x 700 by 1000: 67 us, stored directly 99
    typedef ResultRows<T, TN> Out;
    constexpr int STRIPS = 2;
    static_assert(TM % STRIPS == 0 && 4 * STRIPS * Out::BYTES + 12 * BN <= S * NP * 1024, "the ring holds them");
    Out out(reinterpret_cast<uint8_t*>(first + BN) + wave * (STRIPS * Out::BYTES), lane);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int q = 0; q < TN / D::FI; ++q) {
        float z[D::XE];
        results(i, q, z);
        out.put(q, z, left - q * 16 * D::FI, i % STRIPS);
      }
      if ((i + 1) % STRIPS == 0) out.template store<STRIPS>(p, row0 + ((wave >> 1) * TM + i + 1 - STRIPS) * 16, col0 + c0);
    }
    most = out.most;
  } else {                                                 // 32768 x 2048 by 2048: 160 us, through LDS 165
    // lanes past the last row hold that row's results and store them again
    T* dst[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i)
      dst[i] = static_cast<T*>(p.S) + min(row0 + ((wave >> 1) * TM + i) * 16 + l16, p.n - 1) * p.ld_s + col0 + c0 + D::XE * lg;
#pragma unroll
    for (int q = 0; q < TN / D::FI; ++q) {
      const int lq = left - q * 16 * D::FI;
      if (lq <= 0) continue;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float z[D::XE];
        results(i, q, z);
        if (lq < D::XE) {
#pragma unroll
          for (int e = 0; e < D::XE; ++e) z[e] = e < lq ? z[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < D::XE; ++e) most = fmaxf(most, fabsf(z[e]));
        stg16(dst[i] + q * 16 * D::FI, pack<T>(z));
      }
    }
  }
  if (bad || most >= too_large<T>()) raise_flag(p.flag);
}

constexpr int64_t ROWS_OUT = 4 * 16 * 128;                 // bytes of LDS for four waves' results

template <typename T, int NT, int GK>
hipError_t rows_ntgk(const ProductQ8Params& p, int groups, int64_t wgs, hipStream_t s) {
  const size_t lds = (size_t)groups * GK * NT * 1024 + 16 * NT * 12 + ROWS_OUT;
  auto k = product_rows_kernel<T, NT, GK>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)wgs, (unsigned)((p.N + 16 * NT - 1) / (16 * NT)));
  hipLaunchKernelGGL(k, grid, dim3(256), lds, s, p, groups);
  return hipGetLastError();
}
template <typename T, int NT>
hipError_t rows_nt(const ProductQ8Params& p, int64_t wgs, hipStream_t s) {
  const int steps = (int)((p.K + 63) / 64);
  if (steps == 1) return rows_ntgk<T, NT, 1>(p, 1, wgs, s);
  if (steps == 2) return rows_ntgk<T, NT, 2>(p, 1, wgs, s);
  return rows_ntgk<T, NT, 4>(p, (steps + 3) / 4, wgs, s);
}

// 80 KB of LDS a workgroup at most, so that two share a compute unit.
bool rows_fit(int64_t bn, int64_t kb) { return bn * (kb + 12) + ROWS_OUT <= 80 * 1024; }

template <typename T, int TM, int TN>
hipError_t mm_t(const ProductQ8Params& p, hipStream_t s) {
  const int64_t tiles = (p.n + 32 * TM - 1) / (32 * TM) * ((p.N + 32 * TN - 1) / (32 * TN)), per_xcd = (tiles + XCDS - 1) / XCDS;
  hipLaunchKernelGGL((product_mm_kernel<T, TM, TN>), dim3((unsigned)(per_xcd * XCDS)), dim3(256), 0, s, p, tiles, per_xcd);
  return hipGetLastError();
}

// Which kernel, by price in microseconds.  Up to 64 rows: few.  Below eight steps
// of k: rows (any width's weights then fit LDS).  Otherwise the cheapest of
//  * mm: rounds of one tile a compute unit (tiles of 128 rows run two at a time
//    at half the pace each), each `step` for 64 bytes of k and `ends` for its
//    start and its results;
//  * rows: every column block reads all codes, from HBM or the caches alike at
//    4.6 TB/s with the results' writes, and fills LDS with its weights first;
//  * few: one round per 256 workgroups of 32 rows.
// Measured (us, with the call; few, rows, mm 256 x 256, 256 x 128, 128 x 128, 128
// x 64; fp16 results, ReLU codes, 2048 columns of H): 256 rows, 2048 columns of
// weights 11, 16, 31, 20, 14, 11; 2048 rows 70, 70, 31, 21, 16, 20; 8192 rows 279,
// 174, 42, 58, 58, 80; 32768 rows 1094, 658, 160, 231, 221, 311; 2^18 rows, 64
// columns of weights 316, 234, 139, 128, 132, 127; 32 columns -, 120, 129, 115,
// 116, 111; 32768 rows, 16 columns 21, 17, 37, 29, 20, 18.  512 columns of H, 2^18
// rows, 256 columns of weights -, 84, 89, 110, 112, 137; 128 columns -, 44, 81, 66,
// 64, 77.
struct MmTile { int rows, cols; double step, ends; };
constexpr MmTile MM_TILES[] = {{256, 256, 0.75, 14.0}, {256, 128, 0.55, 11.0}, {128, 128, 0.30, 4.0}, {128, 64, 0.22, 2.0}};

template <typename T>
hipError_t product_t(const ProductQ8Params& p, hipStream_t s) {
  constexpr int64_t WIDTH = 16 * Deal<T>::FI;              // columns of the narrowest block
  const int64_t steps = (p.K + 63) / 64, kb = steps <= 2 ? steps * 64 : (steps + 3) / 4 * 256;   // bytes of a column in LDS
  auto cut = [](int64_t x, int64_t by) { return (x + by - 1) / by; };
  // rows: the widest block that fits LDS, narrower where few rows leave compute units idle
  int64_t bn = WIDTH;
  while (bn < 128 && bn < p.N && rows_fit(2 * bn, kb)) bn *= 2;
  while (bn > WIDTH && cut(p.n, 64) * cut(p.N, bn) < 256) bn /= 2;
  const int64_t blocks = cut(p.N, bn);
  enum { ROWS = 4, FEW = 5 };
  int kind = p.n <= 64 ? FEW : ROWS;
  if (kind == ROWS && p.K >= 64 * MM_MIN_STEPS) {
    double best = rows_fit(bn, kb) ? (double)p.n * (double)(p.K * blocks + p.N * (int64_t)sizeof(T)) / 4.6e6 + (double)(bn * kb) / 1.6e4
                                   : 1e30;
    auto offer = [&](int k, double us) { if (us < best) { best = us; kind = k; } };
    offer(FEW, (double)cut(cut(p.N, WIDTH) * cut(p.n, 32), 256) * (0.11 * steps + 1.5));
    for (int i = 0; i < 4; ++i)
      offer(i, (double)cut(cut(p.n, MM_TILES[i].rows) * cut(p.N, MM_TILES[i].cols), 256) * (MM_TILES[i].step * steps + MM_TILES[i].ends));
  }
  switch (kind) {
    case 0: return mm_t<T, 8, 8>(p, s);
    case 1: return mm_t<T, 8, 4>(p, s);
    case 2: return mm_t<T, 4, 4>(p, s);
    case 3: return mm_t<T, 4, 2>(p, s);
    case FEW:
      if (p.n <= 16) hipLaunchKernelGGL((product_few_kernel<T, 1>), dim3((unsigned)cut(p.N, WIDTH)), dim3(64 * FEW_WAVES), 0, s, p);
      else hipLaunchKernelGGL((product_few_kernel<T, 2>), dim3((unsigned)cut(p.N, WIDTH), (unsigned)cut(p.n, 32)), dim3(64 * FEW_WAVES), 0, s, p);
      return hipGetLastError();
  }
  const int64_t wgs = std::min(cut(p.n, 64), std::max<int64_t>(32, 512 * (128 / bn) / blocks));
  if constexpr (WIDTH == 16)
    if (bn == 16) return rows_nt<T, 1>(p, wgs, s);
  if (bn == 32) return rows_nt<T, 2>(p, wgs, s);
  if (bn == 64) return rows_nt<T, 4>(p, wgs, s);
  return rows_nt<T, 8>(p, wgs, s);
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
