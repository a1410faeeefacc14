// Distillation from a teacher's top scores: the loss of every row and its
// scaled gradient in one call.
//   x_c = (z_c - max z) / T,  s = sum exp x_c,        p_c = exp(x_c) / s
//   y_j = (t_j - max t) / T,  r = sum exp y_j,        q_j = exp(y_j) / r
//   KL = sum_j q_j (y_j - x_{c_j}) - ln r + ln s      (the q_j sum to 1)
//   d_c = p_c - sum of the q_j whose class is c
// Rows of up to 64 vectors of 16 bytes stay in the registers of a lane group
// (distill_group_kernel); longer rows are taken by a workgroup each, or in
// segments.
//
// Bound by the read of the scores (and the base) and the write of the gradient.
// Measured on MI355X, whole calls, against what a copy of as many bytes takes:
// 2^21 rows of 64 classes, fp16, 8 entries, with base and column sums 203 us
// (175); 2048 rows of 50001, bf16 111 us (79); 200000 rows of 40, fp32, with
// base and column sums 34 us (21); 12 rows of 131072, fp32 15 us, two of its
// three launches the segments' two passes.
#include "internal.h"
#include "lanes.h"
#include "rows.h"

namespace gcn {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float load_as_f32(int prec, const void* p, int64_t i) {
  if (prec == 0) return reinterpret_cast<const float*>(p)[i];
  if (prec == 1) return (float)reinterpret_cast<const f16*>(p)[i];
  return (float)reinterpret_cast<const bf16*>(p)[i];
}

// A group of LPR lanes owns a row, 16 bytes of classes a lane.  The entries'
// weights q_j are scattered into the group's line of shared memory, one float
// a class, from where each lane reads the classes it owns: a few shared-memory
// instructions instead of K comparisons for every class.  First every entry
// marks its class with its number; where an entry finds another's number the
// same class occurs twice, and one lane adds the row's weights in the order
// of the entries, so that the sum does not depend on timing.
// KPL > 0: K <= KPL LPR, entries li, li + LPR, ... of the row are held by lane
// li, loaded with the row; KPL = 0: they are read (from the caches) whenever
// they are needed.
template <typename T, int LPR, int R, int KPL>
__global__ __launch_bounds__(256) void distill_group_kernel(DistillParams p) {
  constexpr int VE = Vec<T>::N;
  constexpr int G = 64 / LPR;
  constexpr int RG = 4 * G;                          // rows per workgroup and sub-step
  __shared__ float s_loss[RG];
  __shared__ __align__(16) float s_slot[RG][LPR * VE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane / LPR, li = lane % LPR;
  const int slot = wave * G + g;
  float* mine = s_slot[slot];
  const int col0 = li * VE;
  const bool col_ok = col0 < p.C;
  const int nv = (int)(p.C - col0 < VE ? (p.C - col0 > 0 ? p.C - col0 : 0) : VE);   // classes of this lane
  const T* __restrict__ logits = reinterpret_cast<const T*>(p.logits);
  float acc_loss = 0.f;
  float acc_cs[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) { acc_cs[i] = 0.f; mine[col0 + i] = 0.f; }
  wave_sync();
  const float k = LOG2E * p.inv_T;
  const float sc = p.scale * (p.loss_scale ? *p.loss_scale : 1.f);
  bool bad = false;
  // class of entry j of a row (-1: none), its score, and whether it was refused
  auto entry = [&](int64_t row, int j, int32_t& c, float& tv) {
    c = p.top_classes[row * p.ld_top + j];
    tv = load_as_f32(p.top_prec, p.top_values, row * p.ld_top + j);
  };
  auto accept = [&](int32_t& c, float& tv) {
    if (c >= p.C) bad = true;
    if (c < 0 || c >= p.C || tv == -INFINITY) { c = -1; tv = -INFINITY; }
  };
  for (int64_t first = (int64_t)blockIdx.x * (R * RG); first < p.n; first += (int64_t)gridDim.x * (R * RG)) {
    uint4 raw[R], braw[R];
    constexpr int KE = KPL > 0 ? KPL : 1;
    int32_t cls[R][KE];
    float tvs[R][KE];
    bool on[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int64_t row = first + r * RG + slot;
      row = row < p.n ? row : p.n - 1;               // in bounds; not counted below
      raw[r] = ldg16(logits + row * p.ld + (col_ok ? col0 : 0));
      if (p.base) braw[r] = ldg16(reinterpret_cast<const T*>(p.base) + row * p.ld + (col_ok ? col0 : 0));
      on[r] = !p.mask || p.mask[row] != 0;
#pragma unroll
      for (int i = 0; i < KPL; ++i) entry(row, li + i * LPR < p.K ? li + i * LPR : 0, cls[r][i], tvs[r][i]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * RG + slot;
      const bool row_ok = row < p.n;
      const bool in = row_ok && on[r];
      // the teacher's side
      float tmax = -INFINITY;
      bool some = false;
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        if (in && li + i * LPR < p.K) accept(cls[r][i], tvs[r][i]);
        else { cls[r][i] = -1; tvs[r][i] = -INFINITY; }
        some |= cls[r][i] >= 0;
        tmax = tvs[r][i] > tmax || tvs[r][i] != tvs[r][i] ? tvs[r][i] : tmax;
      }
      if (KPL == 0 && in) {
        for (int j = li; j < p.K; j += LPR) {
          int32_t c; float tv;
          entry(row, j, c, tv);
          accept(c, tv);
          some |= c >= 0;
          tmax = tv > tmax || tv != tv ? tv : tmax;
        }
      }
      tmax = group_max<LPR>(tmax);
      const bool counts = group_any<LPR>(some);
      float er = 0.f, a = 0.f;                       // sum of exponentials, and of exponentials times y T
      const float tm = counts ? tmax : 0.f;
      float ej[KE];
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        const int32_t c = cls[r][i];
        const float y = tvs[r][i] - tm;
        ej[i] = c >= 0 ? __builtin_amdgcn_exp2f(y * k) : 0.f;
        er += ej[i];
        a += ej[i] > 0.f || ej[i] != ej[i] ? ej[i] * y : 0.f;
        if (c >= 0) mine[c] = __int_as_float(li + i * LPR + 1);
      }
      if (KPL == 0 && counts) {
        for (int j = li; j < p.K; j += LPR) {
          int32_t c; float tv;
          entry(row, j, c, tv);
          accept(c, tv);
          if (c < 0) continue;
          const float e = __builtin_amdgcn_exp2f((tv - tm) * k);
          er += e;
          a += e > 0.f || e != e ? e * (tv - tm) : 0.f;
          mine[c] = __int_as_float(j + 1);
        }
      }
      wave_sync();
      bool twice = false;
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        const int32_t c = cls[r][i];
        twice |= c >= 0 && __float_as_int(mine[c >= 0 ? c : 0]) != li + i * LPR + 1;
      }
      if (KPL == 0 && counts) {
        for (int j = li; j < p.K; j += LPR) {
          int32_t c; float tv;
          entry(row, j, c, tv);
          accept(c, tv);
          twice |= c >= 0 && __float_as_int(mine[c]) != j + 1;
        }
      }
      twice = group_any<LPR>(twice);
      er = group_sum<LPR>(er);
      const float inv_er = counts ? 1.f / er : 0.f;
      wave_sync();
      if (!twice) {
#pragma unroll
        for (int i = 0; i < KPL; ++i)
          if (cls[r][i] >= 0) mine[cls[r][i]] = ej[i] * inv_er;
        if (KPL == 0 && counts) {
          for (int j = li; j < p.K; j += LPR) {
            int32_t c; float tv;
            entry(row, j, c, tv);
            accept(c, tv);
            if (c >= 0) mine[c] = __builtin_amdgcn_exp2f((tv - tm) * k) * inv_er;
          }
        }
      } else if (li == 0) {
        for (int pass = 0; pass < 2; ++pass)
          for (int j = 0; j < p.K; ++j) {
            int32_t c; float tv;
            entry(row, j, c, tv);
            accept(c, tv);
            if (c < 0) continue;
            if (pass == 0) mine[c] = 0.f;
            else mine[c] += __builtin_amdgcn_exp2f((tv - tm) * k) * inv_er;
          }
      }
      wave_sync();
      float qs[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) { qs[i] = mine[col0 + i]; mine[col0 + i] = 0.f; }
      wave_sync();
      // the student's side
      float z[VE];
      unpack<T>(raw[r], z);
#pragma unroll
      for (int i = 0; i < VE; ++i) z[i] = i < nv ? z[i] : -INFINITY;
      float mx = z[0];
#pragma unroll
      for (int i = 1; i < VE; ++i) mx = fmaxf(mx, z[i]);
      mx = group_max<LPR>(mx);
      float ez[VE];
      float se = 0.f, b = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float x = z[i] - mx;
        ez[i] = i < nv ? __builtin_amdgcn_exp2f(x * k) : 0.f;
        se += ez[i];
        b += qs[i] > 0.f || qs[i] != qs[i] ? qs[i] * x : 0.f;
      }
      se = group_sum<LPR>(se);
      const float ab = group_sum<LPR>(a * inv_er - b);
      if (counts) acc_loss += ab * p.inv_T - logf(er) + logf(se);
      if (p.dlogits && row_ok && col_ok) {
        const float inv_se = 1.f / se;
        float d[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) d[i] = counts && i < nv ? (ez[i] * inv_se - qs[i]) * sc : 0.f;
        if (p.base) {
          float bv[VE];
          unpack<T>(braw[r], bv);
#pragma unroll
          for (int i = 0; i < VE; ++i) d[i] += i < nv ? bv[i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < VE; ++i) acc_cs[i] += d[i];
        const uint4 o = pack<T>(d);
        stg16_nt(reinterpret_cast<T*>(p.dlogits) + row * p.ld + col0, o);
        bad |= packed_nonfinite<T>(o);
      }
    }
  }
  if (bad) raise_flag(p.flag);
  if (li == 0) s_loss[slot] = acc_loss;
  if (p.part_cs) {
#pragma unroll
    for (int i = 0; i < VE; ++i) mine[col0 + i] = acc_cs[i];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float a = 0.f;
    for (int i = 0; i < RG; ++i) a += s_loss[i];
    p.part_loss[blockIdx.x] = a;
  }
  if (p.part_cs) {
    // the workgroup's column sums: its row slots added in slot order
    for (int c = threadIdx.x; c < p.C; c += 256) {
      float a = s_slot[0][c];
      for (int i = 1; i < RG; ++i) a += s_slot[i][c];
      p.part_cs[(int64_t)blockIdx.x * p.ldcs + c] = a;
    }
  }
}

// ---------------------------------------------------------- longer rows ----
//
// distill_row_kernel: a workgroup owns a row and holds it in its registers (NV
// vectors a thread): one read, one write.  Thread j has the teacher's entry j
// and writes its class after the row.
//
// distill_part_kernel and distill_segment_kernel: rows that do not fit, and
// rows too few to fill the chip, are cut into segments of `seg` vectors, a
// workgroup each: first every segment's maximum and sum of exponentials, then,
// from those of the whole row, its part of the gradient.

// With k = log2(e) / T powers are of 2: p_c = 2^((z_c - M) k) / S, M = max z.  The
// difference is taken before the product: z k could leave the range (the lowest
// finite number is a score), and M k rounded on its own would be off by more than
// the powers' own exponents where |M| / T is large.  In fp16 neither can happen far
// enough to matter (|z k| < 2^27): there the product is joined with the
// subtraction, M k rounded, in one instruction with the conversion, and what the
// rounding left, M k - fl(M k), at most 4 and exact, goes into a factor of the row
// (16384 rows of 4001 classes with base: 102 us instead of 106).
template <typename T>
struct Power {
  float m, k;
  __device__ __forceinline__ Power(float M, float k_) : m(M), k(k_) {}
  __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f((z - m) * k); }
  __device__ __forceinline__ float factor() const { return 1.f; }
};
template <>
struct Power<f16> {
  float mk, k, rest;
  __device__ __forceinline__ Power(float M, float k_) : mk(M * k_), k(k_), rest(fmaf(M, k_, -mk)) {}
  __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, k, -mk)); }
  __device__ __forceinline__ float factor() const { return __builtin_amdgcn_exp2f(-rest); }
};

// A reference m and a sum of powers 2^((z - m) k) relative to it (0 where m is
// -inf).
struct MaxSum { float m, s; };
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float k) {
  const float m = fmaxf(a.m, b.m);
  const float fa = a.m > -INFINITY ? __builtin_amdgcn_exp2f((a.m - m) * k) : 0.f;
  const float fb = b.m > -INFINITY ? __builtin_amdgcn_exp2f((b.m - m) * k) : 0.f;
  return {m, a.s * fa + b.s * fb};                   // a NaN stays in s
}
// All of the waves' parts at once: a power for each.
template <int N>
__device__ __forceinline__ MaxSum join_all(const MaxSum (&part)[N], float k) {
  float m = part[0].m;
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, part[i].m);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s += part[i].m > -INFINITY ? part[i].s * __builtin_amdgcn_exp2f((part[i].m - m) * k) : part[i].s * 0.f;
  return {m, s};
}
__device__ __forceinline__ MaxSum wave_join(MaxSum v, float k) {
  const float m = group_max<64>(v.m);
  v.s *= v.m > -INFINITY ? __builtin_amdgcn_exp2f((v.m - m) * k) : 0.f;
  return {m, group_sum<64>(v.s)};
}

template <typename T>
__device__ __forceinline__ float vector_max(uint4 raw) {
  float v[Vec<T>::N];
  unpack<T>(raw, v);
  float m = v[0];
#pragma unroll
  for (int i = 1; i < Vec<T>::N; ++i) m = fmaxf(m, v[i]);
  return m;
}
// Sum of 2^((z - M) k), without the factor; a lane that has seen only -inf takes
// M = 0.
template <typename T>
__device__ __forceinline__ float vector_sum(uint4 raw, Power<T> power) {
  float v[Vec<T>::N];
  unpack<T>(raw, v);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) s += power(v[i]);
  return s;
}
// Keeps the compiler from holding unpacked scores between two passes.
__device__ __forceinline__ void forget(uint4& r) {
  asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w));
}

// The teacher's entries of a workgroup's row: thread j has entry j, the first
// waves join their references and sums through shared memory, as the row's.
constexpr int TW = GCN_MAX_TOP / 64;
struct EntryTable {
  int32_t c[GCN_MAX_TOP];
  float q[GCN_MAX_TOP];
  MaxSum part[TW];
  float loss[TW];
  int some[TW];
};
template <typename T>
struct Entry {
  int32_t c;               // class, -1: none
  float t, z;              // the teacher's score, and the student's for the class

  // Returns whether the entry is refused.
  __device__ __forceinline__ bool load(const DistillParams& p, int64_t row, const T* __restrict__ zrow) {
    const int j = threadIdx.x;
    const bool in = j < p.K && (!p.mask || p.mask[row] != 0);
    c = -1;
    t = -INFINITY;
    z = 0.f;
    bool bad = false;
    if (in) {
      c = p.top_classes[row * p.ld_top + j];
      t = load_as_f32(p.top_prec, p.top_values, row * p.ld_top + j);
      bad = c >= p.C;
      if (c < 0 || bad || t == -INFINITY) { c = -1; t = -INFINITY; }
      if (c >= 0) z = to_f32<T>(zrow[c]);
    }
    return bad;
  }
  // To shared memory; a barrier later every thread may ask counts().
  __device__ __forceinline__ void share(EntryTable& tab, float k) const {
    const int w = threadIdx.x >> 6;
    if (w >= TW) return;
    const bool some = __ballot(c >= 0) != 0;
    const MaxSum a = wave_join(MaxSum{t, c < 0 ? 0.f : t == t ? 1.f : t}, k);   // absent: t = -inf
    if ((threadIdx.x & 63) == 0) { tab.part[w] = a; tab.some[w] = some ? 1 : 0; }
    tab.c[threadIdx.x] = c;
  }
  static __device__ __forceinline__ bool counts(const EntryTable& tab) {
    return (tab.some[0] | tab.some[1] | tab.some[2] | tab.some[3]) != 0;
  }
  // The weights, and the waves' parts of the row's loss, to shared memory.
  __device__ __forceinline__ void weigh(EntryTable& tab, MaxSum row, float k, float inv_T) const {
    const int w = threadIdx.x >> 6;
    if (w >= TW) return;
    const MaxSum r = join_all(tab.part, k);
    // Subtracted first, as in the sum: t k rounded on its own would be off by
    // 2^-24 t k, another amount in q than in the sum, and the q would not sum to
    // 1 (fp16 scores near 60000 at the lowest temperature: one entry's q was 16)
    const float y = (t - r.m) * k;                     // log2 of q r
    const float q = c >= 0 ? __builtin_amdgcn_exp2f(y) / r.s : 0.f;
    tab.q[threadIdx.x] = q;
    // T times the sum of q (ln q r - ln p s): an entry of weight 0 adds nothing
    const float a = q > 0.f || q != q ? q * ((t - r.m) - (z - row.m)) : 0.f;
    const float sum = group_sum<64>(a) * inv_T;
    if ((threadIdx.x & 63) == 0) tab.loss[w] = w == 0 ? sum - logf(r.s) + logf(row.s) : sum;
  }
  // After a barrier: the row's loss.
  static __device__ __forceinline__ float loss(const EntryTable& tab) {
    return (tab.loss[0] + tab.loss[1]) + (tab.loss[2] + tab.loss[3]);
  }
  // After the row is written: what the entry's class gets.
  __device__ __forceinline__ bool store(const DistillParams& p, const EntryTable& tab, T* d, float base, float M, float k,
                                        float inv_s, float sc) const {
    float qs = 0.f;
    for (int j = 0; j < p.K; ++j) qs += tab.c[j] == c ? tab.q[j] : 0.f;
    const T o = from_f32<T>((__builtin_amdgcn_exp2f((z - M) * k) * inv_s - qs) * sc + base);
    d[c] = o;
    return !finite_f32(to_f32<T>(o));
  }
};
static_assert(TW == 4, "the waves' parts are joined by hand");

// 2^((z - M) k) f, added to the base, of a vector from class c0 on; f holds the
// power's factor.  Returns whether an element is not finite.
template <typename T>
__device__ __forceinline__ bool store_gradient(T* d, const T* base, int c0, int C, uint4 raw, Power<T> power, float f) {
  constexpr int VE = Vec<T>::N;
  float g[VE], v[VE];
  unpack<T>(raw, v);
#pragma unroll
  for (int i = 0; i < VE; ++i) g[i] = power(v[i]) * f;
  if (base) {
    float bv[VE];
    unpack<T>(load_row(base, c0, C, 0.f), bv);
#pragma unroll
    for (int i = 0; i < VE; ++i) g[i] += bv[i];
  }
  const uint4 o = pack<T>(g);
  stg16_nt(d + c0, o);
  return packed_nonfinite<T>(o);
}
// The gradient of a row that is not counted.
template <typename T>
__device__ __forceinline__ bool store_base(T* d, const T* base, int c0, int C) {
  const uint4 o = base ? load_row(base, c0, C, 0.f) : make_uint4(0, 0, 0, 0);
  stg16(d + c0, o);
  return packed_nonfinite<T>(o);
}

// Four waves a SIMD: one row's loads and stores under another's arithmetic.  2048
// rows of 50001 classes, bf16: 512 threads of 16 vectors 130 us, 1024 of 8 (two
// rows a compute unit at 64 registers, with spills) 149, 256 of 32 170, segments
// 146; with streaming stores 117, with the
// waves' parts joined by a power each instead of two 111.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_row_kernel(DistillParams p) {
  constexpr int VE = Vec<T>::N;
  constexpr int NW = NT / 64;
  __shared__ MaxSum s_part[NW];
  __shared__ EntryTable s_tab;
  const int64_t row = p.row0 + blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int C = (int)p.C;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  const T* base = p.base ? reinterpret_cast<const T*>(p.base) + row * p.ld : nullptr;
  T* d = p.dlogits ? reinterpret_cast<T*>(p.dlogits) + row * p.ld : nullptr;
  const float k = LOG2E * p.inv_T;
  uint4 raw[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) raw[v] = load_row(z, (v * NT + t) * VE, C, -INFINITY);
  Entry<T> e;
  bool bad = e.load(p, row, z);
  // read before the row is written over (the base may be the gradient's buffer)
  const float base_c = base && e.c >= 0 ? to_f32<T>(base[e.c]) : 0.f;
  e.share(s_tab, k);
  MaxSum mine{-INFINITY, 0.f};
#pragma unroll
  for (int v = 0; v < NV; ++v) mine.m = fmaxf(mine.m, vector_max<T>(raw[v]));
  const Power<T> own(mine.m > -INFINITY ? mine.m : 0.f, k);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    forget(raw[v]);
    mine.s += vector_sum<T>(raw[v], own);
    forget(raw[v]);
  }
  mine.s *= own.factor();
  mine = wave_join(mine, k);
  if (lane == 0) s_part[wave] = mine;
  __syncthreads();
  const MaxSum all = join_all(s_part, k);
  const bool counts = e.counts(s_tab);
  e.weigh(s_tab, all, k, p.inv_T);
  const float sc = p.scale * (p.loss_scale ? *p.loss_scale : 1.f);
  const float inv_s = 1.f / all.s;
  if (d) {
    const Power<T> power(all.m, k);
    const float f = inv_s * sc * power.factor();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c0 = (v * NT + t) * VE;
      if (c0 >= C) break;
      bad |= counts ? store_gradient(d, base, c0, C, raw[v], power, f) : store_base(d, base, c0, C);
    }
  }
  __syncthreads();                                   // the row is written, the weights known
  if (t == 0) p.part_loss[row] = counts ? e.loss(s_tab) : 0.f;
  if (d && e.c >= 0) bad |= e.store(p, s_tab, d, base_c, all.m, k, inv_s, sc);
  if (bad) raise_flag(p.flag);
}

// Segments: workgroup (row, s) = (row0 + blockIdx.x / segs, blockIdx.x % segs).
struct Segment {
  int64_t row;
  int s, lo, hi;                                     // vectors [lo, hi)
  __device__ __forceinline__ Segment(const DistillParams& p, int VE)
      : row(p.row0 + blockIdx.x / p.segs), s((int)(blockIdx.x % p.segs)), lo(s * p.seg) {
    const int nvec = (int)((p.C + VE - 1) / VE);
    hi = lo + p.seg < nvec ? lo + p.seg : nvec;
  }
};

template <typename T>
__global__ __launch_bounds__(256) void distill_part_kernel(DistillParams p) {
  constexpr int VE = Vec<T>::N;
  __shared__ MaxSum s_part[4];
  const Segment g(p, VE);
  const int t = threadIdx.x;
  const int C = (int)p.C;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + g.row * p.ld;
  const float k = LOG2E * p.inv_T;
  MaxSum mine{-INFINITY, 0.f};
  for (int b = g.lo + t; b < g.hi; b += 4 * 256) {
    uint4 raw[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) raw[q] = load_row(z, b + q * 256 < g.hi ? (b + q * 256) * VE : C, C, -INFINITY);
    float m = vector_max<T>(raw[0]);
#pragma unroll
    for (int q = 1; q < 4; ++q) m = fmaxf(m, vector_max<T>(raw[q]));
    m = fmaxf(mine.m, m);
    const Power<T> power(m > -INFINITY ? m : 0.f, k);
    mine.s *= mine.m > -INFINITY ? __builtin_amdgcn_exp2f((mine.m - m) * k) : 1.f;
    mine.m = m;
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) s += vector_sum<T>(raw[q], power);
    mine.s += s * power.factor();
  }
  mine = wave_join(mine, k);
  if ((t & 63) == 0) s_part[t >> 6] = mine;
  __syncthreads();
  if (t == 0) reinterpret_cast<MaxSum*>(p.part_ms)[g.row * p.segs + g.s] = join_all(s_part, k);
}

template <typename T>
__global__ __launch_bounds__(256) void distill_segment_kernel(DistillParams p) {
  constexpr int VE = Vec<T>::N;
  __shared__ EntryTable s_tab;
  const Segment g(p, VE);
  const int t = threadIdx.x;
  const int C = (int)p.C;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + g.row * p.ld;
  const T* base = p.base ? reinterpret_cast<const T*>(p.base) + g.row * p.ld : nullptr;
  T* d = p.dlogits ? reinterpret_cast<T*>(p.dlogits) + g.row * p.ld : nullptr;
  const float k = LOG2E * p.inv_T;
  Entry<T> e;
  bool bad = e.load(p, g.row, z);
  const bool mine = e.c >= g.lo * VE && e.c < g.hi * VE;
  const float base_c = base && mine ? to_f32<T>(base[e.c]) : 0.f;
  e.share(s_tab, k);
  // the row's reference and sum, by every wave: its segments a lane each, in turn
  const MaxSum* part = reinterpret_cast<const MaxSum*>(p.part_ms) + g.row * p.segs;
  MaxSum all{-INFINITY, 0.f};
  for (int i = t & 63; i < p.segs; i += 64) all = join(all, part[i], k);
  all = wave_join(all, k);
  __syncthreads();                                   // the table is there, the base's entries are read
  const bool counts = e.counts(s_tab);
  e.weigh(s_tab, all, k, p.inv_T);
  const float sc = p.scale * (p.loss_scale ? *p.loss_scale : 1.f);
  const float inv_s = 1.f / all.s;
  if (d) {
    const Power<T> power(all.m, k);
    const float f = inv_s * sc * power.factor();
    for (int b = g.lo + t; b < g.hi; b += 4 * 256) {
      uint4 raw[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) raw[q] = load_row(z, b + q * 256 < g.hi ? (b + q * 256) * VE : C, C, -INFINITY);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c0 = (b + q * 256) * VE;
        if (b + q * 256 >= g.hi) continue;
        bad |= counts ? store_gradient(d, base, c0, C, raw[q], power, f) : store_base(d, base, c0, C);
      }
    }
  }
  __syncthreads();                                   // the segment is written, the weights known
  if (g.s == 0 && t == 0) p.part_loss[g.row] = counts ? e.loss(s_tab) : 0.f;
  if (d && mine) bad |= e.store(p, s_tab, d, base_c, all.m, k, inv_s, sc);
  if (bad) raise_flag(p.flag);
}

// Workgroup 0, the loss: thread t adds partials t, t + 1024, ... in that order
// (eight loads in flight), then the threads' sums are added in a fixed order.
// Workgroups b > 0 (few partials): the column sums of classes 64 (b - 1) on, 16
// threads a column; classes [C, ld) get 0.
__global__ __launch_bounds__(1024) void distill_final_kernel(const float* __restrict__ part, int64_t nb, float scale,
                                                             float* loss, int32_t* flag, const float* __restrict__ part_cs,
                                                             int64_t ldcs, int64_t C, int64_t ld, float* colsum) {
  __shared__ float sh[16];
  __shared__ float s_cs[16][64];
  if (blockIdx.x > 0) {
    const int col = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int64_t c = (int64_t)(blockIdx.x - 1) * 64 + col;
    float a = 0.f;
    if (c < C)
      for (int64_t i = g; i < nb; i += 16) a += part_cs[i * ldcs + c];
    s_cs[g][col] = a;
    __syncthreads();
    if (g == 0 && c < ld) {
      a = s_cs[0][col];
#pragma unroll
      for (int i = 1; i < 16; ++i) a += s_cs[i][col];
      colsum[c] = a;
      if (!finite_f32(a)) raise_flag(flag);
    }
    return;
  }
  float a = 0.f;
  for (int64_t i = threadIdx.x; i < nb; i += 8 * 1024) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = i + u * 1024 < nb ? part[i + u * 1024] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) a += v[u];
  }
  a = block_reduce<16>(a, sh, AddF());
  if (threadIdx.x == 0) {
    const float l = a * scale;
    *loss = l;
    if (!finite_f32(l)) raise_flag(flag);
  }
}

// Entries a lane holds: up to 4 (2^21 rows of 64 classes, 32 entries, fp16: 292 us,
// read again whenever needed about twice that).
// Rows a group takes per iteration: 2 when one would give more than 16384
// workgroups, and at most 65536 workgroups, each walking on.  Two and one, us: 2^21
// x 64 fp16 203 and 207 (four 214: fewer waves hold their registers), with 32
// entries 294 and 331, 2^18 x 512 222 and 240; with fewer workgroups 2^17 x 64 16.7
// and 15.9, 2^19 x 64 52.5 and 51.6, 200000 x 40 fp32 33 and 35.
constexpr int64_t R2_GROUPS = 16384, MAX_BLOCKS = 65536;

int vec_elems(int prec) { return prec == 0 ? 4 : 8; }
bool in_group(int prec, int64_t C) { return C <= 64 * vec_elems(prec); }
int lanes_per_row(int prec, int64_t C) {
  const int64_t nvec = (C + vec_elems(prec) - 1) / vec_elems(prec);
  int l = 1;
  while (l < nvec && l < 64) l <<= 1;
  return l;
}
int64_t blocks_of(int64_t n, int64_t rows) {
  const int64_t nb = (n + rows - 1) / rows;
  return nb < MAX_BLOCKS ? nb : MAX_BLOCKS;
}
int rows_per_group(int64_t n, int64_t rg) { return (n + rg - 1) / rg > R2_GROUPS ? 2 : 1; }
int64_t group_blocks(int prec, int64_t n, int64_t C) {
  const int64_t rg = 4 * (64 / lanes_per_row(prec, C));
  return blocks_of(n, rows_per_group(n, rg) * rg);
}

template <typename T, int LPR, int KPL>
hipError_t launch_one(const DistillParams& p, int64_t nb, hipStream_t s) {
  constexpr int64_t RG = 4 * (64 / LPR);
  if (rows_per_group(p.n, RG) == 2)
    hipLaunchKernelGGL((distill_group_kernel<T, LPR, 2, KPL>), dim3((unsigned)nb), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((distill_group_kernel<T, LPR, 1, KPL>), dim3((unsigned)nb), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_lpr(const DistillParams& p, int64_t nb, hipStream_t s) {
  if (p.K <= LPR) return launch_one<T, LPR, 1>(p, nb, s);
  if (p.K <= 2 * LPR) return launch_one<T, LPR, 2>(p, nb, s);
  if (p.K <= 4 * LPR) return launch_one<T, LPR, 4>(p, nb, s);
  return launch_one<T, LPR, 0>(p, nb, s);
}
template <typename T>
hipError_t launch_group(int lpr, const DistillParams& p, int64_t nb, hipStream_t s) {
  switch (lpr) {
    case 1: return launch_lpr<T, 1>(p, nb, s);
    case 2: return launch_lpr<T, 2>(p, nb, s);
    case 4: return launch_lpr<T, 4>(p, nb, s);
    case 8: return launch_lpr<T, 8>(p, nb, s);
    case 16: return launch_lpr<T, 16>(p, nb, s);
    case 32: return launch_lpr<T, 32>(p, nb, s);
    default: return launch_lpr<T, 64>(p, nb, s);
  }
}

// Long rows: a workgroup each where a row fits its registers (512 threads, 16
// vectors); rows longer than that, and rows of more than 32768 classes (16-bit) too
// few for most compute units, in segments of at least 1024 vectors (4 a thread),
// SEGMENT_GROUPS workgroups in all if the rows allow, and at most 8192 vectors each
// (12 rows of 131072 fp32 classes: a workgroup a row 220 us, segments 16.5 us).  A
// workgroup a row and segments, us: 4 x 9001 fp32 13.5 and 16.7, 64 x 32001 fp32
// 14.6 and 16.5, 64 x 30001 bf16 13.6 and 16.7, 64 x 50001 bf16 19.1 and 16.9, 128 x
// 50001 20.4 and 18.7, 192 x 50001 21.5 and 23.1, 4 x 60001 19.5 and 16.8.
constexpr int64_t ROW_VECS = 8192, ROW_CLASSES = 32768, SEG_VECS = 1024, ROW_WORKGROUPS = 192, SEGMENT_GROUPS = 512;
struct LongPlan { int segs, seg; };                  // segs = 0: a workgroup a row
LongPlan long_plan(int prec, int64_t n, int64_t C) {
  const int64_t nvec = (C + vec_elems(prec) - 1) / vec_elems(prec);
  if (nvec <= ROW_VECS && (C <= ROW_CLASSES || n >= ROW_WORKGROUPS)) return {0, 0};
  const int64_t want = (SEGMENT_GROUPS + n - 1) / n;
  const int64_t most = (nvec + SEG_VECS - 1) / SEG_VECS, least = (nvec + ROW_VECS - 1) / ROW_VECS;
  const int64_t segs = want > most ? most : want < least ? least : want;
  const int64_t seg = (nvec + segs - 1) / segs;
  return {(int)((nvec + seg - 1) / seg), (int)seg};
}

template <typename T>
hipError_t launch_rows(const DistillParams& params, hipStream_t s) {
  const int64_t nvec = (params.C + Vec<T>::N - 1) / Vec<T>::N;
  return launch_long_rows(params, params.segs > 0 ? params.segs : 1, [&](const DistillParams& p, int64_t rows) {
    if (p.segs == 0) {
      const dim3 grid((unsigned)rows);
      if (nvec <= 4 * 256) hipLaunchKernelGGL((distill_row_kernel<T, 256, 4>), grid, dim3(256), 0, s, p);
      else if (nvec <= 8 * 256) hipLaunchKernelGGL((distill_row_kernel<T, 256, 8>), grid, dim3(256), 0, s, p);
      else if (nvec <= 8 * 512) hipLaunchKernelGGL((distill_row_kernel<T, 512, 8>), grid, dim3(512), 0, s, p);
      else hipLaunchKernelGGL((distill_row_kernel<T, 512, 16>), grid, dim3(512), 0, s, p);
      return hipGetLastError();
    }
    const dim3 grid((unsigned)(rows * p.segs));
    hipLaunchKernelGGL((distill_part_kernel<T>), grid, dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((distill_segment_kernel<T>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
  });
}

size_t up256(size_t b) { return (b + 255) & ~size_t(255); }
int64_t cs_ld(int64_t C) { return (C + 7) / 8 * 8; }

}  // namespace

bool distill_colsum_supported(int prec, int64_t C) { return in_group(prec, C); }

// Lane groups: [loss partials][column-sum partials (blocks x cs_ld)][their
// block sums].  Longer rows: [a loss a row][a maximum and sum a
// segment].
size_t distill_workspace_bytes(int prec, int64_t n, int64_t C, int64_t K) {
  if (!in_group(prec, C))
    return up256((size_t)n * sizeof(float)) + up256((size_t)n * long_plan(prec, n, C).segs * sizeof(MaxSum));
  const int64_t nb = group_blocks(prec, n, C);
  return up256((size_t)nb * sizeof(float)) + up256((size_t)nb * (size_t)cs_ld(C) * sizeof(float)) +
         up256((size_t)colsum_partials_floats(nb, cs_ld(C)) * sizeof(float));
}

// Up to this many column-sum partial rows are added by the loss's last launch
// (16 rows at a time for a column: 32 rounds).
constexpr int64_t CS_TOGETHER = 512;
// More than this are first summed in blocks of
// consecutive rows, then the blocks' rows (as for the cross-entropy).
constexpr int64_t CS_ONE_STAGE = 4096;

hipError_t distill_launch(int prec, DistillParams p, float* loss, float* colsum, void* ws, hipStream_t s) {
  char* w = reinterpret_cast<char*>(ws);
  p.part_loss = reinterpret_cast<float*>(w);
  p.part_cs = nullptr;
  p.ldcs = cs_ld(p.C);
  hipError_t e;
  int64_t nb = p.n;
  float* cs_blocks = nullptr;
  if (in_group(prec, p.C)) {
    nb = group_blocks(prec, p.n, p.C);
    w += up256((size_t)nb * sizeof(float));
    if (colsum) p.part_cs = reinterpret_cast<float*>(w);
    w += up256((size_t)nb * (size_t)p.ldcs * sizeof(float));
    cs_blocks = reinterpret_cast<float*>(w);
    const int lpr = lanes_per_row(prec, p.C);
    e = prec == 0 ? launch_group<float>(lpr, p, nb, s)
                  : prec == 1 ? launch_group<f16>(lpr, p, nb, s) : launch_group<bf16>(lpr, p, nb, s);
  } else {
    const LongPlan lp = long_plan(prec, p.n, p.C);
    p.segs = lp.segs;
    p.seg = lp.seg;
    p.part_ms = w + up256((size_t)p.n * sizeof(float));
    e = prec == 0 ? launch_rows<float>(p, s) : prec == 1 ? launch_rows<f16>(p, s) : launch_rows<bf16>(p, s);
  }
  if (e != hipSuccess) return e;
  // few partials: the column sums in the launch that adds up the loss
  const bool together = colsum && nb <= CS_TOGETHER;
  hipLaunchKernelGGL(distill_final_kernel, dim3(together ? 1 + (unsigned)((p.ld + 63) / 64) : 1), dim3(1024), 0, s,
                     p.part_loss, nb, p.loss_factor, loss, p.flag, p.part_cs, p.ldcs, p.C, p.ld, colsum);
  e = hipGetLastError();
  if (e != hipSuccess || !colsum || together) return e;
  Epilogue eb{};
  eb.out = colsum; eb.ldo = p.ld; eb.rows = 1; eb.cols = p.C; eb.mode = EPI_F32; eb.flag = p.flag;
  eb.keep_scale = 1.f;
  if (nb <= CS_ONE_STAGE)
    return reduce_partials2(prec, make_job_ld(p.part_cs, (int)nb, 1, p.C, p.ldcs, eb), nullptr, s);
  int blocks = 0;
  e = colsum_partial_launch(0, p.part_cs, nb, p.C, p.ldcs, cs_blocks, p.ldcs, &blocks, s);
  if (e != hipSuccess) return e;
  return reduce_partials2(prec, make_job_ld(cs_blocks, blocks, 1, p.C, p.ldcs, eb), nullptr, s);
}

}  // namespace gcn
