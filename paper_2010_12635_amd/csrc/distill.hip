// Distillation from a teacher's top scores: the loss of every row and its
// scaled gradient in one call.
//   x_c = (z_c - max z) / T,  s = sum exp x_c,        p_c = exp(x_c) / s
//   y_j = (t_j - max t) / T,  r = sum exp y_j,        q_j = exp(y_j) / r
//   KL = sum_j q_j (y_j - x_{c_j}) - ln r + ln s      (the q_j sum to 1)
//   d_c = p_c - sum of the q_j whose class is c
// Rows of up to 64 vectors of 16 bytes stay in the registers of a lane group
// (distill_group_kernel); longer rows are taken by a workgroup each.
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
// ONE: K <= LPR, an entry a lane at most, loaded with the row; else entries
// li, li + LPR, ... are read (from the caches) whenever they are needed.
template <typename T, int LPR, int R, bool ONE>
__global__ __launch_bounds__(256) void distill_group_kernel(DistillParams p) {
  constexpr int VE = Vec<T>::N;
  constexpr int G = 64 / LPR;
  constexpr int RG = 4 * G;                          // rows per workgroup and sub-step
  __shared__ float s_loss[RG];
  __shared__ __align__(16) float s_slot[RG][LPR * VE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane / LPR, li = lane % LPR;
  const int slot = wave * G + g;
  float* __restrict__ mine = s_slot[slot];
  const int col0 = li * VE;
  const bool col_ok = col0 < p.C;
  const int nv = (int)(p.C - col0 < VE ? (p.C - col0 > 0 ? p.C - col0 : 0) : VE);   // classes of this lane
  const T* __restrict__ logits = reinterpret_cast<const T*>(p.logits);
  float acc_loss = 0.f;
  float acc_cs[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) { acc_cs[i] = 0.f; mine[col0 + i] = 0.f; }
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
    int32_t cls[R];
    float tvs[R];
    bool on[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int64_t row = first + r * RG + slot;
      row = row < p.n ? row : p.n - 1;               // in bounds; not counted below
      raw[r] = ldg16(logits + row * p.ld + (col_ok ? col0 : 0));
      if (p.base) braw[r] = ldg16(reinterpret_cast<const T*>(p.base) + row * p.ld + (col_ok ? col0 : 0));
      on[r] = !p.mask || p.mask[row] != 0;
      if (ONE) entry(row, li < p.K ? li : 0, cls[r], tvs[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * RG + slot;
      const bool row_ok = row < p.n;
      const bool in = row_ok && on[r];
      // the teacher's side
      int32_t c1 = -1;
      float t1 = -INFINITY;
      float tmax = -INFINITY;
      bool some = false;
      if (ONE) {
        if (in && li < p.K) { c1 = cls[r]; t1 = tvs[r]; accept(c1, t1); }
        some = c1 >= 0;
        tmax = t1;
      } else if (in) {
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
      float e1 = 0.f;
      if (ONE) {
        e1 = c1 >= 0 ? __builtin_amdgcn_exp2f((t1 - tm) * k) : 0.f;
        er = e1;
        a = e1 > 0.f || e1 != e1 ? e1 * (t1 - tm) : 0.f;
        if (c1 >= 0) mine[c1] = __int_as_float(li + 1);
      } else if (counts) {
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
      if (ONE) {
        twice = c1 >= 0 && __float_as_int(mine[c1 >= 0 ? c1 : 0]) != li + 1;
      } else if (counts) {
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
        if (ONE) {
          if (c1 >= 0) mine[c1] = e1 * inv_er;
        } else if (counts) {
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
        stg16(reinterpret_cast<T*>(p.dlogits) + row * p.ld + col0, o);
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

// A workgroup owns a row; entry j belongs to thread j.
template <typename T>
__global__ __launch_bounds__(256) void distill_row_kernel(DistillParams p) {
  __shared__ float shf[4];
  __shared__ int32_t s_cls[GCN_MAX_TOP];
  __shared__ float s_q[GCN_MAX_TOP];
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  const T* base = p.base ? reinterpret_cast<const T*>(p.base) + row * p.ld : nullptr;
  T* d = p.dlogits ? reinterpret_cast<T*>(p.dlogits) + row * p.ld : nullptr;
  const float k = LOG2E * p.inv_T;
  // the teacher's entries: one a thread
  int32_t cls = -1;
  float tv = -INFINITY;
  const bool in_mask = !p.mask || p.mask[row] != 0;
  bool bad = false;
  if (in_mask && t < p.K) {
    cls = p.top_classes[row * p.ld_top + t];
    if (cls >= p.C) { cls = -1; bad = true; }
    if (cls >= 0) tv = load_as_f32(p.top_prec, p.top_values, row * p.ld_top + t);
    if (tv == -INFINITY) cls = -1;
  }
  const float tmax = block_reduce<4>(cls >= 0 ? tv : -INFINITY, shf, MaxF());
  const int any = __syncthreads_or(cls >= 0);
  if (!any) {                                        // nothing to learn from: the gradient is the base
    if (d)
      for (int64_t c = t; c < p.C; c += 256) d[c] = base ? base[c] : from_f32<T>(0.f);
    if (t == 0) p.part_loss[row] = 0.f;
    if (bad) raise_flag(p.flag);
    return;
  }
  const float y = cls >= 0 ? (tv - tmax) * p.inv_T : 0.f;
  const float ey = cls >= 0 ? __builtin_amdgcn_exp2f((tv - tmax) * k) : 0.f;
  const float r = block_reduce<4>(ey, shf, AddF());
  const float q = ey / r;
  if (t < p.K) { s_cls[t] = cls; s_q[t] = q; }
  float mx = -INFINITY;
  for (int64_t c = t; c < p.C; c += 256) {
    const float v = to_f32<T>(z[c]);
    mx = v > mx || v != v ? v : mx;
  }
  if (__syncthreads_or(mx != mx)) mx = NAN;
  mx = block_reduce<4>(mx, shf, MaxF());
  float se = 0.f;
  for (int64_t c = t; c < p.C; c += 256) se += __builtin_amdgcn_exp2f((to_f32<T>(z[c]) - mx) * k);
  se = block_reduce<4>(se, shf, AddF());
  // q (y - x) of this thread's entry; an entry of weight 0 adds nothing
  float zc = cls >= 0 ? to_f32<T>(z[cls]) : 0.f;
  const float kl_j = q > 0.f || q != q ? q * (y - (zc - mx) * p.inv_T) : 0.f;
  const float kl = block_reduce<4>(kl_j, shf, AddF()) - logf(r) + logf(se);
  if (t == 0) p.part_loss[row] = kl;
  if (!d) {
    if (bad) raise_flag(p.flag);
    return;
  }
  const float sc = p.scale * (p.loss_scale ? *p.loss_scale : 1.f);
  const float inv_se = 1.f / se;
  // the entry's own element, read before the row is written over (the base
  // may be the gradient's buffer)
  float own = 0.f;
  if (cls >= 0) {
    float qs = 0.f;
    for (int j = 0; j < p.K; ++j) qs += s_cls[j] == cls ? s_q[j] : 0.f;
    own = (__builtin_amdgcn_exp2f((zc - mx) * k) * inv_se - qs) * sc;
    if (base) own += to_f32<T>(base[cls]);
  }
  __syncthreads();
  for (int64_t c = t; c < p.C; c += 256) {
    float g = __builtin_amdgcn_exp2f((to_f32<T>(z[c]) - mx) * k) * inv_se * sc;
    if (base) g += to_f32<T>(base[c]);
    const T o = from_f32<T>(g);
    d[c] = o;
    bad |= !finite_f32(to_f32<T>(o));
  }
  __syncthreads();
  if (cls >= 0) {
    const T o = from_f32<T>(own);
    d[cls] = o;
    bad |= !finite_f32(to_f32<T>(o));
  }
  if (bad) raise_flag(p.flag);
}

__global__ __launch_bounds__(256) void distill_final_kernel(const float* __restrict__ part, int64_t nb, float scale,
                                                            float* loss, int32_t* flag) {
  __shared__ float sh[4];
  float a = 0.f;
  for (int64_t i = threadIdx.x; i < nb; i += 256) a += part[i];
  a = block_reduce<4>(a, sh, AddF());
  if (threadIdx.x == 0) {
    const float l = a * scale;
    *loss = l;
    if (!finite_f32(l)) raise_flag(flag);
  }
}

// Workgroups and rows per iteration as in the cross-entropy kernel: R = 4
// rows a group when one would give more than 16384 workgroups, and at most
// 65536 workgroups, each walking on.
constexpr int64_t R4_GROUPS = 16384, MAX_BLOCKS = 65536;

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
int rows_per_group(int64_t n, int64_t rg) { return (n + rg - 1) / rg > R4_GROUPS ? 4 : 1; }
int64_t group_blocks(int prec, int64_t n, int64_t C) {
  const int64_t rg = 4 * (64 / lanes_per_row(prec, C));
  return blocks_of(n, rows_per_group(n, rg) * rg);
}

template <typename T, int LPR, bool ONE>
hipError_t launch_one(const DistillParams& p, int64_t nb, hipStream_t s) {
  constexpr int64_t RG = 4 * (64 / LPR);
  if (rows_per_group(p.n, RG) == 4)
    hipLaunchKernelGGL((distill_group_kernel<T, LPR, 4, ONE>), dim3((unsigned)nb), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((distill_group_kernel<T, LPR, 1, ONE>), dim3((unsigned)nb), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_lpr(const DistillParams& p, int64_t nb, hipStream_t s) {
  return p.K <= LPR ? launch_one<T, LPR, true>(p, nb, s) : launch_one<T, LPR, false>(p, nb, s);
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

size_t up256(size_t b) { return (b + 255) & ~size_t(255); }
int64_t cs_ld(int64_t C) { return (C + 7) / 8 * 8; }

}  // namespace

bool distill_colsum_supported(int prec, int64_t C) { return in_group(prec, C); }

// Lane groups: [loss partials][column-sum partials (blocks x cs_ld)][their
// block sums].  Workgroup rows: a loss a row.
size_t distill_workspace_bytes(int prec, int64_t n, int64_t C, int64_t K) {
  if (!in_group(prec, C)) return up256((size_t)n * sizeof(float));
  const int64_t nb = group_blocks(prec, n, C);
  return up256((size_t)nb * sizeof(float)) + up256((size_t)nb * (size_t)cs_ld(C) * sizeof(float)) +
         up256((size_t)colsum_partials_floats(nb, cs_ld(C)) * sizeof(float));
}

// More column-sum partial rows than this are first summed in blocks of
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
    const dim3 grid((unsigned)p.n);
    if (prec == 0) hipLaunchKernelGGL((distill_row_kernel<float>), grid, dim3(256), 0, s, p);
    else if (prec == 1) hipLaunchKernelGGL((distill_row_kernel<f16>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((distill_row_kernel<bf16>), grid, dim3(256), 0, s, p);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(distill_final_kernel, dim3(1), dim3(256), 0, s, p.part_loss, nb, p.loss_factor, loss, p.flag);
  e = hipGetLastError();
  if (e != hipSuccess || !colsum) return e;
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
