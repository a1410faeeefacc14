// Labels drawn from the rows' own distributions under temperature, top-k,
// top-p and min-p, from given uniform numbers.
//
// The classes of a row are ordered by falling score, the lower class first
// among equals; each filter keeps a prefix of that order, so what is kept is a
// prefix too and is described by a key, and by how many classes of exactly
// that key belong to it (the lowest ones).  The drawn class is the first kept
// one, in class order, at which the running sum of the weights
// w_c = exp((z_c - max z) / T) passes u times their sum.
#include <algorithm>

#include "internal.h"
#include "lanes.h"
#include "rows.h"
#include "sorted.h"

namespace gcn {

namespace {

// The weights in 64 bits, each sum in a fixed order, for a row taken by NW
// waves.  The borders of top-k and top-p are found by bisection of the key:
// every step counts (or sums) the classes whose key lies in half of what is
// left.
template <typename T, int NW>
struct ExactRow {
  const SampleParams& p;
  const T* __restrict__ z;
  double* shd;        // [NW] shared
  int64_t* shi;       // [NW] shared
  uint32_t* shu;      // [NW] shared
  float zmax;
  static constexpr int NT = 64 * NW;

  __device__ int tid() const { return NW == 1 ? threadIdx.x & 63 : threadIdx.x; }
  __device__ double weight(float v) const { return exp(((double)v - (double)zmax) / p.T); }

  // Classes with lo < key <= hi.
  __device__ int64_t count(uint32_t lo, uint32_t hi) const {
    int64_t m = 0;
    for (int64_t c = tid(); c < p.C; c += NT) {
      const uint32_t key = score_key(to_f32<T>(z[c]));
      m += key > lo && key <= hi ? 1 : 0;
    }
    return block_reduce<NW>(m, shi, AddF());
  }
  // Their weights.
  __device__ double mass(uint32_t lo, uint32_t hi) const {
    double m = 0;
    for (int64_t c = tid(); c < p.C; c += NT) {
      const float v = to_f32<T>(z[c]);
      const uint32_t key = score_key(v);
      if (key > lo && key <= hi) m += weight(v);
    }
    return block_reduce<NW>(m, shd, AddF());
  }

  // Draws for a row whose maximum is finite and whose scores are not NaN.
  __device__ void draw(float u, int32_t* label, float* prob) {
    const uint32_t top = score_key(zmax);
    uint32_t border = KEY_NEG_INF + 1;   // smallest key kept
    int64_t take = p.C;                  // classes of that key kept
    if (p.top_k < p.C) {
      // the largest key that at least top_k classes reach; with fewer finite
      // scores than top_k every one is kept
      if (count(KEY_NEG_INF, top) > p.top_k) {
        uint32_t lo = KEY_NEG_INF + 1, hi = top;
        int64_t above = 0;               // classes with key > hi
        while (lo < hi) {
          const uint32_t mid = lo + (hi - lo) / 2;
          const int64_t m = count(mid, hi);
          if (above + m >= p.top_k) lo = mid + 1;
          else { hi = mid; above += m; }
        }
        border = lo;
        take = p.top_k - above;
      }
    }
    if (p.top_p < 1.0) {
      const int64_t here = count(border - 1, border);
      const int64_t avail = take < here ? take : here;
      const double w_border = weight(key_score(border));
      const double kept = mass(border, top) + (double)avail * w_border;
      const double want = p.top_p * kept;
      // the largest key whose classes, and those above, reach `want`
      uint32_t lo = border, hi = top;
      double above = 0;                  // weight of the keys > hi
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const double m = mass(mid, hi);
        if (above + m >= want) lo = mid + 1;
        else { hi = mid; above += m; }
      }
      const int64_t ties = lo == border ? avail : count(lo - 1, lo);
      double r = ceil((want - above) / weight(key_score(lo)));
      r = r < 1.0 ? 1.0 : r;
      border = lo;
      take = r < (double)ties ? (int64_t)r : ties;
    }
    // each wave owns a range of classes; how many classes of the border's key
    // come before it, then the weight it keeps
    const int lane = threadIdx.x & 63;
    const int wave = NW == 1 ? 0 : threadIdx.x >> 6;
    const int64_t per = (p.C + NT - 1) / NT * 64;
    const int64_t c0 = wave * per, c1 = c0 + per < p.C ? c0 + per : p.C;
    int64_t t = 0;
    for (int64_t c = c0 + lane; c < c1; c += 64) t += score_key(to_f32<T>(z[c])) == border ? 1 : 0;
    t = block_reduce<1>(t, (int64_t*)nullptr, AddF());
    int64_t rank = 0;
    if constexpr (NW > 1) {
      if (lane == 0) shi[wave] = t;
      __syncthreads();
      for (int i = 0; i < wave; ++i) rank += shi[i];
      __syncthreads();
    }
    double run = 0, before = 0, total = 0;
    int64_t last = -1;                   // last class kept in this wave's range
    for (int pass = 0; pass < 2; ++pass) {
      int64_t rk = rank;
      double at = before;
      for (int64_t b = c0; b < c1; b += 64) {
        const int64_t c = b + lane;
        const float v = c < c1 ? to_f32<T>(z[c]) : -INFINITY;
        const uint32_t key = score_key(v);
        const uint64_t tie = __ballot(c < c1 && key == border);
        const int64_t my = rk + __popcll(tie & ((1ull << lane) - 1));
        rk += __popcll(tie);
        const double x = ((double)v - (double)zmax) / p.T;
        const bool kept = c < c1 && (key > border || (key == border && my < take)) && x >= p.ln_min_p;
        const double w = kept ? exp(x) : 0.0;
        const double s = wave_scan(w);
        if (pass == 0) {
          const uint64_t k = __ballot(w > 0.0);
          if (k) last = b + 63 - __clzll(k);
        } else {
          const uint64_t hit = __ballot(w > 0.0 && at + s > (double)u * total);
          if (hit || (last >= b && last < b + 64)) {
            const int64_t c = hit ? b + __ffsll((unsigned long long)hit) - 1 : last;
            if (lane == (int)(c - b)) {
              *label = (int32_t)c;
              if (prob) *prob = (float)(w / total);
            }
            return;
          }
        }
        at += __shfl(s, 63);
      }
      if (pass == 0) {
        run = at;
        total = run;
        if constexpr (NW > 1) {
          if (lane == 0) { shd[wave] = run; shi[wave] = last; }
          __syncthreads();
          total = 0;
          int owner = -1, last_kept = 0;
          for (int i = 0; i < NW; ++i) total += shd[i];
          double acc = 0;
          for (int i = 0; i < NW; ++i) {
            if (shi[i] >= 0) last_kept = i;
            if (owner < 0 && shi[i] >= 0 && acc + shd[i] > (double)u * total) owner = i;
            if (i < wave) before += shd[i];
            acc += shd[i];
          }
          if (owner < 0) owner = last_kept;
          __syncthreads();
          if (owner != wave) return;
        }
      }
    }
  }
};

// ------------------------------------------------ rows in lane groups ----
//
// A group of LPR lanes holds a row, VE classes a lane.  With top-k or top-p the
// row's items are sorted over the group (sorted.h): the weights in that order
// and their running sum give the number of classes kept, and the last kept
// item the border.  The draw then runs over the classes in their own order.
//
// Weights and sums are in 32 bits (W = float); a border is believed only where
// no running sum lies within DRAW_EPS of it.  With e = 2^-24: a weight's
// exponent x = (z - max) log2(e) / T carries 3 e |x| (difference, constant,
// product), so a sum S of weights is off by at most S (3 e ln C / ln 2 + 4 e)
// with the base-2 exponential's 4 e (the mean of |x| under the weights is at
// most log2 C), its VE + 6 adds by (VE + 6) e, and p S or u S by 2 e: below
// 2^-18 S for C <= 512.  Where one does, W = double settles it, for the wave:
// about one wave in a thousand for 64 classes a row.
constexpr float DRAW_EPS = 3.814697265625e-6f;           // 2^-18

template <typename W> struct Draw;
template <> struct Draw<float> {
  static __device__ __forceinline__ float weight(float z, float zmax, const SampleParams& p) {
    return __builtin_amdgcn_exp2f((z - zmax) * p.k);
  }
  static constexpr float EPS = DRAW_EPS;
};
template <> struct Draw<double> {
  static __device__ __forceinline__ double weight(float z, float zmax, const SampleParams& p) {
    return exp(((double)z - (double)zmax) / p.T);
  }
  static constexpr double EPS = 0.0;
};

// The smallest score that min-p keeps.  (double)z >= max + T ln(min_p) holds
// for the same 32-bit z as z >= the bound rounded up to 32 bits.
__device__ __forceinline__ float least_kept(const SampleParams& p, float zmax) {
  const double b = (double)zmax + p.T * p.ln_min_p;
  float f = (float)b;
  if ((double)f < b) f = nextafterf(f, INFINITY);
  return f;
}

// The draw of a group's row.  a: the row's items in class order, s: sorted
// (with FILTER).  Returns whether the answer is certain.
template <typename W, typename T, int LPR, bool FILTER, typename I, int VE>
__device__ __forceinline__ bool group_draw(const SampleParams& p, const I (&a)[VE], const I (&s)[VE], int li, float zmax,
                                           float u, int32_t& label, float& prob) {
  typedef Draw<W> D;
  const int col0 = li * VE;
  bool sure = true;
  I border{0};
  if constexpr (FILTER) {
    W w[VE], sum = 0;
    int n = 0;                                           // this lane's classes under top-k
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const bool in = item_present<T>(s[i]) && col0 + i < p.top_k;
      w[i] = in ? D::weight(to_f32<T>(item_score<T>(s[i])), zmax, p) : W(0);
      sum += w[i];
      n += in ? 1 : 0;
    }
    int m;
    if (p.top_p < 1.0) {
      const W total = group_sum<LPR>(sum);
      W run = group_sum_before<LPR>(sum, li);
      const W want = (W)p.top_p * total;
      const W lo = want - D::EPS * total, hi = want + D::EPS * total;
      int n_lo = 0, n_hi = 0;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const bool in = i < n;                           // what is in comes first
        n_lo += in && run < lo ? 1 : 0;
        n_hi += in && run < hi ? 1 : 0;
        run += w[i];
      }
      const int both = group_sum<LPR>(n_lo | n_hi << 16);
      m = both & 0xffff;
      sure = m == both >> 16 && m > 0;
    } else {
      m = group_sum<LPR>(n);
    }
    // the m-th item, from the lane that holds it
    I mine{0};
#pragma unroll
    for (int i = 0; i < VE; ++i) mine = item_pick(col0 + i == m - 1, s[i], mine);
    border = group_max_item<LPR>(mine);
  }
  const float zmin = least_kept(p, zmax);
  W w[VE], sum = 0;
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    const float z = to_f32<T>(item_score<T>(a[i]));
    const bool kept = item_present<T>(a[i]) && !item_above(border, a[i]) && z >= zmin;
    w[i] = kept ? D::weight(z, zmax, p) : W(0);
    sum += w[i];
  }
  const W total = group_sum<LPR>(sum);
  const W want = (W)u * total;
  const W lo = want - D::EPS * total, hi = want + D::EPS * total;
  W run = group_sum_before<LPR>(sum, li);
  int at;
  if constexpr (sizeof(W) == 4) {
    int n_lo = 0, n_hi = 0;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      run += w[i];
      n_lo += run <= lo ? 1 : 0;
      n_hi += run <= hi ? 1 : 0;
    }
    const int both = group_sum<LPR>(n_lo | n_hi << 16);
    at = both & 0xffff;
    sure &= at == both >> 16;
  } else {
    // the first kept class whose sum passes; the last kept one where rounding
    // leaves none
    int first = LPR * VE, last = -1;
#pragma unroll
    for (int i = VE - 1; i >= 0; --i) last = w[i] > 0 && last < 0 ? col0 + i : last;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      run += w[i];
      if (w[i] > 0 && run > want && first == LPR * VE) first = col0 + i;
    }
    first = -group_max_int<LPR>(-first);
    last = group_max_int<LPR>(last);
    at = first < last ? first : last;
  }
  W mine = 0;
#pragma unroll
  for (int i = 0; i < VE; ++i) mine = col0 + i == at ? w[i] : mine;
  label = at;
  prob = (float)(group_sum<LPR>(mine) / total);
  return sure;
}

template <typename T, int LPR, int R, bool FILTER>
__global__ __launch_bounds__(256) void sample_group_kernel(SampleParams p) {
  constexpr int VE = Vec<T>::N;
  constexpr int RG = 4 * (64 / LPR);
  typedef typename ItemOf<T>::type I;
  const int lane = threadIdx.x & 63, li = lane % LPR;
  const int slot = (threadIdx.x >> 6) * (64 / LPR) + lane / LPR;
  const int col0 = li * VE;
  const bool col_ok = col0 < p.C;
  const int nv = (int)(p.C - col0 < VE ? (p.C - col0 > 0 ? p.C - col0 : 0) : VE);
  const T* __restrict__ logits = reinterpret_cast<const T*>(p.logits);
  bool report = false;
  for (int64_t first = (int64_t)blockIdx.x * (R * RG); first < p.n; first += (int64_t)gridDim.x * (R * RG)) {
    uint4 raw[R];
    float us[R];
    bool on[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * RG + slot;
      on[r] = row < p.n && (!p.mask || p.mask[row] != 0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * RG + slot;
      raw[r] = make_uint4(0, 0, 0, 0);
      us[r] = 0.f;
      if (on[r]) {                                       // rows left out are not read
        raw[r] = ldg16(logits + row * p.ld + (col_ok ? col0 : 0));
        if (!p.greedy) us[r] = p.u[row];
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!__ballot(on[r])) continue;
      const int64_t row = first + r * RG + slot;
      I a[VE], s[VE];
      const bool bad = group_any<LPR>(make_items<T>(raw[r], col0, nv, a)) || !(us[r] >= 0.f && us[r] < 1.f);
      I top{0};
#pragma unroll
      for (int i = 0; i < VE; ++i) top = item_max(top, s[i] = a[i]);
      if constexpr (FILTER) group_sort<LPR, VE>(s, li);
      top = group_max_item<LPR>(top);
      const bool none = bad || !item_present<T>(top);
      const float zmax = none ? 0.f : to_f32<T>(item_score<T>(top));
      int32_t label;
      float prob;
      const bool sure = group_draw<float, T, LPR, FILTER>(p, a, s, li, zmax, us[r], label, prob);
      if (__ballot(on[r] && !none && !sure)) {
        int32_t l2;
        float p2;
        group_draw<double, T, LPR, FILTER>(p, a, s, li, zmax, us[r], l2, p2);
        if (!sure) { label = l2; prob = p2; }
      }
      if (on[r] && li == 0) {
        p.labels[row] = none ? -1 : label;
        if (p.prob) p.prob[row] = none ? 0.f : prob;
        report |= bad;
      }
    }
  }
  if (report) raise_flag(p.flag);
}

template <typename T>
__global__ __launch_bounds__(256) void sample_exact_kernel(SampleParams p) {
  __shared__ double shd[4];
  __shared__ int64_t shi[4];
  __shared__ uint32_t shu[4];
  const int64_t row = blockIdx.x;
  if (p.mask && p.mask[row] == 0) return;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  float mx = -INFINITY;
  bool bad = false;
  for (int64_t c = threadIdx.x; c < p.C; c += 256) {
    const float v = to_f32<T>(z[c]);
    bad |= !(v < INFINITY);
    mx = v > mx ? v : mx;
  }
  const float u = p.greedy ? 0.f : p.u[row];
  bad = __syncthreads_or(bad) || !(u >= 0.f && u < 1.f);
  const float zmax = block_reduce<4>(mx, reinterpret_cast<float*>(shu), MaxF());
  int32_t* label = p.labels + row;
  float* prob = p.prob ? p.prob + row : nullptr;
  if (bad || zmax == -INFINITY) {
    if (threadIdx.x == 0) {
      *label = -1;
      if (prob) *prob = 0.f;
      if (bad) raise_flag(p.flag);
    }
    return;
  }
  ExactRow<T, 4> r{p, z, shd, shi, shu, zmax};
  r.draw(u, label, prob);
}

// ------------------------------------------------------------- launches ----

constexpr int64_t MAX_BLOCKS = 65536;
constexpr int64_t R4_GROUPS = 16384;      // 4 rows a group and iteration from this many workgroups on

template <typename T, int LPR, bool FILTER>
hipError_t launch_filter(const SampleParams& p, hipStream_t s) {
  constexpr int64_t RG = 4 * (64 / LPR);
  const int r = (p.n + RG - 1) / RG > R4_GROUPS ? 4 : 1;
  const int64_t nb = std::min<int64_t>((p.n + r * RG - 1) / (r * RG), MAX_BLOCKS);
  if (r == 4)
    hipLaunchKernelGGL((sample_group_kernel<T, LPR, 4, FILTER>), dim3((unsigned)nb), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((sample_group_kernel<T, LPR, 1, FILTER>), dim3((unsigned)nb), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_lpr(const SampleParams& p, hipStream_t s) {
  return p.top_k < p.C || p.top_p < 1.0 ? launch_filter<T, LPR, true>(p, s) : launch_filter<T, LPR, false>(p, s);
}
template <typename T>
hipError_t launch_t(const SampleParams& p, hipStream_t s) {
  const int64_t nvec = (p.C + Vec<T>::N - 1) / Vec<T>::N;
  if (nvec <= 1) return launch_lpr<T, 1>(p, s);
  if (nvec <= 2) return launch_lpr<T, 2>(p, s);
  if (nvec <= 4) return launch_lpr<T, 4>(p, s);
  if (nvec <= 8) return launch_lpr<T, 8>(p, s);
  if (nvec <= 16) return launch_lpr<T, 16>(p, s);
  if (nvec <= 32) return launch_lpr<T, 32>(p, s);
  if (nvec <= 64) return launch_lpr<T, 64>(p, s);
  hipLaunchKernelGGL((sample_exact_kernel<T>), dim3((unsigned)p.n), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int, int64_t, int64_t) { return 256; }

hipError_t sample_launch(int prec, const SampleParams& p, void*, hipStream_t s) {
  switch (prec) {
    case 0: return launch_t<float>(p, s);
    case 1: return launch_t<f16>(p, s);
    case 2: return launch_t<bf16>(p, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace gcn
