// Labels drawn from the rows' own distributions under temperature, top-k,
// top-p and min-p, from given uniform numbers.
//
// The classes of a row are ordered by falling score, the lower class first
// among equals; each filter keeps a prefix of that order, so what is kept is a
// prefix too and is described by a key, and by how many classes of exactly
// that key belong to it (the lowest ones).  The drawn class is the first kept
// one, in class order, at which the running sum of the weights
// w_c = exp((z_c - max z) / T) passes u times their sum.
#include "internal.h"
#include "lanes.h"
#include "rows.h"

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

template <typename T>
__global__ __launch_bounds__(256) void sample_exact_kernel(SampleParams p) {
  __shared__ double shd[4];
  __shared__ int64_t shi[4];
  __shared__ uint32_t shu[4];
  const int64_t row = blockIdx.x;
  if (p.mask && p.mask[row] == 0) return;
  const T* __restrict__ z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  float mx = -INFINITY;
  int64_t at = -1;
  bool bad = false;
  for (int64_t c = threadIdx.x; c < p.C; c += 256) {
    const float v = to_f32<T>(z[c]);
    bad |= !(v < INFINITY);
    if (v > mx) { mx = v; at = c; }
  }
  const float u = p.u[row];
  bad = __syncthreads_or(bad) || (p.T != 0.0 && !(u >= 0.f && u < 1.f));
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
  if (p.T == 0.0) {
    const int64_t first = block_reduce<4>(at >= 0 && mx == zmax ? at : INT64_MAX, shi, MinF());
    if (threadIdx.x == 0) {
      *label = (int32_t)first;
      if (prob) *prob = 1.f;
    }
    return;
  }
  ExactRow<T, 4> r{p, z, shd, shi, shu, zmax};
  r.draw(u, label, prob);
}

}  // namespace

size_t sample_workspace_bytes(int prec, int64_t n, int64_t C) { return 256; }

hipError_t sample_launch(int prec, const SampleParams& p, void* ws, hipStream_t s) {
  const dim3 grid((unsigned)p.n);
  switch (prec) {
    case 0: hipLaunchKernelGGL((sample_exact_kernel<float>), grid, dim3(256), 0, s, p); break;
    case 1: hipLaunchKernelGGL((sample_exact_kernel<f16>), grid, dim3(256), 0, s, p); break;
    case 2: hipLaunchKernelGGL((sample_exact_kernel<bf16>), grid, dim3(256), 0, s, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace gcn
