// Labels drawn from the rows' own distributions under temperature, top-k,
// top-p and min-p, from given uniform numbers.
//
// The classes of a row are ordered by falling score, the lower class first
// among equals; each filter keeps a prefix of that order, so what is kept is a
// prefix too and is described by its last item (sorted.h).  The drawn class is
// the first kept one, in class order, at which the running sum of the weights
// w_c = exp((z_c - max z) / T) passes u times their sum.
//
// The label is the one that 64-bit arithmetic gives: 32 bits decide where their
// error bound lets them, and the few rows in doubt are done again.
//
// Narrow rows are bound by the arithmetic of the sort and of two exponentials a
// class, long ones by their passes over the row.  Measured on MI355X, whole
// calls, against what a copy of as many bytes takes: 2^21 rows of 64 classes,
// fp16, every filter 268 us (51), without filters 101 us (57); 2048 rows of 7
// classes, fp32 8.5 us; 1024 rows of 50001, bf16, top-p 102-115 us (20), top-k and
// top-p 45 us; one row of 131072, fp32, top-k and top-p 20 us.
#include <algorithm>

#include "internal.h"
#include "longrow.h"
#include "sorted.h"

namespace gcn {

namespace {

// ------------------------------------------------ rows in lane groups ----
//
// A group of LPR lanes holds a row, N classes a lane (two vectors: half the
// exchanges between lanes and half the work a group does once, against one).
// With top-k or top-p the row's items are sorted over the group (sorted.h): the
// weights in that order and their running sum give the number of classes kept,
// and the last kept item the border.  The draw then runs over the classes in
// their own order.
//
// Weights and sums are in 32 bits (W = float); a border is believed only where
// no running sum lies within draw_eps() of it, relative to the total S.  With e =
// 2^-24, what a comparison of a running sum with a share q of S may be off by:
//   weights: an exponent x = (z - max) log2(e) / T carries 3 e |x| (difference,
//     constant, product), the base-2 exponential 4 e.  The sum up to a border
//     less q S has every weight with a factor of at most 1, and the mean of |x|
//     ln 2 under the weights is at most ln C: S (3 ln C + 4) e;
//   additions, L = log2 LPR: N - 1 in the lane, L over the lanes and N on the way
//     through the lane's own for the running sum; N - 1 and L for S;
//   the share's product and the bound's own addition: 2 e S.
// That is 85 e S for 1024 16-bit classes, 69 e S for 64 (and a thousandth for
// products of errors).  Where a sum does come as close, W = double settles it, for
// the wave: with 128 e for every width 2^21 rows of 64 take 279 us instead of 271.
constexpr float draw_eps(int N, int LPR) {
  double ln_c = 0.0;
  int L = 0;
  for (int l = LPR; l > 1; l /= 2) ++L;
  for (int c = LPR * N; c > 1; c /= 2) ln_c += 0.69314718056;
  const double in_e = 3.0 * ln_c + 4.0 + (2 * N - 1 + L) + (N - 1 + L) + 2.0;
  return (float)(in_e * 1.001 / (1 << 24));
}

template <typename W> struct Draw;
template <> struct Draw<float> {
  static __device__ __forceinline__ float weight(float z, float zmax, const SampleParams& p) {
    return __builtin_amdgcn_exp2f((z - zmax) * p.k);
  }
};
template <> struct Draw<double> {
  static __device__ __forceinline__ double weight(float z, float zmax, const SampleParams& p) {
    return exp(((double)z - (double)zmax) / p.T);
  }
};

// The smallest score that min-p keeps.  (double)z >= max + T ln(min_p) holds
// for the same 32-bit z as z >= the bound rounded up to 32 bits.
__device__ __forceinline__ float least_kept(const SampleParams& p, float zmax) {
  const double b = (double)zmax + p.T * p.ln_min_p;
  float f = (float)b;
  if ((double)f < b) f = nextafterf(f, INFINITY);
  return f;
}

// The draw of a group's row.  z, a: the row's scores and items in class order,
// s: the items sorted (with FILTER); absent classes have z = -inf and so weight
// 0.  Returns whether the answer is certain.
template <typename W, typename T, int LPR, bool FILTER, typename I, int N>
__device__ __forceinline__ bool group_draw(const SampleParams& p, const float (&z)[N], const I (&a)[N], const I (&s)[N],
                                           int li, float zmax, float u, int32_t& label, float& prob) {
  typedef Draw<W> D;
  constexpr W EPS = sizeof(W) == 4 ? (W)draw_eps(N, LPR) : W(0);
  const int col0 = li * N;
  bool sure = true;
  I border{0};
  if constexpr (FILTER) {
    const int64_t limit = p.top_k - col0;                // this lane's items under top-k
    const int k = limit < N ? (int)limit : N;
    int m = (int)p.top_k;                                // the items kept; past the last present one: all
    if (p.top_p < 1.0) {
      W w[N], sum = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        w[i] = D::weight(to_f32<T>(item_score<T>(s[i])), zmax, p);
        w[i] = i < k ? w[i] : W(0);
        sum += w[i];
      }
      const W total = group_sum<LPR>(sum);
      W run = group_sum_before<LPR>(sum, li);
      const W want = (W)p.top_p * total;
      const W lo = want - EPS * total, hi = want + EPS * total;
      int n_lo = 0, n_hi = 0;                            // past the last weight the sum is the total
#pragma unroll
      for (int i = 0; i < N; ++i) {
        n_lo += run < lo ? 1 : 0;
        n_hi += run < hi ? 1 : 0;
        run += w[i];
      }
      const int both = group_sum<LPR>(n_lo | n_hi << 16);
      m = both & 0xffff;
      sure = m == both >> 16 && m > 0;
    }
    // the m-th item, from the lane that holds it
    I mine{0};
#pragma unroll
    for (int i = 0; i < N; ++i) mine = item_pick(i == m - 1 - col0, s[i], mine);
    border = group_max_item<LPR>(mine);
  }
  const float zmin = least_kept(p, zmax);
  W w[N], sum = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool kept = (!FILTER || !item_above(border, a[i])) && z[i] >= zmin;
    w[i] = kept ? D::weight(z[i], zmax, p) : W(0);
    sum += w[i];
  }
  const W total = group_sum<LPR>(sum);
  const W want = (W)u * total;
  W run = group_sum_before<LPR>(sum, li);
  int at;
  if constexpr (sizeof(W) == 4) {
    const W lo = want - EPS * total, hi = want + EPS * total;
    int n_lo = 0, n_hi = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
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
    int first = LPR * N, last = -1;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) last = w[i] > 0 && last < 0 ? col0 + i : last;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      run += w[i];
      if (w[i] > 0 && run > want && first == LPR * N) first = col0 + i;
    }
    first = -group_max_int<LPR>(-first);
    last = group_max_int<LPR>(last);
    at = first < last ? first : last;
  }
  W mine = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) mine = i == at - col0 ? w[i] : mine;
  label = at;
  prob = (float)(group_sum<LPR>(mine) / total);
  return sure;
}

// R rows a group and iteration, their loads going out together.
template <typename T, int LPR, int R, bool FILTER>
__global__ __launch_bounds__(256) void sample_group_kernel(SampleParams p) {
  constexpr int VE = Vec<T>::N, N = 2 * VE;
  constexpr int RG = 4 * (64 / LPR);
  typedef typename ItemOf<T>::type I;
  const int lane = threadIdx.x & 63, li = lane % LPR;
  const int slot = (threadIdx.x >> 6) * (64 / LPR) + lane / LPR;
  const int col0 = li * N;
  const int C = (int)p.C;
  const T* __restrict__ logits = reinterpret_cast<const T*>(p.logits);
  bool report = false;
  for (int64_t first = (int64_t)blockIdx.x * (R * RG); first < p.n; first += (int64_t)gridDim.x * (R * RG)) {
    uint4 raw[R][2];
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
      raw[r][0] = raw[r][1] = make_uint4(0, 0, 0, 0);
      us[r] = 0.5f;                                      // greedy: half of one class's weight, no border near
      if (on[r]) {                                       // rows left out are not read
        raw[r][0] = load_row(logits + row * p.ld, col0, C, -INFINITY);
        raw[r][1] = load_row(logits + row * p.ld, col0 + VE, C, -INFINITY);
        if (!p.greedy) us[r] = p.u[row];
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!__ballot(on[r])) continue;
      const int64_t row = first + r * RG + slot;
      I a[N], s[N];
      float z[N];
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        order_items<T>(raw[r][v], col0 + v * VE, a + v * VE);
        unpack<T>(raw[r][v], z + v * VE);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = a[i];
      I most = a[0], least = a[0];
      if constexpr (FILTER) {
        group_sort<LPR, N>(s, li);
        most = s[0];
        least = s[N - 1];
      } else {
#pragma unroll
        for (int i = 1; i < N; ++i) {
          most = item_max(most, a[i]);
          least = item_min(least, a[i]);
        }
      }
      most = group_max_item<LPR>(most);
      least = group_min_item<LPR>(least);
      const bool bad = !items_regular<T>(most, least) || !(us[r] >= 0.f && us[r] < 1.f);
      const bool none = bad || !item_present<T>(most);
      const float zmax = none ? 0.f : to_f32<T>(item_score<T>(most));
      int32_t label;
      float prob;
      const bool sure = group_draw<float, T, LPR, FILTER>(p, z, a, s, li, zmax, us[r], label, prob);
      if (__ballot(on[r] && !none && !sure)) {
        int32_t l2;
        float p2;
        group_draw<double, T, LPR, FILTER>(p, z, a, s, li, zmax, us[r], l2, p2);
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

// ---------------------------------------------------------- longer rows ----

// A workgroup's row: whether it can be drawn from, else its answer is written.
__device__ __forceinline__ bool row_answerable(const SampleParams& p, int64_t row, bool bad, float zmax) {
  if (!bad && zmax > -INFINITY) return true;
  if (threadIdx.x == 0) {
    p.labels[row] = -1;
    if (p.prob) p.prob[row] = 0.f;
    if (bad) raise_flag(p.flag);
  }
  return false;
}

// top_k <= GCN_MAX_TOP: the first top_k items of the row are listed and put in
// order (longrow.h); what follows concerns at most 256 numbers, all in 64 bits.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_top_kernel(SampleParams p) {
  constexpr int NW = NT / 64;
  __shared__ TopList<NT> sh;
  __shared__ double s_item[GCN_MAX_TOP], s_w[GCN_MAX_TOP], s_d[NW];
  __shared__ int s_cls[GCN_MAX_TOP];
  const int64_t row = p.row0 + blockIdx.x;
  if (p.mask && p.mask[row] == 0) return;
  const int t = threadIdx.x;
  const LongRow<T, NT> r(reinterpret_cast<const T*>(p.logits) + row * p.ld, (int)p.C);
  const float u = p.greedy ? 0.f : p.u[row];
  const int K = (int)p.top_k;
  float mx;
  bool bad;
  const int cnt = list_top(r, K, sh, mx, bad);
  rank_list<NT>(sh, cnt, K, [&](int place, double e) { s_item[place] = e; });
  const float zmax = block_reduce<NW>(mx, sh.b, MaxF());
  bad = __syncthreads_or(bad) || !(u >= 0.f && u < 1.f);
  if (!row_answerable(p, row, bad, zmax)) return;
  int m = cnt < K ? cnt : K;
  // item t of the order; NT >= GCN_MAX_TOP
  const float z = t < m ? key_score(item_key(Item64{s_item[t < m ? t : 0]})) : 0.f;
  const int cls = t < m ? item_class(Item64{s_item[t < m ? t : 0]}) : 0;
  const double w = t < m ? Draw<double>::weight(z, zmax, p) : 0.0;
  if (t < m) s_w[t] = w;
  if (p.top_p < 1.0) {
    const double total = block_reduce<NW>(w, s_d, AddF());
    double before = 0.0;
    for (int j = 0; j < t && j < m; ++j) before += s_w[j];
    m = block_reduce<NW>(t < m && before < p.top_p * total ? 1 : 0, sh.n, AddF());
    m = m > 1 ? m : 1;
  }
  const bool kept = t < m && z >= least_kept(p, zmax);
  const double wk = kept ? w : 0.0;
  __syncthreads();
  if (t < m) { s_w[t] = wk; s_cls[t] = cls; }
  const double total = block_reduce<NW>(wk, s_d, AddF());
  double run = 0.0;
  if (wk > 0.0)
    for (int j = 0; j < m; ++j) run += s_cls[j] <= cls ? s_w[j] : 0.0;
  // the lowest class that passes, or the last one where rounding leaves none
  const int first = block_reduce<NW>(wk > 0.0 && run > (double)u * total ? cls : INT32_MAX, sh.n, MinF());
  const int last = block_reduce<NW>(wk > 0.0 ? cls : -1, sh.n, MaxF());
  if (wk > 0.0 && cls == (first < last ? first : last)) {
    p.labels[row] = cls;
    if (p.prob) p.prob[row] = (float)(w / total);
  }
}

// Other limits.  The classes kept are described by the last of them, the border
// item, found by histograms in shared memory: the members of a range of scores
// fall into 1024 bins by score, each with the sum of its members' weights; the
// bin in which the running sum reaches what is wanted is the next range, until
// its members are few enough to be compared with one another or all have the
// same score.  The first histogram is linear in max - z, the next ones in the
// key.  Then the classes are walked in their own order, a range of them a
// wave.  For top_k the weights are 1.
//
// Under top_p the first histogram (and before it the list of run_listed) takes
// weights above 2^-13 only: the others are many, add up to little, and an atomic
// each would cost more than the rest of the pass; where the border is not among
// them it is done again down to (1 - top_p) / (2 C), below which it cannot lie
// (what weighs less adds up to (1 - top_p) / 2 at most, the whole to 1 at least).
//
// W = float: weights carry 2^-22 (the exponent in 64 bits, the base-2
// exponential in 32: one unit in its last place and a rounding), those below the
// histogram REST_EPS = 2^-17: with e = 2^-24 an exponent x of three roundings
// carries 3 e |x|, a weight 3 e |x| ln 2 + 4 e, eight of them added 8 e more,
// below 128 e for |x| <= 55, and what lies beyond weighs next to nothing.  Other
// sums are in 64 bits.  Where a running sum comes within its bound of a border
// the row is done again with W = double.
//
// Sums that several threads add to in no fixed order are whole numbers, so that
// the order cannot show: the bins' in one word of 64 bits with frac() of them
// behind the point, what is rounded away in the bound, or, where that has to be
// exact, in two words, 31 bits and 32 more; a border's members, MEMBERS at most,
// in one word with 54.  (64-bit float atomics, whose sums differ from run to run:
// 1024 rows of 50001 nearly equal classes 469 us instead of 480, 16384 of 4001
// 201 instead of 204.)
constexpr double REST_EPS = 7.62939453125e-6;            // 2^-17
template <typename W> struct LongDraw;
template <> struct LongDraw<float> {
  static __device__ __forceinline__ double weight(float z, float zmax, const SampleParams& p) {
    const double y = ((double)z - (double)zmax) * p.kd;
    if (!(y > -140.0)) return 0.0;                       // below the smallest normal weight
    const double n = rint(y);
    return (double)ldexpf(__builtin_amdgcn_exp2f((float)(y - n)), (int)n);
  }
  static constexpr double EPS = 4.76837158203125e-7;     // 2^-21
};
template <> struct LongDraw<double> {
  static __device__ __forceinline__ double weight(float z, float zmax, const SampleParams& p) {
    return Draw<double>::weight(z, zmax, p);
  }
  static constexpr double EPS = 0.0;
};

constexpr int BINS = 1024, MEMBERS = 256, NEAR_CAP = 512;

enum Sums { COUNTS, WORD, PAIR };                        // what a bin holds

template <int NT>
struct LongShared {
  uint64_t bin[BINS], fine[BINS];                        // fine: the second words of PAIR
  double item[MEMBERS];
  uint64_t weight[MEMBERS];
  double d[NT / 64], rest[NT / 64];
  float f[NT / 64];                                      // the waves' maxima: written once a row
  float low[NT / 64];
  uint32_t u[NT / 64];
  int n[NT / 64];
  int count, hit, doubt;
  uint64_t least, most;
  double above, mass;
  // classes of large weight, those of each wave in the order of the classes
  float near_z[NT / 64][NEAR_CAP];
  int near_c[NT / 64][NEAR_CAP];
  int near_n[NT / 64];
};

// Weights above 2^-NEAR take part in the first histogram, and in the first list of
// run_listed.  10, 13 and 16, us, top-p 0.9 and trained scores: 1024 x 50001 bf16
// at T = 0.5 56, 58, 60, at T = 1 247, 117, 199, at T = 2 421, 350, 369, nearly
// equal scores 397, 478, 531; 2048 x 20011 fp32 172, 98, 125; 16384 x 4001 fp16 189,
// 204, 240.
constexpr float NEAR = 13.f;
// Where the border is not on the list, and where the list is too short for a wave.
// GROW 1.2, 1.4 and 1.8: 16384 x 4001 at top-p 0.99 278, 376, 389, 1024 x 50001 558,
// 542, 544; SHRINK 0.7, 0.8 and 0.9: 1024 x 50001 at T = 1 164, 117, 108, at T = 1.4
// 350, 354, 359.
constexpr float GROW = 1.2f, SHRINK = 0.9f;

template <typename W, typename Row>
struct LongSample {
  typedef LongDraw<W> D;
  static constexpr int VE = Row::VE;
  static constexpr int NT = Row::NT;
  static constexpr int NW = NT / 64;
  const SampleParams& p;
  const Row r;
  LongShared<NT>& sh;
  float zmax;

  static constexpr Sums WEIGHTS = sizeof(W) == 4 ? WORD : PAIR;
  // Bits behind the point of a word: C 2^frac is below 2^62, 2^frac below 2^52.
  __device__ __forceinline__ int frac() const { return min(51, 30 + __clz((int)p.C)); }
  // w <= 1 as a word: the number's last 52 bits when 2^52 is added.
  __device__ __forceinline__ uint64_t word(double w) const {
    const double x = fma(w, ldexp(1.0, frac()), 0x1p52);
    return (uint64_t)__double_as_longlong(x) & 0xfffffffffffffull;
  }

  template <Sums S>
  __device__ __forceinline__ void clear_bins() {
    for (int i = threadIdx.x; i < BINS; i += NT) {
      sh.bin[i] = 0;
      if (S == PAIR) sh.fine[i] = 0;
    }
    if (threadIdx.x == 0) { sh.hit = -1; sh.count = 0; }
  }
  __device__ __forceinline__ void add_pair(int b, double w) {
    const double hi = w * 2147483648.0;                  // w <= 1
    const uint32_t h = (uint32_t)hi;
    lds_add(&sh.bin[b], h);
    lds_add(&sh.fine[b], (uint32_t)((hi - (double)h) * 4294967296.0));
  }
  template <Sums S>
  __device__ __forceinline__ void add_score(int b, float z) {
    if constexpr (S == COUNTS) lds_add(&sh.bin[b], 1);
    else if constexpr (S == WORD) lds_add(&sh.bin[b], word(D::weight(z, zmax, p)));
    else add_pair(b, Draw<double>::weight(z, zmax, p));
  }
  template <Sums S>
  __device__ __forceinline__ double bin_sum(int b) const {
    const double x = (double)sh.bin[b];
    if constexpr (S == COUNTS) return x;
    else if constexpr (S == WORD) return ldexp(x, -frac());
    else return x * 0x1p-31 + (double)sh.fine[b] * 0x1p-63;
  }

  // With the histogram complete (a barrier since): the last bin that holds
  // something and before which the running sum from `above` on is below want,
  // where want = share (above + the sum of the bins + rest): its number, the sum
  // before it and its own.  rest: this wave's part.
  struct Found { int bin; double above, mass, want, sum, rest; };
  template <Sums S>
  __device__ __forceinline__ Found find_bin(double above, double rest, double share, double want) {
    constexpr int PER = BINS / NT;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    double own[PER], sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += own[i] = bin_sum<S>(t * PER + i);
    const double upto = wave_scan(sum);
    if (lane == 63) { sh.d[wave] = upto; sh.rest[wave] = rest; }
    __syncthreads();
    Found r;
    double run = above + wave_before(upto);
    r.sum = 0.0;
    r.rest = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      run += i < wave ? sh.d[i] : 0.0;
      r.sum += sh.d[i];
      r.rest += sh.rest[i];
    }
    r.want = share > 0.0 ? share * (r.sum + r.rest) : want;
    int held = -1;
    double start = 0.0, mass = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (own[i] > 0.0 && run < r.want) { held = t * PER + i; start = run; mass = own[i]; }
      run += own[i];
    }
    const int most = wave_reduce(held, MaxF());
    if (held >= 0 && held == most) atomicMax(&sh.hit, held);
    __syncthreads();
    r.bin = sh.hit;
    if (held >= 0 && held == r.bin) { sh.above = start; sh.mass = mass; }
    __syncthreads();
    r.above = sh.above;
    r.mass = sh.mass;
    return r;
  }

  static __device__ __forceinline__ uint64_t member_weight(double w) { return (uint64_t)(w * 0x1p54); }

  // The n listed members of a bin: one is kept if what comes before it is below
  // f.want.  Returns whether that is certain for all.
  __device__ __forceinline__ bool settle(const Found& f, int n, double eps, double& border) {
    const int t = threadIdx.x;
    if (t < n) {
      const double mine = sh.item[t];
      uint64_t ahead = 0;                                // listed in no fixed order
      for (int j = 0; j < n; ++j) ahead += sh.item[j] > mine ? sh.weight[j] : 0;
      const double before = f.above + (double)ahead * 0x1p-54;
      const uint64_t bits = (uint64_t)__double_as_longlong(mine);
      if (before < f.want) atomicMin((unsigned long long*)&sh.least, (unsigned long long)bits);
      atomicMax((unsigned long long*)&sh.most, (unsigned long long)bits);
      if (eps > 0.0 && !(fabs(before - f.want) > eps && fabs(f.above + f.mass - f.want) > eps)) sh.doubt = 1;
    }
    __syncthreads();
    border = __longlong_as_double((long long)(sh.least != ~0ull ? sh.least : sh.most));
    return sh.doubt == 0;
  }

  // Moves `border` to the last item that top_k (COUNT) or top_p keeps among
  // the items from `border` on (LIMIT; else among all).  Returns whether that is
  // certain.
  template <bool COUNT, bool LIMIT>
  __device__ __forceinline__ bool select(double& border) {
    constexpr Sums S = COUNT ? COUNTS : WEIGHTS;
    const float zl = key_score(item_key(Item64{border}));
    const int cl = item_class(Item64{border});
    auto weight = [&](float z) -> double { return COUNT ? 1.0 : D::weight(z, zmax, p); };
    auto inside = [&](float z, int c) { return LIMIT ? z > zl || (z == zl && c <= cl) : z > -INFINITY; };
    // The first histogram: bin floor((zmax - z) scale), BINS below it.  With COUNT
    // the last bin takes what is below, and what a range past fp32 makes of the
    // product (scale 0 times an infinite difference).
    float scale, near = NEAR;
    auto first_bin = [&](float z) {
      const float x = (zmax - z) * scale;
      return x < (float)BINS ? (int)x : COUNT ? BINS - 1 : BINS;
    };
    if (COUNT) {
      float low = INFINITY;
      r.each([&](const float (&v)[VE], int) {
#pragma unroll
        for (int i = 0; i < VE; ++i) low = v[i] > -INFINITY ? fminf(low, v[i]) : low;
      });
      // not in sh.f: a wave may still be reading the maxima there
      const float range = zmax - block_reduce<NW>(low, sh.low, MinF());
      scale = range > 0.f && range < INFINITY ? (float)BINS / range : 0.f;
      scale = scale < INFINITY ? scale : 0.f;
    }
    const float far = 1.f + log2f((float)p.C) - log2f((float)(1.0 - p.top_p));
    Found f;
    double eps = 0.0;
    for (;;) {
      if (!COUNT) scale = p.k * ((float)BINS / near);
      clear_bins<S>();
      __syncthreads();
      double rest = 0.0;
      r.each([&](const float (&v)[VE], int c0) {
        float low_rest = 0.f;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const int b = first_bin(v[i]);
          if (COUNT) {
            if (inside(v[i], c0 + i)) add_score<S>(b, v[i]);
          } else {
            const bool in = !LIMIT || inside(v[i], c0 + i);   // -inf weighs nothing
            const bool close = b < BINS;
            if (sizeof(W) == 4) low_rest += in && !close ? __builtin_amdgcn_exp2f((v[i] - zmax) * p.k) : 0.f;
            else if (in && !close) rest += weight(v[i]);
            if (in && close) add_score<S>(b, v[i]);
          }
        }
        rest += (double)low_rest;
      });
      if (!COUNT) rest = wave_reduce(rest, AddF());
      __syncthreads();
      f = find_bin<S>(0.0, rest, COUNT ? 0.0 : p.top_p, (double)p.top_k);
      if (COUNT) break;
      eps = D::EPS > 0.0 ? D::EPS * f.sum + REST_EPS * f.rest + ldexp((double)p.C, -frac()) : 0.0;
      if (f.want + eps < f.sum || near >= far) break;
      near = far;
    }
    const double want = f.want;
    uint32_t klo = 0, khi = 0;                           // the range of keys, from the first histogram on
    int shift = -1;
    for (;;) {
      const int hit = f.bin;
      // the members of the bin: how many, and the first MEMBERS
      auto member = [&](float z, int c) {
        bool m;
        if (shift < 0) {
          m = first_bin(z) == hit;
        } else {
          const uint32_t key = score_key(z);
          m = key >= klo && key <= khi && (int)((khi - key) >> shift) == hit;
        }
        return m && inside(z, c);
      };
      if (threadIdx.x == 0) { sh.least = ~0ull; sh.most = 0; sh.doubt = 0; }
      r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          if (!member(v[i], c0 + i)) continue;
          const int at = atomicAdd(&sh.count, 1);
          if (at < MEMBERS) {
            sh.item[at] = score_item(v[i], c0 + i).v;
            sh.weight[at] = member_weight(weight(v[i]));
          }
        }
      });
      __syncthreads();
      const int n = sh.count;
      if (n <= MEMBERS) {
        return settle(f, n, eps, border);
      }
      uint32_t lo = 0xffffffffu, hi = 0;
      r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          if (!member(v[i], c0 + i)) continue;
          const uint32_t key = score_key(v[i]);
          lo = key < lo ? key : lo;
          hi = key > hi ? key : hi;
        }
      });
      lo = block_reduce<NW>(lo, sh.u, MinF());
      hi = block_reduce<NW>(hi, sh.u, MaxF());
      if (lo == hi) {
        // equal scores: the lowest `take` classes
        const double w = weight(key_score(lo));
        const double q = (want - f.above) / w;
        double take = ceil(q);
        take = take < 1.0 ? 1.0 : take > (double)n ? (double)n : take;
        const bool sure = eps == 0.0 || fabs(q - rint(q)) * w > eps;
        int a = 0, b = r.C - 1;                          // the class up to which they are `take`
        while (a < b) {
          const int mid = a + (b - a) / 2;
          int m = 0;
          r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
            for (int i = 0; i < VE; ++i)
              m += c0 + i <= mid && score_key(v[i]) == lo && inside(v[i], c0 + i) ? 1 : 0;
          });
          m = block_reduce<NW>(m, sh.n, AddF());
          if ((double)m >= take) b = mid;
          else a = mid + 1;
        }
        border = item64(lo, (uint32_t)a).v;
        return sure;
      }
      // the next histogram, of the members' keys
      klo = lo;
      khi = hi;
      shift = 0;
      while ((hi - lo) >> shift >= (uint32_t)BINS) ++shift;
      clear_bins<S>();
      __syncthreads();
      r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const uint32_t key = score_key(v[i]);
          if (key >= klo && key <= khi && inside(v[i], c0 + i)) add_score<S>((int)((khi - key) >> shift), v[i]);
        }
      });
      __syncthreads();
      f = find_bin<S>(f.above, 0.0, 0.0, want);
    }
  }

  // The draw among the items from `border` on that min-p keeps.
  __device__ __forceinline__ bool draw(double border, float u, int32_t* label, float* prob) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const float zb = key_score(item_key(Item64{border}));
    const int cb = item_class(Item64{border});
    const float least = fmaxf(least_kept(p, zmax), zb);
    auto weight = [&](float z, int c) -> double {
      return z >= least && (z > zb || c <= cb) ? D::weight(z, zmax, p) : 0.0;
    };
    double sum = 0.0;
    int last = -1;
    r.each([&](const float (&v)[VE], int c0) {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        if (!(v[i] >= least)) continue;
        const double w = weight(v[i], c0 + i);
        sum += w;
        last = w > 0.0 ? c0 + i : last;
      }
    });
    sum = wave_reduce(sum, AddF());
    last = wave_reduce(last, MaxF());
    if (lane == 0) { sh.d[wave] = sum; sh.n[wave] = last; }
    if (t == 0) sh.doubt = 0;
    __syncthreads();
    double total = 0.0, run = 0.0;
    for (int i = 0; i < NW; ++i) total += sh.d[i];
    const double want = (double)u * total;               // below the total: u <= 1 - 2^-24
    int owner = -1;                                      // some wave: the sums end with the total
    double before = 0.0;
    for (int i = 0; i < NW; ++i) {
      if (owner < 0 && sh.n[i] >= 0 && run + sh.d[i] > want) { owner = i; before = run; }
      run += sh.d[i];
    }
    if (wave == owner) {
      const double eps = D::EPS * total;
      bool done = false;
      r.each([&](const float (&v)[VE], int c0) {
        // every lane comes here for every vector of the wave; done and before are the wave's
        if (done) return;
        double w[VE], own = 0.0;
#pragma unroll
        for (int i = 0; i < VE; ++i) own += w[i] = weight(v[i], c0 + i);
        if (!__ballot(own > 0.0)) return;
        const double upto = wave_scan(own);
        double x = before + wave_before(upto);
        const uint64_t hits = __ballot(own > 0.0 && before + upto > want);
        // the class in this lane: its sum passes `want`; where the order of
        // additions leaves none, the lane's last kept one, unless in doubt
        if (hits && lane == __ffsll((unsigned long long)hits) - 1) {
          int at = -1;
          double w_at = 0.0;
          bool passed = false, sure = false;
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            if (w[i] > 0.0 && !passed) {
              const double y = x + w[i];
              at = c0 + i;
              w_at = w[i];
              passed = y > want;
              sure = passed && fabs(x - want) > eps && fabs(y - want) > eps;
              x = y;
            }
          }
          if (sure || D::EPS == 0.0) {
            *label = at;
            if (prob) *prob = (float)(w_at / total);
          } else {
            sh.doubt = 1;
          }
        }
        done = hits != 0;
        before += from_lane(upto, 63);
      });
      // sums of the walk and of the wave may differ by a rounding: the wave's last
      if (!done && lane == 0) {
        if (D::EPS == 0.0) {
          *label = sh.n[owner];
          if (prob) *prob = (float)(D::weight(to_f32<typename Row::Elem>(r.z[sh.n[owner]]), zmax, p) / total);
        } else {
          sh.doubt = 1;
        }
      }
    }
    __syncthreads();
    return sh.doubt == 0;
  }

  // Rows whose mass lies on few classes: those of weights above 2^-near are
  // listed, in the order of the classes, and everything else is done on the
  // list, in 64 bits; the other weights enter by their sum alone, in 32 bits
  // (good to REST_EPS of itself) or, exact, in 64.
  enum Listed {
    DONE,
    BEYOND,                                              // the border is among the others
    LONG, FAR_LONG,                                      // the list is too short, by more than a factor of 2
    DOUBT,                                               // the sum of the others is not known well enough
    TIES                                                 // too many equal or nearly equal scores at the border
  };
  __device__ __forceinline__ Listed run_listed(float near, bool exact, float u, int32_t* label, float* prob) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    if (exact) clear_bins<PAIR>();
    else clear_bins<WORD>();
    int n = 0;                                           // the wave's entries
    double rest = 0.0;
    r.each([&](const float (&v)[VE], int c0) {
      bool in[VE];
      int own = 0;
      float low_rest = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float x = (zmax - v[i]) * p.k;
        in[i] = x < near;
        own += in[i] ? 1 : 0;
        low_rest += in[i] ? 0.f : __builtin_amdgcn_exp2f(-x);
      }
      if (exact) {
        for (int i = 0; i < VE; ++i) rest += in[i] ? 0.0 : Draw<double>::weight(v[i], zmax, p);
      } else {
        rest += (double)low_rest;
      }
      if (!__ballot(own > 0)) return;
      const int upto = wave_scan(own);
      int at = n + upto - own;
      n += from_lane(upto, 63);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        if (!in[i]) continue;
        if (at < NEAR_CAP) { sh.near_z[wave][at] = v[i]; sh.near_c[wave][at] = c0 + i; }
        ++at;
      }
    });
    if (t == 0) { sh.least = ~0ull; sh.most = 0; sh.doubt = 0; }
    if (lane == 0) sh.near_n[wave] = n;
    __syncthreads();
    int longest = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) longest = sh.near_n[i] > longest ? sh.near_n[i] : longest;
    if (longest > NEAR_CAP) return longest > 2 * NEAR_CAP ? FAR_LONG : LONG;
    // this lane's entries: lane, lane + 64, ...
    constexpr int PER = NEAR_CAP / 64;
    float z[PER];
    int c[PER];
    double w[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = i * 64 + lane;
      z[i] = e < n ? sh.near_z[wave][e] : -INFINITY;
      c[i] = e < n ? sh.near_c[wave][e] : 0;
      w[i] = e < n ? Draw<double>::weight(z[i], zmax, p) : 0.0;
    }
    double border = item64(KEY_NEG_INF + 1, 0x3fffffff).v;
    if (p.top_p < 1.0) {
      const float scale = p.k * ((float)BINS / near);
      auto bin = [&](float z) { const float x = (zmax - z) * scale; return x < (float)BINS ? (int)x : BINS - 1; };
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < n) {
          if (exact) add_pair(bin(z[i]), w[i]);
          else lds_add(&sh.bin[bin(z[i])], word(w[i]));
        }
      __syncthreads();
      rest = wave_reduce(rest, AddF());
      const Found f = exact ? find_bin<PAIR>(0.0, rest, p.top_p, 0.0) : find_bin<WORD>(0.0, rest, p.top_p, 0.0);
      const double eps = exact ? 0.0 : REST_EPS * f.rest + 1e-12 * f.sum + ldexp((double)(NW * NEAR_CAP), -frac());
      if (!(f.want + eps < f.sum)) return BEYOND;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < n && bin(z[i]) == f.bin) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < MEMBERS) { sh.item[at] = score_item(z[i], c[i]).v; sh.weight[at] = member_weight(w[i]); }
        }
      __syncthreads();
      const int members = sh.count;
      if (members > MEMBERS) return TIES;
      if (!settle(f, members, eps, border)) return DOUBT;
    }
    const float least = least_kept(p, zmax);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (!(z[i] >= least && score_item(z[i], c[i]).v >= border)) w[i] = 0.0;
      sum += w[i];
    }
    sum = wave_reduce(sum, AddF());
    if (lane == 0) sh.d[wave] = sum;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) total += sh.d[i];
    const double want = (double)u * total;
    int owner = -1;
    double before = 0.0, run = 0.0;
    for (int i = 0; i < NW; ++i) {                       // the last that keeps anything where rounding leaves none
      if (sh.d[i] > 0.0 && run <= want) { owner = i; before = run; }
      run += sh.d[i];
    }
    if (wave != owner) return DONE;
    int at = -1;
    double w_at = 0.0;
    bool passed = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const double upto = before + wave_scan(w[i]);
      const uint64_t kept = __ballot(w[i] > 0.0), hits = __ballot(w[i] > 0.0 && upto > want);
      if (kept && !passed) {
        const int l = hits ? __ffsll((unsigned long long)hits) - 1 : 63 - __clzll(kept);
        at = from_lane(c[i], l);
        w_at = from_lane(w[i], l);
        passed = hits != 0;
      }
      before = from_lane(upto, 63);
    }
    if (lane == 0) {
      *label = at;
      if (prob) *prob = (float)(w_at / total);
    }
    return DONE;
  }

  __device__ __forceinline__ bool run(float u, int32_t* label, float* prob) {
    double border = item64(KEY_NEG_INF + 1, 0x3fffffff).v;   // every score's item is above
    bool sure = true;
    if (p.top_k < p.C) {
      sure &= select<true, false>(border);
      if (p.top_p < 1.0) sure &= select<false, true>(border);
    } else if (p.top_p < 1.0) {
      sure &= select<false, false>(border);
    }
    return sure && draw(border, u, label, prob);
  }
};

template <typename T, int NT>
__global__ __launch_bounds__(NT, 4) void sample_row_kernel(SampleParams p) {
  typedef LongRow<T, NT, true> Row;
  constexpr int NW = NT / 64;
  __shared__ LongShared<NT> sh;
  const int64_t row = p.row0 + blockIdx.x;
  if (p.mask && p.mask[row] == 0) return;
  const Row r(reinterpret_cast<const T*>(p.logits) + row * p.ld, (int)p.C);
  const float u = p.u[row];
  float mx = -INFINITY;
  bool bad = false;
  r.each([&](const float (&v)[Row::VE], int) {
#pragma unroll
    for (int i = 0; i < Row::VE; ++i) {
      bad |= !(v[i] < INFINITY);
      mx = fmaxf(mx, v[i]);
    }
  });
  mx = wave_reduce(mx, MaxF());
  const bool wave_bad = __ballot(bad) != 0;
  if ((threadIdx.x & 63) == 0) sh.f[threadIdx.x >> 6] = wave_bad ? INFINITY : mx;
  __syncthreads();
  float zmax = sh.f[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) zmax = fmaxf(zmax, sh.f[i]);
  if (!row_answerable(p, row, zmax == INFINITY || !(u >= 0.f && u < 1.f), zmax)) return;
  int32_t* label = p.labels + row;
  float* prob = p.prob ? p.prob + row : nullptr;
  LongSample<float, Row> q{p, r, sh, zmax};
  // worth trying where the filters may leave few classes: with more of them
  // where the border is not on the list, with fewer where it is too short by
  // less than a factor of 2
  if (p.top_k == p.C && (p.top_p < 1.0 || p.ln_min_p > -8.0)) {
    float near = p.top_p < 1.0 ? NEAR : (float)(-p.ln_min_p * 1.4426950408889634) + 0.01f;
    bool grown = false, exact = false;
    for (int i = 0; i < 4; ++i) {
      const auto did = q.run_listed(near, exact, u, label, prob);
      if (did == q.DONE) return;
      __syncthreads();
      if (did == q.FAR_LONG || did == q.TIES || p.top_p == 1.0 || (did == q.LONG && grown)) break;
      exact = did == q.DOUBT;
      grown |= did == q.BEYOND;
      near *= did == q.BEYOND ? GROW : did == q.LONG ? SHRINK : 1.f;
    }
  }
  if (q.run(u, label, prob)) return;
  __syncthreads();                                       // every wave has seen the doubt: it is cleared next
  LongSample<double, Row>{p, r, sh, zmax}.run(u, label, prob);
}

// ------------------------------------------------------------- launches ----

constexpr int64_t MAX_BLOCKS = 65536;
// Rows a lane group takes per iteration: 2 where one would give more than
// R2_GROUPS workgroups and two rows' registers leave waves enough, else 1.  Two
// and one, us: without filters 2^21 x 64 fp16 101 and 112, 2^20 x 64 fp32 67 and
// 71, 2^18 x 512 fp16 116 and 122; with them 2^21 x 32 fp16 126 and 134, x 64 271
// and 283, 2^20 x 128 299 and 316, but 2^19 x 256 397 and 356, 2^18 x 512 489 and
// 413, 2^17 x 1000 618 and 647; 2^20 x 64 fp32 189 and 176, 2^19 x 128 238 and
// 217, 2^18 x 256 298 and 299.  Fewer workgroups: 200000 x 40 fp32 43 and 39.
constexpr int64_t R2_GROUPS = 16384;
template <typename T, int LPR, bool FILTER>
constexpr bool two_rows() { return !FILTER || (sizeof(T) == 2 && LPR != 16 && LPR != 32); }

template <typename T, int LPR, bool FILTER>
hipError_t launch_filter(const SampleParams& p, hipStream_t s) {
  constexpr int64_t RG = 4 * (64 / LPR);
  const int r = two_rows<T, LPR, FILTER>() && (p.n + RG - 1) / RG > R2_GROUPS ? 2 : 1;
  const int64_t nb = std::min<int64_t>((p.n + r * RG - 1) / (r * RG), MAX_BLOCKS);
  if constexpr (two_rows<T, LPR, FILTER>()) {
    if (r == 2) {
      hipLaunchKernelGGL((sample_group_kernel<T, LPR, 2, FILTER>), dim3((unsigned)nb), dim3(256), 0, s, p);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((sample_group_kernel<T, LPR, 1, FILTER>), dim3((unsigned)nb), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_lpr(const SampleParams& p, hipStream_t s) {
  return p.top_k < p.C || p.top_p < 1.0 ? launch_filter<T, LPR, true>(p, s) : launch_filter<T, LPR, false>(p, s);
}
// Threads of a long row's workgroup, from both sides of each rule, us.
// Up to GCN_MAX_TOP classes, 256 and 1024 threads:
//   16384 x  4001 fp16  k = 20  94  385   k = 64  154  556   k = 128  314  837
//    2048 x 30001 fp16  k = 64  56   86   k = 128  94  126   k = 256  474  241
//    1024 x 50001 bf16  k = 50  45   56   k = 200 155  116
//     256 x 50001 bf16  k = 50  31   25;  2048 x 131072 fp32, k = 50  354  318
// (as for top scores, the list grows with k against the threads).
bool small_top(int64_t n, int64_t nvec, int64_t k) { return k <= 128 && (nvec <= 2048 || (nvec <= 8192 && n > 512)); }
// Other limits, 256 and 512 threads: 16384 x 1100 fp16 174 and 334, x 4001 203 and
// 358; 4096 x 16001 114 and 123, 2048 x 30001 147 and 103; 512 x 4001 13.0 and
// 14.4, 512 x 16001 37 and 22.
bool small_row(int64_t n, int64_t nvec) { return nvec <= 512 || (nvec <= 2048 && n > 1024); }

template <typename T>
hipError_t launch_rows(const SampleParams& params, hipStream_t s) {
  const int64_t nvec = (params.C + Vec<T>::N - 1) / Vec<T>::N;
  return launch_long_rows(params, 1, [&](const SampleParams& p, int64_t rows) {
    const dim3 grid((unsigned)rows);
    if (p.top_k <= GCN_MAX_TOP) {
      if (small_top(p.n, nvec, p.top_k)) hipLaunchKernelGGL((sample_top_kernel<T, 256>), grid, dim3(256), 0, s, p);
      else hipLaunchKernelGGL((sample_top_kernel<T, 1024>), grid, dim3(1024), 0, s, p);
    } else {
      if (small_row(p.n, nvec)) hipLaunchKernelGGL((sample_row_kernel<T, 256>), grid, dim3(256), 0, s, p);
      else hipLaunchKernelGGL((sample_row_kernel<T, 512>), grid, dim3(512), 0, s, p);
    }
    return hipGetLastError();
  });
}
template <typename T>
hipError_t launch_t(const SampleParams& p, hipStream_t s) {
  const int64_t pairs = (p.C + 2 * Vec<T>::N - 1) / (2 * Vec<T>::N);
  if (pairs <= 1) return launch_lpr<T, 1>(p, s);
  if (pairs <= 2) return launch_lpr<T, 2>(p, s);
  if (pairs <= 4) return launch_lpr<T, 4>(p, s);
  if (pairs <= 8) return launch_lpr<T, 8>(p, s);
  if (pairs <= 16) return launch_lpr<T, 16>(p, s);
  if (pairs <= 32) return launch_lpr<T, 32>(p, s);
  if (pairs <= 64) return launch_lpr<T, 64>(p, s);
  return launch_rows<T>(p, s);
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
