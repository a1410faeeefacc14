// The K largest scores of every row with their classes, in falling order, the
// lower class first among equals.  Scores are turned into items (sorted.h), of
// which no two are equal, so that ties need no care.
//
// Bound by the read of the scores; what has to be kept small is the number of
// comparisons a score takes part in.  Measured on MI355X, whole calls, against
// what a copy of as many bytes takes: 2^21 rows of 64 classes, fp16, K = 8 86 us
// (71); 200000 rows of 40, fp32, K = 5 16 us (8); 2048 rows of 50001, bf16, K =
// 64 72 us (40; two passes, the second from L2); one row of 131072, fp32, K = 100
// 17.6 us, what one compute unit takes to read it (cut into 16 segments whose
// lists a second launch joins: 21 us).
#include <algorithm>

#include "internal.h"
#include "longrow.h"
#include "sorted.h"

namespace gcn {

namespace {

template <typename T, typename I>
__device__ __forceinline__ void put_entry(const TopParams& p, int64_t row, int64_t j, I a) {
  const bool here = item_present<T>(a);
  reinterpret_cast<T*>(p.values)[row * p.ld_top + j] = here ? item_score<T>(a) : from_f32<T>(-INFINITY);
  p.classes[row * p.ld_top + j] = here ? item_class(a) : -1;
}

// Joins the lists of lanes W apart, W = 1, 2, 4, ...: H items are in use.
template <int LPR, int L, int W, int H, typename I>
__device__ __forceinline__ void list_levels(I (&a)[L]) {
  if constexpr (W < LPR) {
    if constexpr (2 * H <= L) {
      // both lists whole: the larger halves of the pairs, then the smaller
      I hi[H], lo[H];
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const I o = lane_xor<W>(a[H - 1 - i]);
        hi[i] = item_max(a[i], o);
        lo[i] = item_min(a[i], o);
      }
      merge_bitonic<H>(hi);
      merge_bitonic<H>(lo);
#pragma unroll
      for (int i = 0; i < H; ++i) { a[i] = hi[i]; a[H + i] = lo[i]; }
      list_levels<LPR, L, 2 * W, 2 * H>(a);
    } else {
      static_assert(H == L, "list lengths are powers of two");
      I hi[L];
#pragma unroll
      for (int i = 0; i < L; ++i) hi[i] = item_max(a[i], lane_xor<W>(a[L - 1 - i]));
      merge_bitonic<L>(hi);
#pragma unroll
      for (int i = 0; i < L; ++i) a[i] = hi[i];
      list_levels<LPR, L, 2 * W, L>(a);
    }
  }
}

// Rows of up to 128 vectors of 16 bytes: a group of LPR lanes owns a row, two
// vectors a lane.
//
// L > 0: the first L >= K items only.  Each lane sorts its own, then lists are
// merged pairwise across lanes: of two sorted lists of L, the larger of item
// i of one and item L - 1 - i of the other are the L largest of both, in
// bitonic order, so a merge costs L maxima and log2 L steps; every lane of the
// group ends with the row's list.  (Shorter lists are joined whole until they
// have L items.)
// L = 0: the row is sorted over the group.
//
// For 2^21 rows of 64 fp16 classes, K = 8: two vectors a lane 90 us, one 117 (twice
// the exchanges between lanes); with the test for NaN at the ends of the sorted
// vectors, where it costs two comparisons, instead of at every score 86.
template <typename T, int LPR, int L, int R>
__global__ __launch_bounds__(256) void top_group_kernel(TopParams p) {
  constexpr int VE = Vec<T>::N, N = 2 * VE;
  constexpr int RG = 4 * (64 / LPR);
  typedef typename ItemOf<T>::type I;
  const int lane = threadIdx.x & 63, li = lane % LPR;
  const int slot = (threadIdx.x >> 6) * (64 / LPR) + lane / LPR;
  const int col0 = li * N;
  const int C = (int)p.C;
  const T* __restrict__ logits = reinterpret_cast<const T*>(p.logits);
  bool bad = false;
  for (int64_t first = (int64_t)blockIdx.x * (R * RG); first < p.n; first += (int64_t)gridDim.x * (R * RG)) {
    uint4 raw[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int64_t row = first + r * RG + slot;
      row = row < p.n ? row : p.n - 1;               // in bounds; not stored below
#pragma unroll
      for (int v = 0; v < 2; ++v) raw[r][v] = load_row(logits + row * p.ld, col0 + v * VE, C, -INFINITY);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = first + r * RG + slot;
      const bool row_ok = row < p.n;
      // both vectors in order; what is not a score stands at an end: +inf and
      // NaN without sign in front, NaN with a sign behind (absent already)
      I a[2][VE];
      bool odd = false;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        order_items<T>(raw[r][v], col0 + v * VE, a[v]);
        sort_items<VE>(a[v]);
        odd |= !items_regular<T>(a[v][0], a[v][VE - 1]);
      }
      if (__ballot(odd)) {                           // rare: again, without NaN
        bad |= odd;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          make_items<T>(raw[r][v], col0 + v * VE, a[v]);
          sort_items<VE>(a[v]);
        }
      }
      if constexpr (L > 0) {
        I list[L];
        // the lane's own list: its two halves joined, or the larger part of both
        constexpr int H = N < L ? N : L;             // items in use
        if constexpr (L > VE) {
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            list[i] = item_max(a[0][i], a[1][VE - 1 - i]);
            list[VE + i] = item_min(a[0][i], a[1][VE - 1 - i]);
          }
          merge_bitonic<VE>(list);
          merge_bitonic<VE>(list + VE);
#pragma unroll
          for (int i = N; i < L; ++i) list[i] = I{0};
        } else {
          static_assert(L == VE, "lists of whole vectors");
#pragma unroll
          for (int i = 0; i < VE; ++i) list[i] = item_max(a[0][i], a[1][VE - 1 - i]);
          merge_bitonic<VE>(list);
        }
        list_levels<LPR, L, 1, H>(list);
        // entry j is written by lane j mod LPR
#pragma unroll
        for (int q = 0; q < (L + LPR - 1) / LPR; ++q) {
          const int j = q * LPR + li;
          I e = list[q * LPR < L ? q * LPR : 0];
#pragma unroll
          for (int i = 1; i < LPR && q * LPR + i < L; ++i) e = item_pick(li == i, list[q * LPR + i], e);
          if (row_ok && j < L && j < p.K) put_entry<T>(p, row, j, e);
        }
      } else {
        I s[N];
#pragma unroll
        for (int i = 0; i < VE; ++i) {               // the second half mirrored: larger parts in front
          s[i] = item_max(a[0][i], a[1][VE - 1 - i]);
          s[VE + i] = item_min(a[0][i], a[1][VE - 1 - i]);
        }
        merge_bitonic<VE>(s);
        merge_bitonic<VE>(s + VE);
        group_merge_levels<LPR, N, 2>(s, li);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (row_ok && col0 + i < p.K) put_entry<T>(p, row, col0 + i, s[i]);
      }
      // entries past the classes the group holds
      constexpr int HELD = L > 0 ? L : LPR * N;
      if (HELD < GCN_MAX_TOP && row_ok)
        for (int64_t j = HELD + li; j < p.K; j += LPR) put_entry<T>(p, row, j, I{0});
    }
  }
  if (bad) raise_flag(p.flag);
}

// Longer rows: a workgroup lists what reaches a bound (longrow.h) and counts
// every listed item into its place.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void top_row_kernel(TopParams p) {
  __shared__ TopList<NT> sh;
  const int64_t row = p.row0 + blockIdx.x;
  const LongRow<T, NT> r(reinterpret_cast<const T*>(p.logits) + row * p.ld, (int)p.C);
  const int K = (int)p.K;
  float mx;
  bool bad;
  const int cnt = list_top(r, K, sh, mx, bad);
  if (bad) raise_flag(p.flag);
  rank_list<NT>(sh, cnt, K, [&](int place, double e) { put_entry<T>(p, row, place, Item64{e}); });
  for (int j = cnt + (int)threadIdx.x; j < K; j += NT) put_entry<T>(p, row, j, Item64{0.0});
}

// ------------------------------------------------------------- launches ----

constexpr int64_t MAX_BLOCKS = 65536;
// Rows a lane group takes per iteration (their loads go out together): 2 where one
// would give more than this many workgroups, else 1.  Above, two and one: 2^21 x
// 64 fp16 85 and 86 us, 2^20 x 64 fp32 76 and 79 (2^18 x 512 fp16, sorted: 237 and
// 233); below: 200000 x 40 fp32 16.9 and 16.2, 2^18 x 64 fp16 12.6 and 12.3.
constexpr int64_t R2_GROUPS = 16384;
// Threads of a long row's workgroup.  256, 512 and 1024 threads, us:
//   16384 x  1100 fp16  K = 64  131  225  428   K = 128  990 1210 1664
//    8192 x  4001 fp32  K = 64   58   78  140   K = 256  822  400  473
//    4096 x 16001 fp16  K = 20   41   39   76   K = 256  546  271  323
//    2048 x 50001 bf16  K = 64   76   72   77   K = 256  691  192  182
//     128 x 50001 bf16  K = 64   28   18   14
//    2048 x 131072 fp32 K = 8   346  331  316
// Few threads where the pass is short and the bound of list_top close enough
// (its list grows with K against the threads), many where a row is long or there
// are not two rows a compute unit.
constexpr int64_t SHORT_VECS = 1024, MIDDLE_VECS = 4096, LONG_VECS = 8192, FEW_ROWS = 512, SMALL_K = 128;
int row_threads(int64_t n, int64_t nvec, int64_t K) {
  if (nvec <= SHORT_VECS && K <= SMALL_K) return 256;
  return nvec <= MIDDLE_VECS || (nvec <= LONG_VECS && n > FEW_ROWS) ? 512 : 1024;
}

template <typename T, int LPR, int L>
hipError_t launch_l(const TopParams& p, hipStream_t s) {
  constexpr int64_t RG = 4 * (64 / LPR);
  const int r = (p.n + RG - 1) / RG > R2_GROUPS ? 2 : 1;
  const int64_t nb = std::min<int64_t>((p.n + r * RG - 1) / (r * RG), MAX_BLOCKS);
  if (r == 2)
    hipLaunchKernelGGL((top_group_kernel<T, LPR, L, 2>), dim3((unsigned)nb), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((top_group_kernel<T, LPR, L, 1>), dim3((unsigned)nb), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_lpr(const TopParams& p, hipStream_t s) {
  if (p.K <= 8) return launch_l<T, LPR, 8>(p, s);
  if (p.K <= 16) return launch_l<T, LPR, 16>(p, s);
  return launch_l<T, LPR, 0>(p, s);
}
template <typename T>
hipError_t launch_rows(const TopParams& params, hipStream_t s) {
  const int64_t nvec = (params.C + Vec<T>::N - 1) / Vec<T>::N;
  return launch_long_rows(params, 1, [&](const TopParams& p, int64_t rows) {
    const dim3 grid((unsigned)rows);
    switch (row_threads(p.n, nvec, p.K)) {
      case 256: hipLaunchKernelGGL((top_row_kernel<T, 256>), grid, dim3(256), 0, s, p); break;
      case 512: hipLaunchKernelGGL((top_row_kernel<T, 512>), grid, dim3(512), 0, s, p); break;
      default: hipLaunchKernelGGL((top_row_kernel<T, 1024>), grid, dim3(1024), 0, s, p);
    }
    return hipGetLastError();
  });
}
template <typename T>
hipError_t launch_t(const TopParams& p, hipStream_t s) {
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

size_t top_workspace_bytes(int, int64_t, int64_t, int64_t) { return 256; }

hipError_t top_launch(int prec, const TopParams& p, void*, hipStream_t s) {
  switch (prec) {
    case 0: return launch_t<float>(p, s);
    case 1: return launch_t<f16>(p, s);
    case 2: return launch_t<bf16>(p, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace gcn
