// The foremost pages of one (sequence, KV head), picked by the threads of one CTA: forced pages first, then by score, then the
// lower page.  The candidates for the last places are narrowed down: the range of their scores is cut into equal parts (the part
// is a monotone function of the score), those in parts above the one that holds the last place are in, those below are out, and
// what is left goes round again until it is few enough to be ranked by comparing all with all.
#pragma once
#include "rkv_internal.h"

namespace rkv {

constexpr int kMostPages = kSelectCluster * kSelectMaxKeysPerCta / 16;   // longest context in pages of 16
constexpr int kRanked = 64;

template <int NT>
struct PickShared {
  double range[NT / 32][2], cand[kRanked];
  int at[kRanked], scan[NT / 32], bins[2 * NT], pick[3];
  uint32_t in[(kMostPages + 31) / 32];       // the pages that are in
};

template <int NT>
__device__ __forceinline__ void block_range(double& lo, double& hi, PickShared<NT>& sh, int tid) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = fmin(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmax(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  if ((tid & 31) == 0) {
    sh.range[tid >> 5][0] = lo;
    sh.range[tid >> 5][1] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    lo = fmin(lo, sh.range[w][0]);
    hi = fmax(hi, sh.range[w][1]);
  }
  __syncthreads();
}

template <int NT>
__device__ __forceinline__ int block_scan(int x, PickShared<NT>& sh, int tid, int* total) {   // exclusive
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if ((tid & 31) >= o) inc += y;
  }
  if ((tid & 31) == 31) sh.scan[tid >> 5] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    const int y = sh.scan[w];
    if (w < (tid >> 5)) before += y;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + inc - x;
}

// put(k, page): the k-th of the m = min(top, pages) picked ones in ascending order, from any thread.  score: finite, [pages];
// sm_s: room for `pages` of them.  All NT threads call it.
template <int NT, typename Put>
__device__ __forceinline__ void pick_pages(const double* score, int pages, int top, int force_first, int force_last, double* sm_s,
                                           PickShared<NT>& sh, int tid, Put put) {
  const int lane = tid & 31, m = min(top, pages);
  if (m == pages) {
    for (int i = tid; i < m; i += NT) put(i, i);
    return;
  }
  const int first = min(force_first, pages), last = min(force_last, pages - first);
  if (first + last >= m) {   // no room beside the forced pages: the lower ones
    for (int i = tid; i < m; i += NT) put(i, i < first ? i : pages - last + (i - first));
    return;
  }
  const int lo_i = first, hi_i = pages - last;   // the pages that compete
  int want = m - first - last;
  double c_lo = INFINITY, c_hi = -INFINITY;      // the candidates: those with a score of c_lo .. c_hi
#pragma unroll 4
  for (int i = lo_i + tid; i < hi_i; i += NT) {
    const double s = __ldcg(score + i);
    sm_s[i] = s;
    c_lo = fmin(c_lo, s);
    c_hi = fmax(c_hi, s);
  }
  sh.bins[2 * tid] = sh.bins[2 * tid + 1] = 0;
  block_range<NT>(c_lo, c_hi, sh, tid);
  int count = hi_i - lo_i;
  while (count > kRanked && count != want && c_lo < c_hi) {
    const double f = 2 * NT / (c_hi - c_lo);
    auto bin = [&](double s) { return min(2 * NT - 1, (int)((c_hi - s) * f)); };
    for (int i = lo_i + tid; i < hi_i; i += NT) {
      const double s = sm_s[i];
      if (s >= c_lo && s <= c_hi) atomicAdd(&sh.bins[bin(s)], 1);
    }
    __syncthreads();
    const int a0 = sh.bins[2 * tid], a1 = sh.bins[2 * tid + 1];
    sh.bins[2 * tid] = sh.bins[2 * tid + 1] = 0;   // (for the next round)
    int all;
    const int at = block_scan<NT>(a0 + a1, sh, tid, &all);
    if (at < want && want <= at + a0 + a1) {       // one thread's
      const bool second = want > at + a0;
      sh.pick[0] = 2 * tid + second;
      sh.pick[1] = second ? at + a0 : at;
      sh.pick[2] = second ? a1 : a0;
    }
    __syncthreads();
    const int pick = sh.pick[0];
    want -= sh.pick[1];
    count = sh.pick[2];
    double n_lo = INFINITY, n_hi = -INFINITY;
    for (int i = lo_i + tid; i < hi_i; i += NT) {
      const double s = sm_s[i];
      if (s >= c_lo && s <= c_hi && bin(s) == pick) {
        n_lo = fmin(n_lo, s);
        n_hi = fmax(n_hi, s);
      }
    }
    block_range<NT>(n_lo, n_hi, sh, tid);
    c_lo = n_lo;
    c_hi = n_hi;
  }
  // in: the forced ones and those above the candidates
  const int words = (pages + 31) >> 5;
  if (tid == 0) sh.pick[0] = 0;
  __syncthreads();
  const bool ties = count > kRanked && count != want;      // more candidates of one score than are ranked
  for (int i0 = (tid >> 5) * 32; i0 < words * 32; i0 += NT) {
    const int i = i0 + lane;
    const bool competes = i >= lo_i && i < hi_i;
    const double s = competes ? sm_s[i] : 0.0;
    const bool in = i < pages && (!competes || s > c_hi || (count == want && s >= c_lo));
    const uint32_t mask = __ballot_sync(0xffffffffu, in);
    if (lane == 0) sh.in[i0 >> 5] = mask;
    if (competes && count != want && !ties && s >= c_lo && s <= c_hi) {
      const int k = atomicAdd(&sh.pick[0], 1);             // (any order: they are ranked)
      sh.cand[k] = s;
      sh.at[k] = i;
    }
  }
  __syncthreads();
  if (count != want && !ties) {
    if (tid < count) {
      const double s = sh.cand[tid];
      const int i = sh.at[tid];
      int rank = 0;
      for (int k = 0; k < count; ++k) rank += sh.cand[k] > s || (sh.cand[k] == s && sh.at[k] < i);
      if (rank < want) atomicOr(&sh.in[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
  }
  if (ties) {   // the first `want` of them
    int before = 0;
    for (int i0 = 0; i0 < pages; i0 += NT) {
      const int i = i0 + tid;
      const bool c = i >= lo_i && i < hi_i && sm_s[i] >= c_lo && sm_s[i] <= c_hi;
      int all;
      const int at = before + block_scan<NT>(c ? 1 : 0, sh, tid, &all);
      if (c && at < want) atomicOr(&sh.in[i >> 5], 1u << (i & 31));
      before += all;
    }
    __syncthreads();
  }
  int before = 0;
  for (int w0 = 0; w0 < words; w0 += NT) {
    uint32_t mask = w0 + tid < words ? sh.in[w0 + tid] : 0u;
    int all;
    int at = before + block_scan<NT>(__popc(mask), sh, tid, &all);
    for (; mask != 0u; mask &= mask - 1u) put(at++, (w0 + tid) * 32 + __ffs(mask) - 1);
    before += all;
  }
}

}  // namespace rkv
