// The foremost pages of one (sequence, KV head), picked by the threads of one CTA: forced pages first, then by score, then the
// lower page.  Scores come as unsigned 64-bit keys of the same order.  The candidates for the last places are narrowed down: the
// range of their keys is cut into equal parts, those in parts above the one that holds the last place are in, those below are out,
// and what is left goes round again until it is few enough to be ranked by comparing all with all.
#pragma once
#include <limits.h>

#include "rkv_internal.h"

namespace rkv {

constexpr int kMostPages = kSelectCluster * kSelectMaxKeysPerCta / 16;   // longest context in pages of 16
constexpr int kRanked = 64;

// A score as an unsigned number of the same order.
__device__ __forceinline__ uint64_t score_key(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s == 0.0 ? 0.0 : s);   // (one zero)
  return (u >> 63) != 0 ? ~u : u | (1ull << 63);
}

template <int NT>
struct PickShared {
  uint64_t lo[NT / 32], hi[NT / 32], cand[kRanked];
  int at[kRanked], scan[NT / 32], bins[2 * NT], pick[3];
  uint32_t in[(kMostPages + 31) / 32];       // the pages that are in
};

__device__ __forceinline__ uint64_t warp_max(uint64_t x) {
  const uint32_t h = (uint32_t)(x >> 32), m = __reduce_max_sync(0xffffffffu, h);
  return (uint64_t)m << 32 | __reduce_max_sync(0xffffffffu, h == m ? (uint32_t)x : 0u);
}

template <int NT>
__device__ __forceinline__ void block_range(uint64_t& lo, uint64_t& hi, PickShared<NT>& sh, int tid) {
  lo = ~warp_max(~lo);
  hi = warp_max(hi);
  if ((tid & 31) == 0) {
    sh.lo[tid >> 5] = lo;
    sh.hi[tid >> 5] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    lo = min(lo, sh.lo[w]);
    hi = max(hi, sh.hi[w]);
  }
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
  *total = all;
  return before + inc - x;
}

// put(k, page): the k-th of the m = min(top, pages) picked ones in ascending order, from any thread.  keys: [pages]; sm_k:
// room for `pages` of them; also(i): called for every page while its key is on its way.  All NT threads call it.
template <int NT, typename Put, typename Also>
__device__ __forceinline__ void pick_pages(const uint64_t* keys, int pages, int top, int force_first, int force_last, uint64_t* sm_k,
                                           PickShared<NT>& sh, int tid, Put put, Also also) {
  const int lane = tid & 31, m = min(top, pages);
  const int first = min(force_first, pages), last = min(force_last, pages - first);
  if (m == pages || first + last >= m) {   // all of them, or no room beside the forced ones: the lower of these
    for (int i = tid; i < m; i += NT) put(i, m == pages || i < first ? i : pages - last + (i - first));
    return;
  }
  const int lo_i = first, hi_i = pages - last;   // the pages that compete
  int want = m - first - last;
  uint64_t c_lo = ~0ull, c_hi = 0ull;            // the candidates: those with a key of c_lo .. c_hi
#pragma unroll 4
  for (int i = tid; i < pages; i += NT) {
    const uint64_t s = __ldcg(reinterpret_cast<const unsigned long long*>(keys) + i);
    also(i);
    sm_k[i] = s;
    if (i >= lo_i && i < hi_i) {
      c_lo = min(c_lo, s);
      c_hi = max(c_hi, s);
    }
  }
  sh.bins[2 * tid] = sh.bins[2 * tid + 1] = 0;
  block_range<NT>(c_lo, c_hi, sh, tid);
  int count = hi_i - lo_i;
  while (count > kRanked && count != want && c_lo < c_hi) {
    // 2^shift keys to a part, so that there are at least NT / 2 parts in use and no more than there are bins
    constexpr int kLog = NT >= 512 ? 10 : NT >= 256 ? 9 : 8;
    static_assert(1 << kLog <= 2 * NT, "a bin for each part");
    const int bits = 64 - __clzll((long long)(c_hi - c_lo)), shift = bits > kLog ? bits - kLog : 0;
    for (int i = lo_i + tid; i < hi_i; i += NT) {
      const uint64_t s = sm_k[i];
      if (s >= c_lo && s <= c_hi) atomicAdd(&sh.bins[(int)((c_hi - s) >> shift)], 1);
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
    // the part's own range, without another look at the keys where the candidates can be ranked already
    const uint64_t n_hi = c_hi - ((uint64_t)pick << shift);
    const uint64_t width = (1ull << shift) - 1, n_lo = n_hi - c_lo < width ? c_lo : n_hi - width;
    if (count <= kRanked || count == want) {
      c_lo = n_lo;
      c_hi = n_hi;
      break;
    }
    uint64_t e_lo = ~0ull, e_hi = 0ull;
    for (int i = lo_i + tid; i < hi_i; i += NT) {
      const uint64_t s = sm_k[i];
      if (s >= n_lo && s <= n_hi) {
        e_lo = min(e_lo, s);
        e_hi = max(e_hi, s);
      }
    }
    block_range<NT>(e_lo, e_hi, sh, tid);
    c_lo = e_lo;
    c_hi = e_hi;
  }
  // in: the forced ones and those above the candidates
  const int words = (pages + 31) >> 5;
  __syncthreads();                                         // (pick[] is no longer read)
  if (tid == 0) sh.pick[0] = 0;
  __syncthreads();
  const bool whole = count == want, ties = count > kRanked && !whole;   // all candidates; more of one score than are ranked
  for (int i0 = (tid >> 5) * 32; i0 < words * 32; i0 += NT) {
    const int i = i0 + lane;
    const bool competes = i >= lo_i && i < hi_i;
    const uint64_t s = competes ? sm_k[i] : 0ull;
    const bool in = i < pages && (!competes || s > c_hi || (whole && s >= c_lo));
    const uint32_t mask = __ballot_sync(0xffffffffu, in);
    if (lane == 0) sh.in[i0 >> 5] = mask;
    if (competes && !whole && !ties && s >= c_lo && s <= c_hi) {
      const int k = atomicAdd(&sh.pick[0], 1);             // (any order: they are ranked)
      sh.cand[k] = s;
      sh.at[k] = i;
    }
  }
  __syncthreads();
  if (!whole && !ties) {   // a warp per candidate, two of the others to a lane
    static_assert(kRanked == 64, "two to a lane");
    const uint64_t k0 = lane < count ? sh.cand[lane] : 0ull, k1 = lane + 32 < count ? sh.cand[lane + 32] : 0ull;
    const int a0 = lane < count ? sh.at[lane] : INT_MAX, a1 = lane + 32 < count ? sh.at[lane + 32] : INT_MAX;
    for (int c = tid >> 5; c < count; c += NT / 32) {
      const uint64_t s = sh.cand[c];
      const int i = sh.at[c];
      const int rank = __popc(__ballot_sync(0xffffffffu, k0 > s || (k0 == s && a0 < i))) +
                       __popc(__ballot_sync(0xffffffffu, k1 > s || (k1 == s && a1 < i)));
      if (lane == 0 && rank < want) atomicOr(&sh.in[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
  }
  if (ties) {   // the first `want` of them
    int before = 0;
    for (int i0 = 0; i0 < pages; i0 += NT) {
      const int i = i0 + tid;
      const bool c = i >= lo_i && i < hi_i && sm_k[i] >= c_lo && sm_k[i] <= c_hi;
      int all;
      const int at = before + block_scan<NT>(c ? 1 : 0, sh, tid, &all);
      if (c && at < want) atomicOr(&sh.in[i >> 5], 1u << (i & 31));
      before += all;
      __syncthreads();
    }
  }
  int before = 0;
  for (int w0 = 0; w0 < words; w0 += NT) {
    uint32_t mask = w0 + tid < words ? sh.in[w0 + tid] : 0u;
    int all;
    int at = before + block_scan<NT>(__popc(mask), sh, tid, &all);
    for (; mask != 0u; mask &= mask - 1u) put(at++, (w0 + tid) * 32 + __ffs(mask) - 1);
    before += all;
    __syncthreads();
  }
}

}  // namespace rkv
