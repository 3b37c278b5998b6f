// Split-K grouped-query decode attention over a paged cache (sm_100a): all positions of a sequence, those behind a shared
// prefix, or the pages that the selection has listed.
//
//   s[h][j] = scale <q[h], K[j]>,  p = softmax_j s,  out[h] = sum_j p[h][j] V[j],   h in the group of one KV head.
//
// What bounds it: 512 bytes per position and KV head from HBM.  The shape is that of the packed caches' passes: one CTA per
// (sequence, KV head, split), two to an SM, four MMA warps with 16 positions of a 64-position tile each, a copy warp that
// keeps a ring of three 32 KB stages full.  A tile is gathered piece by piece: a piece is a page, or 64 positions of a larger
// one, and lands by one tensor-map copy as [half][rows][64 channels] with the 128-byte swizzle; the lanes of the copy warp
// look up 32 pieces at a time and each issues its own, so that pages of 16 (eight copies a tile) cost the warp no more
// issue time than pages of 64.  The copy warp also leaves, per 16-row block, how many of its rows count.
// S^T = K Q^T and O^T += V^T P^T run as m16n8k16 bf16 MMAs, the heads of the group being the N = 8 dimension, with fp32
// accumulators and the softmax statistics in fp32; the probabilities meet V as bf16 (2^-8 relative at most, the one rounding
// but the output's), and the sums that divide the output are those of the rounded values, so that what all values have in common
// comes through unrounded.
//
// The splits of a (sequence, KV head) meet in one of two ways: as a thread-block cluster of up to eight CTAs that finish the output
// through distributed shared memory, or through partials in the workspace and a fold launch.  The first kernel below serves one
// sequence and what clusters are fast enough for, the second the other batches and those behind a shared prefix; the rule, with both
// sides measured, is where they are launched.  Measured (one cache again
// and again, so part of it comes from L2): 32768 positions of 8 heads 24.6 us, 64 sequences of 2048 positions of 8 heads 78,
// 2048 listed positions of one sequence 8.7 with the selection.
#include <cuda_bf16.h>

#include "rkv_internal.h"
#include "rkv_pick.cuh"
#include "rkv_ptx.cuh"

namespace rkv {
namespace {

constexpr int kPHalfBytes = kTile * kHeadDim * 2;       // K (or V) of one tile
constexpr int kPStageBytes = 2 * kPHalfBytes;
constexpr int kPTileWarps = 4;                          // MMA warps that share a tile
constexpr int kPOPad = 132;                             // floats per head row in the merge buffer
constexpr int kPQPad = 68;                              // words per query row

// Merge buffer of W MMA warps, in floats: o [W][8][kPOPad], l [W][8], m [8].
template <int W>
struct Merge {
  static constexpr int kL = W * kMaxGroup * kPOPad, kM = kL + W * kMaxGroup, kBytes = (kM + kMaxGroup) * 4;
};

// Buffers of the first kernel.  Its wide form, for few CTAs, has a whole SM: two groups of MMA warps take alternate tiles.
// (Stages are a multiple of the groups: a stage must always be consumed by the same group, since a warp may only wait for its second
// phase after it has seen the first.)
template <bool kWide>
struct Lay {
  static constexpr int kStages = kWide ? 6 : 3, kGroups = kWide ? 2 : 1, kWarps = kPTileWarps * kGroups;
  static constexpr int kThreads = 32 * (kWarps + 1);    // warp kWarps is the copy warp
  static constexpr int kBarsAt = kStages * kPStageBytes;                     // full, empty [stages], peers' shares
  static constexpr int kRowsAt = (kBarsAt + 8 * (2 * kStages + 1) + 15) & ~15;   // int [stages][4]: rows that count in each block
  static constexpr int kQAt = kRowsAt + kStages * 16;
  static constexpr int kMaxAt = kQAt + kMaxGroup * kPQPad * 4;
  static constexpr int kListAt = kMaxAt + kWarps * kMaxGroup * 4;            // int [kMaxPicked]: pages picked by this CTA
  static constexpr int kRecvAt = kListAt + kMaxPicked * 4;   // cluster: float [sources][heads][128 / C], then (m, l) [sources][heads]
  static constexpr int kSmem = kRecvAt + (kMaxGroup * kHeadDim + kAttnCluster * kMaxGroup * 2) * 4 + 1024;
  static constexpr int kPickSharedAt = kMaxPickFrom * 8;     // behind the keys, in the stages
  static_assert(kStages % kGroups == 0 && kListAt % 16 == 0, "stages of one group, aligned buffers");
  static_assert(kPickSharedAt + (int)sizeof(PickShared<kThreads>) <= kStages * kPStageBytes, "selection in the stages");
  static_assert(Merge<kWarps>::kBytes <= kStages * kPStageBytes, "merge buffer in the stages");
};
static_assert(2 * (Lay<false>::kSmem + 1024) <= 228 * 1024, "two CTAs per SM");
static_assert(Lay<true>::kSmem <= 227 * 1024, "one CTA per SM");

// the balanced form: its merge buffer beside the stages (the next head's tiles are in them), and the sequences' tables
constexpr int kBStages = 2, kPWarps = kPTileWarps, kPThreads = 32 * (kPWarps + 1);
constexpr int kBBarsAt = kBStages * kPStageBytes;
constexpr int kBRowsAt = kBBarsAt + 64;
constexpr int kBQAt = kBRowsAt + 64;
constexpr int kBMaxAt = kBQAt + kMaxGroup * kPQPad * 4;
constexpr int kBMergeAt = (kBMaxAt + kPWarps * kMaxGroup * 4 + 15) & ~15;
constexpr int kBTablesAt = (kBMergeAt + Merge<kPWarps>::kBytes + 15) & ~15;
constexpr int kBSmem = kBTablesAt + kBalancedMaxSeq * 5 * 4 + 16 + 1024;
static_assert(2 * (kBSmem + 1024) <= 228 * 1024, "two CTAs per SM");
static_assert((kBalancedMaxSeq & (kBalancedMaxSeq - 1)) == 0, "binary search over the sequences");

// What a (sequence, KV head) attends: virtual positions 0 .. count - 1, either from .. n - 1 or the listed pages' one
// behind the other.
struct Span { int n, from, count; bool cut; };

__device__ __forceinline__ Span span_of(const PagedAttnParams& p, int b, bool listed) {
  const int64_t room = (int64_t)p.c.table_stride << p.c.page_shift;
  const int lim = room < p.max_len ? (int)room : p.max_len;
  Span s;
  const int len = __ldcg(p.c.len + b);
  s.n = min(max(len, 0), lim);
  s.cut = len > lim;
  if (listed) {
    const int pages = (s.n + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
    s.from = 0;
    s.count = min(p.top, pages) << p.c.page_shift;
  } else {
    s.from = s.n >= p.from ? p.from : 0;
    s.count = s.n - s.from;
  }
  return s;
}

// State and steps of an MMA warp.  One (sequence, KV head) at a time: queries(), tile() for each of its tiles, merge().
template <int W>   // MMA warps of the CTA
struct Consumer {
  uint32_t qb[8][2];              // B fragments of Q^T: [16-channel segment][k half]
  float m0, m1, l0, l1;           // running maximum (log 2) and sum of heads qc, qc + 1
  float o[8][4];                  // [16-channel segment]: O^T rows qd, qd + 8, heads qc, qc + 1

  __device__ __forceinline__ void reset() {
    m0 = m1 = -INFINITY;
    l0 = l1 = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }

  // qv: this thread's 16 bytes of the group's query rows (16 threads to a head; zeros for heads beyond the group)
  __device__ __forceinline__ void queries(uint4 qv, uint32_t* sm_q, int tid) {
    const int lane = tid & 31;
    if (tid < kMaxGroup * 16) *reinterpret_cast<uint4*>(sm_q + (tid >> 4) * kPQPad + (tid & 15) * 4) = qv;
    consumer_bar_n<32 * W>();
    const uint32_t q_at = smem_u32(sm_q) + (uint32_t)(lane & 7) * (kPQPad * 4) + (uint32_t)(lane >> 3) * 16u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t r[4];
      ldsm_x4(r, q_at + 64u * i);
      qb[2 * i][0] = r[0];
      qb[2 * i][1] = r[1];
      qb[2 * i + 1][0] = r[2];
      qb[2 * i + 1][1] = r[3];
    }
  }

  // The warp's 16-row block of a tile, of which `rows` > 0 count.  at: the block's first row (K; V lies kPHalfBytes on), of
  // channels 0 - 63; `half` bytes further those of channels 64 - 127.  sc: softmax scale in units of log 2.
  __device__ __forceinline__ void tile(uint32_t at, uint32_t half, int rows, float sc, int lane) {
    const float ninf = -INFINITY;
    const int qd = lane >> 2, qc = (lane & 3) * 2;   // row of an 8-row group; first of the two heads this lane holds
    float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};   // two accumulator chains
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const int chunk = 2 * ks + (lane >> 4);
      uint32_t a[4];
      ldsm_x4(a, at + (lane & 15) * 128 + (chunk >> 3) * half + (((chunk & 7) ^ (lane & 7)) << 4));
      if (ks & 1) mma_bf16(c2, a, qb[ks][0], qb[ks][1]);
      else mma_bf16(c, a, qb[ks][0], qb[ks][1]);
    }
    float x0 = (c[0] + c2[0]) * sc, x1 = (c[1] + c2[1]) * sc, x2 = (c[2] + c2[2]) * sc, x3 = (c[3] + c2[3]) * sc;
    if (qd >= rows) x0 = x1 = ninf;
    if (qd + 8 >= rows) x2 = x3 = ninf;
    float t0 = fmaxf(x0, x2), t1 = fmaxf(x1, x3);
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
      t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, sh));
      t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, sh));
    }
    const float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
    if (__any_sync(0xffffffffu, (n0 > m0) || (n1 > m1))) {
      const float a0 = (n0 == m0) ? 1.f : ex2(m0 - n0), a1 = (n1 == m1) ? 1.f : ex2(m1 - n1);
      l0 *= a0;
      l1 *= a1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i][0] *= a0;
        o[i][1] *= a1;
        o[i][2] *= a0;
        o[i][3] *= a1;
      }
      m0 = n0;
      m1 = n1;
    }
    const float z0 = (m0 == ninf) ? 0.f : m0, z1 = (m1 == ninf) ? 0.f : m1;
    const uint32_t pl = pack_bf16(ex2(x0 - z0), ex2(x1 - z1)), ph = pack_bf16(ex2(x2 - z0), ex2(x3 - z1));
    l0 += __uint_as_float(pl << 16) + __uint_as_float(ph << 16);
    l1 += __uint_as_float(pl & 0xffff0000u) + __uint_as_float(ph & 0xffff0000u);
    // P^T as the B operand: the two 8x8 [position][head] blocks transposed inside the warp
    const uint32_t b0 = movmatrix_t(pl), b1 = movmatrix_t(ph);
    // rows past the end may hold anything (even NaN): their values are cleared so that 0 * x stays 0
    uint32_t mk0 = 0xffffffffu, mk1 = 0xffffffffu;
    if (rows < 16) {
      mk0 = (qc < rows ? 0x0000ffffu : 0u) | (qc + 1 < rows ? 0xffff0000u : 0u);
      mk1 = (qc + 8 < rows ? 0x0000ffffu : 0u) | (qc + 9 < rows ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {                // V^T: 16 channels x 16 positions
      // blocks of the transposed load: (positions 0-7, channels 0-7), (0-7, 8-15), (8-15, 0-7), (8-15, 8-15)
      const int chunk = 2 * i + ((lane >> 3) & 1), vr = (lane & 7) + ((lane >> 4) << 3);
      uint32_t a[4];
      ldsm_x4_t(a, at + kPHalfBytes + vr * 128 + (chunk >> 3) * half + (((chunk & 7) ^ (vr & 7)) << 4));
      if (rows < 16) {
        a[0] &= mk0;
        a[1] &= mk0;
        a[2] &= mk1;
        a[3] &= mk1;
      }
      mma_bf16(o[i], a, b0, b1);
    }
  }

  // The warps' accumulators, scaled to the CTA-wide maximum, into sm (Merge<W>); sm_wm: [warps][8].
  __device__ __forceinline__ void merge(float* sm, float* sm_wm, int warp, int lane) {
    const float ninf = -INFINITY;
    const int qd = lane >> 2, qc = (lane & 3) * 2;
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, sh);
      l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
    }
    if (lane < 4) *reinterpret_cast<float2*>(sm_wm + warp * kMaxGroup + qc) = make_float2(m0, m1);
    consumer_bar_n<32 * W>();   // every warp's maxima are visible, and nobody reads the stages any more
    float M0 = ninf, M1 = ninf;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 mw = *reinterpret_cast<const float2*>(sm_wm + w * kMaxGroup + qc);
      M0 = fmaxf(M0, mw.x);
      M1 = fmaxf(M1, mw.y);
    }
    const float e0 = (m0 == ninf) ? 0.f : ex2(m0 - M0), e1 = (m1 == ninf) ? 0.f : ex2(m1 - M1);
    float* to = sm + (warp * kMaxGroup + qc) * kPOPad + qd;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      to[16 * i] = o[i][0] * e0;
      to[16 * i + 8] = o[i][2] * e0;
      to[kPOPad + 16 * i] = o[i][1] * e1;
      to[kPOPad + 16 * i + 8] = o[i][3] * e1;
    }
    if (lane < 4) {
      sm[Merge<W>::kL + warp * kMaxGroup + qc] = l0 * e0;
      sm[Merge<W>::kL + warp * kMaxGroup + qc + 1] = l1 * e1;
      if (warp == 0) {
        sm[Merge<W>::kM + qc] = M0;
        sm[Merge<W>::kM + qc + 1] = M1;
      }
    }
    consumer_bar_n<32 * W>();
  }
};

// Sums over the warps of what merge() left: item = (head, four channels); o into to[head][128]; (m, l) of one head.
template <int W>
__device__ __forceinline__ float4 warps_sum(const float* sm, int item) {
  const float* src = sm + (item >> 5) * kPOPad + (item & 31) * 4;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float4 v = *reinterpret_cast<const float4*>(src + w * kMaxGroup * kPOPad);
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  return acc;
}
template <int W>
__device__ __forceinline__ void publish(const float* sm, int G, int tid, float* to) {
  for (int item = tid; item < G * 32; item += 32 * W)
    *reinterpret_cast<float4*>(to + (item >> 5) * kHeadDim + (item & 31) * 4) = warps_sum<W>(sm, item);
}
template <int W>
__device__ __forceinline__ float2 head_ml(const float* sm, int h) {
  float2 ml = make_float2(sm[Merge<W>::kM + h], 0.f);
#pragma unroll
  for (int w = 0; w < W; ++w) ml.y += sm[Merge<W>::kL + w * kMaxGroup + h];
  return ml;
}

// The pieces of 32 / pieces tiles, one to a lane of the copy warp.
struct Pieces {
  int y, live;                     // first row in the pool, positions that count
  // virtual position v of a (sequence, KV head) that attends s (v >= s.count: nothing there)
  __device__ __forceinline__ void look_up(const PagedAttnParams& p, const Span& s, int b, int g, int v, bool listed,
                                          const int* picked = nullptr) {
    const int shift = p.c.page_shift, n_kv = p.c.n_kv_heads, piece = min(1 << shift, kTile);
    live = 0;
    if (v >= s.count) return;
    const int i = !listed             ? (s.from + v) >> shift
                  : picked != nullptr ? picked[v >> shift]
                                      : __ldcg(p.page_idx + ((int64_t)b * n_kv + g) * p.top + (v >> shift));
    const int off = (listed ? v : s.from + v) & ((1 << shift) - 1);
    if (i < 0) return;
    const int left = s.n - ((i << shift) + off);
    if (left <= 0) return;
    const int pg = __ldcg(p.c.table + (int64_t)b * p.c.table_stride + i);
    if ((unsigned)pg >= (unsigned)p.c.n_pages) {
      atomicOr(p.status, RKV_DEV_BAD_INDEX);
      return;
    }
    live = min(left, piece);
    y = ((pg * n_kv + g) << shift) + off;      // (below 2^31: checked on the host)
  }
};

// Requests the tile whose pieces the lanes from, from + 1, ... have looked up, into a stage; all lanes call it.
__device__ __forceinline__ void request_tile(const Pieces& pc, int from, int piece, uint32_t stage, int* rows, uint32_t bar,
                                             const CUtensorMap* tm_k, const CUtensorMap* tm_v, uint64_t policy, int lane) {
  const int pieces = kTile / piece;
  const bool mine = lane >= from && lane < from + pieces && pc.live > 0;
  const uint32_t who = __ballot_sync(0xffffffffu, mine);
  const int block_live = __shfl_sync(0xffffffffu, pc.live, from + 16 * (lane & 3) / piece);
  if (lane < 4) rows[lane] = min(max(block_live - 16 * lane % piece, 0), 16);
  __syncwarp();
  if (lane == 0) mbar_expect_tx(bar, (uint32_t)__popc(who) * piece * kHeadDim * 4);
  __syncwarp();
  if (mine) {
    const uint32_t dst = stage + (lane - from) * piece * kHeadDim * 2;
    tma_load_tile(dst, tm_k, pc.y, bar, policy);
    tma_load_tile(dst + kPHalfBytes, tm_v, pc.y, bar, policy);
  }
}

// After a wait that ran out: waits, again with a limit, until what was requested of the first `issued` tiles has landed.  Shared memory
// is another CTA's as soon as this one has gone.  (Where all waits end, the MMA warps have seen every tile land.)
template <int kStages>
__device__ __forceinline__ void await_tiles(uint32_t bar_full, int issued) {
#pragma unroll 1
  for (int s = 0; s < kStages; ++s) {
    const int uses = (issued - s + kStages - 1) / kStages;
    if (uses > 0) mbar_wait(bar_full + 8 * s, (uses - 1) & 1);
  }
}

__device__ __forceinline__ uint4 load_query(const PagedAttnParams& p, int b, int g, int tid) {
  uint4 qv = make_uint4(0u, 0u, 0u, 0u);
  const int64_t head0 = ((int64_t)b * p.n_q_heads + (int64_t)g * p.group) * kHeadDim;
  if (tid < p.group * 16) qv = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + head0) + tid);
  return qv;
}

// kPick: every CTA picks the pages of its (sequence, KV head) from their scores, all CTAs of a cluster the same ones, before it
// attends its share of them (a launch of the selection's own takes as long as the attention).
template <bool kCluster, bool kListed, bool kPick, bool kWide>
__global__ void __launch_bounds__(Lay<kWide>::kThreads, kWide ? 1 : 2)
paged_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const PagedAttnParams p) {
  using L = Lay<kWide>;
  constexpr int kStg = L::kStages, W = L::kWarps, NT = L::kThreads;
  extern __shared__ uint8_t smem_raw[];
  const int b = blockIdx.z, g = blockIdx.y, split = blockIdx.x, n_cta = gridDim.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + L::kBarsAt, bar_empty = bar_full + 8 * kStg, bar_recv = bar_empty + 8 * kStg;
  int* sm_rows = reinterpret_cast<int*>(smem + L::kRowsAt);
  uint32_t* sm_q = reinterpret_cast<uint32_t*>(smem + L::kQAt);
  float* sm_wm = reinterpret_cast<float*>(smem + L::kMaxAt);
  if (tid == 0) {
    for (int s = 0; s < kStg; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, kPTileWarps);
    }
    if (kCluster) mbar_init(bar_recv, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * W) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  const int G = p.group, n_kv = p.c.n_kv_heads;
  const int piece = min(1 << p.c.page_shift, kTile), pieces = kTile / piece;   // positions of a piece, pieces of a tile
  const int64_t head0 = ((int64_t)b * p.n_q_heads + (int64_t)g * G) * kHeadDim;
  __syncthreads();
  if (kCluster && n_cta > 1) {
    // Every CTA sends each of its peers that peer's share of the channels, with stores that credit the receiver's barrier.  It
    // is armed before the one cluster-wide barrier of the kernel, up here where it costs nothing.
    if (tid == 0) mbar_expect_tx(bar_recv, (uint32_t)(G * kHeadDim * 4 + n_cta * G * 8));
    __syncwarp();
    cluster_sync_alive();
  }
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  const uint4 qv = load_query(p, b, g, tid);
  const Span sp = span_of(p, b, kListed);
  if (act == 0) return;
  if (sp.cut && tid == 0 && split == 0 && g == 0) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
  if (sp.count <= 0 && (kCluster || sp.n == 0)) {   // nothing cached (the fold knows of it by itself)
    if (kPick && split == 0)
      for (int i = tid; i < p.top; i += NT) p.page_idx[((int64_t)b * n_kv + g) * p.top + i] = -1;
    if (kCluster && split == 0 && tid < kHeadDim)
      for (int h = 0; h < G; ++h) static_cast<__nv_bfloat16*>(p.out)[head0 + h * kHeadDim + tid] = __float2bfloat16(0.f);
    return;
  }
  int* picked = kPick ? reinterpret_cast<int*>(smem + L::kListAt) : nullptr;
  if constexpr (kPick) {   // in the stages, which are empty yet
    const int pages = (sp.n + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
    int32_t* idx = p.page_idx + ((int64_t)b * n_kv + g) * p.top;
    if (split == 0)
      for (int i = min(p.top, pages) + tid; i < p.top; i += NT) idx[i] = -1;
    pick_pages<NT>(p.keys + ((int64_t)b * n_kv + g) * p.key_stride, pages, p.top, p.first, p.last,
                          reinterpret_cast<uint64_t*>(smem), *reinterpret_cast<PickShared<NT>*>(smem + L::kPickSharedAt), tid,
                          [&](int k, int page) {
                            picked[k] = page;
                            if (split == 0) idx[k] = page;
                          },
                          [](int) {});
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // tiles will be copied to where the scores were
    __syncthreads();
  }
  const int total_tiles = (sp.count + kTile - 1) / kTile;
  const int n_tiles = total_tiles > split ? (total_tiles - split + n_cta - 1) / n_cta : 0;
  if (!kCluster && n_tiles == 0) return;   // (in a cluster an idle CTA still owns channels of the output)

  if (warp == W) {
    // ------------------------------------------------------------ copy warp
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    const int per = 32 / pieces;             // tiles that 32 looked-up pieces make
    Pieces pc;
    pc.y = pc.live = 0;
    for (int t = 0; t < n_tiles; ++t) {
      if (t % per == 0) {
        const int tt = t + lane / pieces;
        pc.look_up(p, sp, b, g, tt < n_tiles ? (split + tt * n_cta) * kTile + (lane & (pieces - 1)) * piece : sp.count, kListed,
                   picked);
        __syncwarp();
      }
      const int s = t % kStg, use = t / kStg;
      if (use > 0 && !mbar_wait(bar_empty + 8 * s, (use - 1) & 1)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        await_tiles<kStg>(bar_full, t);
        break;
      }
      request_tile(pc, (t % per) * pieces, piece, smem_base + s * kPStageBytes, sm_rows + 4 * s, bar_full + 8 * s, &tm_k, &tm_v,
                   policy, lane);
    }
    return;
  }

  // ---------------------------------------------------------------- MMA warps
  Consumer<W> mma;
  mma.queries(qv, sm_q, tid);
  mma.reset();
  // This warp's 16 rows lie in one piece, the piece's second half of channels `half` bytes further on.
  const uint32_t half = piece * 128;
  const int wb = warp % kPTileWarps, grp = warp / kPTileWarps;
  const uint32_t block_at = (16 * wb / piece) * piece * kHeadDim * 2 + (16 * wb % piece) * 128;
  const float sc = p.scale * kLog2e;               // scores in units of log 2
  for (int t = grp; t < n_tiles; t += L::kGroups) {
    const int s = t % kStg;
    if (!mbar_wait(bar_full + 8 * s, (t / kStg) & 1)) {
      if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
      await_tiles<kStg>(bar_full, min(t + kStg, n_tiles));
      break;
    }
    const int rows = sm_rows[4 * s + wb];          // of this warp's block
    if (rows > 0) mma.tile(smem_base + s * kPStageBytes + block_at, half, rows, sc, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_empty + 8 * s);
  }
  float* sm = reinterpret_cast<float*>(smem);      // (the stages are free by then)
  mma.merge(sm, sm_wm, warp, lane);
  if (!kCluster) {
    const int64_t bg = (int64_t)b * n_kv + g;
    const int slot = p.first_slot + split;
    publish<W>(sm, G, tid, p.partials + (bg * p.max_splits + slot) * PartialLayout::kFloats);
    if (tid < G) {
      const float2 v = head_ml<W>(sm, tid);
      float* ml = p.ml_t + bg * 16 * p.max_splits + slot;
      ml[(int64_t)tid * p.max_splits] = v.x;
      ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = v.y;
    }
    return;
  }
  // C = 1, 2, 4 or 8 CTAs; each finishes 128 / C channels of every head
  const int c_sh = __ffs(n_cta) - 1, own = kHeadDim >> c_sh;
  float* recv = reinterpret_cast<float*>(smem + L::kRecvAt);
  float* recv_ml = recv + kMaxGroup * kHeadDim;
  for (int item = tid; item < G * 32; item += 32 * W) {   // (head, four channels)
    const float4 acc = warps_sum<W>(sm, item);
    const int h = item >> 5, ch = (item & 31) * 4, to = ch / own;
    float* at = recv + (split * G + h) * own + (ch & (own - 1));
    if (n_cta == 1) *reinterpret_cast<float4*>(at) = acc;
    else st_async_f32x4(map_rank(smem_u32(at), to), acc, map_rank(bar_recv, to));
  }
  for (int i = tid; i < (G << c_sh); i += 32 * W) {
    const int h = i >> c_sh, to = i & (n_cta - 1);
    const float2 v = head_ml<W>(sm, h);
    float* at = recv_ml + 2 * (split * G + h);
    if (n_cta == 1) *reinterpret_cast<float2*>(at) = v;
    else st_async_f32x2(map_rank(smem_u32(at), to), v.x, v.y, map_rank(bar_recv, to));
  }
  if (n_cta == 1) {
    consumer_bar_n<32 * W>();
  } else if (!mbar_wait(bar_recv, 0)) {
    if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
    return;
  }
  const int per_sh = 5 - c_sh;                     // log2 of the items per head
  for (int item = tid; item < (G << per_sh); item += 32 * W) {
    const int h = item >> per_sh, ch = (item & ((1 << per_sh) - 1)) * 4;
    const float ninf = -INFINITY;
    float M = ninf, sum = 0.f;
    for (int r = 0; r < n_cta; ++r) M = fmaxf(M, recv_ml[2 * (r * G + h)]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = 0; r < n_cta; ++r) {
      const float2 e = *reinterpret_cast<const float2*>(recv_ml + 2 * (r * G + h));
      const float4 v = *reinterpret_cast<const float4*>(recv + (r * G + h) * own + ch);
      const float w = (e.x == ninf) ? 0.f : ex2(e.x - M);
      sum = fmaf(e.y, w, sum);
      acc.x = fmaf(v.x, w, acc.x);
      acc.y = fmaf(v.y, w, acc.y);
      acc.z = fmaf(v.z, w, acc.z);
      acc.w = fmaf(v.w, w, acc.w);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (every page of the sequence may be missing)
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + head0 + h * kHeadDim + split * own + ch) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
}

// ---------------------------------------------------------------------------------------------- batches: balanced form
// The tiles of all heads of all sequences, in order, are cut into equal runs, one per CTA, in a single wave, whatever the
// lengths (a head of m tiles counts as m + 1 units, the first of them empty, for what beginning and ending it costs).  The lengths are
// on the device, so every CTA sums them up itself.  A run covers the end of one head and the beginning of the next, or
// several whole ones; each piece of it leaves one split partial, slot = first_slot + CTA - first CTA of that head, and the head's first
// CTA records how many there are.  The copy warp walks the tiles without stopping at heads.
struct Run {   // the tiles of one (sequence, KV head) in a CTA's run, and the unit behind them
  int b, g, tile, count, next;
};

// The first tiles at or behind unit x of a run that ends at `end`; count = 0 when there are none.
__device__ __forceinline__ Run run_at(int x, int end, int b, const int* pref, const int* tiles) {
  Run s;
  s.count = 0;
  while (x < end && s.count == 0) {
    while (pref[b + 1] <= x) ++b;          // (sequences without tiles are stepped over)
    const int units = tiles[b] + 1, rem = x - pref[b];
    s.b = b;
    s.g = rem / units;
    const int unit = rem - s.g * units;
    s.next = min(x + units - unit, end);
    s.tile = max(unit - 1, 0);
    s.count = s.next - x - (unit == 0 ? 1 : 0);
    x = s.next;
  }
  return s;
}

template <bool kListed>
__global__ void __launch_bounds__(kPThreads, 2)
paged_balanced_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                      const PagedAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kBBarsAt, bar_empty = bar_full + 8 * kBStages;
  int* sm_rows = reinterpret_cast<int*>(smem + kBRowsAt);
  uint32_t* sm_q = reinterpret_cast<uint32_t*>(smem + kBQAt);
  float* sm_wm = reinterpret_cast<float*>(smem + kBMaxAt);
  float* sm_merge = reinterpret_cast<float*>(smem + kBMergeAt);
  int* sm_n = reinterpret_cast<int*>(smem + kBTablesAt);    // what a sequence attends (Span)
  int* sm_from = sm_n + kBalancedMaxSeq;
  int* sm_count = sm_from + kBalancedMaxSeq;
  int* sm_tiles = sm_count + kBalancedMaxSeq;               // of one head
  int* sm_pref = sm_tiles + kBalancedMaxSeq;                // units of all heads of the sequences before
  int* sm_most = sm_pref + kBalancedMaxSeq + 1;
  if (tid == 0) {
    for (int s = 0; s < kBStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, kPWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * kPWarps) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int n_kv = p.c.n_kv_heads, n_bg = p.n_seq * n_kv;
  for (int b = tid; b < p.n_seq; b += kPThreads) {
    const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
    Span sp = span_of(p, b, kListed);
    if (act == 0) sp.count = 0;
    else if (sp.cut && cta == 0) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
    sm_n[b] = sp.n;
    sm_from[b] = sp.from;
    sm_count[b] = sp.count;
    sm_tiles[b] = (sp.count + kTile - 1) / kTile;
  }
  __syncthreads();
  if (warp == 0) {
    int sum = 0, most = 0;
    for (int b0 = 0; b0 < p.n_seq; b0 += 32) {
      const int b = b0 + lane, mine = b < p.n_seq ? sm_tiles[b] : 0;
      most = max(most, mine);
      const int units = mine > 0 ? (mine + 1) * n_kv : 0;
      int inc = units;
#pragma unroll
      for (int sh = 1; sh < 32; sh <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, sh);
        if (lane >= sh) inc += up;
      }
      if (b < p.n_seq) sm_pref[b] = sum + inc - units;
      sum += __shfl_sync(0xffffffffu, inc, 31);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
      sm_pref[p.n_seq] = sum;
      *sm_most = most;
    }
  }
  __syncthreads();
  const uint32_t total = sm_pref[p.n_seq], most = *sm_most;   // (total * gridDim.x fits 32 bits: checked on the host)
  for (int i = cta * kPThreads + tid; i < n_bg; i += gridDim.x * kPThreads)
    if (sm_tiles[i / n_kv] == 0) p.counts[i] = 0;
  // No more CTAs than units, and no more than leave any head at most `room` partials (a head of m tiles touches at
  // most (m + 1) C / total + 2 runs; and at most m, each with a tile of it).
  const uint32_t room = p.max_splits - p.first_slot;
  uint32_t C = min(gridDim.x, total);
  if (most > room) C = min(C, room > 2 ? max((room - 2) * total / (most + 1), 1u) : 1u);
  if ((uint32_t)cta >= C) return;
  const int t0 = (int)(total * (uint32_t)cta / C), t1 = (int)(total * (uint32_t)(cta + 1) / C);
  int b = 0;   // the last sequence whose units begin at or before t0
  for (int step = kBalancedMaxSeq / 2; step > 0; step >>= 1)
    if (b + step < p.n_seq && sm_pref[b + step] <= t0) b += step;
  const int piece = min(1 << p.c.page_shift, kTile), pieces = kTile / piece;

  if (warp == kPWarps) {
    // ------------------------------------------------------------ copy warp
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    const int per = 32 / pieces;
    int it = 0;
    for (Run s = run_at(t0, t1, b, sm_pref, sm_tiles); s.count > 0; s = run_at(s.next, t1, s.b, sm_pref, sm_tiles)) {
      const Span sp = {sm_n[s.b], sm_from[s.b], sm_count[s.b], false};
      Pieces pc;
      pc.y = pc.live = 0;
      for (int i = 0; i < s.count; ++i, ++it) {
        if (i % per == 0) {
          const int ii = i + lane / pieces;
          pc.look_up(p, sp, s.b, s.g, ii < s.count ? (s.tile + ii) * kTile + (lane & (pieces - 1)) * piece : sp.count, kListed);
          __syncwarp();
        }
        const int st = it % kBStages, use = it / kBStages;
        if (use > 0 && !mbar_wait(bar_empty + 8 * st, (use - 1) & 1)) {
          if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
          await_tiles<kBStages>(bar_full, it);
          return;
        }
        request_tile(pc, (i % per) * pieces, piece, smem_base + st * kPStageBytes, sm_rows + 4 * st, bar_full + 8 * st, &tm_k,
                     &tm_v, policy, lane);
      }
    }
    return;
  }

  // ---------------------------------------------------------------- MMA warps
  const uint32_t half = piece * 128;
  const uint32_t block_at = (16 * warp / piece) * piece * kHeadDim * 2 + (16 * warp % piece) * 128;
  const float sc = p.scale * kLog2e;
  Consumer<kPWarps> mma;
  Run s = run_at(t0, t1, b, sm_pref, sm_tiles);
  if (s.count == 0) return;
  uint4 qv = load_query(p, s.b, s.g, tid);
  int it = 0;
  bool lost = false;
  for (;;) {
    mma.queries(qv, sm_q, tid);
    mma.reset();
    const Run next = run_at(s.next, t1, s.b, sm_pref, sm_tiles);
    if (next.count > 0) qv = load_query(p, next.b, next.g, tid);   // on its way while this piece's tiles are worked on
    for (int i = 0; i < s.count && !lost; ++i, ++it) {
      const int st = it % kBStages;
      if (!mbar_wait(bar_full + 8 * st, (it / kBStages) & 1)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        await_tiles<kBStages>(bar_full, it + kBStages);
        lost = true;   // a copy that never came: no further waits, but the warps still meet at the merges
        break;
      }
      const int rows = sm_rows[4 * st + warp];
      if (rows > 0) mma.tile(smem_base + st * kPStageBytes + block_at, half, rows, sc, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * st);
    }
    mma.merge(sm_merge, sm_wm, warp, lane);
    // runs [total c / C, total (c + 1) / C): unit y lies in the one of c = ((y + 1) C - 1) / total
    const int bg = s.b * n_kv + s.g;
    const uint32_t units = sm_tiles[s.b] + 1, head_at = sm_pref[s.b] + s.g * units;
    const int first = (int)(((head_at + 2) * C - 1) / total);   // the run of the head's first tile
    const int slot = p.first_slot + cta - first;
    publish<kPWarps>(sm_merge, p.group, tid, p.partials + ((int64_t)bg * p.max_splits + slot) * PartialLayout::kFloats);
    if (tid < p.group) {
      const float2 v = head_ml<kPWarps>(sm_merge, tid);
      float* ml = p.ml_t + (int64_t)bg * 16 * p.max_splits + slot;
      ml[(int64_t)tid * p.max_splits] = v.x;
      ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = v.y;
    }
    if (tid == 0 && s.tile == 0)
      p.counts[bg] = (int)(((head_at + units) * C - 1) / total) - first + 1;
    if (next.count == 0) return;
    s = next;
  }
}

// The output from the split partials: those of the shared positions, slots 0 .. first_slot - 1, where the sequence has them all,
// and its own behind them.  One CTA per (head, sequence): warp w takes every fourth partial, a lane four channels.
constexpr int kPFoldWarps = 4;
template <bool kListed>
__global__ void __launch_bounds__(32 * kPFoldWarps) paged_fold_kernel(const PagedAttnParams p, int grid_x) {
  __shared__ float sm_w[kMaxSplits], sm_red[2][kPFoldWarps];
  __shared__ __align__(16) float sm_o[kPFoldWarps][kHeadDim];
  const int h = blockIdx.x, g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t bg = (int64_t)b * p.c.n_kv_heads + g;
  const float* po = p.partials + bg * p.max_splits * PartialLayout::kFloats + h * kHeadDim + 4 * lane;
  const float* pm = p.ml_t + (bg * 16 + h) * p.max_splits;
  const float* pl = pm + (int64_t)kMaxGroup * p.max_splits;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  const Span sp = span_of(p, b, kListed);
  const int own = p.counts != nullptr ? __ldcg(p.counts + bg) : 0;
  float m = tid < p.max_splits ? __ldcg(pm + tid) : -INFINITY, l = tid < p.max_splits ? __ldcg(pl + tid) : 0.f;
  if (act == 0) return;
  __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.out) + ((int64_t)b * p.n_q_heads + (int64_t)g * p.group + h) * kHeadDim;
  const int s0 = sp.from > 0 ? 0 : p.first_slot;               // the sequence's partials: slots s0 .. s1 - 1
  const int s1 = p.first_slot + (p.counts != nullptr ? own : min(grid_x, (sp.count + kTile - 1) / kTile));
  if (tid < s0 || tid >= s1) {   // slots of older passes
    m = -INFINITY;
    l = 0.f;
  }
  float M = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) sm_red[0][warp] = M;
  __syncthreads();
  M = fmaxf(fmaxf(sm_red[0][0], sm_red[0][1]), fmaxf(sm_red[0][2], sm_red[0][3]));
  const float w = (m == -INFINITY) ? 0.f : ex2(m - M);
  sm_w[tid] = w;
  float L = l * w;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  if (lane == 0) sm_red[1][warp] = L;
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int s = s0 + warp; s < s1; s += kPFoldWarps) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(po + (int64_t)s * PartialLayout::kFloats));
    const float e = sm_w[s];
    if (e == 0.f) continue;      // (a partial without positions)
    acc.x = fmaf(x.x, e, acc.x);
    acc.y = fmaf(x.y, e, acc.y);
    acc.z = fmaf(x.z, e, acc.z);
    acc.w = fmaf(x.w, e, acc.w);
  }
  *reinterpret_cast<float4*>(&sm_o[warp][4 * lane]) = acc;
  __syncthreads();
  L = (sm_red[1][0] + sm_red[1][1]) + (sm_red[1][2] + sm_red[1][3]);
  const float x = (sm_o[0][tid] + sm_o[1][tid]) + (sm_o[2][tid] + sm_o[3][tid]);
  to[tid] = __float2bfloat16(L == 0.f ? 0.f : x / L);   // nothing cached, or no page there: zeros
}

}  // namespace

cudaError_t prepare_paged_attention() {
  cudaError_t e = cudaSuccess;
  for (auto kernel : {paged_attn_kernel<true, false, false, false>, paged_attn_kernel<false, false, false, false>,
                      paged_attn_kernel<true, true, false, false>, paged_attn_kernel<false, true, false, false>,
                      paged_attn_kernel<true, true, true, false>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<false>::kSmem);
  for (auto kernel : {paged_attn_kernel<true, false, false, true>, paged_attn_kernel<true, true, false, true>,
                      paged_attn_kernel<true, true, true, true>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<true>::kSmem);
  for (auto kernel : {paged_balanced_kernel<true>, paged_balanced_kernel<false>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBSmem);
  return e;
}

cudaError_t launch_paged_attention(const PagedAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int n_seq,
                                   int grid_x, bool cluster, bool wide, cudaStream_t st) {
  const bool listed = p.page_idx != nullptr, pick = p.keys != nullptr;
  const dim3 grid(grid_x, p.c.n_kv_heads, n_seq);
  if (wide) {
    auto kernel = pick     ? paged_attn_kernel<true, true, true, true>
                  : listed ? paged_attn_kernel<true, true, false, true>
                           : paged_attn_kernel<true, false, false, true>;
    return launch_ex(kernel, grid, dim3(Lay<true>::kThreads), (size_t)Lay<true>::kSmem, st, grid_x, tm_k, tm_v, p);
  }
  auto kernel = pick      ? paged_attn_kernel<true, true, true, false>
                : cluster ? (listed ? paged_attn_kernel<true, true, false, false> : paged_attn_kernel<true, false, false, false>)
                          : (listed ? paged_attn_kernel<false, true, false, false> : paged_attn_kernel<false, false, false, false>);
  return launch_ex(kernel, grid, dim3(Lay<false>::kThreads), (size_t)Lay<false>::kSmem, st, cluster ? grid_x : 1, tm_k, tm_v, p);
}

cudaError_t launch_paged_balanced(const PagedAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int n_cta,
                                  cudaStream_t st) {
  return launch_ex(p.page_idx != nullptr ? paged_balanced_kernel<true> : paged_balanced_kernel<false>, dim3(n_cta),
                   dim3(kPThreads), (size_t)kBSmem, st, 1, tm_k, tm_v, p);
}

cudaError_t launch_paged_fold(const PagedAttnParams& p, int n_seq, int grid_x, cudaStream_t st) {
  static_assert(kMaxSplits <= 32 * kPFoldWarps && kHeadDim == 32 * kPFoldWarps, "one thread per partial, one per channel");
  return launch_ex(p.page_idx != nullptr ? paged_fold_kernel<true> : paged_fold_kernel<false>,
                   dim3(p.group, p.c.n_kv_heads, n_seq), dim3(32 * kPFoldWarps), 0, st, 1, p, grid_x);
}

}  // namespace rkv
