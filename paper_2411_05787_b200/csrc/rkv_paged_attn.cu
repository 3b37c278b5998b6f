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
// through distributed shared memory, or through partials in the workspace and a fold launch.
#include <cuda_bf16.h>

#include "rkv_internal.h"
#include "rkv_ptx.cuh"

namespace rkv {
namespace {

constexpr int kPStages = 3;
constexpr int kPHalfBytes = kTile * kHeadDim * 2;       // K (or V) of one tile
constexpr int kPStageBytes = 2 * kPHalfBytes;
constexpr int kPWarps = 4;                              // MMA warps; warp kPWarps is the copy warp
constexpr int kPThreads = 32 * (kPWarps + 1);
constexpr int kPOPad = 132;                             // floats per head row in the merge buffer
constexpr int kPQPad = 68;                              // words per query row
constexpr int kPBarsAt = kPStages * kPStageBytes;
constexpr int kPRowsAt = kPBarsAt + 64;                 // int [stages][4]: rows that count in each 16-row block
constexpr int kPQAt = kPRowsAt + kPStages * 16 + 16;
constexpr int kPMaxAt = kPQAt + kMaxGroup * kPQPad * 4;
constexpr int kPSmem = kPMaxAt + kPWarps * kMaxGroup * 4 + 1024;
static_assert(kPQAt % 16 == 0, "ldmatrix rows");
static_assert(2 * (kPSmem + 1024) <= 228 * 1024, "two CTAs per SM");
constexpr int kPMergeL = kPWarps * kMaxGroup * kPOPad;  // merge buffer, in floats, over the stages
constexpr int kPMergeM = kPMergeL + kPWarps * kMaxGroup;
constexpr int kPSumAt = kPStageBytes;                   // cluster: this CTA's share, [8][128] and [8][2] floats
static_assert((kPMergeM + kMaxGroup) * 4 <= kPStageBytes, "merge buffer in one stage");

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}

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

template <bool kCluster, bool kListed>
__global__ void __launch_bounds__(kPThreads, 2)
paged_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const PagedAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int b = blockIdx.z, g = blockIdx.y, split = blockIdx.x, n_cta = gridDim.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kPBarsAt, bar_empty = bar_full + 8 * kPStages;
  int* sm_rows = reinterpret_cast<int*>(smem + kPRowsAt);
  uint32_t* sm_q = reinterpret_cast<uint32_t*>(smem + kPQAt);
  float* sm_wm = reinterpret_cast<float*>(smem + kPMaxAt);
  if (tid == 0) {
    for (int s = 0; s < kPStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, kPWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * kPWarps) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  const int G = p.group, n_kv = p.c.n_kv_heads, shift = p.c.page_shift;
  const int piece = min(1 << shift, kTile), pieces = kTile / piece;   // positions of a piece, pieces of a tile
  const int64_t head0 = ((int64_t)b * p.n_q_heads + (int64_t)g * G) * kHeadDim;
  __syncthreads();
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  uint4 qv = make_uint4(0u, 0u, 0u, 0u);
  if (tid < G * 16) qv = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + head0) + tid);
  const Span sp = span_of(p, b, kListed);
  if (act == 0) return;
  if (sp.cut && tid == 0 && split == 0 && g == 0) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
  if (sp.count <= 0 && (kCluster || sp.n == 0)) {   // nothing cached (the fold knows of it by itself)
    if (kCluster && split == 0 && tid < kHeadDim)
      for (int h = 0; h < G; ++h) static_cast<__nv_bfloat16*>(p.out)[head0 + h * kHeadDim + tid] = __float2bfloat16(0.f);
    return;
  }
  const int total_tiles = (sp.count + kTile - 1) / kTile;
  const int n_tiles = total_tiles > split ? (total_tiles - split + n_cta - 1) / n_cta : 0;
  if (!kCluster && n_tiles == 0) return;   // (in a cluster an idle CTA still owns channels of the output)

  if (warp == kPWarps) {
    // ------------------------------------------------------------ copy warp
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    const int32_t* row = p.c.table + (int64_t)b * p.c.table_stride;
    const int32_t* list = kListed ? p.page_idx + ((int64_t)b * n_kv + g) * p.top : nullptr;
    const int per = 32 / pieces;             // tiles that 32 looked-up pieces make
    int y = 0, live = 0;                     // this lane's piece: its first row in the pool, positions of it that count
    for (int t = 0; t < n_tiles; ++t) {
      if (t % per == 0) {
        const int tt = t + lane / pieces;
        live = 0;
        if (tt < n_tiles) {
          const int v = (split + tt * n_cta) * kTile + (lane & (pieces - 1)) * piece;   // virtual position
          int i = -1, off = 0;
          if (v < sp.count) {
            i = kListed ? __ldcg(list + (v >> shift)) : (sp.from + v) >> shift;
            off = (kListed ? v : sp.from + v) & ((1 << shift) - 1);
          }
          if (i >= 0) {
            const int left = sp.n - ((i << shift) + off);
            const int pg = left > 0 ? __ldg(row + i) : 0;
            if ((unsigned)pg >= (unsigned)p.c.n_pages) {
              atomicOr(p.status, RKV_DEV_BAD_INDEX);
            } else {
              live = min(max(left, 0), piece);
              y = ((pg * n_kv + g) << shift) + off;      // (below 2^31: checked on the host)
            }
          }
        }
      }
      const int s = t % kPStages, use = t / kPStages;
      if (use > 0 && !mbar_wait(bar_empty + 8 * s, (use - 1) & 1)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        break;
      }
      const int from = (t % per) * pieces;     // the lanes of this tile's pieces
      const bool mine = lane >= from && lane < from + pieces && live > 0;
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      const int block_live = __shfl_sync(0xffffffffu, live, from + 16 * (lane & 3) / piece);
      if (lane < 4) sm_rows[4 * s + lane] = min(max(block_live - 16 * lane % piece, 0), 16);
      __syncwarp();
      const uint32_t bar = bar_full + 8 * s;
      if (lane == 0) mbar_expect_tx(bar, (uint32_t)__popc(who) * piece * kHeadDim * 4);
      __syncwarp();
      if (mine) {
        const uint32_t dst = smem_base + s * kPStageBytes + (lane - from) * piece * kHeadDim * 2;
        tma_load_tile(dst, &tm_k, y, bar, policy);
        tma_load_tile(dst + kPHalfBytes, &tm_v, y, bar, policy);
      }
    }
    return;
  }

  // ---------------------------------------------------------------- MMA warps
  const float ninf = -INFINITY;
  const int qd = lane >> 2, qc = (lane & 3) * 2;   // row of an 8-row group; first of the two heads this lane holds
  *reinterpret_cast<uint4*>(sm_q + (tid >> 4) * kPQPad + (tid & 15) * 4) = qv;   // (zeros for heads beyond the group)
  consumer_bar_n<32 * kPWarps>();
  uint32_t qb[8][2];                               // B fragments of Q^T: [16-channel segment][k half]
  {
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
  float m0 = ninf, m1 = ninf, l0 = 0.f, l1 = 0.f;
  float o[8][4];                                   // [16-channel segment]: O^T rows qd, qd + 8, heads qc, qc + 1
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  // This warp's 16 rows lie in one piece: rows  at  .. of its block, the piece's second half of channels `half` further on.
  const uint32_t half = piece * 128;
  const uint32_t block_at = (16 * warp / piece) * piece * kHeadDim * 2 + (16 * warp % piece) * 128;
  const uint32_t lane_at = block_at + (lane & 15) * 128;
  const float sc = p.scale * kLog2e;               // scores in units of log 2

  for (int t = 0; t < n_tiles; ++t) {
    const int s = t % kPStages;
    if (!mbar_wait(bar_full + 8 * s, (t / kPStages) & 1)) {
      if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
      break;
    }
    const int rows = sm_rows[4 * s + warp];        // of this warp's block
    if (rows > 0) {
      const uint32_t at = smem_base + s * kPStageBytes + lane_at;
      float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};   // two accumulator chains
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const int chunk = 2 * ks + (lane >> 4);
        uint32_t a[4];
        ldsm_x4(a, at + (chunk >> 3) * half + (((chunk & 7) ^ (lane & 7)) << 4));
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
        ldsm_x4_t(a, smem_base + s * kPStageBytes + kPHalfBytes + block_at + vr * 128 + (chunk >> 3) * half +
                         (((chunk & 7) ^ (vr & 7)) << 4));
        if (rows < 16) {
          a[0] &= mk0;
          a[1] &= mk0;
          a[2] &= mk1;
          a[3] &= mk1;
        }
        mma_bf16(o[i], a, b0, b1);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_empty + 8 * s);
  }

  // The warps' accumulators, scaled to the CTA-wide maximum, summed up in shared memory.
#pragma unroll
  for (int sh = 4; sh <= 16; sh <<= 1) {
    l0 += __shfl_xor_sync(0xffffffffu, l0, sh);
    l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
  }
  if (lane < 4) *reinterpret_cast<float2*>(sm_wm + warp * kMaxGroup + qc) = make_float2(m0, m1);
  consumer_bar_n<32 * kPWarps>();   // every warp's maxima are visible, and nobody reads the stages any more
  float* sm = reinterpret_cast<float*>(smem);
  float M0 = ninf, M1 = ninf;
#pragma unroll
  for (int w = 0; w < kPWarps; ++w) {
    const float2 mw = *reinterpret_cast<const float2*>(sm_wm + w * kMaxGroup + qc);
    M0 = fmaxf(M0, mw.x);
    M1 = fmaxf(M1, mw.y);
  }
  const float e0 = (m0 == ninf) ? 0.f : ex2(m0 - M0), e1 = (m1 == ninf) ? 0.f : ex2(m1 - M1);
  {
    float* to = sm + (warp * kMaxGroup + qc) * kPOPad + qd;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      to[16 * i] = o[i][0] * e0;
      to[16 * i + 8] = o[i][2] * e0;
      to[kPOPad + 16 * i] = o[i][1] * e1;
      to[kPOPad + 16 * i + 8] = o[i][3] * e1;
    }
  }
  if (lane < 4) {
    sm[kPMergeL + warp * kMaxGroup + qc] = l0 * e0;
    sm[kPMergeL + warp * kMaxGroup + qc + 1] = l1 * e1;
    if (warp == 0) {
      sm[kPMergeM + qc] = M0;
      sm[kPMergeM + qc + 1] = M1;
    }
  }
  consumer_bar_n<32 * kPWarps>();
  const int64_t bg = (int64_t)b * n_kv + g;
  const int slot = p.first_slot + split;
  float* sm_sum = reinterpret_cast<float*>(smem + kPSumAt);
  float* part = kCluster ? sm_sum : p.partials + (bg * p.max_splits + slot) * PartialLayout::kFloats;
  for (int item = tid; item < G * 32; item += 32 * kPWarps) {   // (head, four channels)
    const float* src = sm + (item >> 5) * kPOPad + (item & 31) * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kPWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(src + w * kMaxGroup * kPOPad);
      acc.x += v.x;
      acc.y += v.y;
      acc.z += v.z;
      acc.w += v.w;
    }
    *reinterpret_cast<float4*>(part + (item >> 5) * kHeadDim + (item & 31) * 4) = acc;
  }
  float* sm_ml = sm_sum + kMaxGroup * kHeadDim;
  if (tid < G) {
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kPWarps; ++w) l += sm[kPMergeL + w * kMaxGroup + tid];
    const float m = sm[kPMergeM + tid];
    if (kCluster) {
      *reinterpret_cast<float2*>(sm_ml + 2 * tid) = make_float2(m, l);
    } else {
      float* ml = p.ml_t + bg * 16 * p.max_splits + slot;
      ml[(int64_t)tid * p.max_splits] = m;
      ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = l;
    }
  }
  if (kCluster) {
    // Every CTA finishes 128 / C channels of every head from its peers' shared memory; the second barrier keeps that
    // memory until the last reader is done.  (Threads that have left count as arrived.)
    __syncwarp();
    cluster_sync_alive();
    const int c_sh = __ffs(n_cta) - 1, per_sh = 5 - c_sh;      // C = 1, 2, 4 or 8; log2 of the items per head
    const int ch = (split << (7 - c_sh)) + (tid & ((1 << per_sh) - 1)) * 4;
    for (int h = tid >> per_sh; h < G; h += (32 * kPWarps) >> per_sh) {
      const uint32_t at = smem_u32(sm_sum + h * kHeadDim + ch), ml_at = smem_u32(sm_ml + 2 * h);
      float4 v[kAttnCluster];
      float2 e[kAttnCluster];
      float M = ninf, L = 0.f;
#pragma unroll
      for (int r = 0; r < kAttnCluster; ++r) {
        if (r < n_cta) {
          v[r] = ld_cluster4(map_rank(at, r));
          e[r] = ld_cluster2(map_rank(ml_at, r));
        }
      }
#pragma unroll
      for (int r = 0; r < kAttnCluster; ++r)
        if (r < n_cta) M = fmaxf(M, e[r].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < kAttnCluster; ++r) {
        if (r < n_cta) {
          const float w = (e[r].x == ninf) ? 0.f : ex2(e[r].x - M);
          L = fmaf(e[r].y, w, L);
          acc.x = fmaf(v[r].x, w, acc.x);
          acc.y = fmaf(v[r].y, w, acc.y);
          acc.z = fmaf(v[r].z, w, acc.z);
          acc.w = fmaf(v[r].w, w, acc.w);
        }
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;   // (every page of the sequence may be missing)
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + head0 + h * kHeadDim + ch) =
          make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    }
    __syncwarp();
    cluster_sync_alive();
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
  float m = tid < p.max_splits ? __ldcg(pm + tid) : -INFINITY, l = tid < p.max_splits ? __ldcg(pl + tid) : 0.f;
  if (act == 0) return;
  __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.out) + ((int64_t)b * p.n_q_heads + (int64_t)g * p.group + h) * kHeadDim;
  const int s0 = sp.from > 0 ? 0 : p.first_slot;               // the sequence's partials: slots s0 .. s1 - 1
  const int s1 = p.first_slot + min(grid_x, (sp.count + kTile - 1) / kTile);
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
  for (auto kernel : {paged_attn_kernel<true, false>, paged_attn_kernel<false, false>, paged_attn_kernel<true, true>,
                      paged_attn_kernel<false, true>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPSmem);
  return e;
}

cudaError_t launch_paged_attention(const PagedAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int n_seq,
                                   int grid_x, bool cluster, cudaStream_t st) {
  const bool listed = p.page_idx != nullptr;
  auto kernel = cluster ? (listed ? paged_attn_kernel<true, true> : paged_attn_kernel<true, false>)
                        : (listed ? paged_attn_kernel<false, true> : paged_attn_kernel<false, false>);
  return launch_ex(kernel, dim3(grid_x, p.c.n_kv_heads, n_seq), dim3(kPThreads), (size_t)kPSmem, st, cluster ? grid_x : 1,
                   tm_k, tm_v, p);
}

cudaError_t launch_paged_fold(const PagedAttnParams& p, int n_seq, int grid_x, cudaStream_t st) {
  static_assert(kMaxSplits <= 32 * kPFoldWarps && kHeadDim == 32 * kPFoldWarps, "one thread per partial, one per channel");
  return launch_ex(p.page_idx != nullptr ? paged_fold_kernel<true> : paged_fold_kernel<false>,
                   dim3(p.group, p.c.n_kv_heads, n_seq), dim3(32 * kPFoldWarps), 0, st, 1, p, grid_x);
}

}  // namespace rkv
