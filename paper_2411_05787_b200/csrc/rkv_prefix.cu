// Attention of a whole batch over the positions that all its sequences share, read once (sm_100a, 5th-generation tensor cores).
//
// The query rows of one KV head, (sequence, head of the group) for all sequences, are up to 128 rows of one tile:
//   S = Q K^T  [128 rows x 128 positions],   P = 2^(S scale log2 e - m),   O += P V  [128 rows x 128 channels].
// A CTA takes 128 rows and every n-th tile of 128 positions, and leaves one split partial (O, m, l) per row; the fold that
// joins them with each sequence's own positions is that of rkv_paged_attn.cu.
//
// What bounds it: 512 bytes per position and KV head from HBM while there are few rows; from about 200 rows a KV head on, the
// tensor cores and the exponentials, 1024 clocks each per tile (4 x 128^3 products at 8192 a clock; 16384 exponentials at 16).
// So the steps of a tile run beside those of its neighbours: a copy warp keeps a ring of three 64 KB stages full, one thread
// issues tcgen05.mma, and two groups of four warps take alternate tiles, each with an S and an O of its own in tensor memory
// (512 columns in all): while one group is at its exponentials, the products of the other's tile run.  A thread has one row:
// maxima and sums need no exchange.  P goes back to tensor memory as bf16 over its S and is the A operand of O += P V;
// V, with its channels contiguous, is an MN-major B operand.  The accumulators are rescaled only when a row's maximum
// has grown by more than 2^8 since the last time, which keeps P below 2^8 and l exact to fp32; P is rounded to bf16
// (2^-8 relative at most), and l adds the rounded values up.
//
// A tile is gathered page by page, each of the four (K | V) x (channels 0-63 | 64-127) parts of a piece by one copy, so that
// the tile lies in shared memory as [part][128 rows][64 channels] with the 128-byte swizzle, whatever the page.  Pieces that
// are not there (behind the end, or a bad page number) are copied from behind the pool's last row, that is filled with zeros, and masked.
#include <cuda_bf16.h>

#include "rkv_internal.h"
#include "rkv_ptx.cuh"

namespace rkv {
namespace {

constexpr int kXStages = 3;
constexpr int kXRows = 128, kXTile = kPrefixTile;               // rows and positions of a tile
constexpr int kXPart = kXTile * 128;                    // bytes of one part: 128 rows of 64 channels
constexpr int kXStageBytes = 4 * kXPart;                // K lo, K hi, V lo, V hi
constexpr int kXQAt = kXStages * kXStageBytes;          // Q lo, Q hi
constexpr int kXBarsAt = kXQAt + 2 * kXPart;            // full [3], empty [3], s_full [2], p_ready [2], done
constexpr int kXLiveAt = kXBarsAt + 8 * (2 * kXStages + 5);   // [stages] blocks of 16 positions that count
constexpr int kXTmemAt = kXLiveAt + 4 * kXStages;
constexpr int kXSmem = kXTmemAt + 4 + 1024;
constexpr int kXThreads = 320;                          // two groups of four warps, copy warp, MMA warp
static_assert(kXSmem <= 227 * 1024, "shared memory of an SM");
constexpr float kXSlack = 8.f;                          // how far (log 2) a maximum may be above the accumulators'

__device__ __forceinline__ void tma_load_part(uint32_t dst, const CUtensorMap* tm, int y, int half, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(dst),
      "l"(tm), "r"(0), "r"(y), "r"(half), "r"(bar), "l"(policy)
      : "memory");
}
// Shared-memory operand of tcgen05.mma with the 128-byte swizzle: start address, and in units of 16 bytes the distance of
// 8-row groups and, for operands that are contiguous in M or N, that of 64-element columns of them.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t column_step) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(column_step >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// fp32 accumulators, bf16 operands, M = N = 128; bit 16: B is contiguous in N
constexpr uint32_t kMmaS = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t kMmaO = kMmaS | (1u << 16);

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {   // the barrier is told when the products issued so far are done
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
      "r"(r[31])
      : "memory");
}

// The registers of loads issued so far are there (and are not used above this point).
template <int N>
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[N][32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 32; ++j) asm volatile("" : "+r"(r[i][j]));
}

__global__ void __launch_bounds__(kXThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const PrefixAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row0 = blockIdx.x * kXRows, split = blockIdx.y, g = blockIdx.z, n_cta = gridDim.y;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kXBarsAt, bar_empty = bar_full + 8 * kXStages, bar_s = bar_empty + 8 * kXStages,
                 bar_p = bar_s + 16, bar_done = bar_p + 16;
  volatile int* sm_live = reinterpret_cast<int*>(smem + kXLiveAt);
  if (tid == 0) {
    for (int s = 0; s < kXStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(bar_s + 8 * w, 1);
      mbar_init(bar_p + 8 * w, kXRows);
    }
    mbar_init(bar_done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * 8) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_base + kXTmemAt) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int G = p.group, n_kv = p.c.n_kv_heads, shift = p.c.page_shift;
  const int rows = p.n_seq * G;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int positions = p.n_shared << shift;
  const int n_all = (positions + kXTile - 1) / kXTile;
  const int n_tiles = (n_all - split + n_cta - 1) / n_cta;   // (at least one: no more CTAs than tiles)

  if (warp < 8) {   // the query rows, swizzled; zeros behind the last one
    for (int i = tid; i < kXRows * 16; i += 256) {
      const int r = i >> 4, c = i & 15, row = row0 + r;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (row < rows) {
        const int b = row / G, h = row - b * G;
        x = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) +
                                                  ((int64_t)b * p.n_q_heads + g * G + h) * kHeadDim) + c);
      }
      *reinterpret_cast<uint4*>(smem + kXQAt + (c >> 3) * kXPart + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = x;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // what tcgen05.mma will read
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kXTmemAt);

  if (warp == 8) {
    // ------------------------------------------------------------ copy warp: lane = (piece, part)
    uint64_t policy;
    if (gridDim.x == 1) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));   // (other rows read it too)
    const int piece = min(1 << shift, kXTile), pieces = kXTile / piece;   // positions of a piece, pieces of a tile
    const int mine = lane >> 2, part = lane & 3;
    bool ok = true;
    for (int t = 0; t < n_tiles; ++t) {
      const int s = t % kXStages, use = t / kXStages;
      const int pos = (split + t * n_cta) * kXTile + mine * piece;
      int y = (int)p.n_rows;                 // behind the last row: zeros
      bool live = false;
      if (mine < pieces && pos < positions) {
        const int pg = __ldg(p.shared + (pos >> shift));
        if ((unsigned)pg < (unsigned)p.c.n_pages) {
          y = ((pg * n_kv + g) << shift);
          live = true;
        } else if (part == 0 && blockIdx.x == 0 && g == 0) {
          atomicOr(p.status, RKV_DEV_BAD_INDEX);
        }
      }
      const uint32_t who = __ballot_sync(0xffffffffu, live && part == 0);
      if (use > 0 && !mbar_wait(bar_empty + 8 * s, (use - 1) & 1)) {
        ok = false;
      }
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        break;
      }
      if (lane == 0) {
        int blocks = 0;                      // of 16 positions
        for (int i = 0; i < pieces; ++i)
          if ((who >> (4 * i)) & 1) blocks |= ((1 << (piece / 16)) - 1) << (i * (piece / 16));
        sm_live[s] = blocks;
        mbar_expect_tx(bar_full + 8 * s, kXStageBytes);
      }
      __syncwarp();
      if (mine < pieces)
        tma_load_part(smem_base + s * kXStageBytes + part * kXPart + mine * piece * 128, part < 2 ? &tm_k : &tm_v, y, part & 1,
                      bar_full + 8 * s, policy);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------ products
    if (lane == 0) {
      bool ok = true;
      const uint64_t q_at = operand(smem_base + kXQAt, 16);
      auto products_s = [&](int t) {         // S of tile t
        const int s = t % kXStages, w = t & 1;
        ok = ok && mbar_wait(bar_full + 8 * s, (t / kXStages) & 1);
        if (!ok) return;
        tmem_after();
        const uint64_t k_at = operand(smem_base + s * kXStageBytes, 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {        // 16 channels: 32 bytes on, every fourth time the other part
          const uint64_t step = (uint64_t)((i >> 2) * (kXPart >> 4) + (i & 3) * 2);
          mma_ss(tmem + 128 * w, q_at + step, k_at + step, kMmaS, i > 0);
        }
        mma_commit(bar_s + 8 * w);
      };
      auto products_o = [&](int t) {         // O += P V of tile t
        const int s = t % kXStages, w = t & 1;
        ok = ok && mbar_wait(bar_p + 8 * w, (t >> 1) & 1);
        if (!ok) return;
        tmem_after();
        const uint64_t v_at = operand(smem_base + s * kXStageBytes + 2 * kXPart, kXPart);
#pragma unroll
        for (int i = 0; i < 8; ++i)          // 16 positions: 2048 bytes on, 8 columns of P
          mma_ts(tmem + 256 + 128 * w, tmem + 128 * w + 8 * i, v_at + (uint64_t)(i * (2048 >> 4)), kMmaO, t > 1 || i > 0);
        mma_commit(bar_empty + 8 * s);
      };
      products_s(0);
      for (int t = 0; t < n_tiles && ok; ++t) {
        if (t + 1 < n_tiles) {
          // S of tile t + 1 goes where P of tile t - 1 is: that one's product has to be done
          if (t > 0) ok = ok && mbar_wait(bar_empty + 8 * ((t - 1) % kXStages), ((t - 1) / kXStages) & 1);
          products_s(t + 1);
        }
        products_o(t);
      }
      if (!ok) atomicOr(p.status, RKV_DEV_TIMEOUT);
      mma_commit(bar_done);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: thread = row, group w = tiles w, w + 2, ...
    const int w = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;      // the warp's 32 lanes of tensor memory
    const uint32_t s_at = tmem + lanes + 128 * w, o_at = tmem + lanes + 256 + 128 * w;
    const float c = p.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int t = w; t < n_tiles; t += 2) {
      ok = mbar_wait(bar_s + 8 * w, (t >> 1) & 1) && mbar_wait(bar_full + 8 * (t % kXStages), (t / kXStages) & 1);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        break;
      }
      tmem_after();
      uint32_t x[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32(x[i], s_at + 32 * i);
      tmem_wait_ld(x);
      const int live = sm_live[t % kXStages];
      if (live != 0xff) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!((live >> i) & 1)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[i >> 1][16 * (i & 1) + j] = 0xff800000u;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 32; ++j) top = fmaxf(top, __uint_as_float(x[i][j]));
      top *= c;
      const bool grows = top > m + kXSlack || (m == -INFINITY && top > m);
      if (__any_sync(0xffffffffu, grows)) {   // (S of this tile being there, the group's O is at rest)
        const float m_new = grows ? top : m;
        const float a = m_new == m ? 1.f : ex2(m - m_new);
        if (t > 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t o[1][32];
            tmem_ld32(o[0], o_at + 32 * i);
            tmem_wait_ld(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[0][j] = __float_as_uint(__uint_as_float(o[0][j]) * a);
            tmem_st32(o_at + 32 * i, o[0]);
          }
        }
        l *= a;
        m = m_new;
      }
      const float z = m == -INFINITY ? 0.f : -m;
      float l2 = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {           // 64 positions: 32 columns of P
        uint32_t y[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float a = ex2(fmaf(__uint_as_float(x[2 * i + (j >> 4)][2 * (j & 15)]), c, z));
          const float b = ex2(fmaf(__uint_as_float(x[2 * i + (j >> 4)][2 * (j & 15) + 1]), c, z));
          y[j] = pack_bf16(a, b);
          l += __uint_as_float(y[j] << 16);
          l2 += __uint_as_float(y[j] & 0xffff0000u);
        }
        tmem_st32(s_at + 32 * i, y);
      }
      l += l2;
      tmem_wait_st();
      tmem_before();
      mbar_arrive(bar_p + 8 * w);
    }
    // The two groups' accumulators of a row meet: each finishes 64 channels and hands the other 64 over in shared memory.
    if (!mbar_wait(bar_done, 0) && lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
    __syncwarp();
    tmem_after();
    float* sm_ml = reinterpret_cast<float*>(smem);                              // [2 groups][m, l][128 rows]
    float4* sm_o = reinterpret_cast<float4*>(smem + 2048) + w * 16 * kXRows;    // [group][16 x four channels][128 rows]
    const bool any = w < n_tiles;             // (the second group of a CTA with one tile has nothing)
    uint32_t mine[2][32];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t o[1][32];
      tmem_ld32(o[0], o_at + 64 * (1 - w) + 32 * i);
      tmem_wait_ld(o);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        sm_o[(8 * i + j) * kXRows + r] = make_float4(__uint_as_float(o[0][4 * j]), __uint_as_float(o[0][4 * j + 1]),
                                                     __uint_as_float(o[0][4 * j + 2]), __uint_as_float(o[0][4 * j + 3]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) tmem_ld32(mine[i], o_at + 64 * w + 32 * i);
    tmem_wait_ld(mine);
    sm_ml[(2 * w) * kXRows + r] = any ? m : -INFINITY;
    sm_ml[(2 * w + 1) * kXRows + r] = l;
    tmem_before();
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const float m_o = sm_ml[(2 * (1 - w)) * kXRows + r], l_o = sm_ml[(2 * (1 - w) + 1) * kXRows + r];
    const float M = fmaxf(any ? m : -INFINITY, m_o);
    const float e = !any || m == -INFINITY ? 0.f : ex2(m - M), e_o = m_o == -INFINITY ? 0.f : ex2(m_o - M);
    const float4* other = reinterpret_cast<const float4*>(smem + 2048) + (1 - w) * 16 * kXRows;
    const int row = row0 + r;
    if (row < rows) {
      const int b = row / G, h = row - b * G;
      const int64_t bg = (int64_t)b * n_kv + g;
      float* part = p.partials + (bg * p.max_splits + split) * PartialLayout::kFloats + h * kHeadDim + 64 * w;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float4 v = other[i * kXRows + r];
        const uint32_t* o = &mine[i >> 3][4 * (i & 7)];
        float4 sum;                           // (what a group without positions has left counts for nothing, whatever it is)
        sum.x = (e == 0.f ? 0.f : __uint_as_float(o[0]) * e) + (e_o == 0.f ? 0.f : v.x * e_o);
        sum.y = (e == 0.f ? 0.f : __uint_as_float(o[1]) * e) + (e_o == 0.f ? 0.f : v.y * e_o);
        sum.z = (e == 0.f ? 0.f : __uint_as_float(o[2]) * e) + (e_o == 0.f ? 0.f : v.z * e_o);
        sum.w = (e == 0.f ? 0.f : __uint_as_float(o[3]) * e) + (e_o == 0.f ? 0.f : v.w * e_o);
        *reinterpret_cast<float4*>(part + 4 * i) = sum;
      }
      if (w == 0) {
        float* ml = p.ml_t + bg * 16 * p.max_splits + split;
        ml[(int64_t)h * p.max_splits] = M;
        ml[(int64_t)(kMaxGroup + h) * p.max_splits] = l * e + l_o * e_o;
      }
    }
  }
  __syncthreads();
  if (warp == 8 && lane == 0) {   // after a wait that ran out copies may be under way: they land before the CTA goes
    for (int s = 0; s < kXStages; ++s) {
      const int uses = (n_tiles - s + kXStages - 1) / kXStages;
      if (uses > 0) mbar_wait(bar_full + 8 * s, (uses - 1) & 1);
    }
  }
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace

cudaError_t prepare_prefix_attention() {
  return cudaFuncSetAttribute(prefix_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kXSmem);
}

cudaError_t launch_prefix_attention(const PrefixAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int splits,
                                    cudaStream_t st) {
  const int blocks = (p.n_seq * p.group + kXRows - 1) / kXRows;
  return launch_ex(prefix_attn_kernel, dim3(blocks, splits, p.c.n_kv_heads), dim3(kXThreads), (size_t)kXSmem, st, 1, tm_k,
                   tm_v, p);
}

}  // namespace rkv
