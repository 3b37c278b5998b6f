// Attention of a whole batch over the positions that all its sequences share, read once (sm_100a, 5th-generation tensor cores).
//
// The query rows of one KV head, (sequence, head of the group) for all sequences, are cut into blocks of 128:
//   S = Q K^T  [128 rows x 64 positions],   P = 2^(S scale log2 e - m),   O += P V  [128 rows x 128 channels].
// A CTA takes one block or two and every n-th tile of 64 positions, and leaves one split partial (O, m, l) per row; the fold
// that joins them with each sequence's own positions is that of rkv_paged_attn.cu.
//
// What bounds it: 512 bytes per position and KV head from HBM while there are few rows; beyond, the tensor cores (256 clocks a
// tile and block for O, 384 for S, whose operands are read from shared memory, 6 KB per 32 clocks of products at 128 bytes a
// clock) and the exponentials (8192 at 16 a clock: 512).  So the steps of a tile run beside those of its neighbours: a copy warp
// keeps a ring of five 32 KB stages full, and two groups of four warps do the softmax, each with a warp of its own that issues
// its tcgen05.mma.  With one block of rows the groups take alternate tiles, each into an O of its own, and their halves meet at
// the end; with two each group has its block, and a tile that is in shared memory serves 256 rows (that every block fetched K and V
// for itself would need more than L2 can deliver).  Tensor memory holds an O and two S of 64 columns per group: S of task
// k + 1 is there when the exponentials of task k are done; S of task k + 2 goes where P of task k is, when that has been multiplied.
// Measured, 64 sequences of 4 heads behind 32768 positions of 8 KV heads: 43 us, where HBM would allow 20.5, the tensor cores 30;
// a group's chain is the rest (S of a task is waited for and read 450 clocks, its maximum 500, the exponentials 750), and what
// stands before the first tile and behind the last (3 us and 4).  The copy warp begins while the others stage the queries: 47
// when it waited for them.  On the way, at 47: one warp that issues for both groups, in a fixed order or polling, 62 (every wait and
// issue of one group delays the other); both groups at their exponentials at the same time 50; S of 128 columns, one per group, 59;
// half a row per thread with 16 softmax warps 103 (96 registers, spilled beside a shared memory that leaves no L1).
// A thread has one row: maxima and sums need no exchange.  P goes back to tensor memory as bf16 over its S and is the A operand
// of O += P V; V, with its channels contiguous, is an MN-major B operand.  The accumulators are rescaled only when a row's
// maximum has grown by more than 2^8 since the last time, which keeps P below 2^8; P is rounded to bf16 (2^-8 relative
// at most) where it meets V, and l adds up the rounded values, in fp32, so that what all values have in common comes through
// unrounded, as in the other passes (a sharp row's largest probability is not 1 beside an older maximum, and is rounded too).
//
// A tile is gathered page by page, each of the four (K | V) x (channels 0-63 | 64-127) parts of a piece by one copy, so that
// the tile lies in shared memory as [part][64 rows][64 channels] with the 128-byte swizzle, whatever the page.  Pieces that
// are not there (behind the end, or a bad page number) are copied from behind the pool's last row, that is filled with zeros, and masked.
#include <cuda_bf16.h>

#include "rkv_internal.h"
#include "rkv_ptx.cuh"

namespace rkv {
namespace {

constexpr int kXStages = 5;
constexpr int kXRows = 128, kXTile = kPrefixTile;       // rows of a block, positions of a tile
constexpr int kXPart = kXTile * 128;                    // bytes of one part of a tile: 64 channels of its rows
constexpr int kXStageBytes = 4 * kXPart;                // K lo, K hi, V lo, V hi
constexpr int kXQPart = kXRows * 128;
constexpr int kXQAt = kXStages * kXStageBytes;          // [2 blocks][Q lo, Q hi]
constexpr int kXBarsAt = kXQAt + 4 * kXQPart;           // full, empty [stages]; S there, P there, O added to [2 groups][2]; turn [2]; done
constexpr int kXLiveAt = kXBarsAt + 8 * (2 * kXStages + 15);   // [stages] blocks of 16 positions that count
constexpr int kXTmemAt = kXLiveAt + 4 * kXStages;
constexpr int kXSmem = kXTmemAt + 4 + 1024;
constexpr int kXThreads = 352;                          // two groups of four warps, copy warp, an MMA warp per group
static_assert(kXSmem <= 227 * 1024, "shared memory of an SM");
static_assert(kXTile == 64, "two 32-column loads a tile");
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
// fp32 accumulators, bf16 operands, M = 128, N; bit 16: B is contiguous in N
constexpr uint32_t kMma128 = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
constexpr uint32_t kMmaS = kMma128 | (((uint32_t)kXTile >> 3) << 17), kMmaO = kMma128 | ((128u >> 3) << 17) | (1u << 16);

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
// Pairs of floats: one instruction for two.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ void pair_to(uint64_t d, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(d));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ bool elect_one() {   // one lane of a converged warp, always the same
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
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

__device__ __forceinline__ void st_global8(float* to, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

__global__ void __launch_bounds__(kXThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const PrefixAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row0 = blockIdx.x * 2 * kXRows, split = blockIdx.y, g = blockIdx.z, n_cta = gridDim.y;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kXBarsAt, bar_empty = bar_full + 8 * kXStages, bar_s = bar_empty + 8 * kXStages,
                 bar_p = bar_s + 32, bar_o = bar_p + 32, bar_turn = bar_o + 32, bar_done = bar_turn + 16;
  volatile int* sm_live = reinterpret_cast<int*>(smem + kXLiveAt);
  const int G = p.group, n_kv = p.c.n_kv_heads, shift = p.c.page_shift;
  const int rows = p.n_seq * G;
  const int pair = row0 + kXRows < rows ? 1 : 0;          // two blocks of rows
  if (tid == 0) {
    for (int s = 0; s < kXStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1 + pair);             // groups that use a tile
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, kXRows);
      mbar_init(bar_o + 8 * i, 1);
    }
    for (int w = 0; w < 2; ++w) mbar_init(bar_turn + 8 * w, kXRows);
    mbar_init(bar_done, 2);
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
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kXTmemAt);   // S [2 groups][2] of 64 columns, O [2] of 128
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int positions = p.n_shared << shift;
  const int n_all = (positions + kXTile - 1) / kXTile;
  const int n_tiles = (n_all - split + n_cta - 1) / n_cta;   // (at least one: no more CTAs than tiles)

  if (warp < 8) {   // the query rows, swizzled; zeros behind the last one.  (The copy warp is at the first tiles meanwhile.)
    const int c = tid & 15;
    for (int r0 = tid >> 4; r0 < (kXRows << pair); r0 += kXRows) {
      uint4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = row0 + r0 + 16 * i, b = min(row, rows - 1) / G, h = min(row, rows - 1) - b * G;
        x[i] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) +
                                                     ((int64_t)b * p.n_q_heads + g * G + h) * kHeadDim) + c);
        if (row >= rows) x[i] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        *reinterpret_cast<uint4*>(smem + kXQAt + (2 * (r >> 7) + (c >> 3)) * kXQPart + (r & 127) * 128 +
                                  (((c & 7) ^ (r & 7)) << 4)) = x[i];
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // what tcgen05.mma will read
  }
  if (warp != 8) asm volatile("bar.sync 2, 320;" ::: "memory");    // the softmax warps and those that issue products

  if (warp == 8) {
    // ------------------------------------------------------------ copy warp: lane = (piece, part)
    uint64_t policy;
    if (gridDim.x == 1) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));   // (other rows read it too)
    const int piece = min(1 << shift, kXTile), pieces = kXTile / piece;   // positions of a piece, pieces of a tile
    const int mine = lane >> 2, part = lane & 3;
    auto page_of = [&](int t) {              // of this lane's piece; -1: none
      const int pos = (split + t * n_cta) * kXTile + mine * piece;
      return t < n_tiles && mine < pieces && pos < positions ? __ldcg(p.shared + (pos >> shift)) : -1;
    };
    bool ok = true;
    int pg = page_of(0), issued = 0;
    for (int t = 0; t < n_tiles; ++t) {
      const int s = t % kXStages, use = t / kXStages;
      const int pos = (split + t * n_cta) * kXTile + mine * piece;
      const bool there = mine < pieces && pos < positions, live = there && (unsigned)pg < (unsigned)p.c.n_pages;
      int y = (int)p.n_rows;                 // behind the last row: zeros
      if (live) y = ((pg * n_kv + g) << shift) + (pos & ((1 << shift) - 1));
      if (there && !live && part == 0 && blockIdx.x == 0 && g == 0) atomicOr(p.status, RKV_DEV_BAD_INDEX);
      pg = page_of(t + 1);
      const uint32_t who = __ballot_sync(0xffffffffu, live && part == 0);
      ok = __all_sync(0xffffffffu, use == 0 || mbar_wait(bar_empty + 8 * s, (use - 1) & 1));
      if (!ok) {
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
      issued = t + 1;
    }
    __syncwarp();
    for (int s = 0; s < kXStages; ++s) {     // (after a wait that ran out copies may be under way: they land before the CTA goes)
      const int uses = (issued - s + kXStages - 1) / kXStages;
      if (uses > 0) mbar_wait(bar_full + 8 * s, (uses - 1) & 1);
    }
  } else if (warp >= 9) {
    // ------------------------------------------------------------ products of one group: the warp goes through the steps
    // together, one elected lane issues (from a branch of one lane a product took longer to issue than to run)
    const int w = warp - 9, n = pair ? n_tiles : (n_tiles - w + 1) >> 1;   // the group's tasks
    const uint32_t base = __shfl_sync(0xffffffffu, smem_base, 0), tm = __shfl_sync(0xffffffffu, tmem, 0) + 128 * w;
    const uint32_t s_bar = bar_s + 16 * w, p_bar = bar_p + 16 * w, o_bar = bar_o + 16 * w;
    const uint64_t q_at = operand(base + kXQAt + (pair ? w : 0) * 2 * kXQPart, 16);
    bool ok = true;
    auto products_s = [&](int k) {           // S of task k
      const int t = pair ? k : 2 * k + w, s = t % kXStages;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * s, (t / kXStages) & 1));
      if (!ok) return;
      tmem_after();
      const uint64_t k_at = operand(base + s * kXStageBytes, 16);
      const uint32_t d = tm + 64 * (k & 1);
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < 8; ++i)          // 16 channels: 32 bytes on, from the fourth on in the other part
          mma_ss(d, q_at + (uint64_t)((i >> 2) * (kXQPart >> 4) + (i & 3) * 2),
                 k_at + (uint64_t)((i >> 2) * (kXPart >> 4) + (i & 3) * 2), kMmaS, i > 0);
        mma_commit(s_bar + 8 * (k & 1));
      }
      __syncwarp();
    };
    if (n > 0) products_s(0);
    if (n > 1) products_s(1);
    for (int k = 0; k < n && ok; ++k) {
      const int t = pair ? k : 2 * k + w, s = t % kXStages;
      ok = __all_sync(0xffffffffu, mbar_wait(p_bar + 8 * (k & 1), (k >> 1) & 1));
      if (!ok) break;
      tmem_after();
      const uint64_t v_at = operand(base + s * kXStageBytes + 2 * kXPart, kXPart);
      const uint32_t a = tm + 64 * (k & 1), d = tm + 256;
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < 4; ++i)          // 16 positions: 2048 bytes on, 8 columns of P
          mma_ts(d, a + 8 * i, v_at + (uint64_t)(i * (2048 >> 4)), kMmaO, k > 0 || i > 0);
        mma_commit(o_bar + 8 * (k & 1));
        mma_commit(bar_empty + 8 * s);
      }
      __syncwarp();
      if (k + 2 < n) {                       // S of task k + 2 goes where P of this one is
        ok = __all_sync(0xffffffffu, mbar_wait(o_bar + 8 * (k & 1), (k >> 1) & 1));
        if (ok) products_s(k + 2);
      }
    }
    if (elect_one()) {
      if (!ok) atomicOr(p.status, RKV_DEV_TIMEOUT);
      mma_commit(bar_done);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: thread = row
    const int w = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;      // the warp's 32 lanes of tensor memory
    const uint32_t o_at = tmem + lanes + 256 + 128 * w;
    const float c = p.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    const int t0 = pair ? 0 : w, dt = pair ? 1 : 2;
    for (int t = t0, k = 0; t < n_tiles; t += dt, ++k) {
      const int s = t % kXStages;
      const uint32_t s_at = tmem + lanes + 128 * w + 64 * (k & 1);
      const bool ok = mbar_wait(bar_s + 16 * w + 8 * (k & 1), (k >> 1) & 1) && mbar_wait(bar_full + 8 * s, (t / kXStages) & 1);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        break;
      }
      tmem_after();
      uint32_t x[2][32];
      tmem_ld32(x[0], s_at);
      tmem_ld32(x[1], s_at + 32);
      tmem_wait_ld(x);
      const int live = sm_live[s];
      if (live != 0xf) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (!((live >> q) & 1)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[q >> 1][16 * (q & 1) + e] = 0xff800000u;
          }
      }
      float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < 32; ++e)
        tops[e & 3] = max3(tops[e & 3], __uint_as_float(x[e >> 4][2 * (e & 15)]), __uint_as_float(x[e >> 4][2 * (e & 15) + 1]));
      const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * c;
      const bool grows = top > m + kXSlack || (m == -INFINITY && top > m);
      if (__any_sync(0xffffffffu, grows)) {
        const float m_new = grows ? top : m;
        const float a = m_new == m ? 1.f : ex2(m - m_new);
        if (k > 0) {                          // the group's O is at rest when its last product has ended
          const bool rest = mbar_wait(bar_o + 16 * w + 8 * ((k - 1) & 1), ((k - 1) >> 1) & 1);
          if (!__all_sync(0xffffffffu, rest)) {
            if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
            break;
          }
          tmem_after();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t o[1][32];
            tmem_ld32(o[0], o_at + 32 * i);
            tmem_wait_ld(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[0][e] = __float_as_uint(__uint_as_float(o[0][e]) * a);
            tmem_st32(o_at + 32 * i, o[0]);
          }
        }
        l *= a;
        m = m_new;
      }
      // The groups take turns at the exponentials: at the same time each would take twice as long, and the unit would stand
      // idle while both load and look for their maxima.
      const bool turn = (w == 0 && k == 0) || mbar_wait(bar_turn + 8 * w, (k - 1 + w) & 1);
      if (!__all_sync(0xffffffffu, turn)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        break;
      }
      const float z = m == -INFINITY ? 0.f : -m;
      const uint64_t cc = pair_of(c, c), zz = pair_of(z, z);
      uint64_t sum[2] = {0, 0};
      uint32_t y[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) {          // two positions to a column of P
        float a, b;
        pair_to(fma_pair(pair_of(__uint_as_float(x[e >> 4][2 * (e & 15)]), __uint_as_float(x[e >> 4][2 * (e & 15) + 1])), cc, zz),
                a, b);
        a = ex2(a);
        b = ex2(b);
        y[e] = pack_bf16(a, b);
        sum[e & 1] = add_pair(sum[e & 1], pair_of(__uint_as_float(y[e] << 16), __uint_as_float(y[e] & 0xffff0000u)));
      }
      tmem_st32(s_at, y);
      mbar_arrive(bar_turn + 8 * (1 - w));    // (behind the store, which needs all of them)
      float l0, l1;
      pair_to(add_pair(sum[0], sum[1]), l0, l1);
      l += l0 + l1;
      tmem_wait_st();
      tmem_before();
      mbar_arrive(bar_p + 16 * w + 8 * (k & 1));
    }
    if (!mbar_wait(bar_done, 0) && lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
    __syncwarp();
    tmem_after();
    const int row = row0 + r + (pair ? kXRows * w : 0);
    const int b = row / G, h = row - b * G;
    const int64_t bg = (int64_t)b * n_kv + g;
    float* part = p.partials + (bg * p.max_splits + split) * PartialLayout::kFloats + h * kHeadDim;
    float* ml = p.ml_t + bg * 16 * p.max_splits + split;
    if (pair) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t o[1][32];
        tmem_ld32(o[0], o_at + 32 * k);
        tmem_wait_ld(o);
        if (row < rows)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(o[0][8 * j + e]);
            st_global8(part + 32 * k + 8 * j, v);
          }
      }
      if (row < rows) {
        ml[(int64_t)h * p.max_splits] = m;
        ml[(int64_t)(kMaxGroup + h) * p.max_splits] = l;
      }
    } else {
      // The two groups' accumulators of a row meet: each finishes 64 channels and hands the other 64 over in shared memory.
      float* sm_ml = reinterpret_cast<float*>(smem);                              // [2 groups][m, l][128 rows]
      float4* sm_o = reinterpret_cast<float4*>(smem + 2048) + w * 16 * kXRows;    // [group][16 x four channels][128 rows]
      const bool any = w < n_tiles;           // (the second group of a CTA with one tile has nothing)
      if (!any) m = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t o[1][32];
        tmem_ld32(o[0], o_at + 64 * (1 - w) + 32 * k);
        tmem_wait_ld(o);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          sm_o[(8 * k + j) * kXRows + r] = make_float4(__uint_as_float(o[0][4 * j]), __uint_as_float(o[0][4 * j + 1]),
                                                       __uint_as_float(o[0][4 * j + 2]), __uint_as_float(o[0][4 * j + 3]));
      }
      uint32_t mine[2][32];
#pragma unroll
      for (int k = 0; k < 2; ++k) tmem_ld32(mine[k], o_at + 64 * w + 32 * k);
      tmem_wait_ld(mine);
      sm_ml[(2 * w) * kXRows + r] = m;
      sm_ml[(2 * w + 1) * kXRows + r] = l;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float m_o = sm_ml[(2 * (1 - w)) * kXRows + r], l_o = sm_ml[(2 * (1 - w) + 1) * kXRows + r];
      const float M = fmaxf(m, m_o);
      const float e = m == -INFINITY ? 0.f : ex2(m - M), e_o = m_o == -INFINITY ? 0.f : ex2(m_o - M);
      const float4* other = reinterpret_cast<const float4*>(smem + 2048) + (1 - w) * 16 * kXRows;
      if (row < rows) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float v[8];                         // (what a group without positions has left counts for nothing, whatever it is)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float4 x = other[(2 * k + q) * kXRows + r];
            const uint32_t* o = &mine[k >> 2][8 * (k & 3) + 4 * q];
            v[4 * q] = (e == 0.f ? 0.f : __uint_as_float(o[0]) * e) + (e_o == 0.f ? 0.f : x.x * e_o);
            v[4 * q + 1] = (e == 0.f ? 0.f : __uint_as_float(o[1]) * e) + (e_o == 0.f ? 0.f : x.y * e_o);
            v[4 * q + 2] = (e == 0.f ? 0.f : __uint_as_float(o[2]) * e) + (e_o == 0.f ? 0.f : x.z * e_o);
            v[4 * q + 3] = (e == 0.f ? 0.f : __uint_as_float(o[3]) * e) + (e_o == 0.f ? 0.f : x.w * e_o);
          }
          st_global8(part + 64 * w + 8 * k, v);
        }
        if (w == 0) {
          ml[(int64_t)h * p.max_splits] = M;
          ml[(int64_t)(kMaxGroup + h) * p.max_splits] = l * e + l_o * e_o;
        }
      }
    }
    tmem_before();
  }
  __syncthreads();
  if (warp == 9) {
    tmem_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

}  // namespace

cudaError_t prepare_prefix_attention() {
  return cudaFuncSetAttribute(prefix_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kXSmem);
}

cudaError_t launch_prefix_attention(const PrefixAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int splits,
                                    cudaStream_t st) {
  const int blocks = (p.n_seq * p.group + 2 * kXRows - 1) / (2 * kXRows);
  return launch_ex(prefix_attn_kernel, dim3(blocks, splits, p.c.n_kv_heads), dim3(kXThreads), (size_t)kXSmem, st, 1, tm_k,
                   tm_v, p);
}

}  // namespace rkv
