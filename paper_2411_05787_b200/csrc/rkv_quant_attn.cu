// Split-K grouped-query decode attention over the 8-bit cache (sm_100a).
//
//   s[h][j] = scale ks(j) <q[h], K8[j]>,  p = softmax_j s,  out[h] = sum_j p[h][j] vs(j) V8[j],
// K8, V8 e4m3 codes, ks, vs the scales of position j's block of 64.  The split partials, the softmax statistics and
// the raw logits go to the same workspace, in the same layout, as those of the bf16 pass: the fold kernel, the score
// pass and the selection behind it are the same kernels.  (The first kernel below serves one sequence and short batches,
// the second longer batches; the rule between them is where they are launched.)
//
// What bounds it: 256 bytes per position and KV head from HBM, half of the bf16 pass.  The shape is that pass's: one
// CTA per (sequence, KV head, split), two to an SM, a copy warp that keeps a ring of two 32 KB stages full (one
// tensor-map copy of 128 positions for K and one for V per stage: a copy instruction costs its warp about 100 cycles,
// so tiles are as many bytes as there; two stages put 19 MB in flight over the GPU, three 28 MB, which HBM serves more
// slowly: 46.2 against 42.9 us at 131072 positions of eight heads), four MMA warps with 32 positions of a tile each,
// i.e. half a block, so that a scale is one number per warp and tile.
// Measured (attention alone, fold included): 131072 positions of eight heads 42.9 us, 6.26 TB/s; 32768: 14.7 us; 16
// ragged sequences of up to 65535 positions, four heads of seven queries: 65.8 us, 6.25 TB/s; 1000: 4.1 us.
//
// Arithmetic.  Codes become halves exactly (cvt.e4m3x2) and the products run as m16n8k16 f16 MMAs with fp32
// accumulators; the heads of the group are the N = 8 dimension.  fp8 MMAs would want q and p as e4m3, which is not
// enough for either.  The queries are scaled by a power of two per head so that the largest element is near 2^15 and
// every bf16 query element down to 2^-28 of it is exact as a half.  The probabilities meet V as halves
//   p' = p vs / vref 2^13,   vref = a power of two, at least this block's vs and at most 2^8 times as large,
// so that they are normal halves (relative rounding 2^-11) down to p = 2^-19 at least, 2^-27 usually, and never above
// 2^13; the accumulators are rescaled when vref moves and carry vref 2^-13 until they are published.
// K codes are read with ldmatrix as they lie: a lane holds four consecutive channels of a row, and the order of the
// channels in the k dimension is free as long as the query fragments use the same.  For V^T the transposed ldmatrix
// moves pairs of channels; one byte permutation turns (two positions x two channels) into the two halves the A
// fragment wants, channel 2r in row r and channel 2r + 1 in row r + 8 of the fragment.
#include <float.h>

#include "rkv_ptx.cuh"
#include "rkv_quant.cuh"

namespace rkv {
namespace {

constexpr int kQStages = 2;
constexpr int kQHalfBytes = kQuantTile * kHeadDim;   // codes of K (or V) of one tile
constexpr int kQStageBytes = 2 * kQHalfBytes;
constexpr int kQWarps = 4;                           // MMA warps; warp kQWarps is the copy warp
constexpr int kQThreads = 32 * (kQWarps + 1);
constexpr int kQBand = kQuantTile / kQWarps;         // positions of a tile per warp
constexpr int kQBlocks = kQBand / 16;                // 16-row MMA blocks per band
constexpr int kQRow = 144;                           // halves per query row in shared memory (fragment reads spread over the banks)
constexpr int kQOPad = 132;                          // floats per head row in the merge buffer
constexpr int kQCluster = 8;                         // most CTAs that finish an output together
constexpr float kPBase = 8192.f;                     // 2^13: the largest p'
constexpr float kVrefSlack = 1.f / 256.f;            // how far a block's scale may be below the accumulators'
static_assert(kQuantBlock % kQBand == 0, "a warp's band must not straddle two blocks");

constexpr int kMergeL = kQWarps * kMaxGroup * kQOPad;          // merge buffer, in floats: o [warps][8][kQOPad],
constexpr int kMergeM = kMergeL + kQWarps * kMaxGroup;         // l [warps][8], m [8]
constexpr int kMergeBytes = (kMergeM + kMaxGroup) * 4;
constexpr int kBarsAt = kQStages * kQStageBytes;
constexpr int kQAt = kBarsAt + 64;
constexpr int kQsAt = kQAt + kMaxGroup * kQRow * 2;
constexpr int kWmAt = kQsAt + kMaxGroup * 4;
constexpr int kQSmem = kWmAt + kQWarps * kMaxGroup * 4 + 1024;   // + alignment of the stages
constexpr int kQSmemPair = kQSmem + 20 * 1024;       // as much as lets only two CTAs onto an SM
// the balanced form: its merge buffer beside the stages (the next head's tiles are in them), and the sequences' tables
constexpr int kBMergeAt = kWmAt + kQWarps * kMaxGroup * 4;
constexpr int kBTablesAt = (kBMergeAt + kMergeBytes + 15) & ~15;
constexpr int kBSmem = kBTablesAt + kQuantMaxSeq * (8 + 4 * 4) + 16 + 1024;
static_assert(2 * (kBSmem + 1024) <= 228 * 1024, "two CTAs per SM");
static_assert((kQuantMaxSeq & (kQuantMaxSeq - 1)) == 0, "binary search over the sequences");
static_assert(2 * (kQSmemPair + 1024) <= 228 * 1024 && 3 * (kQSmemPair + 1024) > 228 * 1024, "two CTAs per SM, no third");

__device__ __forceinline__ void tma_load_codes(uint32_t dst, const CUtensorMap* tm, int row, uint32_t bar,
                                               uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
      "l"(tm), "r"(0), "r"(row), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float4 ld_peer4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ float2 ld_peer2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}

// State and steps of an MMA warp.  One (sequence, KV head) at a time: queries(), tile() for each of its tiles, merge().
template <bool kLogits>
struct Consumer {
  uint32_t qb[8][2];              // B fragments of Q^T: [16-channel segment][k half]
  float qs0, qs1;                 // softmax scale over the queries' powers of two, for heads qc and qc + 1
  float m0, m1, l0, l1;           // running maximum and sum of heads qc, qc + 1
  float vref, vrcp;               // scale of the accumulators and its reciprocal
  float o[8][4];                  // [16-channel segment]: (channel 16 s + 2 qd, heads qc, qc + 1), (the next channel, the same heads)

  __device__ __forceinline__ void reset() {
    m0 = m1 = -INFINITY;
    l0 = l1 = 0.f;
    vref = 1.17549435e-38f;       // 2^-126
    vrcp = 8.50705917e37f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }

  // A block of much smaller scale than the accumulators': they are brought down to it, as far as what they hold allows
  // (up to 2^100), so that its probabilities stay normal halves and large values of little weight do not hide small ones
  // of much.  Rare: the scales of a head's blocks seldom differ by more than a factor of a few.
  __device__ __forceinline__ void lower_vref(float vs) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) m = fmaxf(m, fabsf(o[i][j]));
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sh));
    const int have = (int)(__float_as_uint(vref) >> 23);                       // exponent fields: powers of two
    const int want = max((int)((__float_as_uint(vs) + 0x7fffffu) >> 23), 1);
    int k = min(have - want, 126);
    if (m > 0.f) k = min(k, 227 - (int)(__float_as_uint(m) >> 23));            // m 2^k <= 2^101
    if (k <= 0) return;
    const float a = pow2f(k);
    vref = __uint_as_float((uint32_t)(have - k) << 23);
    vrcp = __uint_as_float(0x7f000000u - __float_as_uint(vref));
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] *= a;
  }

  // qv: this thread's 16 bytes of the group's query rows (16 threads to a head; zeros for heads beyond the group)
  __device__ __forceinline__ void queries(uint4 qv, float scale, __half* sm_q, float* sm_qs, int tid) {
    const int h = tid >> 4, lane = tid & 31;
    uint32_t m = __vmaxu2(__vmaxu2(qv.x & 0x7fff7fffu, qv.y & 0x7fff7fffu), __vmaxu2(qv.z & 0x7fff7fffu, qv.w & 0x7fff7fffu));
    m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    // 2^e brings the largest magnitude into [2^14, 2^15); nothing is done for a row that is not finite or zero
    int e = 14 - ((int)(m >> 7) - 127);
    if (m >= 0x7f80u || m == 0u) e = 0;
    if (e > 126) e = 126;
    const float up = pow2f(e);
    const uint32_t x[4] = {qv.x, qv.y, qv.z, qv.w};
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = pack_f16(__uint_as_float(x[i] << 16) * up, __uint_as_float(x[i] & 0xffff0000u) * up);
    *reinterpret_cast<uint4*>(sm_q + h * kQRow + (tid & 15) * 8) = make_uint4(y[0], y[1], y[2], y[3]);
    if ((tid & 15) == 0) sm_qs[h] = scale * pow2f(-e);
    consumer_bar_n<32 * kQWarps>();
#pragma unroll
    for (int s = 0; s < 8; ++s) {   // channels 16 s + 4 t .. + 3 of head qd, t = lane & 3
      const uint2 f = *reinterpret_cast<const uint2*>(sm_q + (lane >> 2) * kQRow + 16 * s + 4 * (lane & 3));
      qb[s][0] = f.x;
      qb[s][1] = f.y;
    }
    qs0 = sm_qs[(lane & 3) * 2];
    qs1 = sm_qs[(lane & 3) * 2 + 1];
  }

  // The warp's band of one tile: codes at kbase (K) and kbase + kQHalfBytes (V), its first position pos_base < n, the
  // two scales of its block.  lg0: logit scratch of the (sequence, KV head), position-major, at this lane's heads.
  __device__ __forceinline__ void tile(uint32_t kbase, int band0, int pos_base, int n, float ks, float vs, float* lg0, int gp,
                                       uint64_t keep_policy, int lane) {
    const float ninf = -INFINITY;
    const int qd = lane >> 2, qc = (lane & 3) * 2;   // row of an 8-row group; first of the two heads this lane holds
    // this lane's row of the band in 16-byte piece  lane >> 4, swizzled (piece ^ row & 7; rows of 128 bytes): piece
    // 2 j + (lane >> 4) is at ^ (j << 5)
    const uint32_t at = kbase + (band0 + (lane & 15)) * kHeadDim + (((lane >> 4) ^ (lane & 7)) << 4);
    const bool full = pos_base + kQBand <= n;
    float c[kQBlocks][4], c2[kQBlocks][4];   // two accumulator chains per block
#pragma unroll
    for (int i = 0; i < kQBlocks; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) c[i][j] = c2[i][j] = 0.f;
#pragma unroll
    for (int cs = 0; cs < 4; ++cs) {   // 32 channels
#pragma unroll
      for (int i = 0; i < kQBlocks; ++i) {
        uint32_t a[4];
        ldsm_x4(a, (at ^ (cs << 5)) + 16 * i * kHeadDim);
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e4m3x4_to_f16x4(a[j], lo[j], hi[j]);
        mma_f16(c[i], lo[0], lo[1], hi[0], hi[1], qb[2 * cs][0], qb[2 * cs][1]);
        mma_f16(c2[i], lo[2], lo[3], hi[2], hi[3], qb[2 * cs + 1][0], qb[2 * cs + 1][1]);
      }
    }
    // one factor per head and tile; kept finite, so that a zero product stays zero (NaN scales pass)
    float f0 = ks * qs0, f1 = ks * qs1;
    f0 = f0 > FLT_MAX ? FLT_MAX : f0;
    f1 = f1 > FLT_MAX ? FLT_MAX : f1;
    float sc[kQBlocks][4];
    float t0 = ninf, t1 = ninf;
#pragma unroll
    for (int i = 0; i < kQBlocks; ++i) {
      const int r0 = pos_base + 16 * i + qd, r1 = r0 + 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[i][j] = (c[i][j] + c2[i][j]) * ((j & 1) ? f1 : f0);
      if (kLogits && qc < gp) {
        if (r0 < n) st_keep_f2(lg0 + (int64_t)r0 * gp, sc[i][0], sc[i][1], keep_policy);
        if (r1 < n) st_keep_f2(lg0 + (int64_t)r1 * gp, sc[i][2], sc[i][3], keep_policy);
      }
      if (!full) {
        if (r0 >= n) sc[i][0] = sc[i][1] = ninf;
        if (r1 >= n) sc[i][2] = sc[i][3] = ninf;
      }
      t0 = fmaxf(t0, fmaxf(sc[i][0], sc[i][2]));
      t1 = fmaxf(t1, fmaxf(sc[i][1], sc[i][3]));
    }
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
      t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, sh));
      t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, sh));
    }
    const float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
    if (__any_sync(0xffffffffu, (n0 > m0) || (n1 > m1))) {
      const float a0 = (n0 == m0) ? 1.f : ex2((m0 - n0) * kLog2e);
      const float a1 = (n1 == m1) ? 1.f : ex2((m1 - n1) * kLog2e);
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
    if (vs > vref) {   // the same for the whole warp
      uint32_t up = (__float_as_uint(vs) + 0x7fffffu) & 0x7f800000u;   // the next power of two, 2^126 at most
      if (up > 0x7e800000u) up = 0x7e800000u;
      const float a = vref * __uint_as_float(0x7f000000u - up);
      vref = __uint_as_float(up);
      vrcp = __uint_as_float(0x7f000000u - up);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] *= a;
    } else if (vs < vref * kVrefSlack && vs > 0.f) lower_vref(vs);
    const float vf = vs * vrcp * kPBase;
    const float nm0 = (m0 == ninf) ? 0.f : -m0 * kLog2e;
    const float nm1 = (m1 == ninf) ? 0.f : -m1 * kLog2e;
#pragma unroll
    for (int i = 0; i < kQBlocks; ++i) {
      const int pos_i = pos_base + 16 * i;
      if (pos_i >= n) continue;   // the whole block lies past the end
      const float p0 = ex2(fmaf(sc[i][0], kLog2e, nm0)), p1 = ex2(fmaf(sc[i][1], kLog2e, nm1));
      const float p2 = ex2(fmaf(sc[i][2], kLog2e, nm0)), p3 = ex2(fmaf(sc[i][3], kLog2e, nm1));
      l0 += p0 + p2;
      l1 += p1 + p3;
      // P^T as the B operand: the two 8x8 [position][head] blocks transposed inside the warp
      const uint32_t b0 = movmatrix_t(pack_f16(p0 * vf, p1 * vf)), b1 = movmatrix_t(pack_f16(p2 * vf, p3 * vf));
      const bool tail = pos_i + 16 > n;
      // rows past the end may hold anything (even NaN): their codes are cleared so that 0 * x stays 0.  A register
      // holds positions 2 t, 2 t + 1 (t = lane & 3) of the first or of the second eight.
      uint32_t mk0 = 0xffffffffu, mk1 = 0xffffffffu;
      if (tail) {
        const int pa = pos_i + qc;
        mk0 = (pa < n ? 0x0000ffffu : 0u) | (pa + 1 < n ? 0xffff0000u : 0u);
        mk1 = (pa + 8 < n ? 0x0000ffffu : 0u) | (pa + 9 < n ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int sp = 0; sp < 4; ++sp) {   // two 16-channel segments
        uint32_t a[4];
        ldsm_x4_t(a, (at ^ (sp << 5)) + kQHalfBytes + 16 * i * kHeadDim);
        if (tail) {
          a[0] &= mk0;
          a[1] &= mk1;
          a[2] &= mk0;
          a[3] &= mk1;
        }
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          e4m3x4_to_f16x4(__byte_perm(a[j], 0u, 0x3120), lo[j], hi[j]);   // (channel, two positions) in each half
        mma_f16(o[2 * sp], lo[0], hi[0], lo[1], hi[1], b0, b1);
        mma_f16(o[2 * sp + 1], lo[2], hi[2], lo[3], hi[3], b0, b1);
      }
    }
  }

  // The four warps' accumulators, scaled to the CTA-wide maximum, into sm (kMergeBytes); sm_wm: [warps][8].
  __device__ __forceinline__ void merge(float* sm, float* sm_wm, int warp, int lane) {
    const float ninf = -INFINITY;
    const int qd = lane >> 2, qc = (lane & 3) * 2;
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, sh);
      l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
    }
    if (lane < 4) *reinterpret_cast<float2*>(sm_wm + warp * kMaxGroup + qc) = make_float2(m0, m1);
    consumer_bar_n<32 * kQWarps>();   // every warp's maxima are visible, and nobody reads the stages any more
    float* sm_l = sm + kMergeL;
    float* sm_M = sm + kMergeM;
    float M0 = ninf, M1 = ninf;
#pragma unroll
    for (int w = 0; w < kQWarps; ++w) {
      const float2 mw = *reinterpret_cast<const float2*>(sm_wm + w * kMaxGroup + qc);
      M0 = fmaxf(M0, mw.x);
      M1 = fmaxf(M1, mw.y);
    }
    const float e0 = (m0 == ninf) ? 0.f : ex2((m0 - M0) * kLog2e);
    const float e1 = (m1 == ninf) ? 0.f : ex2((m1 - M1) * kLog2e);
    const float unit = vref * (1.f / kPBase);
    float* base = sm + (warp * kMaxGroup + qc) * kQOPad + 2 * qd;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      *reinterpret_cast<float2*>(base + 16 * s) = make_float2(o[s][0] * e0 * unit, o[s][2] * e0 * unit);
      *reinterpret_cast<float2*>(base + kQOPad + 16 * s) = make_float2(o[s][1] * e1 * unit, o[s][3] * e1 * unit);
    }
    if (lane < 4) {
      sm_l[warp * kMaxGroup + qc] = l0 * e0;
      sm_l[warp * kMaxGroup + qc + 1] = l1 * e1;
      if (warp == 0) {
        sm_M[qc] = M0;
        sm_M[qc + 1] = M1;
      }
    }
    consumer_bar_n<32 * kQWarps>();
  }
};

// Sums over the warps of what merge() left: o into to[head][128], (m, l) of one head.
__device__ __forceinline__ void publish(const float* sm, int G, int tid, float* to) {
  for (int item = tid; item < G * 32; item += 32 * kQWarps) {   // (head, four channels)
    const float* src = sm + (item >> 5) * kQOPad + (item & 31) * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kQWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(src + w * kMaxGroup * kQOPad);
      acc.x += v.x;
      acc.y += v.y;
      acc.z += v.z;
      acc.w += v.w;
    }
    *reinterpret_cast<float4*>(to + (item >> 5) * kHeadDim + (item & 31) * 4) = acc;
  }
}
__device__ __forceinline__ float2 head_ml(const float* sm, int G, int h) {   // heads beyond the group: (-inf, 0)
  float2 ml = make_float2(-INFINITY, 0.f);
  if (h < G) {
    ml.x = sm[kMergeM + h];
#pragma unroll
    for (int w = 0; w < kQWarps; ++w) ml.y += sm[kMergeL + w * kMaxGroup + h];
  }
  return ml;
}

// kCluster: the CTAs of a (sequence, KV head) are one thread-block cluster and finish the output themselves.
template <bool kLogits, bool kCluster>
__global__ void __launch_bounds__(kQThreads, 2)
quant_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const QuantAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int b = blockIdx.z, g = blockIdx.y, split = blockIdx.x, n_cta = gridDim.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kBarsAt, bar_empty = bar_full + 8 * kQStages;
  if (tid == 0) {
    for (int s = 0; s < kQStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, kQWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * kQWarps) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  const int G = p.group;
  const int64_t head0 = ((int64_t)b * p.n_q_heads + (int64_t)g * G) * kHeadDim;
  // geometry: never written by a kernel, read above the dependency wait
  const int cap = __ldg(p.cap + b);
  const int64_t roff = __ldg(p.row_offset + b);
  const bool layout_ok = quant_layout_ok(roff, cap, p.n_kv_heads, p.n_rows);
  const int64_t row0 = roff + (int64_t)g * cap;
  __syncthreads();

  // The tiles of a (sequence, KV head) are dealt out to its CTAs in turn.
  auto tile_pos = [&](int t) { return (split + t * n_cta) * kQuantTile; };
  auto issue_tile = [&](int t, uint64_t policy) {
    const int s = t % kQStages;
    const uint32_t dst = smem_base + s * kQStageBytes, bar = bar_full + 8 * s;
    const int row = (int)(row0 + tile_pos(t));
    mbar_expect_tx(bar, kQStageBytes);
    tma_load_codes(dst, &tm_k, row, bar, policy);
    tma_load_codes(dst + kQHalfBytes, &tm_v, row, bar, policy);
  };
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  // Without a mask the first tiles are requested before the length has been read, as far as the host's bound says that
  // there are any (rows past the buffer's end arrive as zeros; tiles past the length are ignored), and p.early of them
  // before the dependency wait, when the launch before this one leaves the cache alone.  In a batch one tile only: a
  // sequence may be much shorter than the bound (eight sequences of 2048 positions 10.0 -> 9.0 us, ragged 8.9 -> 8.1).
  int n_spec = 0, n_early = 0;
  if (p.spec != 0 && layout_ok) {
    const int room = cap < p.max_len ? cap : p.max_len;
    const int bound = (room + kQuantTile - 1) / kQuantTile;
    n_spec = bound > split ? (bound - split + n_cta - 1) / n_cta : 0;
    const int most = p.n_seq == 1 ? kQStages : 1;
    if (n_spec > most) n_spec = most;
    n_early = p.early < n_spec ? p.early : n_spec;
  }
  if (tid == 32 * kQWarps)
    for (int t = 0; t < n_early; ++t) issue_tile(t, policy);
  pdl_wait();
  pdl_launch();   // after the wait: at most one predecessor is ever in flight behind a kernel of this library
  if (tid == 32 * kQWarps)
    for (int t = n_early; t < n_spec; ++t) issue_tile(t, policy);

  if (kLogits) {   // the score pass that may follow adds to the keys' histogram: it starts from zero, whatever ran before
    uint32_t* hist = p.hist + ((int64_t)b * p.n_kv_heads + g) * kSelectBins;
    for (int i = split * kQThreads + tid; i < kSelectBins; i += n_cta * kQThreads) hist[i] = 0u;
  }

  // sizes, queries and the first scales: independent loads, one round trip
  const int act = (p.active != nullptr) ? __ldcg(p.active + b) : 1;
  int n = __ldcg(p.len + b);
  // Lane i holds the two scales of the warp's half block in the CTA's tile  t0 + i  for 32 tiles at a time.
  const int band0 = kQBand * warp;
  float ks_all = 0.f, vs_all = 0.f;
  auto load_scales = [&](int t0) {
    const int64_t pos = (int64_t)(split + (int64_t)(t0 + lane) * n_cta) * kQuantTile + band0;
    ks_all = vs_all = 0.f;
    if (layout_ok && pos < cap) {
      ks_all = __ldcg(p.k_scale + (row0 + pos) / kQuantBlock);
      vs_all = __ldcg(p.v_scale + (row0 + pos) / kQuantBlock);
    }
  };
  __half* sm_q = reinterpret_cast<__half*>(smem + kQAt);
  float* sm_qs = reinterpret_cast<float*>(smem + kQsAt);
  float* sm_wm = reinterpret_cast<float*>(smem + kWmAt);
  Consumer<kLogits> mma;
  if (warp < kQWarps) {
    uint4 qv = make_uint4(0u, 0u, 0u, 0u);
    if (tid < G * 16) qv = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + head0) + tid);
    load_scales(0);
    mma.queries(qv, p.scale, sm_q, sm_qs, tid);
  }

  auto drain_spec = [&] {   // tiles requested ahead of the length must land before the CTA may go
    if (n_spec > 0) {
      if (tid == 0)
        for (int t = 0; t < n_spec; ++t)
          if (!mbar_wait(bar_full + 8 * t, 0)) atomicOr(p.status, RKV_DEV_TIMEOUT);
      __syncthreads();
    }
  };
  if (act == 0) return;   // (with a mask nothing is requested ahead)
  const int64_t bg = (int64_t)b * p.n_kv_heads + g;
  float* part = p.partials + (bg * p.max_splits + split) * PartialLayout::kFloats;
  float* ml = p.ml_t + bg * 16 * p.max_splits + split;   // split-contiguous copy of (m, l), for the kernels that read across the splits
  if (!layout_ok) {   // nothing is read; a fold behind this one must come to zero (it knows the length, not the layout)
    if (tid == 0 && split == 0) atomicOr(p.status, RKV_DEV_BAD_LAYOUT);
    for (int i = tid; i < G * kHeadDim; i += kQThreads) part[i] = 0.f;
    if (tid < kMaxGroup) {
      part[kMaxGroup * kHeadDim + tid] = ml[(int64_t)tid * p.max_splits] = 0.f;
      part[kMaxGroup * kHeadDim + kMaxGroup + tid] = ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = 1.f;
    }
    n = 0;
  }
  {
    const int lim = cap < p.max_len ? cap : p.max_len;
    if (n > lim) {
      n = lim;
      if (tid == 0 && split == 0) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
    }
  }
  if (n <= 0) {   // nothing cached: the output is defined as zero
    drain_spec();
    if (split == 0 && tid < kHeadDim)
      for (int h = 0; h < G; ++h) static_cast<__nv_bfloat16*>(p.out)[head0 + h * kHeadDim + tid] = __float2bfloat16(0.f);
    return;
  }
  const int total_tiles = (n + kQuantTile - 1) / kQuantTile;
  const int n_tiles = total_tiles > split ? (total_tiles - split + n_cta - 1) / n_cta : 0;
  if (!kCluster && n_tiles == 0) {   // (in a cluster an idle CTA still owns channels of the output)
    drain_spec();
    return;
  }

  if (warp == kQWarps) {
    // ------------------------------------------------------------ copy warp
    if (lane == 0) {
      for (int t = n_spec; t < n_tiles; ++t) {
        const int s = t % kQStages, use = t / kQStages;
        if (use > 0 && !mbar_wait(bar_empty + 8 * s, (use - 1) & 1)) {
          atomicOr(p.status, RKV_DEV_TIMEOUT);
          break;
        }
        issue_tile(t, policy);
      }
    }
    return;
  }

  // ---------------------------------------------------------------- MMA warps
  mma.reset();
  float* lg0 = kLogits ? p.logits + bg * p.logit_stride * p.gp + (lane & 3) * 2 : nullptr;
  uint64_t keep_policy = 0;
  if (kLogits) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep_policy));

  const int n_wait = n_tiles > n_spec ? n_tiles : n_spec;   // tiles requested ahead of the length are always consumed
  for (int t = 0; t < n_wait; ++t) {
    const int s = t % kQStages;
    if (t > 0 && (t & 31) == 0) load_scales(t);
    const float ks = __shfl_sync(0xffffffffu, ks_all, t & 31), vs = __shfl_sync(0xffffffffu, vs_all, t & 31);
    if (!mbar_wait(bar_full + 8 * s, (t / kQStages) & 1)) {
      if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
      break;
    }
    const int pos_base = tile_pos(t) + band0;
    if (t < n_tiles && pos_base < n)
      mma.tile(smem_base + s * kQStageBytes, band0, pos_base, n, ks, vs, lg0, p.gp, keep_policy, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_empty + 8 * s);
  }

  float* sm_merge = reinterpret_cast<float*>(smem);   // (the stages are free by then)
  mma.merge(sm_merge, sm_wm, warp, lane);
  float* sm_sum = reinterpret_cast<float*>(smem + kQStageBytes);   // cluster: this CTA's share, [8][128] and [8][2]
  float* sm_ml = sm_sum + kMaxGroup * kHeadDim;
  publish(sm_merge, G, tid, kCluster ? sm_sum : part);
  if (tid < kMaxGroup) {
    const float2 v = head_ml(sm_merge, G, tid);
    if (kCluster) {
      *reinterpret_cast<float2*>(sm_ml + 2 * tid) = v;
    } else {
      part[kMaxGroup * kHeadDim + tid] = v.x;
      part[kMaxGroup * kHeadDim + kMaxGroup + tid] = v.y;
    }
    if (kLogits || !kCluster) {
      ml[(int64_t)tid * p.max_splits] = v.x;
      ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = v.y;
    }
  }
  if (kCluster) {
    // Every CTA finishes 128 / C channels of every head from its peers' shared memory; the second barrier keeps that
    // memory until the last reader is done.  (Threads that have left count as arrived.)
    __syncwarp();
    cluster_sync_alive();
    const int c_sh = __ffs(n_cta) - 1, per_sh = 5 - c_sh;      // C = 1, 2, 4 or 8; log2 of the items per head
    const int h = tid >> per_sh, ch = (split << (7 - c_sh)) + (tid & ((1 << per_sh) - 1)) * 4;
    for (int hh = h; hh < G; hh += (32 * kQWarps) >> per_sh) {
      const uint32_t at = smem_u32(sm_sum + hh * kHeadDim + ch), ml_at = smem_u32(sm_ml + 2 * hh);
      float4 v[kQCluster];
      float2 e[kQCluster];
      const float ninf = -INFINITY;
      float M = ninf, L = 0.f;
#pragma unroll
      for (int r = 0; r < kQCluster; ++r) {
        if (r < n_cta) {
          v[r] = ld_peer4(map_rank(at, r));
          e[r] = ld_peer2(map_rank(ml_at, r));
        }
      }
#pragma unroll
      for (int r = 0; r < kQCluster; ++r)
        if (r < n_cta) M = fmaxf(M, e[r].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < kQCluster; ++r) {
        if (r < n_cta) {
          const float w = (e[r].x == ninf) ? 0.f : ex2((e[r].x - M) * kLog2e);
          L = fmaf(e[r].y, w, L);
          acc.x = fmaf(v[r].x, w, acc.x);
          acc.y = fmaf(v[r].y, w, acc.y);
          acc.z = fmaf(v[r].z, w, acc.z);
          acc.w = fmaf(v[r].w, w, acc.w);
        }
      }
      const float inv = 1.f / L;
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + head0 + hh * kHeadDim + ch) =
          make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    }
    __syncwarp();
    cluster_sync_alive();
  }
}


// ---------------------------------------------------------------------------------------------- batches: balanced form
// The tiles of all heads of all sequences, in order, are cut into equal runs, one per CTA, in a single wave: whatever the
// lengths, every CTA has the same work up to a tile (beginning and ending a head costs about as much as a tile, so a
// head of m tiles counts as m + 1 units, the first of them empty).  (With a fixed number of CTAs per (sequence, KV head) a
// ragged batch waits for its longest sequence, and the waves a finer cut needs cost more than they balance: 16 sequences
// of up to 3000 positions, 8 heads: 16.4 us with two CTAs a head, 23.4 with 24.)  The lengths are on the device, so every
// CTA sums them up itself.  A run covers the end of one head and the beginning of the next, or several whole ones; each
// piece leaves one split partial, slot = CTA - first CTA of that head, and the head's first CTA records how many there
// are.  The copy warp walks the tiles without stopping at heads; the next head's queries and scales are requested while
// the current one's tiles are worked on.
struct Piece {   // the tiles of one (sequence, KV head) in a CTA's run, and the unit behind them
  int b, g, tile, count, next;
};

// The first piece with tiles at or behind unit x of a run that ends at `end`; count = 0 when there is none.
__device__ __forceinline__ Piece piece_at(int x, int end, int b, const int* pref, const int* tiles) {
  Piece s;
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

template <bool kLogits>
__global__ void __launch_bounds__(kQThreads, 2)
quant_balanced_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                      const QuantAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bar_full = smem_base + kBarsAt, bar_empty = bar_full + 8 * kQStages;
  __half* sm_q = reinterpret_cast<__half*>(smem + kQAt);
  float* sm_qs = reinterpret_cast<float*>(smem + kQsAt);
  float* sm_wm = reinterpret_cast<float*>(smem + kWmAt);
  float* sm_merge = reinterpret_cast<float*>(smem + kBMergeAt);
  int64_t* sm_row = reinterpret_cast<int64_t*>(smem + kBTablesAt);            // first row of a sequence
  int* sm_cap = reinterpret_cast<int*>(sm_row + kQuantMaxSeq);
  int* sm_len = sm_cap + kQuantMaxSeq;
  int* sm_tiles = sm_len + kQuantMaxSeq;                                      // of one head
  int* sm_pref = sm_tiles + kQuantMaxSeq;                                     // units of all heads of the sequences before
  int* sm_most = sm_pref + kQuantMaxSeq + 1;
  if (tid == 0) {
    for (int s = 0; s < kQStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, kQWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 32 * kQWarps) {
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  for (int b = tid; b < p.n_seq; b += kQThreads) {   // geometry: never written by a kernel, read above the dependency wait
    sm_row[b] = __ldg(p.row_offset + b);
    sm_cap[b] = __ldg(p.cap + b);
  }
  pdl_wait();
  pdl_launch();   // after the wait: at most one predecessor is ever in flight behind a kernel of this library
  const int n_bg = p.n_seq * p.n_kv_heads;
  int flags = 0;
  for (int b = tid; b < p.n_seq; b += kQThreads) {   // (each entry by the thread that wrote its geometry)
    const int act = (p.active != nullptr) ? __ldcg(p.active + b) : 1;
    int n = __ldcg(p.len + b);
    const int cap = sm_cap[b], lim = cap < p.max_len ? cap : p.max_len;
    if (act == 0) {
      n = 0;
    } else if (!quant_layout_ok(sm_row[b], cap, p.n_kv_heads, p.n_rows)) {
      flags |= RKV_DEV_BAD_LAYOUT;
      n = 0;
    } else if (n > lim) {
      flags |= RKV_DEV_LEN_CLAMPED;
      n = lim;
    }
    if (n < 0) n = 0;
    sm_len[b] = n;
    sm_tiles[b] = (n + kQuantTile - 1) / kQuantTile;
  }
  if (cta == 0 && flags != 0) atomicOr(p.status, flags);
  if (kLogits)    // the score pass that may follow adds to the keys' histograms: they start from zero
    for (int bg = cta; bg < n_bg; bg += gridDim.x)
      for (int i = tid; i < kSelectBins; i += kQThreads) p.hist[(int64_t)bg * kSelectBins + i] = 0u;
  __syncthreads();
  if (warp == 0) {
    int sum = 0, most = 0;
    for (int b0 = 0; b0 < p.n_seq; b0 += 32) {
      const int b = b0 + lane, mine = b < p.n_seq ? sm_tiles[b] : 0;
      most = max(most, mine);
      const int units = mine > 0 ? (mine + 1) * p.n_kv_heads : 0;
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
  for (int i = cta * kQThreads + tid; i < n_bg; i += gridDim.x * kQThreads)
    if (sm_tiles[i / p.n_kv_heads] == 0) p.counts[i] = 0;
  // No more CTAs than units, and no more than leave any head at most max_splits partials (a head of m tiles touches at
  // most (m + 1) C / total + 2 runs; and at most m, each with a tile of it).
  uint32_t C = min(gridDim.x, total);
  if (most > (uint32_t)p.max_splits) C = min(C, (uint32_t)(p.max_splits - 2) * total / (most + 1));
  if ((uint32_t)cta >= C) return;
  const int t0 = (int)(total * (uint32_t)cta / C), t1 = (int)(total * (uint32_t)(cta + 1) / C);
  int b = 0;   // the last sequence whose units begin at or before t0
  for (int step = kQuantMaxSeq / 2; step > 0; step >>= 1)
    if (b + step < p.n_seq && sm_pref[b + step] <= t0) b += step;

  if (warp == kQWarps) {
    // ------------------------------------------------------------ copy warp
    if (lane == 0) {
      uint64_t policy;
      asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
      int it = 0;
      for (Piece s = piece_at(t0, t1, b, sm_pref, sm_tiles); s.count > 0; s = piece_at(s.next, t1, s.b, sm_pref, sm_tiles)) {
        const int row = (int)(sm_row[s.b] + (int64_t)s.g * sm_cap[s.b]) + s.tile * kQuantTile;
        for (int i = 0; i < s.count; ++i, ++it) {
          const int st = it % kQStages, use = it / kQStages;
          if (use > 0 && !mbar_wait(bar_empty + 8 * st, (use - 1) & 1)) {
            atomicOr(p.status, RKV_DEV_TIMEOUT);
            return;
          }
          const uint32_t dst = smem_base + st * kQStageBytes, bar = bar_full + 8 * st;
          mbar_expect_tx(bar, kQStageBytes);
          tma_load_codes(dst, &tm_k, row + i * kQuantTile, bar, policy);
          tma_load_codes(dst + kQHalfBytes, &tm_v, row + i * kQuantTile, bar, policy);
        }
      }
    }
    return;
  }

  // ---------------------------------------------------------------- MMA warps
  const int G = p.group, band0 = kQBand * warp;
  Consumer<kLogits> mma;
  uint64_t keep_policy = 0;
  if (kLogits) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep_policy));
  auto load_query = [&](const Piece& s) {
    uint4 qv = make_uint4(0u, 0u, 0u, 0u);
    const int64_t head0 = ((int64_t)s.b * p.n_q_heads + (int64_t)s.g * G) * kHeadDim;
    if (tid < G * 16) qv = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + head0) + tid);
    return qv;
  };
  // lane i: the scales of the warp's half block in the piece's tile  first + i
  auto load_scales = [&](const Piece& s, int first, float& ks, float& vs) {
    ks = vs = 0.f;
    const int64_t pos = (int64_t)(s.tile + first + lane) * kQuantTile + band0;
    if (first + lane < s.count && pos < sm_cap[s.b]) {
      const int64_t blk = (sm_row[s.b] + (int64_t)s.g * sm_cap[s.b] + pos) / kQuantBlock;
      ks = __ldcg(p.k_scale + blk);
      vs = __ldcg(p.v_scale + blk);
    }
  };
  Piece s = piece_at(t0, t1, b, sm_pref, sm_tiles);
  if (s.count == 0) return;
  uint4 qv = load_query(s);
  float ks_all, vs_all;
  load_scales(s, 0, ks_all, vs_all);
  int it = 0;
  bool lost = false;
  for (;;) {
    mma.reset();
    mma.queries(qv, p.scale, sm_q, sm_qs, tid);
    const Piece next = piece_at(s.next, t1, s.b, sm_pref, sm_tiles);
    float ks_next = 0.f, vs_next = 0.f;
    if (next.count > 0) {   // on their way while this piece's tiles are worked on
      qv = load_query(next);
      load_scales(next, 0, ks_next, vs_next);
    }
    const int n = sm_len[s.b];
    const int bg = s.b * p.n_kv_heads + s.g;
    float* lg0 = kLogits ? p.logits + (int64_t)bg * p.logit_stride * p.gp + (lane & 3) * 2 : nullptr;
    for (int i = 0; i < s.count && !lost; ++i, ++it) {
      const int st = it % kQStages;
      if (i > 0 && (i & 31) == 0) load_scales(s, i, ks_all, vs_all);
      const float ks = __shfl_sync(0xffffffffu, ks_all, i & 31), vs = __shfl_sync(0xffffffffu, vs_all, i & 31);
      if (!mbar_wait(bar_full + 8 * st, (it / kQStages) & 1)) {
        if (lane == 0) atomicOr(p.status, RKV_DEV_TIMEOUT);
        lost = true;   // a copy that never came: no further waits, but the warps still meet at the merges
        break;
      }
      const int pos_base = (s.tile + i) * kQuantTile + band0;
      if (pos_base < n)
        mma.tile(smem_base + st * kQStageBytes, band0, pos_base, n, ks, vs, lg0, p.gp, keep_policy, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * st);
    }
    mma.merge(sm_merge, sm_wm, warp, lane);
    // runs [total c / C, total (c + 1) / C): unit y lies in the one of c = ((y + 1) C - 1) / total
    const uint32_t units = sm_tiles[s.b] + 1, head_at = sm_pref[s.b] + s.g * units;
    const int first = (int)(((head_at + 2) * C - 1) / total);   // the run of the head's first tile
    const int slot = cta - first;
    float* part = p.partials + ((int64_t)bg * p.max_splits + slot) * PartialLayout::kFloats;
    publish(sm_merge, G, tid, part);
    if (tid < kMaxGroup) {
      const float2 v = head_ml(sm_merge, G, tid);
      float* ml = p.ml_t + (int64_t)bg * 16 * p.max_splits + slot;
      ml[(int64_t)tid * p.max_splits] = v.x;
      ml[(int64_t)(kMaxGroup + tid) * p.max_splits] = v.y;
    }
    if (tid == 0 && s.tile == 0)
      p.counts[bg] = (int)(((head_at + units) * C - 1) / total) - first + 1;
    if (next.count == 0) return;
    s = next;
    ks_all = ks_next;
    vs_all = vs_next;
  }
}

// The output from the balanced form's partials: one CTA per (head, sequence), warp w takes the partials w, w + 4, ..., a lane
// four channels.  The number of partials, their (m, l) and the first sixteen of them come in one round trip.
constexpr int kFoldWarps = 4, kFoldAhead = 4;
__global__ void __launch_bounds__(32 * kFoldWarps) quant_fold_kernel(const float* __restrict__ partials,
                                                                     const float* __restrict__ ml_t,
                                                                     const int32_t* __restrict__ counts,
                                                                     const int32_t* __restrict__ active, __nv_bfloat16* out,
                                                                     int n_q_heads, int n_kv_heads, int group, int max_splits) {
  __shared__ float sm_w[kMaxSplits], sm_red[2][kFoldWarps];
  __shared__ __align__(16) float sm_o[kFoldWarps][kHeadDim];
  const int h = blockIdx.x, g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t bg = (int64_t)b * n_kv_heads + g;
  const float* po = partials + bg * max_splits * PartialLayout::kFloats + h * kHeadDim + 4 * lane;
  const float* pm = ml_t + (bg * 16 + h) * max_splits;
  const float* pl = pm + (int64_t)kMaxGroup * max_splits;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = active != nullptr ? __ldcg(active + b) : 1;
  const int count = __ldcg(counts + bg);
  float m = tid < max_splits ? __ldcg(pm + tid) : -INFINITY, l = tid < max_splits ? __ldcg(pl + tid) : 0.f;
  auto load = [&](int s) { return __ldcg(reinterpret_cast<const float4*>(po + (int64_t)s * PartialLayout::kFloats)); };
  float4 v[kFoldAhead];
#pragma unroll
  for (int k = 0; k < kFoldAhead; ++k) {
    const int s = warp + kFoldWarps * k;
    v[k] = s < max_splits ? load(s) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (act == 0) return;
  __nv_bfloat16* to = out + ((int64_t)b * n_q_heads + (int64_t)g * group + h) * kHeadDim;
  if (count <= 0) {   // nothing cached: the output is defined as zero
    to[tid] = __float2bfloat16(0.f);
    return;
  }
  if (tid >= count) {   // slots of older passes
    m = -INFINITY;
    l = 0.f;
  }
  float M = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) sm_red[0][warp] = M;
  __syncthreads();
  M = fmaxf(fmaxf(sm_red[0][0], sm_red[0][1]), fmaxf(sm_red[0][2], sm_red[0][3]));
  const float w = (m == -INFINITY) ? 0.f : ex2((m - M) * kLog2e);
  sm_w[tid] = w;
  float L = l * w;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  if (lane == 0) sm_red[1][warp] = L;
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& x, float e) {
    acc.x = fmaf(x.x, e, acc.x);
    acc.y = fmaf(x.y, e, acc.y);
    acc.z = fmaf(x.z, e, acc.z);
    acc.w = fmaf(x.w, e, acc.w);
  };
#pragma unroll
  for (int k = 0; k < kFoldAhead; ++k)
    if (warp + kFoldWarps * k < count) add(v[k], sm_w[warp + kFoldWarps * k]);
#pragma unroll 8
  for (int s = warp + kFoldWarps * kFoldAhead; s < count; s += kFoldWarps) add(load(s), sm_w[s]);
  *reinterpret_cast<float4*>(&sm_o[warp][4 * lane]) = acc;
  __syncthreads();
  L = (sm_red[1][0] + sm_red[1][1]) + (sm_red[1][2] + sm_red[1][3]);
  to[tid] = __float2bfloat16(((sm_o[0][tid] + sm_o[1][tid]) + (sm_o[2][tid] + sm_o[3][tid])) / L);
}

}  // namespace

cudaError_t prepare_quant_attention() {
  cudaError_t e = cudaSuccess;
  for (auto kernel : {quant_attn_kernel<true, false>, quant_attn_kernel<false, false>, quant_attn_kernel<true, true>,
                      quant_attn_kernel<false, true>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kQSmemPair);
  for (auto kernel : {quant_balanced_kernel<true>, quant_balanced_kernel<false>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBSmem);
  return e;
}

cudaError_t launch_quant_balanced(const QuantAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int n_cta,
                                  cudaStream_t st) {
  return launch_ex(p.logits != nullptr ? quant_balanced_kernel<true> : quant_balanced_kernel<false>, dim3(n_cta),
                   dim3(kQThreads), (size_t)kBSmem, st, 1, tm_k, tm_v, p);
}

cudaError_t launch_quant_fold(const QuantAttnParams& p, cudaStream_t st) {
  static_assert(kMaxSplits <= 32 * kFoldWarps && kHeadDim == 32 * kFoldWarps, "one thread per partial, one per channel");
  return launch_ex(quant_fold_kernel, dim3(p.group, p.n_kv_heads, p.n_seq), dim3(32 * kFoldWarps), 0, st, 1, p.partials, p.ml_t,
                   p.counts, p.active, static_cast<__nv_bfloat16*>(p.out), p.n_q_heads, p.n_kv_heads, p.group,
                   p.max_splits);
}

cudaError_t launch_quant_attention(const QuantAttnParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                                   int n_seq, int grid_x, bool cluster, bool one_wave, cudaStream_t st) {
  const bool logits = p.logits != nullptr;
  auto kernel = cluster ? (logits ? quant_attn_kernel<true, true> : quant_attn_kernel<false, true>)
                        : (logits ? quant_attn_kernel<true, false> : quant_attn_kernel<false, false>);
  // A grid that fits two to an SM must not be packed three to an SM beside idle ones (16384 positions of eight
  // sequences: 49.3 us packed, 43.2 spread); one of several waves gains from the third (ragged batch: 74.3, 71.3 us).
  const size_t smem = one_wave ? kQSmemPair : kQSmem;
  return launch_ex(kernel, dim3(grid_x, p.n_kv_heads, n_seq), dim3(kQThreads), smem, st, cluster ? grid_x : 1, tm_k, tm_v, p);
}

}  // namespace rkv
