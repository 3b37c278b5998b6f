// The 8-bit full cache: storing rows (encode, append) and the rebuild of the bf16 small cache from it.
#include "rkv_quant.cuh"

namespace rkv {
namespace {

// ------------------------------------------------------------------------------------------------------------ store
// Rows x (bf16) of sequence b go to positions start .. start + count - 1 of every KV head.  For each block of 64
// positions they touch:  a = max finite |x| over the block's new rows,
//   scale' = max(needed(a), scale)  if the block holds rows below start (they are then encoded again),  needed(a) otherwise,
//   code = rne(x / scale'),  needed(a) = the smallest power of two >= a / 448 (not below 2^-126).
// One CTA per (block, KV head, sequence): all of its new rows, K and V, sit in registers (32 KB per CTA in flight,
// 128 bytes a thread), the two maxima meet once in shared memory, then the codes leave as whole 128-byte rows.
// HBM-bound for prompts (256 bytes read and 128 written per row and cache): 32768 rows of eight heads in 33.2 us,
// 6.06 TB/s (512 threads a CTA 45.8 us, 128: 36.2; without the bound of 64 registers, which costs the fourth CTA of an SM,
// 36.1); 2000-row chunks of four ragged sequences 4.6 us, of which the grid without rows takes 1.8.  For single tokens a
// chain of two round trips (sizes, then rows and scales), three when a block has to be encoded again: 2.2 us.
constexpr int kStoreThreads = 256;
constexpr int kStorePer = kQuantBlock * 16 / kStoreThreads;   // 16-byte pieces of bf16 per thread and cache

struct StoreParams {
  const uint4* k_new; const uint4* v_new;
  int64_t k_seq, k_tok, v_seq, v_tok;   // strides in 16-byte pieces
  const int32_t* start; const int32_t* count;   // [B] or null
  uint8_t* k8; uint8_t* v8; float* k_scale; float* v_scale;
  const int64_t* row_offset; const int32_t* cap; int32_t* len;
  int64_t n_rows;
  int32_t* tickets; int32_t* status;
  int n_kv_heads, n_tok;
};

__device__ __forceinline__ uint32_t max_bits(uint4 w, uint32_t m) {
  m = __vmaxu2(m, w.x & 0x7fff7fffu);
  m = __vmaxu2(m, w.y & 0x7fff7fffu);
  m = __vmaxu2(m, w.z & 0x7fff7fffu);
  return __vmaxu2(m, w.w & 0x7fff7fffu);
}
// Magnitudes that are not finite do not count towards a scale.
__device__ __forceinline__ uint32_t drop_nonfinite(uint32_t w) {
  const uint32_t m = w & 0x7fff7fffu;
  const uint32_t lo = (m & 0xffffu) >= 0x7f80u ? 0u : (m & 0xffffu), hi = (m >> 16) >= 0x7f80u ? 0u : (m & 0xffff0000u);
  return lo | hi;
}
// Infinities become NaN: the code has none, and a magnitude of 448 in their place would go unnoticed.
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) <= 3.4e38f ? x : __int_as_float(0x7fffffff); }

template <bool kFinite>
__device__ __forceinline__ uint2 encode8(uint4 w, float inv) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = __uint_as_float(x[i] << 16), hi = __uint_as_float(x[i] & 0xffff0000u);
    if (!kFinite) {
      lo = finite_or_nan(lo);
      hi = finite_or_nan(hi);
    }
    c[i] = encode2(lo * inv, hi * inv);
  }
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

// Codes of rows below `rows` of a block again, under a scale 1 / ratio times as large.
__device__ __forceinline__ void encode_again(uint8_t* block, int rows, float ratio, int tid) {
  for (int i = tid; i < rows * 8; i += kStoreThreads) {
    uint4 w = __ldcg(reinterpret_cast<const uint4*>(block) + i);
    uint32_t* x = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = f16x2_to_float2(codes_lo_f16x2(x[j])), b = f16x2_to_float2(codes_hi_f16x2(x[j]));
      x[j] = encode2(a.x * ratio, a.y * ratio) | (encode2(b.x * ratio, b.y * ratio) << 16);
    }
    reinterpret_cast<uint4*>(block)[i] = w;
  }
}

__global__ void __launch_bounds__(kStoreThreads, 4) store_kernel(const StoreParams p) {
  __shared__ uint32_t sm_max[2][kStoreThreads / 32];
  __shared__ int sm_sizes[3];
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cap = p.cap[b];               // geometry: constant while calls are in flight
  const int64_t roff = p.row_offset[b];
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  // One thread reads the sizes for its CTA; behind the barrier, where it has had them to hand on, it draws a ticket, the
  // last of which writes the new length.  So a ticket says that nobody in its CTA will read the sizes again - every warp,
  // of idle CTAs too, takes them from shared memory - also where start is the tensor of the lengths itself.  (Were each
  // warp to read for itself, one that comes late could take the new length for its start.)
  if (tid == 0) {
    const int l = __ldcg(p.len + b);
    sm_sizes[0] = l;
    sm_sizes[1] = p.start != nullptr ? __ldcg(p.start + b) : l;
    sm_sizes[2] = p.count != nullptr ? __ldcg(p.count + b) : p.n_tok;
  }
  __syncthreads();
  int ticket = -1;
  if (tid == 0) ticket = atomicAdd(p.tickets + b, 1);
  const int len = sm_sizes[0];
  int start = sm_sizes[1], count = sm_sizes[2];
  int flags = 0;
  if (!quant_layout_ok(roff, cap, p.n_kv_heads, p.n_rows)) {
    flags = RKV_DEV_BAD_LAYOUT;
    count = 0;
  } else if (start < 0 || start > len || start > cap) {
    flags = RKV_DEV_LEN_CLAMPED;
    count = 0;
  }
  const bool sound = flags == 0;
  if (count > p.n_tok) count = p.n_tok;
  if (count < 0) count = 0;
  if (sound && count > cap - start) {
    flags |= RKV_DEV_APPEND_OVERFLOW;
    count = cap - start;
  }
  const int end = start + count;
  const int blk = start / kQuantBlock + (int)blockIdx.x, pos0 = blk * kQuantBlock;
  if (count > 0 && pos0 < end) {
    const int64_t row0 = roff + (int64_t)g * cap + pos0;
    const int sub = tid & 15, slot = tid >> 4;
    uint4 kx[kStorePer], vx[kStorePer];
#pragma unroll
    for (int u = 0; u < kStorePer; ++u) {
      const int pos = pos0 + slot + u * (kStoreThreads / 16);
      kx[u] = vx[u] = make_uint4(0u, 0u, 0u, 0u);
      if (pos >= start && pos < end) {
        const int64_t t = pos - start;
        kx[u] = __ldcg(p.k_new + b * p.k_seq + t * p.k_tok + g * 16 + sub);
        vx[u] = __ldcg(p.v_new + b * p.v_seq + t * p.v_tok + g * 16 + sub);
      }
    }
    const bool joins = pos0 < start;       // the block holds older rows
    float k_old = 0.f, v_old = 0.f;
    if (joins) {
      k_old = __ldcg(p.k_scale + row0 / kQuantBlock);
      v_old = __ldcg(p.v_scale + row0 / kQuantBlock);
    }
    uint32_t mk = 0u, mv = 0u;
#pragma unroll
    for (int u = 0; u < kStorePer; ++u) {
      mk = max_bits(kx[u], mk);
      mv = max_bits(vx[u], mv);
    }
    mk = __reduce_max_sync(0xffffffffu, max(mk & 0xffffu, mk >> 16));
    mv = __reduce_max_sync(0xffffffffu, max(mv & 0xffffu, mv >> 16));
    bool finite = true;
    if (lane == 0) {
      sm_max[0][warp] = mk;
      sm_max[1][warp] = mv;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kStoreThreads / 32; ++w) {
      mk = max(mk, sm_max[0][w]);
      mv = max(mv, sm_max[1][w]);
    }
    if (max(mk, mv) >= 0x7f80u) {          // rare: the maxima once more without what is not finite
      finite = false;
      flags |= RKV_DEV_NONFINITE;
      mk = mv = 0u;
#pragma unroll
      for (int u = 0; u < kStorePer; ++u) {
        const uint4 a = kx[u], c = vx[u];
        mk = max_bits(make_uint4(drop_nonfinite(a.x), drop_nonfinite(a.y), drop_nonfinite(a.z), drop_nonfinite(a.w)), mk);
        mv = max_bits(make_uint4(drop_nonfinite(c.x), drop_nonfinite(c.y), drop_nonfinite(c.z), drop_nonfinite(c.w)), mv);
      }
      mk = __reduce_max_sync(0xffffffffu, max(mk & 0xffffu, mk >> 16));
      mv = __reduce_max_sync(0xffffffffu, max(mv & 0xffffu, mv >> 16));
      __syncthreads();
      if (lane == 0) {
        sm_max[0][warp] = mk;
        sm_max[1][warp] = mv;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kStoreThreads / 32; ++w) {
        mk = max(mk, sm_max[0][w]);
        mv = max(mv, sm_max[1][w]);
      }
    }
    const int ek = scale_exponent(mk), ev = scale_exponent(mv);
    float ks = pow2f(ek), vs = pow2f(ev);
    float k_inv = pow2f(-ek), v_inv = pow2f(-ev);      // -120 <= -e <= 126
    if (joins) {
      if (k_old >= ks) {
        ks = k_old;
        k_inv = 1.f / k_old;                           // exact for the powers of two the library writes
      } else {
        encode_again(p.k8 + row0 * kHeadDim, start - pos0, k_old * k_inv, tid);
      }
      if (v_old >= vs) {
        vs = v_old;
        v_inv = 1.f / v_old;
      } else {
        encode_again(p.v8 + row0 * kHeadDim, start - pos0, v_old * v_inv, tid);
      }
    }
#pragma unroll
    for (int u = 0; u < kStorePer; ++u) {
      const int r = slot + u * (kStoreThreads / 16), pos = pos0 + r;
      if (pos >= start && pos < end) {
        const int64_t at = (row0 + r) * kHeadDim + sub * 8;
        *reinterpret_cast<uint2*>(p.k8 + at) = finite ? encode8<true>(kx[u], k_inv) : encode8<false>(kx[u], k_inv);
        *reinterpret_cast<uint2*>(p.v8 + at) = finite ? encode8<true>(vx[u], v_inv) : encode8<false>(vx[u], v_inv);
      }
    }
    if (tid == 0) {
      p.k_scale[row0 / kQuantBlock] = ks;
      p.v_scale[row0 / kQuantBlock] = vs;
    }
  }
  if (tid == 0) {
    if (flags != 0) atomicOr(p.status, flags);
    if (ticket == (int)gridDim.x * p.n_kv_heads - 1) {
      if (sound) p.len[b] = end;
      p.tickets[b] = 0;   // ready for the next call on this stream
    }
  }
}

// ----------------------------------------------------------------------------------------------------------- rebuild
// small.K[b][g][r] = code * scale of full.K[b][g][idx[b][g][r]] (and V), as bf16: exact for scales that are powers of
// two (a code has four significant bits), rounded once otherwise.  One CTA of 128 threads per 32 output rows,
// eight lanes to a row; a lane moves eight codes from either half of a row, so that what a warp stores are whole 128-byte
// lines (16 neighbouring codes a lane, two half-covered lines per store, took 4.2 us where this takes 3.1 for 2048 rows of
// eight heads, and half as long again for four ragged sequences of up to 4096).  Rows a CTA: 32 take 3.1 and 5.9 us (3.6
// TB/s), 64 take 3.1 and 6.6, 16 take 3.4 and 8.6.  Indices come with the sizes, rows and scales in the round trip behind
// them: two in all, and what is left is their latency.
constexpr int kGatherRows = 32;
constexpr int kGatherThreads = 128;

__device__ __forceinline__ uint32_t decode2(uint32_t f16x2, float scale) {
  const float2 v = f16x2_to_float2(f16x2);
  const __nv_bfloat162 r = __floats2bfloat162_rn(v.x * scale, v.y * scale);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 decode8(uint2 w, float scale) {
  return make_uint4(decode2(codes_lo_f16x2(w.x), scale), decode2(codes_hi_f16x2(w.x), scale),
                    decode2(codes_lo_f16x2(w.y), scale), decode2(codes_hi_f16x2(w.y), scale));
}

__global__ void __launch_bounds__(kGatherThreads) quant_gather_kernel(const int32_t* __restrict__ topk_idx,
                                                                     const int32_t* __restrict__ k_small, int k_max,
                                                                     QuantDev full, CacheDev small_cache, int64_t small_rows,
                                                                     const int32_t* __restrict__ active, int n_kv_heads,
                                                                     int32_t* status) {
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x;
  const int sub = tid & 7, slot = tid >> 3;
  constexpr int kStep = kGatherThreads / 8, kPer = kGatherRows / kStep;
  const int r_base = blockIdx.x * kGatherRows;
  // the caches' geometry is never written by a kernel: read above the dependency wait
  const int cap_s = small_cache.cap[b], cap_f = full.cap[b];
  const int64_t roff_f = full.row_offset[b];
  const int64_t src0 = roff_f + (int64_t)g * cap_f;
  const int64_t roff_s = small_cache.row_offset[b];
  const int64_t dst0 = roff_s + (int64_t)g * cap_s;
  const int32_t* idx = topk_idx + (int64_t)(b * n_kv_heads + g) * k_max;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = active != nullptr ? __ldcg(active + b) : 1;
  int n = __ldcg(full.len + b);
  int m = __ldcg(k_small + b);
  int j[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int r = r_base + slot + u * kStep;
    j[u] = r < k_max ? __ldcg(idx + r) : -1;
  }
  if (act == 0) return;
  const bool fits = roff_s >= 0 && cap_s >= 0 && roff_s + (int64_t)n_kv_heads * cap_s <= small_rows;
  if (!fits || !quant_layout_ok(roff_f, cap_f, n_kv_heads, full.n_rows)) {
    if (tid == 0 && blockIdx.x == 0) atomicOr(status, RKV_DEV_BAD_LAYOUT);
    return;
  }
  if (n > cap_f) {
    n = cap_f;
    if (tid == 0 && blockIdx.x == 0) atomicOr(status, RKV_DEV_LEN_CLAMPED);
  }
  if (m > k_max) m = k_max;
  if (m > n) m = n;
  if (m < 0) m = 0;
  if (m > cap_s) {
    m = cap_s;
    if (tid == 0 && blockIdx.x == 0) atomicOr(status, RKV_DEV_LEN_CLAMPED);
  }
  if (blockIdx.x == 0 && g == 0 && tid == 0) small_cache.len[b] = m;
  if (r_base >= m) return;
  uint2 kc[kPer][2], vc[kPer][2];   // channels 8 sub .. + 7 and 64 + 8 sub .. + 7 of a row: whole 128-byte lines leave
  float ks[kPer], vs[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    ks[u] = vs[u] = 0.f;
    if (r_base + slot + u * kStep >= m) j[u] = -1;
    if (j[u] >= n || j[u] < -1) {                  // -1 is the padding of topk_idx; anything else outside [0, len) is flagged
      if (sub == 0) atomicOr(status, RKV_DEV_BAD_INDEX);
      j[u] = -1;
    }
    if (j[u] >= 0) {
      const int64_t row = src0 + j[u];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        kc[u][i] = __ldcg(reinterpret_cast<const uint2*>(full.k) + row * 16 + 8 * i + sub);
        vc[u][i] = __ldcg(reinterpret_cast<const uint2*>(full.v) + row * 16 + 8 * i + sub);
      }
      ks[u] = __ldcg(full.k_scale + row / kQuantBlock);
      vs[u] = __ldcg(full.v_scale + row / kQuantBlock);
    }
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    if (j[u] >= 0) {
      const int64_t at = (dst0 + r_base + slot + u * kStep) * 16 + sub;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        static_cast<uint4*>(small_cache.k)[at + 8 * i] = decode8(kc[u][i], ks[u]);
        static_cast<uint4*>(small_cache.v)[at + 8 * i] = decode8(vc[u][i], vs[u]);
      }
    }
  }
}

}  // namespace

cudaError_t launch_quant_store(const QuantNew& rows, const int32_t* start, const int32_t* count, const QuantDev& c,
                               int n_seq, int n_kv_heads, int32_t* tickets, int32_t* status, cudaStream_t st) {
  StoreParams p;
  p.k_new = static_cast<const uint4*>(rows.k);
  p.v_new = static_cast<const uint4*>(rows.v);
  p.k_seq = rows.k_seq / 8;
  p.k_tok = rows.k_tok / 8;
  p.v_seq = rows.v_seq / 8;
  p.v_tok = rows.v_tok / 8;
  p.start = start;
  p.count = count;
  p.k8 = c.k;
  p.v8 = c.v;
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.row_offset = c.row_offset;
  p.cap = c.cap;
  p.len = c.len;
  p.n_rows = c.n_rows;
  p.tickets = tickets;
  p.status = status;
  p.n_kv_heads = n_kv_heads;
  p.n_tok = rows.n_tok;
  // blocks that n_tok rows can touch: they may start at the last position of one
  const int blocks = (int)(((int64_t)rows.n_tok + 2 * (kQuantBlock - 1)) / kQuantBlock);
  return launch_ex(store_kernel, dim3(blocks, n_kv_heads, n_seq), dim3(kStoreThreads), 0, st, 1, p);
}

cudaError_t launch_quant_gather(const int32_t* topk_idx, const int32_t* k_small, int k_max, const QuantDev& full,
                                const CacheDev& small_cache, int64_t small_rows, const int32_t* active, int n_seq,
                                int n_kv_heads, int32_t* status, cudaStream_t st) {
  dim3 grid((k_max + kGatherRows - 1) / kGatherRows, n_kv_heads, n_seq);
  return launch_ex(quant_gather_kernel, grid, dim3(kGatherThreads), 0, st, 1, topk_idx, k_small, k_max, full, small_cache,
                   small_rows, active, n_kv_heads, status);
}

}  // namespace rkv
