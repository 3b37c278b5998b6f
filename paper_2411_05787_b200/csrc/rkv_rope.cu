// Rotary positions of a batch of tokens: the fused projection's rows are split into queries, keys and values, and the
// first rot channels of every query and key head are turned.
//
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a) amp,   a = pos f_i,
// pairs (x, y) = channels (i, i + rot/2) or (2i, 2i + 1).  An angle of a far position must not be formed in fp32: at
// position 10^5 its 24 bits leave an error of 10^-2 radians in the fastest pair.  Frequencies come as turns per
// position in 64-bit fixed point, so  pos * f mod 2^64  IS the angle's fraction of a turn, exact up to pos 2^-65 turns,
// for any int32 position; its upper 32 bits go to sincospif as a number in [-1, 1).
//
// HBM-bound: every channel is read once and written once (12 KB + 12 KB per token with 48 bf16 heads).  One CTA of 64
// threads per token.  A thread keeps its 16 channels of a head - eight pairs, or 16 channels that are only copied - for
// all heads, eight heads to a row of the CTA, so the angles are worked out once per (token, pair), one thread apiece
// while the rows are on their way, and its eight sines and cosines then stay in registers.  Six heads of a thread are in
// flight as raw 16-byte pieces.  Measured for 32768 tokens of 48 bf16 heads: 117 us, 6.86 TB/s (four tokens to a CTA:
// 127 us; with three heads in flight 141 us; with rows converted as they arrive, which doubles their registers, 205 us);
// 20000 fp32 tokens 106 us, 6.93 TB/s; 4097 tokens of 36 heads 13.7 us (four to a CTA: 17.2 us); one token 2.1 us.
#include <cuda_bf16.h>

#include "rkv_internal.h"

namespace rkv {
namespace {

constexpr int kRopeThreads = 64;

struct RopeParams {
  const void* qkv; int64_t tok_stride;      // elements
  const int32_t* pos; const unsigned long long* freqs;
  __nv_bfloat16* q; __nv_bfloat16* k; __nv_bfloat16* v;
  int n_q, n_kv, rot;
  float amp;
};

// Eight channels as they come (converted where they are used, so that as many heads as possible are in flight).
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcg(reinterpret_cast<const float4*>(p));
    b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&r);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

constexpr int kBatch = 6;   // heads of a thread whose loads are in flight together

template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
  __shared__ float2 sm_cs[kHeadDim / 2];
  const int tid = threadIdx.x, part = tid & 7, hsub = tid >> 3;
  const int64_t tok = blockIdx.x;
  const int heads = p.n_q + 2 * p.n_kv;
  const int half = p.rot >> 1;
  const bool turn = part < (p.rot >> 4);
  // this thread's two pieces of eight channels in every head
  const int ca = (kInterleaved || !turn) ? 16 * part : 8 * part;
  const int cb = (kInterleaved || !turn) ? 16 * part + 8 : half + 8 * part;
  const T* row = static_cast<const T*>(p.qkv) + tok * p.tok_stride;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  Raw8<T> ra[kBatch], rb[kBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + 8 * i;
      if (h < heads && (p.v != nullptr || h < p.n_q + p.n_kv)) {
        ra[i].load(row + h * kHeadDim + ca);
        rb[i].load(row + h * kHeadDim + cb);
      }
    }
  };
  load(hsub);
  if (tid < half) {
    const long long pos = __ldcg(p.pos + tok);
    const unsigned long long t = (unsigned long long)pos * __ldg(p.freqs + tid);
    float s, c;
    sincospif((float)(int)(t >> 32) * 4.656612873e-10f, &s, &c);   // 2^-31: half turns
    sm_cs[tid] = make_float2(c * p.amp, s * p.amp);
  }
  __syncthreads();
  float c[8], s[8];
  if (turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 cs = sm_cs[8 * part + j];
      c[j] = cs.x;
      s[j] = cs.y;
    }
  }
  for (int h0 = hsub; h0 < heads; h0 += 8 * kBatch) {
    if (h0 != hsub) load(h0);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + 8 * i;
      if (h >= heads || (p.v == nullptr && h >= p.n_q + p.n_kv)) continue;
      float a[8], b[8];
      ra[i].get(a);
      rb[i].get(b);
      __nv_bfloat16* out;
      if (h < p.n_q) out = p.q + (tok * p.n_q + h) * kHeadDim;
      else if (h < p.n_q + p.n_kv) out = p.k + (tok * p.n_kv + h - p.n_q) * kHeadDim;
      else out = p.v + (tok * p.n_kv + h - p.n_q - p.n_kv) * kHeadDim;
      if (turn && h < p.n_q + p.n_kv) {
        if (kInterleaved) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = a[2 * j], y = a[2 * j + 1], z = b[2 * j], w = b[2 * j + 1];
            a[2 * j] = x * c[j] - y * s[j];
            a[2 * j + 1] = x * s[j] + y * c[j];
            b[2 * j] = z * c[4 + j] - w * s[4 + j];
            b[2 * j + 1] = z * s[4 + j] + w * c[4 + j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = a[j], y = b[j];
            a[j] = x * c[j] - y * s[j];
            b[j] = x * s[j] + y * c[j];
          }
        }
      }
      store8(out + ca, a);
      store8(out + cb, b);
    }
  }
}

}  // namespace

cudaError_t launch_rope(const void* qkv, bool is_bf16, int64_t tok_stride, const int32_t* pos, int n_tok, int n_q,
                        int n_kv, const uint64_t* freqs, int rot, bool interleaved, float amp, void* q, void* k, void* v,
                        cudaStream_t st) {
  RopeParams p;
  p.qkv = qkv;
  p.tok_stride = tok_stride;
  p.pos = pos;
  p.freqs = reinterpret_cast<const unsigned long long*>(freqs);
  p.q = static_cast<__nv_bfloat16*>(q);
  p.k = static_cast<__nv_bfloat16*>(k);
  p.v = static_cast<__nv_bfloat16*>(v);
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.rot = rot;
  p.amp = amp;
  const dim3 grid(n_tok), block(kRopeThreads);
  if (is_bf16)
    return interleaved ? launch_ex(rope_kernel<__nv_bfloat16, true>, grid, block, 0, st, 1, p)
                       : launch_ex(rope_kernel<__nv_bfloat16, false>, grid, block, 0, st, 1, p);
  return interleaved ? launch_ex(rope_kernel<float, true>, grid, block, 0, st, 1, p)
                     : launch_ex(rope_kernel<float, false>, grid, block, 0, st, 1, p);
}

}  // namespace rkv
