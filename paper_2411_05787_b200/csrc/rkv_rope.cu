// Rotary positions of a batch of tokens: the fused projection's rows are split into queries, keys and values, and the
// first rot channels of every query and key head are turned.
//
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a) amp,   a = pos f_i,
// pairs (x, y) = channels (i, i + rot/2) or (2i, 2i + 1).  An angle of a far position must not be formed in fp32: at
// position 10^5 its 24 bits leave an error of 10^-2 radians in the fastest pair.  Frequencies come as turns per
// position in 64-bit fixed point, so  pos * f mod 2^64  IS the angle's fraction of a turn, exact up to pos 2^-65 turns,
// for any int32 position; its upper 32 bits go to sincospif as a number in [-1, 1).
//
// HBM-bound: every channel is read once and written once (12 KB + 12 KB per token with 48 bf16 heads).  A CTA takes four
// tokens, 64 threads to a token: the angles are worked out once per (token, pair), a quarter of a warp's lanes apiece,
// while the first rows are on their way, and since a thread keeps its 16 channels (eight pairs, or 16 channels that
// are only copied) for all heads, their sines and cosines stay in its registers.
#include <cuda_bf16.h>

#include "rkv_internal.h"

namespace rkv {
namespace {

constexpr int kRopeTokens = 4;
constexpr int kRopeThreads = 64 * kRopeTokens;
constexpr int kRopePairs = kHeadDim / 2;

struct RopeParams {
  const void* qkv; int64_t tok_stride;      // elements
  const int32_t* pos; const unsigned long long* freqs;
  __nv_bfloat16* q; __nv_bfloat16* k; __nv_bfloat16* v;
  int n_tok, n_q, n_kv, rot;
  float amp;
};

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&r);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

// kBatch: heads of a thread whose loads are in flight together
template <typename T, bool kInterleaved, int kBatch>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
  __shared__ float2 sm_cs[kRopeTokens][kRopePairs];
  const int tid = threadIdx.x, part = tid & 7, hsub = (tid >> 3) & 7;
  const int64_t tok = (int64_t)blockIdx.x * kRopeTokens + (tid >> 6);
  const bool live = tok < p.n_tok;
  const int heads = p.n_q + 2 * p.n_kv;
  const int half = p.rot >> 1;
  const bool turn = part < (p.rot >> 4);
  // this thread's two pieces of eight channels in every head
  const int ca = (kInterleaved || !turn) ? 16 * part : 8 * part;
  const int cb = (kInterleaved || !turn) ? 16 * part + 8 : half + 8 * part;
  const T* row = static_cast<const T*>(p.qkv) + tok * p.tok_stride;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  float a[kBatch][8], b[kBatch][8];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + 8 * i;
      if (live && h < heads && (p.v != nullptr || h < p.n_q + p.n_kv)) {
        load8(row + h * kHeadDim + ca, a[i]);
        load8(row + h * kHeadDim + cb, b[i]);
      }
    }
  };
  load(hsub);
  if (live && (tid & 63) < half) {
    const long long pos = __ldg(p.pos + tok);
    const unsigned long long t = (unsigned long long)pos * __ldg(p.freqs + (tid & 63));
    float s, c;
    sincospif((float)(int)(t >> 32) * 4.656612873e-10f, &s, &c);   // 2^-31: half turns
    sm_cs[tid >> 6][tid & 63] = make_float2(c * p.amp, s * p.amp);
  }
  __syncthreads();
  if (!live) return;
  float c[8], s[8];
  if (turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 cs = sm_cs[tid >> 6][8 * part + j];
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
      __nv_bfloat16* out;
      if (h < p.n_q) out = p.q + (tok * p.n_q + h) * kHeadDim;
      else if (h < p.n_q + p.n_kv) out = p.k + (tok * p.n_kv + h - p.n_q) * kHeadDim;
      else out = p.v + (tok * p.n_kv + h - p.n_q - p.n_kv) * kHeadDim;
      if (turn && h < p.n_q + p.n_kv) {
        if (kInterleaved) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = a[i][2 * j], y = a[i][2 * j + 1], z = b[i][2 * j], w = b[i][2 * j + 1];
            a[i][2 * j] = x * c[j] - y * s[j];
            a[i][2 * j + 1] = x * s[j] + y * c[j];
            b[i][2 * j] = z * c[4 + j] - w * s[4 + j];
            b[i][2 * j + 1] = z * s[4 + j] + w * c[4 + j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = a[i][j], y = b[i][j];
            a[i][j] = x * c[j] - y * s[j];
            b[i][j] = x * s[j] + y * c[j];
          }
        }
      }
      store8(out + ca, a[i]);
      store8(out + cb, b[i]);
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
  p.n_tok = n_tok;
  p.n_q = n_q;
  p.n_kv = n_kv;
  p.rot = rot;
  p.amp = amp;
  const dim3 grid((unsigned)((n_tok + (int64_t)kRopeTokens - 1) / kRopeTokens)), block(kRopeThreads);
  if (is_bf16)
    return interleaved ? launch_ex(rope_kernel<__nv_bfloat16, true, 3>, grid, block, 0, st, 1, p)
                       : launch_ex(rope_kernel<__nv_bfloat16, false, 3>, grid, block, 0, st, 1, p);
  return interleaved ? launch_ex(rope_kernel<float, true, 3>, grid, block, 0, st, 1, p)
                     : launch_ex(rope_kernel<float, false, 3>, grid, block, 0, st, 1, p);
}

}  // namespace rkv
