// Eight channels of a row at a time: as they come out of a projection, as bf16, and their bounds.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace rkv {

// Converted where they are used, so that as many rows as possible are in flight.
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

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&r);
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// Least and largest of eight channels over rows; NaN does not count.
struct Bounds8 {
  __nv_bfloat162 lo[4], hi[4];
  static __device__ __forceinline__ __nv_bfloat162 bits(uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); }
  static __device__ __forceinline__ uint32_t bits(__nv_bfloat162 x) { return *reinterpret_cast<const uint32_t*>(&x); }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = bits(0x7f807f80u);
      hi[i] = bits(0xff80ff80u);
    }
  }
  __device__ __forceinline__ void join(uint4 least, uint4 most) {
    const uint32_t a[4] = {least.x, least.y, least.z, least.w}, b[4] = {most.x, most.y, most.z, most.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __hmin2(lo[i], bits(a[i]));
      hi[i] = __hmax2(hi[i], bits(b[i]));
    }
  }
  __device__ __forceinline__ void take(uint4 x) { join(x, x); }
  __device__ __forceinline__ void over_octets() {   // over the four octets of a warp, which hold the same channels
#pragma unroll
    for (int sh = 8; sh <= 16; sh <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __hmin2(lo[i], bits(__shfl_xor_sync(0xffffffffu, bits(lo[i]), sh)));
        hi[i] = __hmax2(hi[i], bits(__shfl_xor_sync(0xffffffffu, bits(hi[i]), sh)));
      }
  }
  __device__ __forceinline__ uint4 lo4() const { return make_uint4(bits(lo[0]), bits(lo[1]), bits(lo[2]), bits(lo[3])); }
  __device__ __forceinline__ uint4 hi4() const { return make_uint4(bits(hi[0]), bits(hi[1]), bits(hi[2]), bits(hi[3])); }
};

}  // namespace rkv
