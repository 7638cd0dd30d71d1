// Rows of binary32 or bfloat16 values, eight neighbours at a time.
#pragma once

#include <cuda_bf16.h>

#include "tensorcore.cuh"

namespace rtopk {
namespace mat {

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// |v| as a bit pattern: ordered like the magnitudes, a NaN above everything, so that maxima of it are exact and
// independent of their order.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Eight neighbours of a row as they are in memory; those past the end are zero.  `vec`: the row allows 16-byte loads.
template <class T>
struct Eight;
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, int left, bool vec) {
    if (vec && left >= 8) {
      a = *(const float4*)p, b = *(const float4*)(p + 4);
    } else {
      a = make_float4(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
      b = make_float4(left > 4 ? p[4] : 0.f, left > 5 ? p[5] : 0.f, left > 6 ? p[6] : 0.f, left > 7 ? p[7] : 0.f);
    }
  }
  __device__ __forceinline__ void widen_to(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {
    m = max(max(m, magnitude(a.x)), max(magnitude(a.y), max(magnitude(a.z), magnitude(a.w))));
    return max(max(m, magnitude(b.x)), max(magnitude(b.y), max(magnitude(b.z), magnitude(b.w))));
  }
  static __device__ __forceinline__ uint32_t as_magnitude(uint32_t m) { return m; }
  __device__ __forceinline__ float at(int j) const { return j < 4 ? (j < 2 ? (j ? a.y : a.x) : (j == 2 ? a.z : a.w)) : (j < 6 ? (j == 4 ? b.x : b.y) : (j == 6 ? b.z : b.w)); }
};
template <>
struct Eight<__nv_bfloat16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, bool vec) {
    if (vec && left >= 8) {
      const uint4 a = *(const uint4*)p;
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
      const uint16_t* u = (const uint16_t*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (left > 2 * i ? u[2 * i] : 0u) | (left > 2 * i + 1 ? (uint32_t)u[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void widen_to(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  // two 16-bit maxima in a word
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    return m;
  }
  static __device__ __forceinline__ uint32_t as_magnitude(uint32_t m) { return max(m << 16, m & 0xFFFF0000u); }
  __device__ __forceinline__ float at(int j) const { return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16); }
};
template <class T>
__device__ __forceinline__ void load8(const T* p, int left, bool vec, float (&v)[8]) {
  Eight<T> e;
  e.load(p, left, vec);
  e.widen_to(v);
}

}  // namespace mat
}  // namespace rtopk
