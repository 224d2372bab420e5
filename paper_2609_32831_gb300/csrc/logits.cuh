// Rows of logits of any supported type, as 16-byte vectors.
#pragma once

#include "common.cuh"

namespace uc {

constexpr float kLog2e = 1.4426950408889634f;

// A 16-byte vector of logits by type: its elements as fp32, its largest element
// (NaN if there is one).
template <typename T>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int kE = 4;
  static __device__ __forceinline__ float get(const uint4& v, int e) {
    return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
  }
  static __device__ __forceinline__ uint32_t raw(float x) { return __float_as_uint(x); }
  static __device__ __forceinline__ float largest(const uint4& v) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(get(v, 0)), "f"(get(v, 1)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(get(v, 2)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(get(v, 3)));
    return m;
  }
};
template <typename H, typename H2>
struct Logits16 {
  static constexpr int kE = 8;
  static __device__ __forceinline__ H2 pair(uint32_t w) { return *reinterpret_cast<H2*>(&w); }
  static __device__ __forceinline__ H2 largest2(const uint4& v) {
    return __hmax2_nan(__hmax2_nan(pair(v.x), pair(v.y)), __hmax2_nan(pair(v.z), pair(v.w)));
  }
};
template <>
struct Logits<__nv_bfloat16> : Logits16<__nv_bfloat16, __nv_bfloat162> {
  static __device__ __forceinline__ float get(const uint4& v, int e) {
    const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    return e & 1 ? bf16_hi(w) : bf16_lo(w);
  }
  static __device__ __forceinline__ uint32_t raw(float x) { return __float_as_uint(x) >> 16; }  // (exact)
  static __device__ __forceinline__ float largest(const uint4& v) {
    const __nv_bfloat162 m = largest2(v);
    return __bfloat162float(__hmax_nan(m.x, m.y));
  }
};
template <>
struct Logits<__half> : Logits16<__half, __half2> {
  static __device__ __forceinline__ float get(const uint4& v, int e) {
    const __half2 h = pair(e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w);
    return e & 1 ? __high2float(h) : __low2float(h);
  }
  static __device__ __forceinline__ uint32_t raw(float x) { return __half_as_ushort(__float2half_rn(x)); }
  static __device__ __forceinline__ float largest(const uint4& v) {
    const __half2 m = largest2(v);
    return __half2float(__hmax_nan(m.x, m.y));
  }
};
// A vector from its elements (rows' ends, values that are no logits).
template <typename T, typename F>
__device__ __forceinline__ uint4 make_vector(const F& element) {
  constexpr int kE = Logits<T>::kE;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kE == 4)
      w[i] = Logits<T>::raw(element(i));
    else
      w[i] = Logits<T>::raw(element(2 * i)) | (Logits<T>::raw(element(2 * i + 1)) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

}  // namespace uc
