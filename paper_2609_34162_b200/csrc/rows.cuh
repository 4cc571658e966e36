// Rows of BF16 or FP32 values as vectors of V of them.
#pragma once

#include "device_utils.cuh"

namespace slidedp {

template <typename T, int V> struct Raw;
template <> struct Raw<uint16_t, 8> { typedef uint4 type; };
template <> struct Raw<uint16_t, 2> { typedef uint32_t type; };
template <> struct Raw<uint16_t, 1> { typedef uint16_t type; };
template <> struct Raw<float, 4> { typedef uint4 type; };
template <> struct Raw<float, 1> { typedef float type; };

template <typename T, int V>
__device__ __forceinline__ void to_floats(typename Raw<T, V>::type a, float* v) {
  if constexpr (sizeof(T) == 2 && V == 8) {
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
    v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
  } else if constexpr (sizeof(T) == 2 && V == 2) {
    v[0] = bf16_lo(a); v[1] = bf16_hi(a);
  } else if constexpr (sizeof(T) == 2) {
    v[0] = __uint_as_float((uint32_t)a << 16);
  } else if constexpr (V == 4) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  } else {
    v[0] = a;
  }
}
// V values to consecutive elements of either type, aligned to V of them or to 16 bytes.
template <int V>
__device__ __forceinline__ void store_values(float* p, const float* v) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int e = 0; e < V; e += 4)
      st_stream(p + e, make_uint4(__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3])));
  } else if constexpr (V == 2) {
    __stcs(reinterpret_cast<float2*>(p), make_float2(v[0], v[1]));
  } else {
    __stcs(p, v[0]);
  }
}
template <int V>
__device__ __forceinline__ void store_values(uint16_t* p, const float* v) {
  if constexpr (V == 8) {
    st_stream(p, make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])));
  } else if constexpr (V == 4) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])));
  } else if constexpr (V == 2) {
    __stcs(reinterpret_cast<uint32_t*>(p), f32x2_to_bf16x2(v[0], v[1]));
  } else {
    __stcs(p, (uint16_t)f32_to_bf16_bits(v[0]));
  }
}
template <int V, typename T>
__device__ __forceinline__ void load_values(const T* p, float* v) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (sizeof(T) == 4) v[e] = p[e];
    else v[e] = __uint_as_float((uint32_t)p[e] << 16);
  }
}

}  // namespace slidedp
