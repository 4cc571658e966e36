// Rows of logits for the losses: 16-byte chunks of either type, running maximum and sums of exponentials.
#pragma once

#include "device_utils.cuh"
#include "tcgen05.cuh"

namespace slidedp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T> struct Logit;
template <> struct Logit<uint16_t> {
  static constexpr int kPer = 8;   // values per 16 bytes
  static __device__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ void store(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
  // the four pairs of values of a chunk
  static __device__ uint64_t two(uint32_t a) { return pair(bf16_lo(a), bf16_hi(a)); }
  static __device__ void unpack(uint4 a, uint64_t* v) { v[0] = two(a.x); v[1] = two(a.y); v[2] = two(a.z); v[3] = two(a.w); }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
  static __device__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ float largest(uint4 a) {
    const uint32_t m = max2(max2(a.x, a.y), max2(a.z, a.w));
    return fmaxf(bf16_lo(m), bf16_hi(m));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
};
template <> struct Logit<float> {
  static constexpr int kPer = 4;
  static __device__ float load(const float* p) { return *p; }
  static __device__ void store(float* p, float v) { *p = v; }
  static __device__ void unpack(uint4 a, uint64_t* v) {
    v[0] = pair(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = pair(__uint_as_float(a.z), __uint_as_float(a.w));
  }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ float largest(uint4 a) {
    return fmaxf(fmaxf(__uint_as_float(a.x), __uint_as_float(a.y)), fmaxf(__uint_as_float(a.z), __uint_as_float(a.w)));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
};

// A row as 16-byte chunks on the address grid of its first value: chunk c holds values
// first + c * kPer .. of which those outside [0, vocab) do not exist (only in the first and last
// chunk). Whole chunks are one 16-byte access whatever the row's alignment.
template <typename T>
struct Row {
  const T* z;
  int64_t vocab;
  int head;      // values of chunk 0 that lie before the row
  __device__ Row(const T* z_, int64_t vocab_) : z(z_), vocab(vocab_) {
    head = (int)((reinterpret_cast<uintptr_t>(z_) & 15u) / sizeof(T));
  }
  // I: int where all chunks' values are below 2^31, else int64_t
  template <typename I> __device__ I first(I c) const { return c * (I)Logit<T>::kPer - (I)head; }
  template <typename I> __device__ bool whole(I c) const { return first(c) >= 0 && first(c) + (I)Logit<T>::kPer <= (I)vocab; }
  template <typename I> __device__ uint4 load(I c) const {
    const I f = first(c);
    if (f >= 0 && f + (I)Logit<T>::kPer <= (I)vocab) return ld_stream(z + f);
    union { uint4 v; T e[Logit<T>::kPer]; } u;
    u.v = Logit<T>::lowest();     // -inf where there is no value
    for (int i = 0; i < Logit<T>::kPer; ++i)
      if (f + i >= 0 && f + i < (I)vocab) u.e[i] = z[f + i];
    return u.v;
  }
};

__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
  float lo, hi;
  split(x, &lo, &hi);
  return pair(exp2_approx(lo), exp2_approx(hi));
}

// Running maximum and sums of exp2(k (z - m)) for one or two factors k.
struct SoftSum {
  float m, s0, s1;
};
__device__ __forceinline__ float shifted(float z, float m, float k) {
  // z = m = -inf (nothing seen yet, or a row of -inf) counts as no shift rather than NaN
  return z == m ? 0.0f : (z - m) * k;
}
// Where only -inf (or NaN) was seen any finite shift gives the sums, zero (or NaN).
__device__ __forceinline__ float finite_shift(float m) { return m == -INFINITY ? 0.0f : m; }
// Joins the sums of the lanes that differ in the bits below LANES; all of them get the result.
template <int LANES, bool kTwo>
__device__ __forceinline__ SoftSum join_lanes(SoftSum a, float k0, float k1) {
  float m = a.m;   // never NaN: a NaN logit shows in the sums
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  a.s0 *= exp2_approx(shifted(a.m, m, k0));
  if (kTwo) a.s1 *= exp2_approx(shifted(a.m, m, k1));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    a.s0 += __shfl_xor_sync(0xffffffffu, a.s0, o);
    if (kTwo) a.s1 += __shfl_xor_sync(0xffffffffu, a.s1, o);
  }
  a.m = m;
  return a;
}
// Adds N chunks to a thread's sums. Differences are taken before they are scaled: the type's lowest value
// times a factor above one would be -inf.
template <typename T, bool kTwo, int N>
__device__ __forceinline__ void accumulate(SoftSum& mine, const uint4* a, float k0, float k1) {
  float top = mine.m;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, Logit<T>::largest(a[i]));
  const float shift = finite_shift(top);
  mine.s0 *= exp2_approx(shifted(mine.m, top, k0));
  if (kTwo) mine.s1 *= exp2_approx(shifted(mine.m, top, k1));
  mine.m = top;
  const uint64_t minus = pair(-shift, -shift), f0 = pair(k0, k0), f1 = pair(k1, k1);
  uint64_t s0 = 0, s1 = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint64_t v[Logit<T>::kPer / 2];
    Logit<T>::unpack(a[i], v);
#pragma unroll
    for (int e = 0; e < Logit<T>::kPer / 2; ++e) {
      const uint64_t d = add2(v[e], minus);
      s0 = add2(s0, exp2_pair(mul2(d, f0)));
      if (kTwo) s1 = add2(s1, exp2_pair(mul2(d, f1)));
    }
  }
  float x, y;
  split(s0, &x, &y);
  mine.s0 += x + y;
  if (kTwo) {
    split(s1, &x, &y);
    mine.s1 += x + y;
  }
}

}  // namespace slidedp
