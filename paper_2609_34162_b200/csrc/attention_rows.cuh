// Attention rows computed by one warp, lanes over the head's values, one partner row at a time: any
// head_dim up to 256 and any stride. Used by the kernels for views that the tensor-core kernels do not
// take, and by those kernels to redo a row in which a NaN showed up: a masked pair has
// probability zero, but zero times the NaN or infinity of a row that is not visible is NaN in a
// matrix product, and only the visible rows may decide the result.
#pragma once

#include "attention.h"
#include "device_utils.cuh"

namespace slidedp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kLanes = 32;
constexpr int kMaxPer = host::kMaxHeadDim / kLanes;

__device__ __forceinline__ float load_bf16(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

__device__ __forceinline__ void load_row(const AttnView& v, int t, int h, int n, float* x) {
  const uint16_t* row = v.p + t * v.t + h * v.h;
  const int lane = threadIdx.x % kLanes;
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) x[i] = lane + i * kLanes < n ? load_bf16(row + lane + i * kLanes) : 0.0f;
}
__device__ __forceinline__ void store_row(const AttnView& v, int t, int h, int from, int to, const float* x) {
  uint16_t* row = v.p + t * v.t + h * v.h;
  const int lane = threadIdx.x % kLanes;
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i)
    if (lane + i * kLanes >= from && lane + i * kLanes < to) row[lane + i * kLanes] = (uint16_t)f32_to_bf16_bits(x[i]);
}
__device__ __forceinline__ float dot(const float* a, const float* b) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) s = fmaf(a[i], b[i], s);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
// Score of one pair in units of log2 e from the raw product, and d score / d (scale * product).
__device__ __forceinline__ float score(const AttnParams& p, float raw, float slope, int distance, float* grad) {
  float s = raw * p.scale;
  *grad = 1.0f;
  if (p.softcap > 0.0f) {
    const float th = tanhf(s / p.softcap);
    s = p.softcap * th;
    *grad = 1.0f - th * th;
  }
  return (s - slope * (float)abs(distance)) * kLog2e;
}

// One row each, by a whole warp. Not inlined: the tensor-core kernels call them on NaN only.
static __device__ __noinline__ void attention_out_row(const AttnParams& p, int i, int h, bool with_lse) {
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], o[kMaxPer] = {};
  load_row(p.q, i, h, p.head_dim, q);
  int lo, hi;
  p.mask.keys_of(i, p.mask.above(i), &lo, &hi);
  float m = -INFINITY, l = 0.0f;
  for (int j = lo; j < hi; ++j) {
    float x[kMaxPer], g;
    load_row(p.k, j, hk, p.head_dim, x);
    const float s = score(p, dot(q, x), slope, i - j, &g);
    load_row(p.v, j, hk, p.head_dim, x);
    const float top = fmaxf(m, s), shift = top == -INFINITY ? 0.0f : top;   // scores of -inf weigh nothing, also when they come first
    const float keep = exp2f(m - shift), e = exp2f(s - shift);
    m = top;
    l = l * keep + e;
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) o[d] = fmaf(e, x[d], o[d] * keep);
  }
  const float inv = lo < hi ? 1.0f / l : 0.0f;
#pragma unroll
  for (int d = 0; d < kMaxPer; ++d) o[d] *= inv;
  store_row(p.o, i, h, 0, p.head_dim, o);
  if (with_lse && threadIdx.x % kLanes == 0) p.lse[(int64_t)h * p.tokens + i] = lo < hi ? (m + log2f(l)) / kLog2e : -INFINITY;
}

// dq's values [from, to) are stored.
static __device__ __noinline__ void attention_dq_row(const AttnParams& p, int i, int h, int from, int to) {
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], go[kMaxPer], dq[kMaxPer] = {};
  load_row(p.q, i, h, p.head_dim, q);
  load_row(p.dout, i, h, p.head_dim, go);
  const float lse = p.row_lse[h * p.pitch + i], delta = p.row_delta[h * p.pitch + i];
  int lo, hi;
  p.mask.keys_of(i, p.mask.above(i), &lo, &hi);
  for (int j = lo; j < hi; ++j) {
    float k[kMaxPer], v[kMaxPer], g;
    load_row(p.k, j, hk, p.head_dim, k);
    load_row(p.v, j, hk, p.head_dim, v);
    const float pr = exp2f(score(p, dot(q, k), slope, i - j, &g) - lse);
    const float ds = pr * (dot(go, v) - delta) * g * p.scale;
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) dq[d] = fmaf(ds, k[d], dq[d]);
  }
  store_row(p.dq, i, h, from, to, dq);
}

// Values [from, to) of dk, of dv, or of both are stored.
static __device__ __noinline__ void attention_dkv_row(const AttnParams& p, int j, int hk, bool with_dk, bool with_dv, int from, int to) {
  float k[kMaxPer], v[kMaxPer], dk[kMaxPer] = {}, dv[kMaxPer] = {};
  load_row(p.k, j, hk, p.head_dim, k);
  load_row(p.v, j, hk, p.head_dim, v);
  int lo, hi;
  p.mask.queries_of(j, p.mask.above(j), &lo, &hi);
  for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    for (int i = lo; i < hi; ++i) {
      float q[kMaxPer], go[kMaxPer], g;
      load_row(p.q, i, h, p.head_dim, q);
      load_row(p.dout, i, h, p.head_dim, go);
      const float pr = exp2f(score(p, dot(q, k), slope, i - j, &g) - p.row_lse[h * p.pitch + i]);
      const float ds = pr * (dot(go, v) - p.row_delta[h * p.pitch + i]) * g * p.scale;
#pragma unroll
      for (int d = 0; d < kMaxPer; ++d) {
        dv[d] = fmaf(pr, go[d], dv[d]);
        dk[d] = fmaf(ds, q[d], dk[d]);
      }
    }
  }
  if (with_dk) store_row(p.dk, j, hk, from, to, dk);
  if (with_dv) store_row(p.dv, j, hk, from, to, dv);
}

}  // namespace slidedp
