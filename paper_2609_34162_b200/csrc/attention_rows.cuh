// Attention rows computed by one warp, lanes over the head's values, one partner row at a time: any
// head_dim up to 256 and any stride. Used by the kernels for views that the tensor-core kernels do not
// take, and by those kernels to redo a row in which a NaN showed up: a masked pair has
// probability zero, but zero times the NaN or infinity of a row that is not visible is NaN in a
// matrix product, and only the visible rows may decide the result. A NaN that the visible rows account for stays:
// redoing such rows too made one NaN key cost 125 ms forward and 440 ms backward (4096 tokens, 8 + 2 heads of 128, 0.09 and
// 0.14 ms without it).
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
    const float y = s / p.softcap, r = 1.0f / (1.0f + expf(2.0f * fabsf(y)));
    s = p.softcap * tanhf(y);
    *grad = 4.0f * r * (1.0f - r);   // 1 - tanh^2, without the difference that cancels when the score is near the cap
  }
  return (s - slope * (float)abs(distance)) * kLog2e;
}

// ---- one row each, by a whole warp ----------------------------------------------------------------------
//
// WIDE, for the tensor-core kernels' views: 16 lanes per partner with 16 bytes each, two partners at once and four of those
// ahead, because what bounds a warp alone is the latency of its loads and sums (dkv of 4096 queries, 4 heads of 128: 3 ms a
// key row against 14). Otherwise lanes over the head's values and one partner at a time. Not inlined: the tensor-core kernels
// call them on NaN only.
template <bool WIDE>
struct Lanes {
  static constexpr int kPer = WIDE ? 16 : kLanes, kGroups = kLanes / kPer, kAhead = WIDE ? 4 : 1, kStep = kGroups * kAhead;
  static __device__ __forceinline__ int group() { return threadIdx.x % kLanes / kPer; }
  // zeros if !live
  static __device__ __forceinline__ void load(const AttnView& v, int t, int h, int n, bool live, float* x) {
    if constexpr (WIDE) {
      const int d = threadIdx.x % kPer * 8;
      uint4 y = make_uint4(0, 0, 0, 0);
      if (live && d < n) y = *reinterpret_cast<const uint4*>(v.p + t * v.t + h * v.h + d);
      const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
      }
    } else {
      load_row(v, t, h, live ? n : 0, x);
    }
  }
  static __device__ __forceinline__ void store(const AttnView& v, int t, int h, int from, int to, const float* x) {
    if constexpr (WIDE) {
      const int d = threadIdx.x % kLanes * 8;
      if (d >= from && d < to)
        *reinterpret_cast<uint4*>(v.p + t * v.t + h * v.h + d) =
            make_uint4(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]), f32x2_to_bf16x2(x[6], x[7]));
    } else {
      store_row(v, t, h, from, to, x);
    }
  }
  static __device__ __forceinline__ float dot(const float* a, const float* b) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxPer; ++i) s = fmaf(a[i], b[i], s);
#pragma unroll
    for (int o = kPer / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
  }
  // the groups' sums joined
  static __device__ __forceinline__ void join(float* x) {
    if constexpr (kGroups == 2)
#pragma unroll
      for (int i = 0; i < kMaxPer; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], kPer);
  }
};

template <bool WIDE>
static __device__ __noinline__ void attention_out_row(const AttnParams& p, int i, int h, bool with_lse) {
  using L = Lanes<WIDE>;
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], o[kMaxPer] = {};
  L::load(p.q, i, h, p.head_dim, true, q);
  int lo, hi;
  p.mask.keys_of(i, p.mask.above(i), &lo, &hi);
  float m = -INFINITY, l = 0.0f;
  for (int j0 = lo + L::group(); j0 - L::group() < hi; j0 += L::kStep) {
    float x[L::kAhead][kMaxPer], s[L::kAhead], g, top = m;
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) L::load(p.k, j0 + u * L::kGroups, hk, p.head_dim, j0 + u * L::kGroups < hi, x[u]);
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) {
      const int j = j0 + u * L::kGroups;
      s[u] = score(p, L::dot(q, x[u]), slope, i - j, &g);
      if (j >= hi) s[u] = -INFINITY;
      top = fmaxf(top, s[u]);
    }
    const float shift = top == -INFINITY ? 0.0f : top;   // scores of -inf weigh nothing, also when they come first
    const float keep = exp2f(m - shift);
    m = top;
    l *= keep;
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) L::load(p.v, j0 + u * L::kGroups, hk, p.head_dim, j0 + u * L::kGroups < hi, x[u]);
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) o[d] *= keep;
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) {
      const float e = exp2f(s[u] - shift);
      l += e;
#pragma unroll
      for (int d = 0; d < kMaxPer; ++d) o[d] = fmaf(e, x[u][d], o[d]);
    }
  }
  if constexpr (L::kGroups == 2) {
    const float top = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, L::kPer)), keep = exp2f(m - (top == -INFINITY ? 0.0f : top));
    m = top;
    l *= keep;
    l += __shfl_xor_sync(0xffffffffu, l, L::kPer);
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) o[d] *= keep;
    L::join(o);
  }
  const float inv = lo < hi ? 1.0f / l : 0.0f;
#pragma unroll
  for (int d = 0; d < kMaxPer; ++d) o[d] *= inv;
  L::store(p.o, i, h, 0, p.head_dim, o);
  if (with_lse && threadIdx.x % kLanes == 0) p.lse[(int64_t)h * p.tokens + i] = lo < hi ? (m + log2f(l)) / kLog2e : -INFINITY;
}

// dq's values [from, to) are stored.
template <bool WIDE>
static __device__ __noinline__ void attention_dq_row(const AttnParams& p, int i, int h, int from, int to) {
  using L = Lanes<WIDE>;
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], go[kMaxPer], dq[kMaxPer] = {};
  L::load(p.q, i, h, p.head_dim, true, q);
  L::load(p.dout, i, h, p.head_dim, true, go);
  const float lse = p.row_lse[h * p.pitch + i], delta = p.row_delta[h * p.pitch + i];
  int lo, hi;
  p.mask.keys_of(i, p.mask.above(i), &lo, &hi);
  for (int j0 = lo + L::group(); j0 - L::group() < hi; j0 += L::kStep) {
    float k[L::kAhead][kMaxPer], v[L::kAhead][kMaxPer];
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) {
      const int j = j0 + u * L::kGroups;
      L::load(p.k, j, hk, p.head_dim, j < hi, k[u]);
      L::load(p.v, j, hk, p.head_dim, j < hi, v[u]);
    }
#pragma unroll
    for (int u = 0; u < L::kAhead; ++u) {
      const int j = j0 + u * L::kGroups;
      float g;
      const float pr = exp2f(score(p, L::dot(q, k[u]), slope, i - j, &g) - lse);
      const float d = L::dot(go, v[u]), ds = j < hi ? pr * (d - delta) * g * p.scale : 0.0f;
#pragma unroll
      for (int e = 0; e < kMaxPer; ++e) dq[e] = fmaf(ds, k[u][e], dq[e]);
    }
  }
  L::join(dq);
  L::store(p.dq, i, h, from, to, dq);
}

// Values [from, to) of dk, of dv, or of both are stored.
template <bool WIDE>
static __device__ __noinline__ void attention_dkv_row(const AttnParams& p, int j, int hk, bool with_dk, bool with_dv, int from, int to) {
  using L = Lanes<WIDE>;
  float k[kMaxPer], v[kMaxPer], dk[kMaxPer] = {}, dv[kMaxPer] = {};
  L::load(p.k, j, hk, p.head_dim, true, k);
  L::load(p.v, j, hk, p.head_dim, true, v);
  int lo, hi;
  p.mask.queries_of(j, p.mask.above(j), &lo, &hi);
  for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    for (int i0 = lo + L::group(); i0 - L::group() < hi; i0 += L::kStep) {
      float q[L::kAhead][kMaxPer], go[L::kAhead][kMaxPer], lse[L::kAhead], delta[L::kAhead];
#pragma unroll
      for (int u = 0; u < L::kAhead; ++u) {
        const int i = i0 + u * L::kGroups;
        L::load(p.q, i, h, p.head_dim, i < hi, q[u]);
        L::load(p.dout, i, h, p.head_dim, i < hi, go[u]);
        lse[u] = i < hi ? p.row_lse[h * p.pitch + i] : 0.0f;
        delta[u] = i < hi ? p.row_delta[h * p.pitch + i] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < L::kAhead; ++u) {
        const int i = i0 + u * L::kGroups;
        float g, pr = exp2f(score(p, L::dot(q[u], k), slope, i - j, &g) - lse[u]);
        if (i >= hi) pr = 0.0f;
        const float d = L::dot(go[u], v), ds = i < hi ? pr * (d - delta[u]) * g * p.scale : 0.0f;
#pragma unroll
        for (int e = 0; e < kMaxPer; ++e) {
          dv[e] = fmaf(pr, go[u][e], dv[e]);
          dk[e] = fmaf(ds, q[u][e], dk[e]);
        }
      }
    }
  }
  L::join(dk);
  L::join(dv);
  if (with_dk) L::store(p.dk, j, hk, from, to, dk);
  if (with_dv) L::store(p.dv, j, hk, from, to, dv);
}

// ---- which rows of NaN to redo -----------------------------------------------------------------------
//
// A warp looks at its rows row0 + lane, those of `redo`, of which lane holds the partners [lo, hi) that it sees; the
// tensor-core kernels' heads only (head_dim up to 128). Returns the rows with a NaN that no visible partner accounts for.

constexpr int kWords = 128 / kLanes;   // a row's values as bits: bit l of word w is value l + 32 w

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// The stored row's NaN among values [from, to), for lane `row`, past L1: TMA wrote them.
__device__ __forceinline__ void nan_columns(const AttnView& v, int t, int h, int row, int from, int to, uint32_t* words) {
  const uint16_t* at = v.p + t * v.t + h * v.h;
  const int lane = threadIdx.x % kLanes;
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const int d = lane + w * kLanes;
    const uint32_t bits = __ballot_sync(0xffffffffu, d >= from && d < to && (__ldcg(at + d) & 0x7fffu) > 0x7f80u);
    if (lane == row) words[w] = bits;
  }
}
__device__ __forceinline__ uint32_t any_left(const uint32_t* words) { return (words[0] | words[1]) | (words[2] | words[3]); }

// Outputs whose scores gave a sum above zero: they are NaN in the columns where a value that they see is.
static __device__ __noinline__ uint32_t spoiled_out_rows(const AttnParams& p, uint32_t redo, int row0, int h, int lo, int hi) {
  const int hk = h / p.group;
  uint32_t left[kWords] = {};
  for (uint32_t r = redo; r; r &= r - 1) nan_columns(p.o, row0 + __ffs(r) - 1, h, __ffs(r) - 1, 0, p.head_dim, left);
  if (!any_left(left)) lo = hi = 0;
  const int from = __reduce_min_sync(0xffffffffu, lo < hi ? lo : p.tokens), to = __reduce_max_sync(0xffffffffu, hi);
  constexpr int U = 8;
  for (int j = from; j < to && __any_sync(0xffffffffu, any_left(left)); j += U) {
    float x[U][kMaxPer];
#pragma unroll
    for (int u = 0; u < U; ++u) load_row(p.v, min(j + u, to - 1), hk, p.head_dim, x[u]);
    uint32_t bad = 0;   // which of the U keys
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int w = 0; w < kWords; ++w) bad |= x[u][w] == x[u][w] ? 0u : 1u << u;
    bad = __reduce_or_sync(0xffffffffu, bad);
    if (!bad) continue;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const uint32_t columns = __ballot_sync(0xffffffffu, x[u][w] != x[u][w]);
        if (min(j + u, to - 1) >= lo && min(j + u, to - 1) < hi) left[w] &= ~columns;
      }
  }
  return __ballot_sync(0xffffffffu, any_left(left) != 0);
}

// Gradients of keys (or, of_v, of values). A visible query whose lse is not finite makes the whole row of both NaN, as its
// scores hold NaN. One with a NaN in dout has it in its delta, which makes the whole row of dk NaN, and in a column of dv. One whose
// delta is infinite adds infinities of the sign of -delta q to dk: NaN in the columns where two differ. What is not finite in
// the key's own k or v shows in the statistics of every query that sees it.
static __device__ __noinline__ uint32_t spoiled_key_rows(const AttnParams& p, uint32_t redo, int row0, int hk, int lo, int hi, bool of_v,
                                                         int from, int to) {
  const int lane = threadIdx.x % kLanes;
  uint32_t left[kWords] = {}, up[kWords] = {}, down[kWords] = {};
  for (uint32_t r = redo; r; r &= r - 1) nan_columns(of_v ? p.dv : p.dk, row0 + __ffs(r) - 1, hk, __ffs(r) - 1, from, to, left);
  if (!any_left(left)) lo = hi = 0;
  const int first = __reduce_min_sync(0xffffffffu, lo < hi ? lo : p.tokens) & ~(kLanes * 4 - 1), last = __reduce_max_sync(0xffffffffu, hi);
  for (int h = hk * p.group; h < (hk + 1) * p.group; ++h)
    for (int i0 = first; i0 < last && __any_sync(0xffffffffu, any_left(left)); i0 += kLanes * 4) {   // the pitch is a multiple of 128
      const float4 l4 = *reinterpret_cast<const float4*>(p.row_lse + h * p.pitch + i0 + lane * 4);
      const float4 d4 = *reinterpret_cast<const float4*>(p.row_delta + h * p.pitch + i0 + lane * 4);
      const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, ds[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t nans = __ballot_sync(0xffffffffu, !finite(ls[e]) || (!of_v && ds[e] != ds[e]));   // of the whole row
        const uint32_t some = __ballot_sync(0xffffffffu, !finite(ds[e]));
        for (uint32_t rest = nans | some; rest && __any_sync(0xffffffffu, any_left(left)); rest &= rest - 1) {
          const int at = __ffs(rest) - 1, i = i0 + at * 4 + e;
          const bool seen = i >= lo && i < hi;
          if (!__any_sync(0xffffffffu, seen)) continue;
          if (nans >> at & 1) {
            if (seen) left[0] = left[1] = left[2] = left[3] = 0;
            continue;
          }
          float x[kMaxPer];
          load_row(of_v ? p.dout : p.q, i, h, p.head_dim, x);
          const float sign = __shfl_sync(0xffffffffu, ds[e], at);
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            if (of_v) {
              const uint32_t columns = __ballot_sync(0xffffffffu, x[w] != x[w]);
              if (seen) left[w] &= ~columns;
            } else {   // zero times infinity counts as both
              const uint32_t plus = __ballot_sync(0xffffffffu, !(x[w] * sign < 0.0f)), minus = __ballot_sync(0xffffffffu, !(x[w] * sign > 0.0f));
              if (seen) {
                up[w] |= plus;
                down[w] |= minus;
                left[w] &= ~(up[w] & down[w]);
              }
            }
          }
        }
      }
    }
  return __ballot_sync(0xffffffffu, any_left(left) != 0);
}

}  // namespace slidedp
