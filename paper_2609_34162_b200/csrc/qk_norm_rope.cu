// libslidedp: RMS norm of every query and key head with the position rotation in the same pass,
// forward and backward. See include/slidedp_ops.h for the contract.
//
// With r = rsqrt(mean(x^2) + eps), xh = x r, n = xh w and R the rotation of the token:
//   y  = R n
//   dz = R^T dy,  u = w dz,  dx = r (u - xh mean(u xh)),  dw = sum over rows of dz xh
// Bound: HBM. Forward reads x and writes y (4 bytes per BF16 value), backward reads x and dy and
// writes dx (6 bytes); the cos/sin row and w are read once per task and stay in registers.
// Measured, 8192 tokens, 32 + 8 heads of 128, BF16: forward 36 us (4.7 TB/s), backward 63 + 3.6 us (4.1 TB/s);
// 16384 tokens, 40 + 8 heads: forward 83 us (4.9 TB/s).
#include "device_utils.cuh"
#include "ops_internal.h"

namespace slidedp {

constexpr int kQkThreads = 128;
constexpr int kQkForwardHeads = 4;    // heads of one token per task: one cos/sin row serves them all
constexpr int kQkBackwardBlocks = 148 * 4;   // as many as are resident (117 registers); 148 * 8: 65 + 6.8 us against 63 + 3.5

struct QkSide {
  const void* x;
  const void* dy;   // backward
  void* out;        // y, or dx
  const void* w;
  int64_t x_t, x_h, dy_t, dy_h, out_t, out_h;
  int heads;
};

struct QkParams {
  QkSide side[2];   // q, k
  const float* cos_sin;
  const int32_t* positions;
  int64_t table_rows;
  uint32_t tokens;
  int head_dim, rope_dim, interleaved;
  int chunks_q, chunks;   // forward: tasks of a token, the queries' first
  int blocks_q;           // backward: blocks that take queries
  double eps, inv_dim;
  float* partials;  // backward: [block][head_dim], null when no weight gradient is asked for
};

// A run of VW values of type T as they lie in memory.
template <typename T, int VW> struct Run;
template <> struct Run<uint16_t, 8> {
  uint4 r;
  __device__ void load(const uint16_t* p) { r = ld_stream(p); }   // a pass over more than L2 holds: 90 -> 83 us
  __device__ void unpack(float* v) const {
    v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
    v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
  }
  static __device__ void store(uint16_t* p, const float* v) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7]));
  }
};
template <> struct Run<uint16_t, 4> {
  uint2 r;
  __device__ void load(const uint16_t* p) { r = *reinterpret_cast<const uint2*>(p); }
  __device__ void unpack(float* v) const { v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y); }
  static __device__ void store(uint16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
  }
};
template <> struct Run<uint16_t, 1> {
  uint16_t r;
  __device__ void load(const uint16_t* p) { r = *p; }
  __device__ void unpack(float* v) const { v[0] = __uint_as_float((uint32_t)r << 16); }
  static __device__ void store(uint16_t* p, const float* v) { *p = (uint16_t)f32_to_bf16_bits(v[0]); }
};
template <> struct Run<float, 4> {
  float4 r;
  __device__ void load(const float* p) { r = *reinterpret_cast<const float4*>(p); }
  __device__ void unpack(float* v) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ void store(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Run<float, 1> {
  float r;
  __device__ void load(const float* p) { r = *p; }
  __device__ void unpack(float* v) const { v[0] = r; }
  static __device__ void store(float* p, const float* v) { *p = v[0]; }
};

// A lane owns GPL groups of VW pairs of its row, group g = lane + i * L. A group is two runs of VW
// consecutive values at a0 and a1: the two members of its pairs (or, interleaved, the two halves
// of the VW adjacent pairs; or, past rope_dim, two runs of values that are not rotated). So a row
// is loaded, rotated and stored without exchanging values between lanes.
struct Group {
  int a0, a1, pair;   // pair: the first pair's index in the cos/sin row
  bool on0, on1, rotated;
  __device__ Group(const QkParams& p, int g, int vw) {
    const int half = p.rope_dim / 2, first = g * vw;
    rotated = first < half;
    pair = first;
    if (rotated) {
      a0 = p.interleaved ? 2 * first : first;
      a1 = p.interleaved ? 2 * first + vw : first + half;
      on0 = on1 = true;
    } else {
      const int rest = (p.head_dim - p.rope_dim + 1) / 2;
      a0 = p.rope_dim + first - half;
      a1 = a0 + rest;
      on0 = first - half < rest;
      on1 = on0 && a1 < p.head_dim;
    }
  }
};

template <typename T, int VW>
struct Both {   // a group's two runs
  Run<T, VW> lo, hi;
  __device__ __forceinline__ void load(const T* row, const Group& g, bool live) {
    lo = Run<T, VW>();
    hi = Run<T, VW>();
    if (live && g.on0) lo.load(row + g.a0);
    if (live && g.on1) hi.load(row + g.a1);
  }
  __device__ __forceinline__ void unpack(float* v) const { lo.unpack(v); hi.unpack(v + VW); }
  static __device__ __forceinline__ void store(T* row, const Group& g, const float* v) {
    if (g.on0) Run<T, VW>::store(row + g.a0, v);
    if (g.on1) Run<T, VW>::store(row + g.a1, v + VW);
  }
};

// (a, b) -> (a c - b s, b c + a s) for the pairs of a group; s negated gives the transpose.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = a, y = b;
  a = x * c - y * s;
  b = y * c + x * s;
}
template <int VW>
__device__ __forceinline__ void rotate(float* v, const float* c, const float* s, bool interleaved) {
  // two loops rather than selected indices, which would put v in local memory
  if (VW > 1 && interleaved) {
#pragma unroll
    for (int i = 0; i < VW; ++i) turn(v[2 * i], v[2 * i + 1], c[i], s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VW; ++i) turn(v[i], v[VW + i], c[i], s[i]);
  }
}

// The token's cosines and sines for a group; NaN when its position is outside the table.
template <int VW>
__device__ __forceinline__ void load_angles(const QkParams& p, uint32_t t, const Group& g, float* c, float* s) {
  if (!g.rotated) return;
  const int64_t pos = p.positions ? (int64_t)p.positions[t] : t;
  if (pos < 0 || pos >= p.table_rows) {
#pragma unroll
    for (int i = 0; i < VW; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
    return;
  }
  const float* row = p.cos_sin + pos * p.rope_dim + g.pair;
  const int half = p.rope_dim / 2;
  constexpr int R = VW >= 4 ? 4 : 1;
#pragma unroll
  for (int i = 0; i < VW; i += R) {
    Run<float, R> a, b;
    a.load(row + i);
    b.load(row + half + i);
    a.unpack(c + i);
    b.unpack(s + i);
  }
}

// The arithmetic of a row: FP32 for groups of several pairs; FP64 for single pairs, which serve the heads
// of a few values where dx is a small difference (one value: u (1 - xh^2), about eps of u).
template <int VW> struct Acc { using type = float; };
template <> struct Acc<1> { using type = double; };
__device__ __forceinline__ float inverse_root(float x) { return rsqrtf(x); }
__device__ __forceinline__ double inverse_root(double x) { return rsqrt(x); }

template <int L, typename A>
__device__ __forceinline__ A sum_lanes(A x) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// One task = kQkForwardHeads query or key heads of one token for L lanes. The heads' values stay as they were
// loaded between the norm and the rotation: 16 bytes per run in flight and in registers. (Two heads per task: 40
// and 103 us for the sizes above, eight: 43 and 105; 36 and 90 before streaming loads.)
template <typename T, int VW, int L, int GPL>
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_kernel(const __grid_constant__ QkParams p) {
  constexpr int U = kQkForwardHeads, N = 2 * VW;
  const int lane = threadIdx.x % L;
  const uint32_t task = blockIdx.x * (kQkThreads / L) + threadIdx.x / L;
  uint32_t t = task / (uint32_t)p.chunks;
  int chunk = (int)(task - t * (uint32_t)p.chunks);
  const bool is_k = chunk >= p.chunks_q, live = t < p.tokens;
  if (!live) t = 0;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int h0 = (is_k ? chunk - p.chunks_q : chunk) * U;
  const int heads = live ? sd.heads - h0 : 0;
  const T* x = static_cast<const T*>(sd.x) + t * sd.x_t + h0 * sd.x_h;

  Both<T, VW> raw[GPL][U];
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[i][u].load(x + u * sd.x_h, g, u < heads);
  }
  float r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      float v[N];
      raw[i][u].unpack(v);
#pragma unroll
      for (int e = 0; e < N; ++e) sum = fmaf(v[e], v[e], sum);
    }
    r[u] = rsqrtf(fmaf(sum_lanes<L>(sum), (float)p.inv_dim, (float)p.eps));
  }
  T* y = static_cast<T*>(sd.out) + t * sd.out_t + h0 * sd.out_h;
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
    float w[N], c[VW], s[VW];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = 1.0f;
    if (sd.w) {
      Both<T, VW> rw;
      rw.load(static_cast<const T*>(sd.w), g, true);
      rw.unpack(w);
    }
    load_angles<VW>(p, t, g, c, s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      raw[i][u].unpack(v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= r[u] * w[e];
      if (g.rotated) rotate<VW>(v, c, s, p.interleaved);
      if (u < heads) Both<T, VW>::store(y + u * sd.out_h, g, v);
    }
  }
}

// One task = one head of one token, walked by a fixed grid whose first blocks take queries, the others keys;
// the next task's values are on their way while this one's are worked on. Every lane keeps its values' share
// of dw in registers over all its tasks; the block adds its lanes in a fixed order and writes one row of
// partial sums, which qk_weight_grad_kernel adds in a fixed order. So dw has the same bits in every run.
template <typename T, int VW, int L, int GPL>
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_backward_kernel(const __grid_constant__ QkParams p) {
  constexpr int N = 2 * VW, kTasks = kQkThreads / L;
  using A = typename Acc<VW>::type;
  __shared__ float part[kTasks][L * GPL * N + 1];
  const bool is_k = (int)blockIdx.x >= p.blocks_q;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int block = (int)blockIdx.x - (is_k ? p.blocks_q : 0);
  const int blocks = is_k ? (int)gridDim.x - p.blocks_q : p.blocks_q;
  const int lane = threadIdx.x % L;
  const uint32_t heads = (uint32_t)sd.heads, tasks = p.tokens * heads, step = (uint32_t)blocks * kTasks;
  float w[GPL][N], dw[GPL][N];
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
#pragma unroll
    for (int e = 0; e < N; ++e) { w[i][e] = 1.0f; dw[i][e] = 0.0f; }
    if (sd.w) {
      Both<T, VW> rw;
      rw.load(static_cast<const T*>(sd.w), g, true);
      rw.unpack(w[i]);
    }
  }
  Both<T, VW> rx[GPL], rd[GPL];
  const auto fetch = [&](uint32_t task, bool live) {
    const uint32_t t = live ? task / heads : 0, h = live ? task - t * heads : 0;
    const T* x = static_cast<const T*>(sd.x) + t * sd.x_t + h * sd.x_h;
    const T* d = static_cast<const T*>(sd.dy) + t * sd.dy_t + h * sd.dy_h;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      rx[i].load(x, g, live);
      rd[i].load(d, g, live);
    }
  };
  // every lane of a warp takes part in every round, so that the lane sums see whole warps
  const uint32_t mine = (uint32_t)block * kTasks + threadIdx.x / L, rounds = (tasks + step - 1) / step;
  fetch(mine, mine < tasks);
  for (uint32_t k = 0; k < rounds; ++k) {
    const uint32_t task = mine + k * step;
    const bool live = task < tasks && task >= mine;
    const uint32_t t = live ? task / heads : 0, h = live ? task - t * heads : 0;
    float x[GPL][N], d[GPL][N];
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      rx[i].unpack(x[i]);
      rd[i].unpack(d[i]);
    }
    const uint32_t next = task + step;
    if (k + 1 < rounds) fetch(next, live && next < tasks && next > task);
    A xx = 0, xu = 0;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      if (g.rotated && live) {
        float c[VW], s[VW];
        load_angles<VW>(p, t, g, c, s);
#pragma unroll
        for (int e = 0; e < VW; ++e) s[e] = -s[e];
        rotate<VW>(d[i], c, s, p.interleaved);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        xx += (A)x[i][e] * (A)x[i][e];
        xu += (A)x[i][e] * ((A)d[i][e] * (A)w[i][e]);
      }
    }
    const A r = inverse_root(sum_lanes<L>(xx) * (A)p.inv_dim + (A)p.eps);
    const A mean = sum_lanes<L>(xu) * r * (A)p.inv_dim;   // mean(u xh)
    if (!live) continue;
    T* out = static_cast<T*>(sd.out) + t * sd.out_t + h * sd.out_h;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      float o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const A xh = (A)x[i][e] * r;
        dw[i][e] += (float)((A)d[i][e] * xh);
        o[e] = (float)(r * ((A)d[i][e] * (A)w[i][e] - xh * mean));
      }
      Both<T, VW>::store(out, g, o);
    }
  }
  if (!p.partials) return;
#pragma unroll
  for (int i = 0; i < GPL; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) part[threadIdx.x / L][(lane * GPL + i) * N + e] = dw[i][e];
  __syncthreads();
  for (int k = threadIdx.x; k < L * GPL * N; k += kQkThreads) {
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < kTasks; ++s) sum += part[s][k];
    const int e = k % N, i = k / N % GPL;
    const Group g(p, k / (N * GPL) + i * L, VW);
    if (e < VW ? g.on0 : g.on1)
      p.partials[(int64_t)blockIdx.x * p.head_dim + (e < VW ? g.a0 + e : g.a1 + e - VW)] = sum;
  }
}

// dw[d] = sum over the side's blocks of partials[block][d]: 32 columns per block, 32 threads per column,
// each adding every 32nd row, folded in a fixed order.
__global__ void __launch_bounds__(1024) qk_weight_grad_kernel(const float* partials, int head_dim, int blocks_q,
                                                              int blocks, float* dw_q, float* dw_k) {
  __shared__ float part[32][33];
  const int side = blockIdx.y, d = blockIdx.x * 32 + threadIdx.x;
  float* dw = side ? dw_k : dw_q;
  const int lo = side ? blocks_q : 0, hi = side ? blocks : blocks_q;
  float s = 0.0f;
  if (d < head_dim)
    for (int b = lo + (int)threadIdx.y; b < hi; b += 32) s += partials[(int64_t)b * head_dim + d];
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && d < head_dim && dw) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += part[i][threadIdx.x];
    dw[d] = t;
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

int check_qk(const slidedp_qk_args* a) {
  if (!a || a->tokens < 0 || a->tokens > kMaxTokens || a->heads_q < 0 || a->heads_k < 0 || a->heads_q > 65536 ||
      a->heads_k > 65536 || a->head_dim < 1 || a->head_dim > kMaxHeadDim)
    return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens * (a->heads_q > a->heads_k ? a->heads_q : a->heads_k) > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  if (a->rope_dim < 0 || a->rope_dim > a->head_dim || a->rope_dim % 2 != 0 || a->table_rows < 0 ||
      (a->interleaved != 0 && a->interleaved != 1) || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) ||
      !(a->eps >= 0.0) || !is_finite(a->eps))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

// What both directions need of their tensors; fills the common part of the parameters. vec: pairs per group, the
// widest that the lengths are multiples of and all tensors are aligned to (8 only for BF16: 16-byte runs).
// 8192 tokens, 40 heads of 128, BF16, forward / backward: 36 / 63 us in groups of 8 pairs, 37 / 70 in groups of 4.
struct QkPlan {
  QkParams p;
  int vec, lanes;
};
int plan_qk(const slidedp_qk_args* a, const slidedp_heads* const in[2], const slidedp_heads* const dy[2],
            const slidedp_heads* const out[2], const void* const w[2], const float* cos_sin,
            const int32_t* positions, QkPlan* plan) {
  const int64_t elem = a->dtype == SLIDEDP_F32 ? 4 : 2;
  const int heads[2] = {a->heads_q, a->heads_k};
  if (a->rope_dim > 0) {
    if (!cos_sin || reinterpret_cast<uintptr_t>(cos_sin) % 4 != 0) return SLIDEDP_ERR_INVALID_ARG;
    if (!positions && a->tokens > a->table_rows) return SLIDEDP_ERR_INVALID_ARG;
  }
  if (reinterpret_cast<uintptr_t>(positions) % 4 != 0) return SLIDEDP_ERR_INVALID_ARG;
  QkParams& p = plan->p;
  const auto fits = [&](int vec) {
    if (a->rope_dim % (2 * vec) != 0 || (a->head_dim - a->rope_dim) % (2 * vec) != 0) return false;
    if (a->rope_dim > 0 && (reinterpret_cast<uintptr_t>(cos_sin) % 16 != 0 || a->rope_dim % 8 != 0)) return false;
    for (int s = 0; s < 2; ++s) {
      if (heads[s] == 0) continue;
      if (!heads_aligned(in[s], elem, vec * elem, a->tokens, heads[s]) || !heads_aligned(out[s], elem, vec * elem, a->tokens, heads[s]) ||
          (dy && !heads_aligned(dy[s], elem, vec * elem, a->tokens, heads[s])) ||
          reinterpret_cast<uintptr_t>(w[s]) % (uintptr_t)(vec * elem) != 0)
        return false;
    }
    return true;
  };
  for (int s = 0; s < 2; ++s) {
    p.side[s] = QkSide{};
    p.side[s].heads = heads[s];
    if (heads[s] == 0) continue;
    if (!heads_ok(in[s], elem) || !heads_ok(out[s], elem) || (dy && !heads_ok(dy[s], elem)))
      return SLIDEDP_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(w[s]) % (uintptr_t)elem != 0) return SLIDEDP_ERR_INVALID_ARG;
    p.side[s].x = in[s]->data;
    p.side[s].x_t = in[s]->stride_token;
    p.side[s].x_h = in[s]->stride_head;
    if (dy) {
      p.side[s].dy = dy[s]->data;
      p.side[s].dy_t = dy[s]->stride_token;
      p.side[s].dy_h = dy[s]->stride_head;
    }
    p.side[s].out = out[s]->data;
    p.side[s].out_t = out[s]->stride_token;
    p.side[s].out_h = out[s]->stride_head;
    p.side[s].w = w[s];
  }
  p.cos_sin = cos_sin;
  p.positions = positions;
  p.tokens = (uint32_t)a->tokens;
  p.table_rows = a->table_rows;
  p.head_dim = a->head_dim;
  p.rope_dim = a->rope_dim;
  p.interleaved = a->interleaved;
  p.eps = a->eps;
  p.inv_dim = 1.0 / a->head_dim;
  p.partials = nullptr;
  p.blocks_q = 0;
  p.chunks_q = (a->heads_q + kQkForwardHeads - 1) / kQkForwardHeads;
  p.chunks = p.chunks_q + (a->heads_k + kQkForwardHeads - 1) / kQkForwardHeads;
  plan->vec = elem == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
  plan->lanes = 32;
  if (plan->vec > 1)
    for (plan->lanes = 4; plan->lanes * 2 * plan->vec < a->head_dim;) plan->lanes *= 2;
  return SLIDEDP_OK;
}

#define SLIDEDP_QK_LANES(KERNEL, T, VW)                                            \
  switch (plan.lanes) {                                                            \
    case 4: KERNEL<T, VW, 4, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;       \
    case 8: KERNEL<T, VW, 8, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;       \
    case 16: KERNEL<T, VW, 16, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;     \
    default: KERNEL<T, VW, 32, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;     \
  }
#define SLIDEDP_QK_LAUNCH(KERNEL)                                                  \
  do {                                                                             \
    if (plan.vec == 1) {                                                           \
      if (f32) KERNEL<float, 1, 32, 4><<<grid, kQkThreads, 0, st>>>(plan.p);       \
      else KERNEL<uint16_t, 1, 32, 4><<<grid, kQkThreads, 0, st>>>(plan.p);        \
    } else if (f32) {                                                              \
      SLIDEDP_QK_LANES(KERNEL, float, 4)                                           \
    } else if (plan.vec == 8) {                                                    \
      SLIDEDP_QK_LANES(KERNEL, uint16_t, 8)                                        \
    } else {                                                                       \
      SLIDEDP_QK_LANES(KERNEL, uint16_t, 4)                                        \
    }                                                                              \
  } while (0)

}  // namespace

extern "C" {

int slidedp_qk_norm_rope(slidedp_ctx* ctx, const slidedp_qk_args* a, const slidedp_heads* q, const slidedp_heads* k,
                         const void* w_q, const void* w_k, const float* cos_sin, const int32_t* positions,
                         const slidedp_heads* q_out, const slidedp_heads* k_out, void* cuda_stream) {
  if (!ctx || check_qk(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens == 0 || a->heads_q + a->heads_k == 0) return SLIDEDP_OK;
  const slidedp_heads* in[2] = {q, k};
  const slidedp_heads* out[2] = {q_out, k_out};
  const void* w[2] = {w_q, w_k};
  QkPlan plan;
  int rc = plan_qk(a, in, nullptr, out, w, cos_sin, positions, &plan);
  if (rc != SLIDEDP_OK) return rc;
  const int64_t tasks = a->tokens * plan.p.chunks, per_block = kQkThreads / plan.lanes;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  const unsigned grid = (unsigned)((tasks + per_block - 1) / per_block);
  const bool f32 = a->dtype == SLIDEDP_F32;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  FAULT_POINT();
  SLIDEDP_QK_LAUNCH(qk_norm_rope_kernel);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_qk_norm_rope_workspace(const slidedp_qk_args* a) {
  if (check_qk(a) != SLIDEDP_OK) return 0;
  return (size_t)kQkBackwardBlocks * a->head_dim * sizeof(float);
}

int slidedp_qk_norm_rope_backward(slidedp_ctx* ctx, const slidedp_qk_args* a, const slidedp_heads* q,
                                  const slidedp_heads* k, const void* w_q, const void* w_k, const float* cos_sin,
                                  const int32_t* positions, const slidedp_heads* dq_out, const slidedp_heads* dk_out,
                                  const slidedp_heads* dq, const slidedp_heads* dk, float* dw_q, float* dw_k,
                                  void* workspace, void* cuda_stream) {
  if (!ctx || check_qk(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if ((dw_q || dw_k) && !workspace) return SLIDEDP_ERR_INVALID_ARG;
  if (!aligned16(workspace)) return SLIDEDP_ERR_MISALIGNED;
  const slidedp_heads* in[2] = {q, k};
  const slidedp_heads* dy[2] = {dq_out, dk_out};
  const slidedp_heads* out[2] = {dq, dk};
  const void* w[2] = {w_q, w_k};
  QkPlan plan;
  const bool work = a->tokens > 0 && a->heads_q + a->heads_k > 0;
  int rc = work ? plan_qk(a, in, dy, out, w, cos_sin, positions, &plan) : SLIDEDP_OK;
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // a side without rows: its weight gradient is zero
  const size_t dw_bytes = a->head_dim * sizeof(float);
  if (dw_q && (!work || a->heads_q == 0)) { CU(cudaMemsetAsync(dw_q, 0, dw_bytes, st)); dw_q = nullptr; }
  if (dw_k && (!work || a->heads_k == 0)) { CU(cudaMemsetAsync(dw_k, 0, dw_bytes, st)); dw_k = nullptr; }
  if (!work) return SLIDEDP_OK;
  // the fixed grid, split between queries and keys by their share of the heads; each side that has
  // heads gets at least one block and no more than it has work for
  const int64_t per_block = kQkThreads / plan.lanes;
  const int64_t need_q = (a->tokens * a->heads_q + per_block - 1) / per_block, need_k = (a->tokens * a->heads_k + per_block - 1) / per_block;
  int64_t bq = need_q, bk = need_k;
  if (bq + bk > kQkBackwardBlocks) {
    bq = (int64_t)kQkBackwardBlocks * a->heads_q / (a->heads_q + a->heads_k);
    if (a->heads_q > 0 && bq < 1) bq = 1;
    if (a->heads_k > 0 && bq > kQkBackwardBlocks - 1) bq = kQkBackwardBlocks - 1;
    bk = kQkBackwardBlocks - bq;
    if (bq > need_q) bq = need_q;
    if (bk > need_k) bk = need_k;
  }
  plan.p.blocks_q = (int)bq;
  plan.p.partials = (dw_q || dw_k) ? static_cast<float*>(workspace) : nullptr;
  const unsigned grid = (unsigned)(bq + bk);
  const bool f32 = a->dtype == SLIDEDP_F32;
  FAULT_POINT();
  SLIDEDP_QK_LAUNCH(qk_norm_rope_backward_kernel);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  if (plan.p.partials) {
    FAULT_POINT();
    qk_weight_grad_kernel<<<dim3((a->head_dim + 31) / 32, 2), dim3(32, 32), 0, st>>>(
        plan.p.partials, a->head_dim, (int)bq, (int)(bq + bk), dw_q, dw_k);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  return SLIDEDP_OK;
}

}  // extern "C"
