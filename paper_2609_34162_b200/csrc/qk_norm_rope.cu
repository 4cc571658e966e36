// libslidedp: RMS norm of every query and key head with the position rotation in the same pass,
// forward and backward. See include/slidedp_ops.h for the contract.
//
// With r = rsqrt(mean(x^2) + eps), xh = x r, n = xh w and R the rotation of the token:
//   y  = R n
//   dz = R^T dy,  u = w dz,  dx = r (u - xh mean(u xh)),  dw = sum over rows of dz xh
// Bound: HBM. Forward reads x and writes y (4 bytes per BF16 value), backward reads x and dy and
// writes dx (6 bytes); the cos/sin row and w are read once per task and stay in registers.
#include "device_utils.cuh"
#include "ops_internal.h"

namespace slidedp {

constexpr int kQkThreads = 128;
constexpr int kQkForwardHeads = 4;    // heads of one token per task: one cos/sin row serves them all
constexpr int kQkBackwardHeads = 2;   // backward holds x and dy of each
constexpr int kQkBackwardBlocks = 148 * 8;

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
  int64_t tokens, table_rows;
  int head_dim, rope_dim, interleaved, blocks_q;
  double eps;
  float* partials;  // backward: [block][head_dim], null when no weight gradient is asked for
};

template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
  static __device__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ void store(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
  static __device__ void load4(const uint16_t* p, float* v) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
  }
  static __device__ void store4(uint16_t* p, const float* v) {
    uint2 a;
    a.x = f32_to_bf16_bits(v[0]) | f32_to_bf16_bits(v[1]) << 16;
    a.y = f32_to_bf16_bits(v[2]) | f32_to_bf16_bits(v[3]) << 16;
    *reinterpret_cast<uint2*>(p) = a;
  }
};
template <> struct Elem<float> {
  static __device__ float load(const float* p) { return *p; }
  static __device__ void store(float* p, float v) { *p = v; }
  static __device__ void load4(const float* p, float* v) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  }
  static __device__ void store4(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};

// A lane owns GPL groups of VW pairs of its row, group g = lane + i * L. A group is two runs of VW
// consecutive values at a0 and a1: the two members of its pairs (or, interleaved, the two halves
// of the VW adjacent pairs; or, past rope_dim, two runs of values that are not rotated). So a row
// is loaded, rotated and stored without exchanging values between lanes.
template <int VW>
struct Group {
  int a0, a1;
  bool on0, on1, rotated;
  int pair;   // first pair's index in the cos/sin row
  __device__ Group(const QkParams& p, int g) {
    const int half = p.rope_dim / 2, first = g * VW;
    rotated = first < half;
    pair = first;
    if (rotated) {
      a0 = p.interleaved ? 2 * first : first;
      a1 = p.interleaved ? 2 * first + VW : first + half;
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
__device__ __forceinline__ void load_group(const T* row, const Group<VW>& g, float* v) {
  if constexpr (VW == 4) {
    if (g.on0) { Elem<T>::load4(row + g.a0, v); Elem<T>::load4(row + g.a1, v + 4); }
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
  } else {
    v[0] = g.on0 ? Elem<T>::load(row + g.a0) : 0.0f;
    v[1] = g.on1 ? Elem<T>::load(row + g.a1) : 0.0f;
  }
}
template <typename T, int VW>
__device__ __forceinline__ void store_group(T* row, const Group<VW>& g, const float* v) {
  if constexpr (VW == 4) {
    if (g.on0) { Elem<T>::store4(row + g.a0, v); Elem<T>::store4(row + g.a1, v + 4); }
  } else {
    if (g.on0) Elem<T>::store(row + g.a0, v[0]);
    if (g.on1) Elem<T>::store(row + g.a1, v[1]);
  }
}
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
__device__ __forceinline__ void load_angles(const QkParams& p, int64_t t, const Group<VW>& g, float* c, float* s) {
  if (!g.rotated) return;
  const int64_t pos = p.positions ? (int64_t)p.positions[t] : t;
  if (pos < 0 || pos >= p.table_rows) {
#pragma unroll
    for (int i = 0; i < VW; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
    return;
  }
  const float* row = p.cos_sin + pos * p.rope_dim + g.pair;
  const int half = p.rope_dim / 2;
  if constexpr (VW == 4) {
    Elem<float>::load4(row, c);
    Elem<float>::load4(row + half, s);
  } else {
    c[0] = row[0];
    s[0] = row[half];
  }
}

// The arithmetic of a row: FP32 for groups of four pairs; FP64 for single pairs, which serve the heads
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

// One task = kQkForwardHeads heads of one token for L lanes; blocks below blocks_q take queries,
// the others keys.
template <typename T, int VW, int L, int GPL>
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_kernel(const __grid_constant__ QkParams p) {
  constexpr int U = kQkForwardHeads, N = 2 * VW;
  const bool is_k = (int)blockIdx.x >= p.blocks_q;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int block = (int)blockIdx.x - (is_k ? p.blocks_q : 0);
  const int lane = threadIdx.x % L;
  const int chunks = (sd.heads + U - 1) / U;
  const int64_t task = (int64_t)block * (kQkThreads / L) + threadIdx.x / L;
  const bool live = task < p.tokens * chunks;
  const int64_t t = live ? task / chunks : 0;
  const int h0 = live ? (int)(task % chunks) * U : sd.heads;   // no heads for lanes past the end

  float v[U][GPL][N];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group<VW> g(p, lane + i * L);
      if (h0 + u < sd.heads) {
        load_group<T, VW>(static_cast<const T*>(sd.x) + t * sd.x_t + (h0 + u) * sd.x_h, g, v[u][i]);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[u][i][e] = 0.0f;
      }
    }
  float r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < GPL; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) s = fmaf(v[u][i][e], v[u][i][e], s);
    r[u] = rsqrtf(sum_lanes<L>(s) / (float)p.head_dim + (float)p.eps);
  }
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group<VW> g(p, lane + i * L);
    float w[N], c[VW], s[VW];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = 1.0f;
    if (sd.w) load_group<T, VW>(static_cast<const T*>(sd.w), g, w);
    load_angles<VW>(p, t, g, c, s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h0 + u >= sd.heads) continue;
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][i][e] *= r[u] * w[e];
      if (g.rotated) rotate<VW>(v[u][i], c, s, p.interleaved);
      store_group<T, VW>(static_cast<T*>(sd.out) + t * sd.out_t + (h0 + u) * sd.out_h, g, v[u][i]);
    }
  }
}

// Same tasks, walked by a fixed grid: every lane keeps its values' share of dw in registers over
// all its tasks; the block adds its lanes in a fixed order and writes one row of partial sums, which
// qk_weight_grad_kernel adds in a fixed order. So dw has the same bits in every run.
template <typename T, int VW, int L, int GPL>
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_backward_kernel(const __grid_constant__ QkParams p) {
  constexpr int U = kQkBackwardHeads, N = 2 * VW, kTasks = kQkThreads / L;
  __shared__ float part[kTasks][L * GPL * N + 1];
  const bool is_k = (int)blockIdx.x >= p.blocks_q;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int block = (int)blockIdx.x - (is_k ? p.blocks_q : 0);
  const int blocks = is_k ? (int)gridDim.x - p.blocks_q : p.blocks_q;
  const int lane = threadIdx.x % L;
  const int chunks = (sd.heads + U - 1) / U;
  const int64_t tasks = p.tokens * chunks;
  float w[GPL][N], dw[GPL][N];
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group<VW> g(p, lane + i * L);
#pragma unroll
    for (int e = 0; e < N; ++e) { w[i][e] = 1.0f; dw[i][e] = 0.0f; }
    if (sd.w) load_group<T, VW>(static_cast<const T*>(sd.w), g, w[i]);
  }
  // every lane of the block takes part in every round, so that the lane sums see whole warps
  for (int64_t base = (int64_t)block * kTasks; base < tasks; base += (int64_t)blocks * kTasks) {
    const int64_t task = base + threadIdx.x / L;
    const bool live = task < tasks;
    const int64_t t = live ? task / chunks : 0;
    const int h0 = live ? (int)(task % chunks) * U : sd.heads;
    float x[U][GPL][N], d[U][GPL][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < GPL; ++i) {
        const Group<VW> g(p, lane + i * L);
        if (h0 + u < sd.heads) {
          load_group<T, VW>(static_cast<const T*>(sd.x) + t * sd.x_t + (h0 + u) * sd.x_h, g, x[u][i]);
          load_group<T, VW>(static_cast<const T*>(sd.dy) + t * sd.dy_t + (h0 + u) * sd.dy_h, g, d[u][i]);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) x[u][i][e] = d[u][i][e] = 0.0f;
        }
      }
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group<VW> g(p, lane + i * L);
      if (!g.rotated || !live) continue;
      float c[VW], s[VW];
      load_angles<VW>(p, t, g, c, s);
#pragma unroll
      for (int e = 0; e < VW; ++e) s[e] = -s[e];
#pragma unroll
      for (int u = 0; u < U; ++u) if (h0 + u < sd.heads) rotate<VW>(d[u][i], c, s, p.interleaved);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      using A = typename Acc<VW>::type;
      A xx = 0, xu = 0;
#pragma unroll
      for (int i = 0; i < GPL; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          xx += (A)x[u][i][e] * (A)x[u][i][e];
          xu += (A)x[u][i][e] * ((A)d[u][i][e] * (A)w[i][e]);
        }
      const A r = inverse_root(sum_lanes<L>(xx) / (A)p.head_dim + (A)p.eps);
      const A mean = sum_lanes<L>(xu) * r / (A)p.head_dim;   // mean(u xh)
      if (h0 + u >= sd.heads) continue;
#pragma unroll
      for (int i = 0; i < GPL; ++i) {
        const Group<VW> g(p, lane + i * L);
        float o[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const A xh = (A)x[u][i][e] * r;
          dw[i][e] += (float)((A)d[u][i][e] * xh);
          o[e] = (float)(r * ((A)d[u][i][e] * (A)w[i][e] - xh * mean));
        }
        store_group<T, VW>(static_cast<T*>(sd.out) + t * sd.out_t + (h0 + u) * sd.out_h, g, o);
      }
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
    const Group<VW> g(p, k / (N * GPL) + i * L);
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
  if (a->rope_dim < 0 || a->rope_dim > a->head_dim || a->rope_dim % 2 != 0 || a->table_rows < 0 ||
      (a->interleaved != 0 && a->interleaved != 1) || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) ||
      !(a->eps >= 0.0) || !is_finite(a->eps))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

// What both directions need of their tensors; fills the common part of the parameters. `vec` says
// whether groups of four pairs can be used: lengths that four pairs divide and 4-element alignment.
struct QkPlan {
  QkParams p;
  bool vec;
  int lanes;
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
  QkParams& p = plan->p;
  plan->vec = a->rope_dim % 8 == 0 && a->head_dim % 8 == 0 &&
              (a->rope_dim == 0 || reinterpret_cast<uintptr_t>(cos_sin) % 16 == 0);
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
    plan->vec = plan->vec && heads_aligned(in[s], elem, 4 * elem, a->tokens, heads[s]) &&
                heads_aligned(out[s], elem, 4 * elem, a->tokens, heads[s]) &&
                (!dy || heads_aligned(dy[s], elem, 4 * elem, a->tokens, heads[s])) &&
                reinterpret_cast<uintptr_t>(w[s]) % (uintptr_t)(4 * elem) == 0;
  }
  p.cos_sin = cos_sin;
  p.positions = positions;
  p.tokens = a->tokens;
  p.table_rows = a->table_rows;
  p.head_dim = a->head_dim;
  p.rope_dim = a->rope_dim;
  p.interleaved = a->interleaved;
  p.eps = a->eps;
  p.partials = nullptr;
  p.blocks_q = 0;
  plan->lanes = 32;
  if (plan->vec) for (plan->lanes = 4; plan->lanes < a->head_dim / 8;) plan->lanes *= 2;
  return SLIDEDP_OK;
}

int64_t qk_blocks(const QkPlan& plan, int heads, int per_task) {
  const int64_t tasks = plan.p.tokens * ((heads + per_task - 1) / per_task);
  const int per_block = kQkThreads / plan.lanes;
  return (tasks + per_block - 1) / per_block;
}

#define SLIDEDP_QK_LAUNCH(KERNEL)                                                                          \
  do {                                                                                                     \
    if (!plan.vec) {                                                                                       \
      if (f32) KERNEL<float, 1, 32, 4><<<grid, kQkThreads, 0, st>>>(plan.p);                               \
      else KERNEL<uint16_t, 1, 32, 4><<<grid, kQkThreads, 0, st>>>(plan.p);                                \
    } else switch (plan.lanes) {                                                                           \
      case 4: if (f32) KERNEL<float, 4, 4, 1><<<grid, kQkThreads, 0, st>>>(plan.p);                        \
              else KERNEL<uint16_t, 4, 4, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;                  \
      case 8: if (f32) KERNEL<float, 4, 8, 1><<<grid, kQkThreads, 0, st>>>(plan.p);                        \
              else KERNEL<uint16_t, 4, 8, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;                  \
      case 16: if (f32) KERNEL<float, 4, 16, 1><<<grid, kQkThreads, 0, st>>>(plan.p);                      \
               else KERNEL<uint16_t, 4, 16, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;                \
      default: if (f32) KERNEL<float, 4, 32, 1><<<grid, kQkThreads, 0, st>>>(plan.p);                      \
               else KERNEL<uint16_t, 4, 32, 1><<<grid, kQkThreads, 0, st>>>(plan.p); break;                \
    }                                                                                                      \
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
  const int64_t bq = qk_blocks(plan, a->heads_q, kQkForwardHeads), bk = qk_blocks(plan, a->heads_k, kQkForwardHeads);
  if (bq + bk > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  plan.p.blocks_q = (int)bq;
  const unsigned grid = (unsigned)(bq + bk);
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
  const int64_t need_q = qk_blocks(plan, a->heads_q, kQkBackwardHeads), need_k = qk_blocks(plan, a->heads_k, kQkBackwardHeads);
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
