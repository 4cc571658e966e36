// libslidedp: the norms before and after a block with its gate and residual. See include/slidedp_ops.h for the contract.
//
// n = y r w_post, x' = x + a g n, h = x' r' w_pre with r = rsqrt(mean y^2 + eps), r' = rsqrt(mean x'^2 + eps). Backward:
//   u = dh w_pre, d = dx' + r' (u - x' r'^2 mean(u x')), dx = d
//   v = a d g w_post, dy = r (v - y r mean(v y r)), dgate = a d n g', dw_pre = sum dh x' r', dw_post = sum a d g y r
// Bound: HBM; every tensor is read or written once. A row is held in the registers of one block, 16 values per thread, its sums are
// joined through shared memory; blocks stay and take every (number of blocks)th row, with the weights and the sums of their
// gradients in registers. One partial row of sums per block, added in a fixed order by a second kernel.
#include "ops_internal.h"
#include "rows.cuh"

#include <type_traits>

namespace slidedp {

struct NormView {
  void* p;
  int64_t stride;
};
struct BlockNormParams {
  NormView x, y, gate, x_out, h_out;          // forward
  NormView dx_out, dh, dx, dy, dgate;         // backward
  const void *w_post, *w_pre;
  float *dw_post, *dw_pre, *dgate_sum;
  float* partial;                             // [blocks][2][hidden]
  int64_t tokens;
  int hidden;
  int has_y, post, pre, gate_kind, sigmoid;
  float alpha, eps, inv_hidden;
};

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }

// Sums of up to two values over the block; each call uses the other half of `sh`, so that one barrier is enough.
struct BlockSums {
  float2 part[2][32];
};
__device__ __forceinline__ float2 block_sums(float a, float b, BlockSums& sh, int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  const int warps = blockDim.x / 32;
  if (warps == 1) return make_float2(a, b);
  turn ^= 1;
  if (threadIdx.x % 32 == 0) sh.part[turn][threadIdx.x / 32] = make_float2(a, b);
  __syncthreads();
  float2 v = threadIdx.x % 32 < warps ? sh.part[turn][threadIdx.x % 32] : make_float2(0.0f, 0.0f);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

// A thread's N values of a row: vectors of V, blockDim vectors apart.
template <typename T, int V, int N>
struct Values {
  typedef typename Raw<T, V>::type R;
  R a[N / V];
  __device__ __forceinline__ void load(const void* p, int64_t at, int hidden) {
#pragma unroll
    for (int k = 0; k < N / V; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * V;
      if (col < hidden) a[k] = *reinterpret_cast<const R*>(static_cast<const T*>(p) + at + col);
      else memset(&a[k], 0, sizeof(R));
    }
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int k = 0; k < N / V; ++k) to_floats<T, V>(a[k], v + k * V);
  }
};
template <typename T, int V, int N>
__device__ __forceinline__ void store_row(void* p, int64_t at, int hidden, const float* v) {
#pragma unroll
  for (int k = 0; k < N / V; ++k) {
    const int col = (k * blockDim.x + threadIdx.x) * V;
    if (col < hidden) store_values<V>(static_cast<T*>(p) + at + col, v + k * V);
  }
}
template <typename T, int V, int N>
__device__ __forceinline__ void weights(const void* w, int hidden, float* v) {
  if (w) {
    Values<T, V, N> raw;
    raw.load(w, 0, hidden);
    raw.get(v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 1.0f;
  }
}

// kToken: the gate is [tokens, hidden].
template <typename T, int V, int N, bool kToken, int kThreads>
__global__ void __launch_bounds__(kThreads) block_norm_kernel(const __grid_constant__ BlockNormParams p) {
  start_after_previous_kernel();
  __shared__ BlockSums sh;
  int turn = 0;
  float w_post[N], w_pre[N];
  weights<T, V, N>(p.w_post, p.hidden, w_post);
  weights<T, V, N>(p.w_pre, p.hidden, w_pre);
  if (!kToken && p.gate_kind) {       // a factor of the weight
    float g[N];
    weights<T, V, N>(p.gate.p, p.hidden, g);
#pragma unroll
    for (int i = 0; i < N; ++i) w_post[i] *= p.sigmoid ? sigmoid(g[i]) : g[i];
  }
  for (int64_t row = blockIdx.x; row < p.tokens; row += gridDim.x) {
    Values<T, V, N> raw, raw_y, raw_g;
    raw.load(p.x.p, row * p.x.stride, p.hidden);
    if (p.has_y) raw_y.load(p.y.p, row * p.y.stride, p.hidden);
    if (kToken) raw_g.load(p.gate.p, row * p.gate.stride, p.hidden);
    float x[N];
    raw.get(x);
    if (p.has_y) {
      float y[N], r = p.alpha;
      raw_y.get(y);
      if (p.post) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(y[i], y[i], s);
        r *= rsqrtf(block_sums(s, 0.0f, sh, turn).x * p.inv_hidden + p.eps);
      }
      float g[N];
      if (kToken) raw_g.get(g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float f = r * w_post[i];
        if (kToken) f *= p.sigmoid ? sigmoid(g[i]) : g[i];
        x[i] = fmaf(f, y[i], x[i]);
      }
      store_row<T, V, N>(p.x_out.p, row * p.x_out.stride, p.hidden, x);
    }
    if (p.pre) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) s = fmaf(x[i], x[i], s);
      const float r = rsqrtf(block_sums(s, 0.0f, sh, turn).x * p.inv_hidden + p.eps);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] *= r * w_pre[i];
      store_row<T, V, N>(p.h_out.p, row * p.h_out.stride, p.hidden, x);
    }
  }
}

template <typename T, int V, int N, bool kToken, int kThreads>
__global__ void __launch_bounds__(kThreads) block_norm_backward_kernel(const __grid_constant__ BlockNormParams p) {
  start_after_previous_kernel();
  __shared__ BlockSums sh;
  int turn = 0;
  Values<T, V, N> raw_w_post, raw_w_pre, raw_gate;
  if (p.w_post) raw_w_post.load(p.w_post, 0, p.hidden);
  if (p.w_pre) raw_w_pre.load(p.w_pre, 0, p.hidden);
  if (!kToken && p.gate_kind) raw_gate.load(p.gate.p, 0, p.hidden);
  float sum_post[N] = {}, sum_pre[N] = {};
  for (int64_t row = blockIdx.x; row < p.tokens; row += gridDim.x) {
    Values<T, V, N> rx, ry, rg, rd, rh;
    rx.load(p.x.p, row * p.x.stride, p.hidden);
    if (p.has_y) ry.load(p.y.p, row * p.y.stride, p.hidden);
    if (kToken) rg.load(p.gate.p, row * p.gate.stride, p.hidden);
    if (p.dx_out.p) rd.load(p.dx_out.p, row * p.dx_out.stride, p.hidden);
    if (p.pre) rh.load(p.dh.p, row * p.dh.stride, p.hidden);
    float y[N], f[N], g[N], x[N], r = 1.0f;      // y r, the factor a g w_post of it, the gate
    rx.get(x);
    if (p.has_y) {
      ry.get(y);
      if (p.post) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(y[i], y[i], s);
        r = rsqrtf(block_sums(s, 0.0f, sh, turn).x * p.inv_hidden + p.eps);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = p.alpha;
      if (p.w_post) {
        raw_w_post.get(f);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] *= p.alpha;
      }
      if (kToken) rg.get(g);
      else if (p.gate_kind) raw_gate.get(g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (kToken || p.gate_kind) {
          if (p.sigmoid) g[i] = sigmoid(g[i]);
          f[i] *= g[i];
        }
        y[i] *= r;
        x[i] = fmaf(f[i], y[i], x[i]);
      }
    }
    float d[N];
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = 0.0f;
    if (p.dx_out.p) rd.get(d);
    if (p.pre) {
      float h[N], u[N], ss = 0.0f, ux = 0.0f;
      rh.get(h);
#pragma unroll
      for (int i = 0; i < N; ++i) u[i] = 1.0f;
      if (p.w_pre) raw_w_pre.get(u);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        u[i] *= h[i];
        ss = fmaf(x[i], x[i], ss);
        ux = fmaf(u[i], x[i], ux);
      }
      const float2 s = block_sums(ss, ux, sh, turn);
      const float r2 = rsqrtf(s.x * p.inv_hidden + p.eps), m = s.y * r2 * p.inv_hidden;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float xh = x[i] * r2;
        sum_pre[i] = fmaf(h[i], xh, sum_pre[i]);
        d[i] = fmaf(r2, fmaf(-xh, m, u[i]), d[i]);
      }
    }
    store_row<T, V, N>(p.dx.p, row * p.dx.stride, p.hidden, d);
    if (p.has_y) {
      float dot = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float ad = p.alpha * d[i];
        sum_post[i] = fmaf(kToken ? ad * g[i] : ad, y[i], sum_post[i]);
        f[i] *= d[i];                          // now v
        dot = fmaf(f[i], y[i], dot);
      }
      if (kToken && p.dgate.p) {               // a d n g', n = y r w_post
        float w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 1.0f;
        if (p.w_post) raw_w_post.get(w);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] *= p.alpha * d[i] * y[i] * (p.sigmoid ? g[i] * (1.0f - g[i]) : 1.0f);
        store_row<T, V, N>(p.dgate.p, row * p.dgate.stride, p.hidden, w);
      }
      if (p.post) {
        const float m = block_sums(dot, 0.0f, sh, turn).x * p.inv_hidden;
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = r * fmaf(-y[i], m, f[i]);
      }
      store_row<T, V, N>(p.dy.p, row * p.dy.stride, p.hidden, f);
    }
  }
  if (p.partial) {
    float* at = p.partial + (int64_t)blockIdx.x * 2 * p.hidden;
    store_row<float, V, N>(at, 0, p.hidden, sum_post);
    store_row<float, V, N>(at, p.hidden, p.hidden, sum_pre);
  }
}

// Adds the blocks' partial rows: 32 columns per block, eight parts of the blocks, joined in order. What the columns of the first
// sum stand for: sum a d y r, times g for w_post and times w_post g' for a gate for all tokens.
constexpr int kNormSumParts = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kNormSumParts) block_norm_sum_kernel(const __grid_constant__ BlockNormParams p, int blocks) {
  start_after_previous_kernel();
  __shared__ float part[kNormSumParts][32];
  const int lane = threadIdx.x % 32, slice = threadIdx.x / 32, col = blockIdx.x * 32 + lane, which = blockIdx.y;
  float s = 0.0f;
  if (col < p.hidden)
    for (int b = slice; b < blocks; b += kNormSumParts) s += p.partial[((int64_t)b * 2 + which) * p.hidden + col];
  part[slice][lane] = s;
  __syncthreads();
  if (slice > 0 || col >= p.hidden) return;
  for (int i = 1; i < kNormSumParts; ++i) s += part[i][lane];
  if (which == 1) {
    if (p.dw_pre) p.dw_pre[col] = s;
    return;
  }
  float g = 1.0f, slope = 1.0f, w = 1.0f, v[1];
  if (p.gate_kind == 1) {
    load_values<1>(static_cast<const T*>(p.gate.p) + col, v);
    g = p.sigmoid ? sigmoid(v[0]) : v[0];
    slope = p.sigmoid ? g * (1.0f - g) : 1.0f;
  }
  if (p.w_post) {
    load_values<1>(static_cast<const T*>(p.w_post) + col, v);
    w = v[0];
  }
  if (p.dw_post) p.dw_post[col] = s * g;
  if (p.dgate_sum) p.dgate_sum[col] = s * (w * slope);
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

constexpr int64_t kMaxNormHidden = 16384;

int check_norm(const slidedp_block_norm_args* a) {
  const auto flag = [](int32_t x) { return x == 0 || x == 1; };
  if (!a || a->tokens < 0 || a->tokens > kMaxTokens || a->hidden < 1 || a->hidden > kMaxNormHidden ||
      (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) || !flag(a->has_y) || !flag(a->post_norm) || !flag(a->pre_norm) ||
      a->gate_kind < 0 || a->gate_kind > 2 || !flag(a->gate_sigmoid) || (!a->has_y && (a->post_norm || a->gate_kind || !a->pre_norm)) ||
      (!a->gate_kind && a->gate_sigmoid) || !fits_f32(a->residual_scale) || !(a->eps >= 0.0) || !fits_f32(a->eps) ||
      (a->eps > 0.0 && (float)a->eps == 0.0f))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

// Values per thread: 16, or 8 where that is as many registers; longer FP32 rows would need more threads than a block has.
int values_per_thread(const slidedp_block_norm_args* a) { return a->dtype == SLIDEDP_F32 && a->hidden <= 4096 ? 8 : 16; }
unsigned norm_threads(const slidedp_block_norm_args* a) {
  const int64_t n = (a->hidden + values_per_thread(a) - 1) / values_per_thread(a);
  return (unsigned)((n + 31) / 32 * 32);
}
// Blocks that stay: about 20 warps per SM, and no more than 16 blocks.
int64_t norm_blocks(const slidedp_block_norm_args* a) {
  const int64_t per_sm = 640 / norm_threads(a), most = 148 * (per_sm < 1 ? 1 : per_sm > 16 ? 16 : per_sm);
  return a->tokens < most ? a->tokens : most;
}

// Whether the outputs may be where they are: not two of them at one address, none at an input's with another stride.
bool places_ok(std::initializer_list<const slidedp_rows*> outs, std::initializer_list<const slidedp_rows*> ins, int64_t rows) {
  for (const slidedp_rows* const* o = outs.begin(); o != outs.end(); ++o) {
    if (!*o) continue;
    for (const slidedp_rows* const* q = outs.begin(); q != o; ++q)
      if (*q && (*q)->data == (*o)->data) return false;
    for (const slidedp_rows* in : ins)
      if (in && in->data == (*o)->data && rows > 1 && in->stride != (*o)->stride) return false;
  }
  return true;
}

bool weight_ok(const void* w, int elem) { return reinterpret_cast<uintptr_t>(w) % elem == 0; }

NormView norm_view(const slidedp_rows* r) { return r ? NormView{r->data, r->stride} : NormView{nullptr, 0}; }

BlockNormParams norm_params(const slidedp_block_norm_args* a) {
  BlockNormParams p = {};
  p.tokens = a->tokens;
  p.hidden = (int)a->hidden;
  p.has_y = a->has_y;
  p.post = a->post_norm;
  p.pre = a->pre_norm;
  p.gate_kind = a->gate_kind;
  p.sigmoid = a->gate_sigmoid;
  p.alpha = (float)a->residual_scale;
  p.eps = (float)a->eps;
  p.inv_hidden = (float)(1.0 / (double)a->hidden);
  return p;
}

// run(T, V, N, threads) as template arguments
template <typename F>
void pick_norm_kernel(const slidedp_block_norm_args* a, int v, F run) {
  typedef std::integral_constant<int, 8> N8;
  typedef std::integral_constant<int, 16> N16;
  const bool wide = norm_threads(a) > 512;
  const auto width = [&](auto type, auto n, auto full) {
    typedef std::integral_constant<int, 512> Up512;
    typedef std::integral_constant<int, 1024> Up1024;
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    const auto threads = [&](auto vector) { wide ? run(type, vector, n, Up1024()) : run(type, vector, n, Up512()); };
    if (v == full) return threads(full);
    if constexpr (sizeof(type) == 2)
      if (v == 2) return threads(Two());
    threads(One());
  };
  if (a->dtype == SLIDEDP_BF16) width(uint16_t(), N16(), std::integral_constant<int, 8>());
  else if (values_per_thread(a) == 8) width(float(), N8(), std::integral_constant<int, 4>());
  else width(float(), N16(), std::integral_constant<int, 4>());
}

}  // namespace

extern "C" {

int slidedp_block_norm(slidedp_ctx* ctx, const slidedp_block_norm_args* a, const slidedp_rows* x, const slidedp_rows* y, const void* w_post,
                       const slidedp_rows* gate, const void* w_pre, const slidedp_rows* x_out, const slidedp_rows* h_out, void* cuda_stream) {
  if (!ctx || check_norm(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens == 0) return SLIDEDP_OK;
  const int elem = elem_bytes(a->dtype);
  const slidedp_rows vector = {gate ? gate->data : nullptr, 0};
  if (!a->has_y) y = x_out = nullptr;
  if (!a->gate_kind) gate = nullptr;
  else if (a->gate_kind == 1) gate = &vector;
  if (!a->post_norm) w_post = nullptr;
  if (!a->pre_norm) w_pre = nullptr, h_out = nullptr;
  const int64_t T = a->tokens, H = a->hidden;
  if (!rows_ok(x, elem, T, H, false) || (a->has_y && (!rows_ok(y, elem, T, H, false) || !rows_ok(x_out, elem, T, H, true))) ||
      (a->gate_kind && !rows_ok(gate, elem, T, H, false)) || (a->pre_norm && !rows_ok(h_out, elem, T, H, true)) || !weight_ok(w_post, elem) ||
      !weight_ok(w_pre, elem) || !places_ok({x_out, h_out}, {x, y, a->gate_kind == 2 ? gate : nullptr}, T))
    return SLIDEDP_ERR_INVALID_ARG;
  BlockNormParams p = norm_params(a);
  p.x = norm_view(x);
  p.y = norm_view(y);
  p.gate = norm_view(gate);
  p.x_out = norm_view(x_out);
  p.h_out = norm_view(h_out);
  p.w_post = w_post;
  p.w_pre = w_pre;
  const slidedp_rows wp = {const_cast<void*>(w_post), 0}, wq = {const_cast<void*>(w_pre), 0};
  const int v = vector_width(H, elem, {{x, elem}, {y, elem}, {gate, elem}, {x_out, elem}, {h_out, elem}, {&wp, elem}, {&wq, elem}});
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  FAULT_POINT();
  pick_norm_kernel(a, v, [&](auto type, auto vec, auto n, auto threads) {
    typedef decltype(type) T_;
    const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)norm_blocks(a)), norm_threads(a), 0, 1, static_cast<cudaStream_t>(cuda_stream), p); };
    a->gate_kind == 2 ? run(block_norm_kernel<T_, vec, n, true, threads>) : run(block_norm_kernel<T_, vec, n, false, threads>);
  });
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_block_norm_workspace(const slidedp_block_norm_args* a) {
  if (check_norm(a) != SLIDEDP_OK) return 0;
  return (size_t)(norm_blocks(a) * 2 * a->hidden) * sizeof(float) + 16;
}

int slidedp_block_norm_backward(slidedp_ctx* ctx, const slidedp_block_norm_args* a, const slidedp_rows* x, const slidedp_rows* y,
                                const void* w_post, const slidedp_rows* gate, const void* w_pre, const slidedp_rows* dx_out,
                                const slidedp_rows* dh_out, const slidedp_rows* dx, const slidedp_rows* dy, const slidedp_rows* dgate,
                                float* dw_post, float* dw_pre, void* workspace, void* cuda_stream) {
  if (!ctx || check_norm(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  const int elem = elem_bytes(a->dtype);
  const slidedp_rows vector = {gate ? gate->data : nullptr, 0};
  float* dgate_sum = nullptr;
  if (dgate && !dgate->data) dgate = nullptr;
  if (dx_out && !dx_out->data) dx_out = nullptr;
  if (!a->has_y) y = dy = nullptr;
  if (!a->gate_kind) gate = dgate = nullptr;
  if (a->gate_kind == 1) {
    gate = &vector;
    if (dgate) dgate_sum = static_cast<float*>(dgate->data);
    dgate = nullptr;
  }
  if (!a->post_norm) w_post = nullptr, dw_post = nullptr;
  if (!a->pre_norm) w_pre = nullptr, dw_pre = nullptr, dh_out = nullptr;
  const bool sums = dw_post || dw_pre || dgate_sum;
  const int64_t T = a->tokens, H = a->hidden;
  if ((T > 0 && (!rows_ok(x, elem, T, H, false) || (a->has_y && (!rows_ok(y, elem, T, H, false) || !rows_ok(dy, elem, T, H, true))) ||
                 (gate && !rows_ok(gate, elem, T, H, false)) || (a->pre_norm && !rows_ok(dh_out, elem, T, H, false)) ||
                 (dx_out && !rows_ok(dx_out, elem, T, H, false)) || !rows_ok(dx, elem, T, H, true) || (dgate && !rows_ok(dgate, elem, T, H, true)) ||
                 !places_ok({dx, dy, dgate}, {x, y, a->gate_kind == 2 ? gate : nullptr, dx_out, dh_out}, T))) ||
      !weight_ok(w_post, elem) || !weight_ok(w_pre, elem) || !weight_ok(dw_post, 4) || !weight_ok(dw_pre, 4) || !weight_ok(dgate_sum, 4) ||
      (sums && !workspace))
    return SLIDEDP_ERR_INVALID_ARG;
  if (sums && !aligned16(workspace)) return SLIDEDP_ERR_MISALIGNED;
  if (T == 0 && !sums) return SLIDEDP_OK;
  BlockNormParams p = norm_params(a);
  p.x = norm_view(x);
  p.y = norm_view(y);
  p.gate = norm_view(gate);
  p.dx_out = norm_view(dx_out);
  p.dh = norm_view(dh_out);
  p.dx = norm_view(dx);
  p.dy = norm_view(dy);
  p.dgate = norm_view(dgate);
  p.w_post = w_post;
  p.w_pre = w_pre;
  p.dw_post = dw_post;
  p.dw_pre = dw_pre;
  p.dgate_sum = dgate_sum;
  p.partial = sums ? static_cast<float*>(workspace) : nullptr;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned blocks = (unsigned)norm_blocks(a);
  if (T > 0) {
    const slidedp_rows wp = {const_cast<void*>(w_post), 0}, wq = {const_cast<void*>(w_pre), 0};
    const int v = vector_width(H, elem, {{x, elem}, {y, elem}, {gate, elem}, {dx_out, elem}, {dh_out, elem}, {dx, elem}, {dy, elem}, {dgate, elem},
                                         {&wp, elem}, {&wq, elem}});
    FAULT_POINT();
    pick_norm_kernel(a, v, [&](auto type, auto vec, auto n, auto threads) {
      typedef decltype(type) T_;
      const auto run = [&](auto kernel) { launch_after(kernel, dim3(blocks), norm_threads(a), 0, 1, st, p); };
      a->gate_kind == 2 ? run(block_norm_backward_kernel<T_, vec, n, true, threads>) : run(block_norm_backward_kernel<T_, vec, n, false, threads>);
    });
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  if (sums) {
    FAULT_POINT();
    const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)((H + 31) / 32), 2), 32 * kNormSumParts, 0, 1, st, p, (int)blocks); };
    elem == 4 ? run(block_norm_sum_kernel<float>) : run(block_norm_sum_kernel<uint16_t>);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  return SLIDEDP_OK;
}

}  // extern "C"
