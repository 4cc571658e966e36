// libslidedp: attention over packed documents: argument checks, dispatch, and the kernels for the views
// that the tensor-core kernels do not take. See include/slidedp_ops.h for the contract.
#include "attention.h"
#include "device_utils.cuh"

namespace slidedp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowTile = 128;            // the row statistics are padded to this many rows per head
constexpr int kGeneralThreads = 128;
constexpr int kLanes = 32;
constexpr int kMaxPer = host::kMaxHeadDim / kLanes;

// ---- kernels without tensor cores -------------------------------------------------------------------
// One warp per row (a query, or a key of the backward pass), lanes over the head's values, one partner
// row at a time with a running maximum: any head_dim and stride, no shared memory. They serve head_dim
// above 128 or not a multiple of 8 and views that are not 16-byte aligned, which TMA cannot address.

__device__ __forceinline__ float load_bf16(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

__device__ __forceinline__ void load_row(const AttnView& v, int t, int h, int n, float* x) {
  const uint16_t* row = v.p + t * v.t + h * v.h;
  const int lane = threadIdx.x % kLanes;
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) x[i] = lane + i * kLanes < n ? load_bf16(row + lane + i * kLanes) : 0.0f;
}
__device__ __forceinline__ void store_row(const AttnView& v, int t, int h, int n, const float* x) {
  uint16_t* row = v.p + t * v.t + h * v.h;
  const int lane = threadIdx.x % kLanes;
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i)
    if (lane + i * kLanes < n) row[lane + i * kLanes] = (uint16_t)f32_to_bf16_bits(x[i]);
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

__global__ void __launch_bounds__(kGeneralThreads) attention_forward_general_kernel(const __grid_constant__ AttnParams p) {
  const int i = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes, h = blockIdx.y;
  if (i >= p.tokens) return;
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], o[kMaxPer] = {};
  load_row(p.q, i, h, p.head_dim, q);
  int lo, hi;
  p.mask.keys_of(i, &lo, &hi);
  float m = -INFINITY, l = 0.0f;
  for (int j = lo; j < hi; ++j) {
    float x[kMaxPer], g;
    load_row(p.k, j, hk, p.head_dim, x);
    const float s = score(p, dot(q, x), slope, i - j, &g);
    load_row(p.v, j, hk, p.head_dim, x);
    const float top = fmaxf(m, s), keep = exp2f(m - top), e = exp2f(s - top);
    m = top;
    l = l * keep + e;
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) o[d] = fmaf(e, x[d], o[d] * keep);
  }
  const float inv = lo < hi ? 1.0f / l : 0.0f;
#pragma unroll
  for (int d = 0; d < kMaxPer; ++d) o[d] *= inv;
  store_row(p.o, i, h, p.head_dim, o);
  if (threadIdx.x % kLanes == 0) p.lse[(int64_t)h * p.tokens + i] = lo < hi ? (m + log2f(l)) / kLog2e : -INFINITY;
}

__global__ void __launch_bounds__(kGeneralThreads) attention_dq_general_kernel(const __grid_constant__ AttnParams p) {
  const int i = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes, h = blockIdx.y;
  if (i >= p.tokens) return;
  const int hk = h / p.group;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  float q[kMaxPer], go[kMaxPer], dq[kMaxPer] = {};
  load_row(p.q, i, h, p.head_dim, q);
  load_row(p.dout, i, h, p.head_dim, go);
  const float2 row = p.rows[h * p.pitch + i];
  int lo, hi;
  p.mask.keys_of(i, &lo, &hi);
  for (int j = lo; j < hi; ++j) {
    float k[kMaxPer], v[kMaxPer], g;
    load_row(p.k, j, hk, p.head_dim, k);
    load_row(p.v, j, hk, p.head_dim, v);
    const float pr = exp2f(score(p, dot(q, k), slope, i - j, &g) - row.x);
    const float ds = pr * (dot(go, v) - row.y) * g * p.scale;
#pragma unroll
    for (int d = 0; d < kMaxPer; ++d) dq[d] = fmaf(ds, k[d], dq[d]);
  }
  store_row(p.dq, i, h, p.head_dim, dq);
}

__global__ void __launch_bounds__(kGeneralThreads) attention_dkv_general_kernel(const __grid_constant__ AttnParams p) {
  const int j = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes, hk = blockIdx.y;
  if (j >= p.tokens) return;
  float k[kMaxPer], v[kMaxPer], dk[kMaxPer] = {}, dv[kMaxPer] = {};
  load_row(p.k, j, hk, p.head_dim, k);
  load_row(p.v, j, hk, p.head_dim, v);
  int lo, hi;
  p.mask.queries_of(j, &lo, &hi);
  for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    for (int i = lo; i < hi; ++i) {
      float q[kMaxPer], go[kMaxPer], g;
      load_row(p.q, i, h, p.head_dim, q);
      load_row(p.dout, i, h, p.head_dim, go);
      const float2 row = p.rows[h * p.pitch + i];
      const float pr = exp2f(score(p, dot(q, k), slope, i - j, &g) - row.x);
      const float ds = pr * (dot(go, v) - row.y) * g * p.scale;
#pragma unroll
      for (int d = 0; d < kMaxPer; ++d) {
        dv[d] = fmaf(pr, go[d], dv[d]);
        dk[d] = fmaf(ds, q[d], dk[d]);
      }
    }
  }
  store_row(p.dk, j, hk, p.head_dim, dk);
  store_row(p.dv, j, hk, p.head_dim, dv);
}

// rows[h][i] = (lse log2 e, sum_d dout out), zeros for the rows of the padding: one warp per row.
// Bound: HBM, one read of out and dout.
__global__ void __launch_bounds__(kGeneralThreads) attention_rows_kernel(const __grid_constant__ AttnParams p) {
  const int64_t i = (int64_t)blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes;
  const int h = blockIdx.y;
  if (i >= p.pitch) return;
  float s = 0.0f, l = 0.0f;
  if (i < p.tokens) {
    float a[kMaxPer], b[kMaxPer];
    load_row(p.o, (int)i, h, p.head_dim, a);
    load_row(p.dout, (int)i, h, p.head_dim, b);
    s = dot(a, b);
    l = p.lse[(int64_t)h * p.tokens + i] * kLog2e;
  }
  if (threadIdx.x % kLanes == 0) p.rows[h * p.pitch + i] = make_float2(l, s);
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

int64_t row_pitch(int64_t tokens) { return (tokens + kRowTile - 1) / kRowTile * kRowTile; }

int check_attn(const slidedp_attn_args* a) {
  if (!a || a->tokens < 0 || a->tokens > kMaxTokens || a->heads_q < 1 || a->heads_kv < 1 || a->heads_q > 65535 ||
      a->heads_q % a->heads_kv != 0 || a->head_dim < 1 || a->head_dim > kMaxHeadDim || (a->causal != 0 && a->causal != 1) ||
      a->docs < 0 || a->docs > kMaxTokens || (!a->cu_docs && (a->docs != 1 || a->prefix)))
    return SLIDEDP_ERR_INVALID_ARG;
  if (!is_finite(a->scale) || !(a->softcap >= 0.0) || !is_finite(a->softcap)) return SLIDEDP_ERR_INVALID_ARG;
  const uintptr_t small = reinterpret_cast<uintptr_t>(a->cu_docs) | reinterpret_cast<uintptr_t>(a->prefix) |
                          reinterpret_cast<uintptr_t>(a->slopes);
  return small % 4 == 0 ? SLIDEDP_OK : SLIDEDP_ERR_INVALID_ARG;
}

AttnView view(const slidedp_heads* v) {
  return AttnView{static_cast<uint16_t*>(v->data), v->stride_token, v->stride_head};
}

AttnParams make_params(const slidedp_attn_args* a, const slidedp_heads* q, const slidedp_heads* k,
                       const slidedp_heads* v, const slidedp_heads* out, const float* lse) {
  AttnParams p = {};
  p.q = view(q);
  p.k = view(k);
  p.v = view(v);
  p.o = view(out);
  p.lse = const_cast<float*>(lse);
  p.pitch = row_pitch(a->tokens);
  p.slopes = a->slopes;
  p.mask = DocMask{a->cu_docs, a->prefix, a->docs, (int)a->tokens, a->causal};
  p.tokens = (int)a->tokens;
  p.heads_q = a->heads_q;
  p.heads_kv = a->heads_kv;
  p.group = a->heads_q / a->heads_kv;
  p.head_dim = a->head_dim;
  p.scale = (float)a->scale;
  p.softcap = (float)a->softcap;
  p.scale_log2 = (float)(a->scale * 1.4426950408889634);
  return p;
}

unsigned general_blocks(int64_t rows) {
  return (unsigned)((rows + kGeneralThreads / kLanes - 1) / (kGeneralThreads / kLanes));
}

}  // namespace

extern "C" {

int slidedp_attention(slidedp_ctx* ctx, const slidedp_attn_args* a, const slidedp_heads* q, const slidedp_heads* k,
                      const slidedp_heads* v, const slidedp_heads* out, float* lse, void* cuda_stream) {
  if (!ctx || check_attn(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens == 0) return SLIDEDP_OK;
  if (!heads_ok(q, 2) || !heads_ok(k, 2) || !heads_ok(v, 2) || !heads_ok(out, 2) || !lse ||
      reinterpret_cast<uintptr_t>(lse) % 4 != 0)
    return SLIDEDP_ERR_INVALID_ARG;
  const AttnParams p = make_params(a, q, k, v, out, lse);
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  FAULT_POINT();
  attention_forward_general_kernel<<<dim3(general_blocks(p.tokens), p.heads_q), kGeneralThreads, 0, st>>>(p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_attention_workspace(const slidedp_attn_args* a) {
  if (check_attn(a) != SLIDEDP_OK) return 0;
  return (size_t)a->heads_q * row_pitch(a->tokens) * sizeof(float2);
}

int slidedp_attention_backward(slidedp_ctx* ctx, const slidedp_attn_args* a, const slidedp_heads* q,
                               const slidedp_heads* k, const slidedp_heads* v, const slidedp_heads* out,
                               const float* lse, const slidedp_heads* d_out, const slidedp_heads* dq,
                               const slidedp_heads* dk, const slidedp_heads* dv, void* workspace, void* cuda_stream) {
  if (!ctx || check_attn(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens == 0) return SLIDEDP_OK;
  if (!heads_ok(q, 2) || !heads_ok(k, 2) || !heads_ok(v, 2) || !heads_ok(out, 2) || !heads_ok(d_out, 2) ||
      !heads_ok(dq, 2) || !heads_ok(dk, 2) || !heads_ok(dv, 2) || !lse || reinterpret_cast<uintptr_t>(lse) % 4 != 0 ||
      !workspace)
    return SLIDEDP_ERR_INVALID_ARG;
  if (!aligned16(workspace)) return SLIDEDP_ERR_MISALIGNED;
  AttnParams p = make_params(a, q, k, v, out, lse);
  p.dout = view(d_out);
  p.dq = view(dq);
  p.dk = view(dk);
  p.dv = view(dv);
  p.rows = static_cast<float2*>(workspace);
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  FAULT_POINT();
  attention_rows_kernel<<<dim3(general_blocks(p.pitch), p.heads_q), kGeneralThreads, 0, st>>>(p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  FAULT_POINT();
  attention_dq_general_kernel<<<dim3(general_blocks(p.tokens), p.heads_q), kGeneralThreads, 0, st>>>(p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  FAULT_POINT();
  attention_dkv_general_kernel<<<dim3(general_blocks(p.tokens), p.heads_kv), kGeneralThreads, 0, st>>>(p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

}  // extern "C"
