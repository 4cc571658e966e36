// libslidedp: attention over packed documents: argument checks, dispatch, and the kernels for the views
// that the tensor-core kernels do not take. See include/slidedp_ops.h for the contract.
#include "attention_rows.cuh"

namespace slidedp {

constexpr int kRowTile = 128;            // the row statistics are padded to this many rows per head
constexpr int kGeneralThreads = 128;

// ---- kernels without tensor cores -------------------------------------------------------------------
// One warp per row. They serve head_dim above 128 or not a multiple of 8 and views that are not 16-byte
// aligned, which TMA cannot address.

__global__ void __launch_bounds__(kGeneralThreads) attention_forward_general_kernel(const __grid_constant__ AttnParams p) {
  start_after_previous_kernel();
  const int i = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes;
  if (i < p.tokens) attention_out_row<false>(p, i, blockIdx.y, true);
}
__global__ void __launch_bounds__(kGeneralThreads) attention_dq_general_kernel(const __grid_constant__ AttnParams p) {
  start_after_previous_kernel();
  const int i = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes;
  if (i < p.tokens) attention_dq_row<false>(p, i, blockIdx.y, 0, p.head_dim);
}
__global__ void __launch_bounds__(kGeneralThreads) attention_dkv_general_kernel(const __grid_constant__ AttnParams p) {
  start_after_previous_kernel();
  const int j = blockIdx.x * (kGeneralThreads / kLanes) + threadIdx.x / kLanes;
  if (j < p.tokens) attention_dkv_row<false>(p, j, blockIdx.y, true, true, 0, p.head_dim);
}

// row_lse[h][i] = lse log2 e, row_delta[h][i] = sum_d dout out, zeros for the rows of the padding: one warp per row.
// Bound: HBM, one read of out and dout.
__global__ void __launch_bounds__(kGeneralThreads) attention_rows_kernel(const __grid_constant__ AttnParams p) {
  start_after_previous_kernel();
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
  if (threadIdx.x % kLanes == 0) {
    p.row_lse[h * p.pitch + i] = l;
    p.row_delta[h * p.pitch + i] = s;
  }
}

// The same for views with 16-byte aligned rows of a multiple of 8 values: L lanes of 16 bytes per row, four tokens of a
// head per group of lanes. 8192 tokens, 32 heads of 128: 28 us against 48 of the kernel above.
template <int L>
__global__ void __launch_bounds__(kGeneralThreads) attention_rows_wide_kernel(const __grid_constant__ AttnParams p) {
  start_after_previous_kernel();
  constexpr int kGroups = kGeneralThreads / L, U = 4;
  const int group = threadIdx.x / L, d = threadIdx.x % L * 8, h = blockIdx.y;
  const int64_t first = (int64_t)blockIdx.x * kGroups * U + group;
  const bool on = d < p.head_dim;
  uint4 o[U], g[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = first + u * kGroups;
    o[u] = g[u] = make_uint4(0, 0, 0, 0);
    if (on && i < p.tokens) {
      o[u] = *reinterpret_cast<const uint4*>(p.o.p + i * p.o.t + h * p.o.h + d);
      g[u] = *reinterpret_cast<const uint4*>(p.dout.p + i * p.dout.t + h * p.dout.h + d);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = first + u * kGroups;
    const uint32_t a[4] = {o[u].x, o[u].y, o[u].z, o[u].w}, b[4] = {g[u].x, g[u].y, g[u].z, g[u].w};
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) s = fmaf(bf16_hi(a[k]), bf16_hi(b[k]), fmaf(bf16_lo(a[k]), bf16_lo(b[k]), s));
#pragma unroll
    for (int k = L / 2; k > 0; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
    if (threadIdx.x % L == 0 && i < p.pitch) {
      p.row_lse[h * p.pitch + i] = i < p.tokens ? p.lse[(int64_t)h * p.tokens + i] * kLog2e : 0.0f;
      p.row_delta[h * p.pitch + i] = s;
    }
  }
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
  if (!fits_f32(a->scale * 1.4426950408889634) || !(a->softcap == 0.0 || (positive_f32(a->softcap) && fits_f32(a->softcap * 1.4426950408889634) &&
                                                                           fits_f32(a->scale / a->softcap))))
    return SLIDEDP_ERR_INVALID_ARG;
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

bool tensor_core_dim(int head_dim) { return head_dim % 8 == 0 && head_dim <= 128; }

// Whether TMA can address a view: 16-byte base and strides, none of them zero where it is used.
bool tma_view(const slidedp_heads* v, int64_t tokens, int heads) {
  return heads_aligned(v, 2, 16, tokens, heads) && (tokens <= 1 || v->stride_token > 0) &&
         (heads <= 1 || v->stride_head > 0) && v->stride_token < (1ll << 38) && v->stride_head < (1ll << 38);
}

// Whether two views start at the same place: outputs that lie over what other blocks still read are refused where that is
// plain to see.
bool same_start(const slidedp_heads* a, const slidedp_heads* b) { return a->data == b->data; }

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
      reinterpret_cast<uintptr_t>(lse) % 4 != 0 || same_start(out, q) || same_start(out, k) || same_start(out, v))
    return SLIDEDP_ERR_INVALID_ARG;
  AttnParams p = make_params(a, q, k, v, out, lse);
  p.error = ctx->kernel_error;
  p.polls = ctx->wait_polls;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (tensor_core_dim(p.head_dim) && tma_view(q, p.tokens, p.heads_q) && tma_view(k, p.tokens, p.heads_kv) &&
      tma_view(v, p.tokens, p.heads_kv) && tma_view(out, p.tokens, p.heads_q))
    return attention_forward_mma(ctx, p, st);
  FAULT_POINT();
  launch_after(attention_forward_general_kernel, dim3(general_blocks(p.tokens), p.heads_q), kGeneralThreads, 0, 1, st, p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_attention_workspace(const slidedp_attn_args* a) {
  if (check_attn(a) != SLIDEDP_OK) return 0;
  return (size_t)a->heads_q * row_pitch(a->tokens) * 2 * sizeof(float);
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
  const slidedp_heads *ins[] = {q, k, v, d_out}, *outs[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const slidedp_heads* in : ins)
      if (same_start(outs[i], in)) return SLIDEDP_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (same_start(outs[i], outs[j])) return SLIDEDP_ERR_INVALID_ARG;
  }
  AttnParams p = make_params(a, q, k, v, out, lse);
  p.dout = view(d_out);
  p.dq = view(dq);
  p.dk = view(dk);
  p.dv = view(dv);
  p.error = ctx->kernel_error;
  p.polls = ctx->wait_polls;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  p.row_lse = static_cast<float*>(workspace);
  p.row_delta = p.row_lse + a->heads_q * p.pitch;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  FAULT_POINT();
  if (p.head_dim % 8 == 0 && heads_aligned(out, 2, 16, p.tokens, p.heads_q) && heads_aligned(d_out, 2, 16, p.tokens, p.heads_q)) {
    const int lanes = p.head_dim <= 64 ? 8 : p.head_dim <= 128 ? 16 : 32;
    const int64_t per_block = (int64_t)kGeneralThreads / lanes * 4;
    const dim3 grid((unsigned)((p.pitch + per_block - 1) / per_block), p.heads_q);
    if (lanes == 8) launch_after(attention_rows_wide_kernel<8>, grid, kGeneralThreads, 0, 1, st, p);
    else if (lanes == 16) launch_after(attention_rows_wide_kernel<16>, grid, kGeneralThreads, 0, 1, st, p);
    else launch_after(attention_rows_wide_kernel<32>, grid, kGeneralThreads, 0, 1, st, p);
  } else {
    launch_after(attention_rows_kernel, dim3(general_blocks(p.pitch), p.heads_q), kGeneralThreads, 0, 1, st, p);
  }
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  if (tensor_core_dim(p.head_dim) && tma_view(q, p.tokens, p.heads_q) && tma_view(k, p.tokens, p.heads_kv) &&
      tma_view(v, p.tokens, p.heads_kv) && tma_view(d_out, p.tokens, p.heads_q) && tma_view(dq, p.tokens, p.heads_q) &&
      tma_view(dk, p.tokens, p.heads_kv) && tma_view(dv, p.tokens, p.heads_kv))
    return attention_backward_mma(ctx, p, st);
  FAULT_POINT();
  launch_after(attention_dq_general_kernel, dim3(general_blocks(p.tokens), p.heads_q), kGeneralThreads, 0, 1, st, p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  FAULT_POINT();
  launch_after(attention_dkv_general_kernel, dim3(general_blocks(p.tokens), p.heads_kv), kGeneralThreads, 0, 1, st, p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

}  // extern "C"
