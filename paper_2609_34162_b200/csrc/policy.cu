// libslidedp: the clipped policy loss with a second term towards a reference model. See include/slidedp_ops.h for the contract.
//
// With c = 1 / temperature, m = max z, s = sum exp(c (z - m)): logp = c (z_y - m) - log s, rho = exp(logp - old), k = ref - logp,
//   loss = -min(rho A, clamp(rho, 1 - lo, 1 + hi) A) + w (e^k - k - 1),   l = -A rho [inside] + w (1 - e^k)
//   dz = g c l (onehot - p)
// Bound: HBM. The logits are all that is large.
#include "ops_internal.h"
#include "logit_rows.cuh"

namespace slidedp {

constexpr int kPolicyThreads = 256;
constexpr int kPolicyWarps = kPolicyThreads / 32;

struct PolicyParams {
  const void* z;
  void* dz;
  const int32_t* labels;
  const float *old_logp, *ref_logp, *advantage, *row_grad;
  const float* saved_logp;
  float *loss, *logp;
  int64_t rows, vocab, z_stride, dz_stride;
  float inv_tau;
  double low, high, kl, inv_tau64;
};

// What a row's log-probability makes of it: its loss, and the factor f of dz = f (onehot - p). In FP64: the ratio is compared
// with the edges of the clipped range, and one thread per row does it.
struct RowTerms {
  double loss;
  float f;
};
__device__ __forceinline__ RowTerms row_terms(const PolicyParams& p, int64_t r, double logp) {
  double loss = 0.0, slope = 0.0;
  const double a = p.advantage ? (double)p.advantage[r] : 0.0;
  if (a != 0.0) {
    const double ratio = p.old_logp ? exp(logp - (double)p.old_logp[r]) : 1.0;
    const bool inside = a > 0.0 ? ratio <= p.high : ratio >= p.low;
    const double clipped = ratio > p.high ? p.high : ratio < p.low ? p.low : ratio;
    loss = -(inside || ratio != ratio || a != a ? ratio : clipped) * a;
    if (inside || ratio != ratio || a != a) slope = -a * ratio;
  }
  if (p.ref_logp) {
    const double k = (double)p.ref_logp[r] - logp, e = exp(k);
    loss += p.kl * (e - k - 1.0);
    slope += p.kl * (1.0 - e);
  }
  const double g = p.row_grad ? (double)p.row_grad[r] : 1.0;
  return RowTerms{loss, g == 0.0 ? 0.0f : (float)(g * slope * p.inv_tau64)};
}

__device__ __forceinline__ int row_label(const PolicyParams& p, int64_t r) {
  const int y = p.labels[r];
  return y >= 0 && y < p.vocab ? y : -1;
}

struct PolicyShared {
  SoftSum warp[kPolicyWarps];
  double loss, logp;
  float f;
};

// Gradient of a chunk of a row: f (onehot - p) with p = exp2(k (z - base) + offset); nothing outside the row is written.
struct PolicyGrad {
  float k, base, offset, f, at_label;
  int label;
};
template <typename T>
__device__ __forceinline__ void policy_chunk(const Row<T>& row, T* dz, int64_t c, uint4 a, const PolicyGrad& g) {
  constexpr int P = Logit<T>::kPer;
  uint64_t v[P / 2];
  float out[P];
  Logit<T>::unpack(a, v);
  const uint64_t minus = pair(-g.base, -g.base);
#pragma unroll
  for (int e = 0; e < P / 2; ++e) {
    float lo, hi;
    split(fma2(add2(v[e], minus), pair(g.k, g.k), pair(g.offset, g.offset)), &lo, &hi);
    out[2 * e] = -g.f * exp2_approx(lo);
    out[2 * e + 1] = -g.f * exp2_approx(hi);
  }
  const int64_t first = row.first(c);
  if (g.label >= first && g.label < first + P) out[g.label - first] = g.at_label;
  const bool same_grid = ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(row.z)) & 15u) == 0;
  if (same_grid && first >= 0 && first + P <= row.vocab) {
    st_stream(dz + first, Logit<T>::pack(out));
  } else {
#pragma unroll
    for (int e = 0; e < P; ++e)
      if (first + e >= 0 && first + e < row.vocab) Logit<T>::store(dz + first + e, out[e]);
  }
}

// A block per row. kForward: log-probability and loss; kGradient: the gradient, from the saved log-probability without kForward.
template <typename T, bool kForward, bool kGradient>
__global__ void __launch_bounds__(kPolicyThreads) policy_row_kernel(const __grid_constant__ PolicyParams p) {
  start_after_previous_kernel();
  __shared__ PolicyShared sh;
  const int64_t r = blockIdx.x;
  const T* z = static_cast<const T*>(p.z) + r * p.z_stride;
  T* dz = static_cast<T*>(p.dz) + r * p.dz_stride;
  const Row<T> row(z, p.vocab);
  const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
  const int label = row_label(p, r);
  const float at = label >= 0 ? Logit<T>::load(z + label) : 0.0f;
  PolicyGrad g;
  g.k = p.inv_tau * kLog2e;
  g.label = label;
  g.f = 0.0f;
  if (kForward) {
    if (label < 0) {
      if (threadIdx.x == 0) {
        if (p.loss) p.loss[r] = 0.0f;
        p.logp[r] = 0.0f;
      }
    } else {
      SoftSum mine = {-INFINITY, 0.0f, 0.0f};
      for (int64_t c = threadIdx.x; c < chunks; c += kPolicyThreads) {
        const uint4 a = row.load(c);
        accumulate<T, false, 1>(mine, &a, g.k, g.k);
      }
      mine = join_lanes<32, false>(mine, g.k, g.k);
      if (threadIdx.x % 32 == 0) sh.warp[threadIdx.x / 32] = mine;
      __syncthreads();
      mine = join_lanes<kPolicyWarps, false>(sh.warp[threadIdx.x % kPolicyWarps], g.k, g.k);
      g.base = finite_shift(mine.m);
      if (threadIdx.x == 0) {
        const double logp = ((double)at - (double)g.base) * p.inv_tau64 - log((double)mine.s0);
        const RowTerms t = row_terms(p, r, logp);
        if (p.loss) p.loss[r] = (float)t.loss;
        p.logp[r] = (float)logp;
        sh.logp = logp;
        sh.f = t.f;
      }
      g.offset = -log2f(mine.s0);
    }
  } else if (label >= 0) {
    g.base = at;
    if (threadIdx.x == 0) {
      const double logp = p.saved_logp[r];
      sh.logp = logp;
      sh.f = row_terms(p, r, logp).f;
    }
    g.offset = p.saved_logp[r] * kLog2e;
  }
  if (kGradient) {
    __syncthreads();
    if (label >= 0) {
      g.f = sh.f;
      g.at_label = g.f * -(float)expm1(sh.logp);
    }
    if (g.f == 0.0f) {
      for (int64_t c = threadIdx.x; c < chunks; c += kPolicyThreads) {
        g.label = -1;
        g.k = g.base = 0.0f;
        g.offset = -INFINITY;
        policy_chunk<T>(row, dz, c, make_uint4(0, 0, 0, 0), g);
      }
    } else {
      for (int64_t c = threadIdx.x; c < chunks; c += kPolicyThreads) policy_chunk<T>(row, dz, c, row.load(c), g);
    }
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

enum PolicyMode { kPolicyForward, kPolicyBackward, kPolicyStep };

int check_policy(const slidedp_policy_args* a) {
  if (!a || a->rows < 0 || a->rows > kMaxTokens || a->vocab < 1 || a->vocab > (1ll << 30) || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) ||
      a->logits_stride < 0 || !positive_f32(a->temperature) || !positive_f32(1.0 / a->temperature) || !fits_f32(1.4426950408889634 / a->temperature) ||
      !(a->clip_low >= 0.0) || !(a->clip_high >= 0.0) || !fits_f32(a->clip_low) || !fits_f32(a->clip_high) || !fits_f32(a->kl_weight))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

int run_policy(slidedp_ctx* ctx, const slidedp_policy_args* a, PolicyMode mode, const void* logits, const int32_t* labels, const float* old_logp,
               const float* ref_logp, const float* advantage, const float* saved, const float* row_grad, float* loss, float* logp, void* dz,
               cudaStream_t st) {
  if (!ctx || check_policy(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->rows == 0) return SLIDEDP_OK;
  const int64_t elem = a->dtype == SLIDEDP_F32 ? 4 : 2;
  const auto odd = [](const void* q, int64_t align) { return reinterpret_cast<uintptr_t>(q) % (uintptr_t)align != 0; };
  if (!logits || odd(logits, elem) || !labels || odd(labels, 4) || odd(old_logp, 4) || odd(ref_logp, 4) || odd(advantage, 4) || odd(row_grad, 4))
    return SLIDEDP_ERR_INVALID_ARG;
  if (mode == kPolicyBackward ? !saved || odd(saved, 4) : !logp || odd(logp, 4) || odd(loss, 4) || (!loss && (old_logp || ref_logp || advantage)))
    return SLIDEDP_ERR_INVALID_ARG;
  if (mode != kPolicyForward && (!dz || odd(dz, elem) || (a->rows > 1 && (a->d_logits_stride < a->vocab || (dz == logits && a->d_logits_stride != a->logits_stride)))))
    return SLIDEDP_ERR_INVALID_ARG;
  PolicyParams p = {};
  p.z = logits;
  p.dz = dz;
  p.labels = labels;
  p.old_logp = old_logp;
  p.ref_logp = a->kl_weight != 0.0 ? ref_logp : nullptr;
  p.advantage = advantage;
  p.row_grad = row_grad;
  p.saved_logp = saved;
  p.loss = loss;
  p.logp = logp;
  p.rows = a->rows;
  p.vocab = a->vocab;
  p.z_stride = a->logits_stride;
  p.dz_stride = a->d_logits_stride;
  p.inv_tau = (float)(1.0 / a->temperature);
  p.inv_tau64 = 1.0 / a->temperature;
  p.low = 1.0 - a->clip_low;
  p.high = 1.0 + a->clip_high;
  p.kl = a->kl_weight;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  FAULT_POINT();
  const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)a->rows), kPolicyThreads, 0, 1, st, p); };
  const bool f32 = a->dtype == SLIDEDP_F32;
  if (mode == kPolicyForward) f32 ? run(policy_row_kernel<float, true, false>) : run(policy_row_kernel<uint16_t, true, false>);
  else if (mode == kPolicyBackward) f32 ? run(policy_row_kernel<float, false, true>) : run(policy_row_kernel<uint16_t, false, true>);
  else f32 ? run(policy_row_kernel<float, true, true>) : run(policy_row_kernel<uint16_t, true, true>);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

}  // namespace

extern "C" {

int slidedp_policy_loss(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits, const int32_t* labels, const float* old_logp,
                        const float* ref_logp, const float* advantage, float* loss, float* logp, void* cuda_stream) {
  return run_policy(ctx, args, kPolicyForward, logits, labels, old_logp, ref_logp, advantage, nullptr, nullptr, loss, logp, nullptr,
                    static_cast<cudaStream_t>(cuda_stream));
}

int slidedp_policy_loss_backward(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits, const int32_t* labels,
                                 const float* old_logp, const float* ref_logp, const float* advantage, const float* logp, const float* row_grad,
                                 void* d_logits, void* cuda_stream) {
  return run_policy(ctx, args, kPolicyBackward, logits, labels, old_logp, ref_logp, advantage, logp, row_grad, nullptr, nullptr, d_logits,
                    static_cast<cudaStream_t>(cuda_stream));
}

int slidedp_policy_step(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits, const int32_t* labels, const float* old_logp,
                        const float* ref_logp, const float* advantage, const float* row_grad, float* loss, float* logp, void* d_logits,
                        void* cuda_stream) {
  return run_policy(ctx, args, kPolicyStep, logits, labels, old_logp, ref_logp, advantage, nullptr, row_grad, loss, logp, d_logits,
                    static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
