// libslidedp: distillation from a teacher's top logits with hard labels beside it: loss, gradient, and
// both in one pass. See include/slidedp_ops.h for the contract.
//
// With c = 1 / temperature, m = max z, s = sum exp(c (z - m)):  lse = c m + log s,  log p = c z - lse and
//   dz = g (w_t tau (p - q) + w_l (p1 - onehot)),   p1 the softmax at temperature 1.
// Bound: HBM. The logits are all that is large: forward reads them once, backward reads them and writes
// the gradient, and the step (both) reads and writes once because a row stays on chip between its two
// uses: a cluster of up to eight blocks holds it in shared memory (a row of 131072 BF16 logits is
// 256 KB, more than one SM has) and exchanges its maximum and sums through distributed shared memory.
#include <cooperative_groups.h>

#include "device_utils.cuh"
#include "ops_internal.h"

namespace cg = cooperative_groups;

namespace slidedp {

constexpr int kMaxEntries = 512;        // teacher entries per row
constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kDistillMaxCluster = 8;
constexpr int kDistillUnroll = 8;       // 16-byte loads in flight per thread
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

enum DistillMode { kForward = 0, kBackward = 1, kStep = 2 };

struct DistillParams {
  const void* z;
  void* dz;
  const int32_t* ids;
  const float* t;
  const int32_t* labels;   // null when the label term is off
  const float* row_grad;
  float* loss;
  float* lse;              // [2][rows]
  int64_t rows, vocab, z_stride, dz_stride;
  int entries;
  int64_t chunks_per_block;  // 16-byte chunks of a row that one block of its cluster takes
  float inv_tau, tau, w_teacher, w_label;
};

template <typename T> struct Logit;
template <> struct Logit<uint16_t> {
  static constexpr int kPer = 8;   // values per 16 bytes
  static __device__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ void store(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
  static __device__ void unpack(uint4 a, float* v) {
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
    v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
  }
  static __device__ uint32_t two(float lo, float hi) {   // one cvt for both: hi in the upper half
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7]));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
};
template <> struct Logit<float> {
  static constexpr int kPer = 4;
  static __device__ float load(const float* p) { return *p; }
  static __device__ void store(float* p, float v) { *p = v; }
  static __device__ void unpack(uint4 a, float* v) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
};

__device__ __forceinline__ float exp2_fast(float x) {   // 2 ulp, and 0 for -inf
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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
  __device__ int64_t first(int64_t c) const { return c * Logit<T>::kPer - head; }
  __device__ bool whole(int64_t c) const { return first(c) >= 0 && first(c) + Logit<T>::kPer <= vocab; }
  __device__ uint4 load(int64_t c) const {
    const int64_t f = first(c);
    if (f >= 0 && f + Logit<T>::kPer <= vocab) return ld_stream(z + f);
    union { uint4 v; T e[Logit<T>::kPer]; } u;
    u.v = Logit<T>::lowest();     // -inf where there is no value
    for (int i = 0; i < Logit<T>::kPer; ++i)
      if (f + i >= 0 && f + i < vocab) u.e[i] = z[f + i];
    return u.v;
  }
};

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
__device__ __forceinline__ SoftSum join(const SoftSum& a, const SoftSum& b, float k0, float k1) {
  SoftSum r;
  r.m = fmaxf(a.m, b.m);   // never NaN: a NaN logit shows in the sums
  r.s0 = a.s0 * exp2_fast(shifted(a.m, r.m, k0)) + b.s0 * exp2_fast(shifted(b.m, r.m, k0));
  r.s1 = a.s1 * exp2_fast(shifted(a.m, r.m, k1)) + b.s1 * exp2_fast(shifted(b.m, r.m, k1));
  return r;
}

struct DistillShared {
  SoftSum warp[kDistillWarps];
  SoftSum block;                 // read by the other blocks of the cluster
  float red[kDistillWarps];
  int ids[kMaxEntries + 1];      // the stored entries, then the label
  float q[kMaxEntries + 1];      // their teacher probability (0 for the label)
  float zat[kMaxEntries + 1];    // the student's logits there
};

__device__ __forceinline__ float block_sum(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = x;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kDistillWarps; ++i) s += red[i];
  return s;
}
__device__ __forceinline__ float block_max(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = x;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int i = 1; i < kDistillWarps; ++i) s = fmaxf(s, red[i]);
  return s;
}

// One cluster per row; block b of it takes chunks [b * chunks_per_block, ...). kTwo: the softmax at
// temperature 1 is needed beside the one at temperature tau (label term, tau != 1).
template <typename T, int MODE, bool kTwo>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const __grid_constant__ DistillParams p) {
  extern __shared__ uint4 keep[];          // kStep: this block's chunks of the row
  __shared__ DistillShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int cluster_size = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int64_t r = blockIdx.x / cluster_size;
  const Row<T> row(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab);
  const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
  const int64_t lo = rank * p.chunks_per_block;
  const int64_t hi = lo + p.chunks_per_block < chunks ? lo + p.chunks_per_block : chunks;
  const float k0 = p.inv_tau * kLog2e, k1 = kLog2e;

  // ---- the teacher's entries and the label; the student's logits at them are read before any
  // gradient is written, which may go to the same memory
  const int label = p.labels ? p.labels[r] : -1;
  const bool hard = label >= 0 && label < p.vocab;
  float tmax = -INFINITY;
  for (int k = threadIdx.x; k <= p.entries; k += kDistillThreads) {
    int id = k < p.entries ? p.ids[r * p.entries + k] : label;
    const bool ok = id >= 0 && id < p.vocab;
    if (!ok) id = -1;
    sh.ids[k] = id;
    sh.zat[k] = ok ? Logit<T>::load(row.z + id) : 0.0f;
    const float t = k < p.entries && ok ? p.t[r * p.entries + k] : -INFINITY;
    sh.q[k] = t;
    tmax = t != t ? INFINITY : fmaxf(tmax, t);   // a NaN logit makes the row NaN below
  }
  tmax = block_max(tmax, sh.red);
  const bool some = tmax > -INFINITY;
  float esum = 0.0f;
  for (int k = threadIdx.x; k < p.entries; k += kDistillThreads)
    esum += sh.q[k] == -INFINITY ? 0.0f : exp2_fast((sh.q[k] - tmax) * k0);
  esum = block_sum(esum, sh.red);
  // log q_k = c (t_k - tmax) - log esum; kept as q_k, with the loss's sum of q (log q - log p) split
  // into the entropy part here and the cross part once the row's maximum and sums are known
  const float log_esum = some ? logf(esum) : 0.0f;
  float negent = 0.0f, qsum = 0.0f;
  for (int k = threadIdx.x; k < p.entries; k += kDistillThreads) {
    const float t = sh.q[k];
    float q = 0.0f;
    if (t != -INFINITY) {
      const float logq = (t - tmax) * p.inv_tau - log_esum;
      q = exp2_fast((t - tmax) * k0) / esum;
      if (q != 0.0f) {
        negent += q * logq;
        qsum += q;
      }
    }
    sh.q[k] = q;
  }
  if (threadIdx.x == 0) sh.q[p.entries] = 0.0f;

  // ---- maximum and sums over the row
  float m = 0.0f, l0 = 0.0f, l1 = 0.0f;   // p = exp2((z - m) k - l)
  if (MODE != kBackward) {
    SoftSum mine = {-INFINITY, 0.0f, 0.0f};
    for (int64_t c0 = lo + threadIdx.x; c0 < hi; c0 += (int64_t)kDistillThreads * kDistillUnroll) {
      uint4 a[kDistillUnroll];
#pragma unroll
      for (int i = 0; i < kDistillUnroll; ++i) {
        const int64_t c = c0 + (int64_t)i * kDistillThreads;
        a[i] = c < hi ? row.load(c) : Logit<T>::lowest();
      }
      float top = mine.m;
#pragma unroll
      for (int i = 0; i < kDistillUnroll; ++i) {
        float v[Logit<T>::kPer];
        Logit<T>::unpack(a[i], v);
#pragma unroll
        for (int e = 0; e < Logit<T>::kPer; ++e) top = fmaxf(top, v[e]);
      }
      if (MODE == kStep) {
#pragma unroll
        for (int i = 0; i < kDistillUnroll; ++i) {
          const int64_t c = c0 + (int64_t)i * kDistillThreads;
          if (c < hi) keep[c - lo] = a[i];
        }
      }
      const float shift = finite_shift(top);
      float s0 = mine.s0 * exp2_fast(shifted(mine.m, top, k0));
      float s1 = kTwo ? mine.s1 * exp2_fast(shifted(mine.m, top, k1)) : 0.0f;
#pragma unroll
      for (int i = 0; i < kDistillUnroll; ++i) {
        float v[Logit<T>::kPer];
        Logit<T>::unpack(a[i], v);
#pragma unroll
        for (int e = 0; e < Logit<T>::kPer; ++e) {
          const float d = v[e] - shift;
          s0 += exp2_fast(d * k0);
          if (kTwo) s1 += exp2_fast(d * k1);
        }
      }
      mine.m = top;
      mine.s0 = s0;
      mine.s1 = s1;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      SoftSum other;
      other.m = __shfl_xor_sync(0xffffffffu, mine.m, o);
      other.s0 = __shfl_xor_sync(0xffffffffu, mine.s0, o);
      other.s1 = __shfl_xor_sync(0xffffffffu, mine.s1, o);
      mine = join(mine, other, k0, k1);
    }
    if (threadIdx.x % 32 == 0) sh.warp[threadIdx.x / 32] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      SoftSum all = sh.warp[0];
      for (int i = 1; i < kDistillWarps; ++i) all = join(all, sh.warp[i], k0, k1);
      sh.block = all;
    }
    cluster.sync();
    SoftSum all = *cluster.map_shared_rank(&sh.block, 0);
    for (int i = 1; i < cluster_size; ++i) all = join(all, *cluster.map_shared_rank(&sh.block, i), k0, k1);
    // no block may leave (or reuse sh.block) before the others have read it
    cluster.sync();
    m = finite_shift(all.m);
    l0 = log2f(all.s0);
    l1 = kTwo ? log2f(all.s1) : l0;
    if (rank == 0) {
      // log p = c (z - m) - log s: differences from the maximum, so that logits far from zero cost
      // the loss no digits
      float cross = 0.0f;
      for (int k = threadIdx.x; k < p.entries; k += kDistillThreads)
        if (sh.q[k] != 0.0f) cross += sh.q[k] * ((sh.zat[k] - m) * p.inv_tau);
      const float total_q = block_sum(qsum, sh.red);
      const float kl = block_sum(negent, sh.red) - block_sum(cross, sh.red) + total_q * (l0 * kLn2);
      if (threadIdx.x == 0) {
        float loss = p.w_teacher != 0.0f && total_q > 0.0f ? p.w_teacher * p.tau * p.tau * kl : 0.0f;
        if (hard) loss += p.w_label * (l1 * kLn2 - (sh.zat[p.entries] - m));
        p.loss[r] = loss;
        p.lse[r] = m * p.inv_tau + l0 * kLn2;
        p.lse[p.rows + r] = p.labels ? m + l1 * kLn2 : 0.0f;
      }
    }
  } else {
    l0 = p.lse[r] * kLog2e;
    l1 = p.labels ? p.lse[p.rows + r] * kLog2e : l0;
    __syncthreads();
  }
  if (MODE == kForward) return;

  // ---- gradient
  const float g = p.row_grad ? p.row_grad[r] : 1.0f;
  const float a0 = some ? g * p.w_teacher * p.tau : 0.0f, a1 = hard ? g * p.w_label : 0.0f;
  // without a second softmax the two terms share p
  const float f0 = kTwo ? a0 : a0 + a1, f1 = kTwo ? a1 : 0.0f;
  T* dz = static_cast<T*>(p.dz) + r * p.dz_stride;
  const bool same_grid = (reinterpret_cast<uintptr_t>(dz) & 15u) == (reinterpret_cast<uintptr_t>(row.z) & 15u);
  for (int64_t c0 = lo + threadIdx.x; c0 < hi; c0 += (int64_t)kDistillThreads * 4) {
    uint4 a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t c = c0 + (int64_t)i * kDistillThreads;
      if (c < hi) a[i] = MODE == kStep ? keep[c - lo] : row.load(c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t c = c0 + (int64_t)i * kDistillThreads;
      if (c >= hi) continue;
      float v[Logit<T>::kPer];
      Logit<T>::unpack(a[i], v);
#pragma unroll
      for (int e = 0; e < Logit<T>::kPer; ++e) {
        const float d = v[e] - m;
        v[e] = f0 * exp2_fast(fmaf(d, k0, -l0)) + (kTwo ? f1 * exp2_fast(fmaf(d, k1, -l1)) : 0.0f);
      }
      const int64_t f = row.first(c);
      if (same_grid && row.whole(c)) {
        st_stream(dz + f, Logit<T>::pack(v));
      } else {
        for (int e = 0; e < Logit<T>::kPer; ++e)
          if (f + e >= 0 && f + e < p.vocab) Logit<T>::store(dz + f + e, v[e]);
      }
    }
  }
  __syncthreads();   // the stores above come before those below
  // the values with a teacher entry or the label: the first entry of each id adds up its repeats
  const int64_t own_lo = row.first(lo), own_hi = row.first(hi);
  for (int k = threadIdx.x; k <= p.entries; k += kDistillThreads) {
    const int id = sh.ids[k];
    if (id < 0 || id < own_lo || id >= own_hi || lo >= hi) continue;
    float q = 0.0f;
    bool leader = true;
    for (int j = 0; j <= p.entries; ++j) {
      const bool same = sh.ids[j] == id;
      if (same && j < k) leader = false;
      if (same) q += sh.q[j];
    }
    if (!leader) continue;
    const float d = sh.zat[k] - m;
    float v = f0 * exp2_fast(fmaf(d, k0, -l0)) + (kTwo ? f1 * exp2_fast(fmaf(d, k1, -l1)) : 0.0f);
    v -= a0 * q;
    if (hard && id == label) v -= a1;
    Logit<T>::store(dz + id, v);
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

int check_distill(const slidedp_distill_args* a) {
  if (!a || a->rows < 0 || a->rows > kMaxTokens || a->vocab < 1 || a->vocab > (1ll << 30) || a->entries < 0 ||
      a->entries > kMaxEntries || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) || a->logits_stride < 0)
    return SLIDEDP_ERR_INVALID_ARG;
  if (!(a->temperature > 0.0) || !is_finite(a->temperature) || !is_finite(1.0 / a->temperature) || !is_finite(a->w_teacher) ||
      !is_finite(a->w_label))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

template <typename T, int MODE, bool kTwo>
cudaError_t launch_distill(const DistillParams& p, unsigned cluster, size_t smem, cudaStream_t st) {
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(distill_kernel<T, MODE, kTwo>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.rows * cluster);
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, distill_kernel<T, MODE, kTwo>, p);
}

// Rows are cut over as many blocks as leave each about 32 KB of logits (several blocks per SM, so that
// one's loads run beside another's arithmetic and stores), up to the portable cluster size.
constexpr int64_t kSliceBytes = 32 * 1024;
constexpr int64_t kMaxSliceBytes = 200 * 1024;

int run_distill(slidedp_ctx* ctx, const slidedp_distill_args* a, int mode, const void* logits,
                const int32_t* ids, const float* t, const int32_t* labels, const float* row_grad, float* loss,
                float* lse, void* dz, cudaStream_t st) {
  if (!ctx || check_distill(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->rows == 0) return SLIDEDP_OK;
  const int64_t elem = a->dtype == SLIDEDP_F32 ? 4 : 2;
  const auto bad = [](const void* q, int64_t align) { return !q || reinterpret_cast<uintptr_t>(q) % (uintptr_t)align != 0; };
  if (bad(logits, elem) || bad(lse, 4) || (a->entries > 0 && (bad(ids, 4) || bad(t, 4)))) return SLIDEDP_ERR_INVALID_ARG;
  if (mode != kBackward && bad(loss, 4)) return SLIDEDP_ERR_INVALID_ARG;
  if (mode != kForward && (bad(dz, elem) || (a->rows > 1 && a->d_logits_stride < a->vocab))) return SLIDEDP_ERR_INVALID_ARG;
  if (labels && reinterpret_cast<uintptr_t>(labels) % 4 != 0) return SLIDEDP_ERR_INVALID_ARG;
  if (row_grad && reinterpret_cast<uintptr_t>(row_grad) % 4 != 0) return SLIDEDP_ERR_INVALID_ARG;

  DistillParams p = {};
  p.z = logits;
  p.dz = dz;
  p.ids = ids;
  p.t = t;
  p.labels = a->w_label != 0.0 ? labels : nullptr;
  p.row_grad = row_grad;
  p.loss = loss;
  p.lse = lse;
  p.rows = a->rows;
  p.vocab = a->vocab;
  p.z_stride = a->logits_stride;
  p.dz_stride = a->d_logits_stride;
  p.entries = a->entries;
  p.inv_tau = (float)(1.0 / a->temperature);
  p.tau = (float)a->temperature;
  p.w_teacher = (float)a->w_teacher;
  p.w_label = (float)a->w_label;
  const int64_t chunks = (a->vocab * elem + 15) / 16 + 1;   // an unaligned row touches one more
  unsigned cluster = 1;
  while (cluster < (unsigned)kDistillMaxCluster && chunks * 16 > kSliceBytes * cluster) cluster *= 2;
  p.chunks_per_block = (chunks + cluster - 1) / cluster;
  if ((int64_t)a->rows * cluster > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  const bool two = p.labels && a->temperature != 1.0;
  const bool f32 = a->dtype == SLIDEDP_F32;

  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  // A row too long for a cluster's shared memory is read twice: forward, then backward.
  if (mode == kStep && p.chunks_per_block * 16 > kMaxSliceBytes) {
    const int rc = run_distill(ctx, a, kForward, logits, ids, t, labels, nullptr, loss, lse, nullptr, st);
    return rc != SLIDEDP_OK ? rc : run_distill(ctx, a, kBackward, logits, ids, t, labels, row_grad, nullptr, lse, dz, st);
  }
  const size_t smem = mode == kStep ? (size_t)p.chunks_per_block * 16 : 0;
  FAULT_POINT();
  cudaError_t e;
#define SLIDEDP_CASE(M)                                                                                     \
  case M:                                                                                                   \
    e = f32 ? (two ? launch_distill<float, M, true>(p, cluster, smem, st)                                   \
                   : launch_distill<float, M, false>(p, cluster, smem, st))                                 \
            : (two ? launch_distill<uint16_t, M, true>(p, cluster, smem, st)                                \
                   : launch_distill<uint16_t, M, false>(p, cluster, smem, st));                             \
    break;
  switch (mode) {
    SLIDEDP_CASE(kForward)
    SLIDEDP_CASE(kBackward)
    default: SLIDEDP_CASE(kStep)
  }
#undef SLIDEDP_CASE
  if (e != cudaSuccess) return cuda_fail(ctx, e);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

}  // namespace

extern "C" {

int slidedp_distill_loss(slidedp_ctx* ctx, const slidedp_distill_args* args, const void* logits,
                         const int32_t* teacher_ids, const float* teacher_logits, const int32_t* labels, float* loss,
                         float* lse, void* cuda_stream) {
  return run_distill(ctx, args, kForward, logits, teacher_ids, teacher_logits, labels, nullptr, loss, lse, nullptr,
                     static_cast<cudaStream_t>(cuda_stream));
}

int slidedp_distill_loss_backward(slidedp_ctx* ctx, const slidedp_distill_args* args, const void* logits,
                                  const int32_t* teacher_ids, const float* teacher_logits, const int32_t* labels,
                                  const float* lse, const float* row_grad, void* d_logits, void* cuda_stream) {
  return run_distill(ctx, args, kBackward, logits, teacher_ids, teacher_logits, labels, row_grad, nullptr,
                     const_cast<float*>(lse), d_logits, static_cast<cudaStream_t>(cuda_stream));
}

int slidedp_distill_step(slidedp_ctx* ctx, const slidedp_distill_args* args, const void* logits,
                         const int32_t* teacher_ids, const float* teacher_logits, const int32_t* labels,
                         const float* row_grad, float* loss, float* lse, void* d_logits, void* cuda_stream) {
  return run_distill(ctx, args, kStep, logits, teacher_ids, teacher_logits, labels, row_grad, loss, lse, d_logits,
                     static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
