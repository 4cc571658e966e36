// libslidedp: the clipped policy loss with a second term towards a reference model. See include/slidedp_ops.h for the contract.
//
// With c = 1 / temperature, m the greatest logit but the label's, s = sum exp(c (z - m)) over all but the label's and o = exp(c (z_y - m)):
// logp = -log(1 + s / o), 1 - p_y = s / (s + o), p = exp(c (z - m)) / (s + o) elsewhere, rho = exp(logp - old), k = ref - logp,
//   loss = -min(rho A, clamp(rho, 1 - lo, 1 + hi) A) + w (e^k - k - 1),   l = -A rho [inside] + w (1 - e^k)
//   dz = g c l (onehot - p)
// The label's own term stays out of the sum, so that a token which is all but certain keeps the digits of what it lacks of one.
// Bound: HBM. The logits are all that is large: a step reads them once and writes the gradient once, forward and backward apart read
// them twice. Rows are held where they are read: in registers up to 64 KB, in shared memory up to 1.1 MB.
#include "ops_internal.h"
#include "logit_rows.cuh"

namespace slidedp {

constexpr int kPolicyThreads = 256;
constexpr int kPolicyWarps = kPolicyThreads / 32;
constexpr int kPolicyMaxCluster = 8;
constexpr int kPolicyUnroll = 4;

struct PolicyParams {
  const void* z;
  void* dz;
  const int32_t* labels;
  const float *old_logp, *ref_logp, *advantage, *row_grad;
  const float* saved_logp;
  float *loss, *logp;
  int64_t rows, vocab, z_stride, dz_stride;
  int64_t chunks_per_block;  // 16-byte chunks of a row that one block of its cluster takes
  int* error;                // pinned host word that a wait which runs out sets
  uint32_t polls;            // and how long it polls
  float inv_tau, low, high, kl;
  double inv_tau64;
};

__device__ __forceinline__ int row_label(const PolicyParams& p, int64_t r) {
  const int y = p.labels[r];
  return y >= 0 && y < p.vocab ? y : -1;
}

// ---- a row's sum and its probabilities ------------------------------------------------------------------------
// With k = log2 e / temperature in FP32 and a shift c in FP32, exp2(fma(z, k, -c)) has one rounding, of the exponent: logits far from
// zero cost no digits as long as the same c goes into what is made of the sum. c = k m, rounded, for the greatest logit m so far.
// Far from zero, where that rounding is no longer small, a logit's difference from m is taken first and then scaled.

struct PolicySum {
  float m, s;
};
// rounded on its own, wherever it is used: no part of a fused multiply-add
__device__ __forceinline__ float shift_of(float m, float k) { return m == -INFINITY ? 0.0f : __fmul_rn(m, k); }
__device__ __forceinline__ bool is_far(float c) { return !(fabsf(c) < 1048576.0f); }
// What the shift of a sum lacks of k m.
__device__ __forceinline__ float shift_error(float m, float k) {
  const float c = shift_of(m, k);
  return is_far(c) ? 0.0f : -fmaf(m, k, -c);
}
// The factor that takes a sum shifted for m to one shifted for the greater `to`.
__device__ __forceinline__ float rescale(float m, float to, float k) {
  if (m == to) return 1.0f;
  return m == -INFINITY ? 0.0f : exp2_approx((m - to) * k + (shift_error(m, k) - shift_error(to, k)));
}
template <int LANES>
__device__ __forceinline__ PolicySum join_sums(PolicySum a, float k) {
  float m = a.m;   // never NaN: a NaN logit shows in the sum
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  a.s *= rescale(a.m, m, k);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
  a.m = m;
  return a;
}
template <typename T, int N>
__device__ __forceinline__ float largest_of(const uint4* a) {
  if constexpr (sizeof(T) == 2) {
    uint4 m = a[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
      m.x = Logit<T>::max2(m.x, a[i].x); m.y = Logit<T>::max2(m.y, a[i].y);
      m.z = Logit<T>::max2(m.z, a[i].z); m.w = Logit<T>::max2(m.w, a[i].w);
    }
    return Logit<T>::largest(m);
  } else {
    float m = Logit<T>::largest(a[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, Logit<T>::largest(a[i]));
    return m;
  }
}
// Adds N chunks to a thread's sum.
template <typename T, int N>
__device__ __forceinline__ void add_chunks(PolicySum& mine, const uint4* a, float k) {
  constexpr int P = Logit<T>::kPer;
  const float top = fmaxf(mine.m, largest_of<T, N>(a));
  mine.s *= rescale(mine.m, top, k);
  mine.m = top;
  const float c = shift_of(top, k);
  uint64_t s0 = 0, s1 = 0;
  const uint64_t kk = pair(k, k), minus = pair(-c, -c);
  if (!is_far(c)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint64_t v[P / 2];
      Logit<T>::unpack(a[i], v);
#pragma unroll
      for (int e = 0; e < P / 2; ++e) {
        const uint64_t x = exp2_pair(fma2(v[e], kk, minus));
        if (e % 2) s1 = add2(s1, x); else s0 = add2(s0, x);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint64_t v[P / 2];
      Logit<T>::unpack(a[i], v);
#pragma unroll
      for (int e = 0; e < P / 2; ++e) {
        s0 = add2(s0, exp2_pair(mul2(add2(v[e], pair(-top, -top)), kk)));
      }
    }
  }
  float x, y;
  split(add2(s0, s1), &x, &y);
  mine.s += x + y;
}

// One value as a sum.
__device__ __forceinline__ PolicySum one_value(float v, float k) {
  const float m = fmaxf(v, -INFINITY), c = shift_of(m, k);     // NaN shows in the sum
  return PolicySum{m, exp2_approx(is_far(c) ? (v - m) * k : fmaf(v, k, -c))};
}
// A chunk without its value number e.
template <typename T>
__device__ __forceinline__ uint4 without(uint4 a, int e) {
  uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if (e == 2 * i) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
      if (e == 2 * i + 1) w[i] = (w[i] & 0xffffu) | 0xff800000u;
    } else {
      if (e == i) w[i] = 0xff800000u;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// N chunks `step` apart from c on, of which number `hot` has the label as its value number e: without it.
template <typename T, int N>
__device__ __forceinline__ void leave_out(uint4* a, int c, int step, int hot, int e) {
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (c + u * step == hot) a[u] = without<T>(a[u], e);
}

// What a row's gradient f (onehot - p) needs: p = exp2(k z - shift) * scale, or far from zero exp2(k (z - shift) + offset) * scale; `factor`
// is -f scale. A gradient that is zero throughout is told by f.
struct RowTerms {
  float shift, offset, factor, at_label, f;
  int far;
  float loss, logp;
};
struct PolicyGrad {
  float k;
  RowTerms t;
  int hot, place;      // the label is value number `place` of chunk `hot`
};
template <typename T>
__device__ __forceinline__ void policy_values(uint4 a, const PolicyGrad& g, float* out) {
  constexpr int P = Logit<T>::kPer;
  uint64_t v[P / 2];
  Logit<T>::unpack(a, v);
  const uint64_t factor = pair(g.t.factor, g.t.factor), kk = pair(g.k, g.k), minus = pair(-g.t.shift, -g.t.shift);
#pragma unroll
  for (int e = 0; e < P / 2; ++e) split(mul2(exp2_pair(fma2(v[e], kk, minus)), factor), &out[2 * e], &out[2 * e + 1]);
}
template <typename T>
__device__ __forceinline__ void policy_values_far(uint4 a, float k, const RowTerms& t, float* out) {
  constexpr int P = Logit<T>::kPer;
  uint64_t v[P / 2];
  Logit<T>::unpack(a, v);
#pragma unroll
  for (int e = 0; e < P / 2; ++e)
    split(mul2(exp2_pair(fma2(add2(v[e], pair(-t.shift, -t.shift)), pair(k, k), pair(t.offset, t.offset))), pair(t.factor, t.factor)), &out[2 * e], &out[2 * e + 1]);
}
// The label is the chunk's value number `at`, if that is one of them.
template <typename T>
__device__ __forceinline__ void put_label(float* out, int at, float v) {
#pragma unroll
  for (int e = 0; e < Logit<T>::kPer; ++e) out[e] = at == e ? v : out[e];
}
// Value by value: partial chunks, and rows whose gradient lies on another address grid.
template <typename T, typename I>
__device__ __forceinline__ void store_chunk(const Row<T>& row, T* dz, I c, const float* out) {
  const I first = row.first(c);
#pragma unroll
  for (int e = 0; e < Logit<T>::kPer; ++e)
    if (first + e >= 0 && first + e < row.vocab) Logit<T>::store(dz + first + e, out[e]);
}
template <typename T, typename I>      // the chunk's number as int where the whole row's are, which takes fewer instructions
__device__ __forceinline__ void policy_chunk(const Row<T>& row, T* dz, bool same_grid, I c, uint4 a, const PolicyGrad& g) {
  float out[Logit<T>::kPer];
  if (g.t.far) policy_values_far<T>(a, g.k, g.t, out);
  else policy_values<T>(a, g, out);
  if (c == g.hot) put_label<T>(out, g.place, g.t.at_label);
  if (same_grid && row.whole(c)) st_stream(dz + row.first(c), Logit<T>::pack(out));
  else store_chunk<T>(row, dz, c, out);
}
// The other values of the label's chunk, by as many lanes of a warp as it has: -inf where there is none.
template <typename T>
__device__ __forceinline__ float beside_label(const Row<T>& row, int hot, int label) {
  const int lane = threadIdx.x % 32, at = row.first(hot) + lane;
  return lane < Logit<T>::kPer && at >= 0 && at < row.vocab && at != label ? Logit<T>::load(row.z + at) : -INFINITY;
}
template <typename T>
__device__ __forceinline__ void zero_chunks(const Row<T>& row, T* dz, bool same_grid, int64_t from, int64_t to, int first, int step) {
  const float zeros[Logit<T>::kPer] = {};
  for (int64_t c = from + first; c < to; c += step) {
    if (same_grid && row.whole(c)) st_stream(dz + row.first(c), make_uint4(0, 0, 0, 0));
    else store_chunk<T>(row, dz, c, zeros);
  }
}
template <typename T>
__device__ __forceinline__ bool on_same_grid(const T* a, const T* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// A row's own numbers, which can be fetched before its sum is known.
struct RowInput {
  float advantage, old_logp, ref_logp, grad;
};
__device__ __forceinline__ RowInput row_input(const PolicyParams& p, int64_t r) {
  return RowInput{p.advantage ? p.advantage[r] : 0.0f, p.old_logp ? p.old_logp[r] : 0.0f, p.ref_logp ? p.ref_logp[r] : 0.0f, p.row_grad ? p.row_grad[r] : 1.0f};
}
// e^k - k - 1 for |k| up to a quarter, by the exponential's series from its second power on: 2^-26 of itself.
__device__ __forceinline__ float beyond_linear(float k) {
  const float k2 = k * k, far = fmaf(1.0f / 5040, k, 1.0f / 720), middle = fmaf(1.0f / 120, k, 1.0f / 24);
  return fmaf(fmaf(far, k2, middle), k2, fmaf(1.0f / 6, k, 0.5f)) * k2;
}
// A row's loss, and the rest of its terms, by one warp: the exponentials that hang on the log-probability are taken by three lanes at
// once. The log-probability comes in FP64, its differences from the old and the reference's one are formed in FP64; `rest` is what the
// label's probability lacks of one, where it is known by itself (kRest).
template <bool kRest>
__device__ __forceinline__ void finish_row(const PolicyParams& p, const RowInput& in, double logp, float rest, float scale, RowTerms* t) {
  const int lane = threadIdx.x % 32;
  const float a = in.advantage, k = p.ref_logp ? (float)((double)in.ref_logp - logp) : 0.0f;
  const float x = lane == 0 ? (p.old_logp && a != 0.0f ? (float)(logp - (double)in.old_logp) : 0.0f) : lane == 1 ? k : (float)logp;
  const float ratio = __shfl_sync(0xffffffffu, expf(x), 0), less_one = expm1f(x);
  const float near = beyond_linear(k), to_ref = __shfl_sync(0xffffffffu, less_one, 1);     // e^k less one
  if (!kRest) rest = -__shfl_sync(0xffffffffu, less_one, 2);
  float loss = 0.0f, slope = 0.0f;
  if (a != 0.0f) {
    const bool inside = !(a > 0.0f ? ratio > p.high : ratio < p.low) || a != a;
    loss = -(inside ? ratio : a > 0.0f ? p.high : p.low) * a;
    if (inside) slope = -a * ratio;
  }
  if (p.ref_logp) {
    loss = fmaf(p.kl, fabsf(k) <= 0.25f ? near : to_ref == INFINITY ? to_ref : to_ref - k, loss);
    slope = fmaf(-p.kl, to_ref, slope);
  }
  t->loss = loss;
  t->logp = (float)logp;
  const float f = in.grad == 0.0f ? 0.0f : in.grad * slope * p.inv_tau;
  t->factor = -f * scale;
  t->at_label = f * rest;
  t->f = f;
}
// From the sum over all but the label, and the label's logit, whose term is 2^e in the sum's units. Where that is above one, all are taken down by
// it, and the log-probability is -log(1 + rest): with the digits of `rest` by log(u) rest / (u - 1), u = 1 + rest as rounded (W. Kahan).
__device__ __forceinline__ RowTerms finish_sum(const PolicyParams& p, const RowInput& in, PolicySum others, float mark, float k) {
  const float c = shift_of(others.m, k);
  RowTerms r;
  r.far = is_far(c);
  r.shift = r.far ? others.m : c;
  r.offset = 0.0f;
  float e = r.far ? (mark - others.m) * k : fmaf(mark, k, -c);
  if (others.m == -INFINITY) e = mark == -INFINITY ? NAN : 0.0f;      // nothing but the label, or not even that
  if (mark == INFINITY) e = NAN;
  const float term = exp2_approx(-fabsf(e)), down = e >= 0.0f ? term : 1.0f;
  const float rest = others.s * down, all = (e >= 0.0f ? 1.0f : term) + rest, less = all - 1.0f, over_all = 1.0f / all;
  const float corrected = less > 0.0f ? __fdividef(rest, less) : 1.0f;
  const int bits = __float_as_int(all);                               // the exponent's part of the log in FP64; NaN stays
  const float log_part = logf(__int_as_float((bits & 0x007fffff) | 0x3f800000)) + (all - all);
  const double own = r.far ? ((double)mark - (double)others.m) * p.inv_tau64 : ((double)k * (double)mark - (double)c) * 0.6931471805599453;
  const double log_all = fma((double)((bits >> 23) - 127), 0.6931471805599453, (double)log_part);
  const double logp = e >= 0.0f && rest < 1.0f ? -(double)(less > 0.0f ? log_part * corrected : rest) : (e >= 0.0f ? 0.0 : own) - log_all;
  finish_row<true>(p, in, logp, rest * over_all, down * over_all, &r);
  return r;
}
__device__ __forceinline__ void write_loss(const PolicyParams& p, int64_t r, const RowTerms& t) {
  if (p.loss) p.loss[r] = t.loss;
  p.logp[r] = t.logp;
}
// From the saved log-probability: the shift is the row's log2 sum, or far from zero the label's logit.
__device__ __forceinline__ RowTerms finish_saved(const PolicyParams& p, const RowInput& in, float mark, float k, float saved) {
  const double logp = saved, log2_p = logp * 1.4426950408889634, exact = (double)k * (double)mark - log2_p;
  RowTerms t;
  t.far = is_far((float)exact) || is_far(mark * k);
  t.shift = t.far ? mark : (float)exact;
  t.offset = (float)log2_p;
  finish_row<false>(p, in, logp, 0.0f, t.far ? 1.0f : exp2f((float)((double)t.shift - exact)), &t);
  return t;
}

// ---- a block, or a cluster of them, per row ----------------------------------------------------------------

struct PolicyShared {
  RowTerms row;
  PolicySum warp[kPolicyWarps];
  alignas(8) float2 part[kPolicyMaxCluster];   // maximum and sum of each block of the cluster
};

// A block's sum to block `to` of its cluster, and the sum of what has come.
__device__ __forceinline__ void store_part(PolicyShared& sh, int rank, int to, PolicySum v) {
  const uint32_t there = peer_addr(smem_addr(&sh.part[rank]), to);
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.m), "f"(v.s) : "memory");
}
__device__ __forceinline__ PolicySum join_parts(const PolicyShared& sh, int cluster, float k) {
  const int i = threadIdx.x % kPolicyMaxCluster;
  return join_sums<kPolicyMaxCluster>(i < cluster ? PolicySum{sh.part[i].x, sh.part[i].y} : PolicySum{-INFINITY, 0.0f}, k);
}
// The sum over chunks [from, to) without the label, by a block; all threads get it.
template <typename T>
__device__ __forceinline__ PolicySum block_sum(const Row<T>& row, int64_t from, int64_t to, int label, float k, PolicySum* warps) {
  constexpr int U = kPolicyUnroll;
  // the label's chunk is not read with the others, but its other values by the last warp
  const int label_chunk = (label + row.head) / Logit<T>::kPer, n = (int)(to - from), hot = label_chunk - (int)from;
  PolicySum mine = {-INFINITY, 0.0f};
  if (threadIdx.x >= kPolicyThreads - 32 && hot >= 0 && hot < n) mine = one_value(beside_label<T>(row, label_chunk, label), k);
  for (int c = threadIdx.x; c < n; c += kPolicyThreads * U) {
    uint4 a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = c + u * kPolicyThreads < n && c + u * kPolicyThreads != hot ? row.load(from + c + u * kPolicyThreads) : Logit<T>::lowest();
    // FP32: all of them before the first is used; the compiler uses each as it comes (1023 x 100003: 72 -> 47 us)
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int u = 0; u < U; ++u) asm volatile("" : "+r"(a[u].x), "+r"(a[u].y), "+r"(a[u].z), "+r"(a[u].w));
    }
    add_chunks<T, U>(mine, a, k);
  }
  mine = join_sums<32>(mine, k);
  if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = mine;
  __syncthreads();
  return join_sums<kPolicyWarps>(warps[threadIdx.x % kPolicyWarps], k);
}

// FP32 holds a log-probability to 2^-24 of itself, by which a row's probabilities are off that are made from it: 4e-6 at -64. Rows with less are
// summed again, a label without any probability among them.
constexpr float kTrustedLogp = -64.0f;

// The row's terms from its logits, by all blocks of a cluster, which have met and have not written any.
template <typename T>
__device__ __forceinline__ void sum_again(const PolicyParams& p, PolicyShared& sh, int64_t r, int rank, int cluster, int64_t from, int64_t to, int label) {
  const Row<T> row(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab);
  const float mark = Logit<T>::load(row.z + label), k = p.inv_tau * kLog2e;
  PolicySum mine = block_sum<T>(row, from, to, label, k, sh.warp);
  if (cluster > 1) {
    if ((int)threadIdx.x < cluster) store_part(sh, rank, threadIdx.x, mine);
    cluster_sync();
    mine = join_parts(sh, cluster, k);
  }
  if (threadIdx.x < 32) {
    const RowTerms t = finish_sum(p, row_input(p, r), mine, mark, k);
    if (threadIdx.x == 0) sh.row = t;
  }
  __syncthreads();
}

// kGradient: the gradient from the saved log-probability, else log-probability and loss. The blocks of a cluster share a row's chunks;
// forward they bring their sums to the first through distributed shared memory. Bound: HBM. 4096 x 131072 BF16: forward 170 us
// (6.3 TB/s), gradient 343 (6.3); with the label's chunk asked for in int64_t, or its label taken out of a chunk that has been read, forward 2 to 4 %
// more.
template <typename T, bool kGradient>
__global__ void __launch_bounds__(kPolicyThreads, 5) policy_row_kernel(const __grid_constant__ PolicyParams p, int cluster) {
  start_after_previous_kernel();
  __shared__ PolicyShared sh;
  const int64_t r = blockIdx.x / cluster;
  const int rank = blockIdx.x % cluster;
  const T* z = static_cast<const T*>(p.z) + r * p.z_stride;
  T* dz = static_cast<T*>(p.dz) + r * p.dz_stride;
  const Row<T> row(z, p.vocab);
  const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
  const int64_t from = rank * p.chunks_per_block < chunks ? rank * p.chunks_per_block : chunks;
  const int64_t to = from + p.chunks_per_block < chunks ? from + p.chunks_per_block : chunks;
  const int label = row_label(p, r);
  const bool same_grid = on_same_grid<T>(z, dz);
  if (label < 0) {      // all blocks of the cluster alike
    if (kGradient) {
      zero_chunks<T>(row, dz, same_grid, from, to, threadIdx.x, kPolicyThreads);
    } else if (rank == 0 && threadIdx.x == 0) {
      if (p.loss) p.loss[r] = 0.0f;
      p.logp[r] = 0.0f;
    }
    return;
  }
  // forward, a block's sums go to the first block's shared memory: that block must have started, which is asked for here and waited
  // for where they are ready
  if (!kGradient && cluster > 1) cluster_arrive();
  const float at = Logit<T>::load(z + label), k = p.inv_tau * kLog2e;
  constexpr int U = kPolicyUnroll;
  if constexpr (kGradient) {
    const float saved = p.saved_logp[r];
    if (threadIdx.x < 32) {
      const RowTerms t = finish_saved(p, row_input(p, r), at, k, saved);
      if (threadIdx.x == 0) sh.row = t;
    }
    // nothing has been read of the row but `at`, which no block may change before all have it
    if (cluster > 1) cluster_sync(); else __syncthreads();
    if (saved < kTrustedLogp) sum_again<T>(p, sh, r, rank, cluster, from, to, label);
    const RowTerms t = sh.row;
    if (t.f == 0.0f) return zero_chunks<T>(row, dz, same_grid, from, to, threadIdx.x, kPolicyThreads);
    const int hot = (label + row.head) / Logit<T>::kPer;
    const PolicyGrad g = {k, t, hot, label - row.first(hot)};
    const int last = (int)to;        // chunks in int: with int64_t registers are spilled (8192 x 1000 BF16 23.5 us in place of 26.3, 4096 x 131072 332 of 345)
    for (int c = (int)from + threadIdx.x; c < last; c += kPolicyThreads * U) {
      uint4 a[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + u * kPolicyThreads < last) a[u] = row.load(c + u * kPolicyThreads);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + u * kPolicyThreads < last) policy_chunk<T>(row, dz, same_grid, c + u * kPolicyThreads, a[u], g);
    }
  } else {
    PolicySum mine = block_sum<T>(row, from, to, label, k, sh.warp);
    if (cluster > 1) {
      cluster_wait();
      if (threadIdx.x == 0) store_part(sh, rank, 0, mine);
      cluster_sync();
      if (rank > 0) return;
      mine = join_parts(sh, cluster, k);
    }
    if (threadIdx.x < 32) {
      const RowTerms t = finish_sum(p, row_input(p, r), mine, at, k);
      if (threadIdx.x == 0) write_loss(p, r, t);
    }
  }
}

// Both for short rows: kRow threads hold a row in registers, U chunks each; a warp, eight of them per block, or a block. Against the ring
// below, which is for rows longer than these: 8192 x 8000 BF16 55 us (a block of 256) and 117, 4096 x 32768 111 (of 512) and 117;
// a warp for 8192 x 1000: 10, where a block takes 28.
// Blocks per SM that the registers allow: four for each chunk as it is read, and what a thread of a row needs besides (8192 x 8000 BF16: six
// blocks 55 us, the five that the compiler would leave 61).
constexpr int held_blocks(int u, int row) { return 65536 / ((row < 256 ? 256 : row) * (4 * u + (row < 256 ? 44 : 24))); }
template <typename T, int U, int kRow>
__global__ void __launch_bounds__(kRow < 256 ? 256 : kRow, held_blocks(U, kRow)) policy_held_kernel(const __grid_constant__ PolicyParams p) {
  start_after_previous_kernel();
  __shared__ RowTerms shared_terms;
  __shared__ PolicySum warps[16];
  constexpr int kRows = kRow < 256 ? 256 / kRow : 1, kWarps = kRow / 32;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kRow;
  const int thread = threadIdx.x % kRow;
  if (r >= p.rows) return;
  const T* z = static_cast<const T*>(p.z) + r * p.z_stride;
  T* dz = static_cast<T*>(p.dz) + r * p.dz_stride;
  const Row<T> row(z, p.vocab);
  const int chunks = (int)((p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer);
  const int label = row_label(p, r);
  const bool same_grid = on_same_grid<T>(z, dz);
  if (label < 0) {
    if (thread == 0) {
      if (p.loss) p.loss[r] = 0.0f;
      p.logp[r] = 0.0f;
    }
    return zero_chunks<T>(row, dz, same_grid, 0, chunks, thread, kRow);
  }
  const float at = Logit<T>::load(z + label), k = p.inv_tau * kLog2e;
  RowInput in = {};
  if (thread < 32) in = row_input(p, r);
  const int hot = (label + row.head) / Logit<T>::kPer;
  uint4 a[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = thread + u * kRow;
    a[u] = c < chunks ? row.load(c) : Logit<T>::lowest();
  }
  const int place = label - row.first(hot);
  leave_out<T, U>(a, thread, kRow, hot, place);       // the gradient does not need it either
  PolicySum mine = {-INFINITY, 0.0f};
  add_chunks<T, U>(mine, a, k);
  mine = join_sums<32>(mine, k);
  RowTerms t;
  if constexpr (kWarps == 1) {
    t = finish_sum(p, in, mine, at, k);      // all lanes read the row before one writes it: they have met in the sums
    if (thread == 0) write_loss(p, r, t);
  } else {
    if (thread % 32 == 0) warps[thread / 32] = mine;
    __syncthreads();
    if (thread < 32) {
      mine = join_sums<kWarps>(warps[thread % kWarps], k);
      t = finish_sum(p, in, mine, at, k);
      if (thread == 0) {
        shared_terms = t;
        write_loss(p, r, t);
      }
    }
    __syncthreads();
    t = shared_terms;
  }
  if (t.f == 0.0f) return zero_chunks<T>(row, dz, same_grid, 0, chunks, thread, kRow);
  const PolicyGrad g = {k, t, hot, place};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (thread + u * kRow < chunks) policy_chunk<T>(row, dz, same_grid, thread + u * kRow, a[u], g);
}

// ---- rows in shared memory -----------------------------------------------------------------------------------
// Both for long rows: blocks, or clusters that share a row, stay, one per SM. A producer copies slice after slice into a ring of
// slots; the sums' warps go through a row as it comes, the gradient's warps follow one row behind them and give the slots back. So
// the next rows are under way while a row's sums are exchanged and made into its loss, by a warp of its own, and every logit is
// read once. A slice is at most as long as leaves part of the ring for the row after it. 4096 x 131072 BF16: 392 us, 2.15 GB at 5.5 TB/s
// (forward and gradient apart: 519). Slower: 12 or 14 warps for each group, 446 and 461 when these took 424; slots of 32 KB, 497; 16 warps
// that do both in turn, 609 to 427; shorter slices in larger clusters, 566; reading the row again from L2, 750.

constexpr int kRingWarps = 8;                       // of each of the two groups
constexpr int kRingGroup = kRingWarps * 32;
constexpr int kRingThreads = 2 * kRingGroup + 64;   // and the producer's and the rows' warps
constexpr int kSlotUnroll = 4;
constexpr int kSlotChunks = kRingGroup * kSlotUnroll;
constexpr int kSlots = 208 * 1024 / (kSlotChunks * 16);
// Rows between the first and the last that any block of a cluster has to do with: a block's sums are at most kSlots rows before its
// gradients, which wait for the other blocks' sums, which are at most kSlots rows before those blocks' gradients.
constexpr int kRowSlots = 32;
static_assert(kRowSlots > 2 * kSlots + 2, "rows that are still looked at would be overwritten");

struct PolicyRing {
  alignas(16) float4 part[kRowSlots][kPolicyMaxCluster];   // maximum, sum, the label's logit where it is known, the sums' number
  RowTerms row[kRowSlots];
  alignas(16) PolicySum warp[2][kRingWarps];
  uint64_t full[kSlots], empty[kSlots];
  uint64_t summed[kRowSlots], known[kRowSlots];
  int sent[kPolicyMaxCluster];                             // the number after that of the last sums that each block sent
  uint32_t dead;
};

// One block's part of a row: chunks [lo, hi), of which [mid, mid + n) are whole.
template <typename T>
struct RingSlice {
  Row<T> row;
  int64_t lo, hi, mid;
  int n;
  __device__ __forceinline__ RingSlice(const PolicyParams& p, int64_t r, int rank) : row(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab) {
    const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
    lo = rank * p.chunks_per_block;
    hi = lo + p.chunks_per_block < chunks ? lo + p.chunks_per_block : chunks;
    if (lo > hi) lo = hi;
    mid = lo < hi && !row.whole(lo) ? lo + 1 : lo;
    n = (int)((hi > mid && !row.whole(hi - 1) ? hi - 1 : hi) - mid);
  }
  // f(chunk) for the partial chunks, each by one thread of a group
  template <typename F>
  __device__ __forceinline__ void edges(int thread, F f) const {
    if (thread == 32 && mid > lo) f(lo);
    if (thread == 64 && mid + n < hi) f(hi - 1);
  }
};
// The place in a ring of N that comes round: its index and the parity of its phase.
template <int N>
struct Place {
  int i = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void next() {
    if (++i == N) i = 0, parity ^= 1;
  }
};

template <typename T>
__global__ void __launch_bounds__(kRingThreads, 1) policy_ring_kernel(const __grid_constant__ PolicyParams p, int cluster) {
  extern __shared__ uint4 slots[];
  __shared__ PolicyRing ring;
  allow_next_kernel();
  const int rank = blockIdx.x % cluster, first = blockIdx.x / cluster, step = gridDim.x / cluster;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_addr(&ring.full[i]), 1);
      mbar_init(smem_addr(&ring.empty[i]), kRingWarps);
    }
    for (int i = 0; i < kRowSlots; ++i) {
      mbar_init(smem_addr(&ring.summed[i]), 1);
      mbar_init(smem_addr(&ring.known[i]), 1);
    }
    ring.dead = 0;
    mbar_init_fence();
  }
  if (threadIdx.x < kRowSlots * kPolicyMaxCluster) ring.part[threadIdx.x / kPolicyMaxCluster][threadIdx.x % kPolicyMaxCluster].w = 0.0f;
  if (cluster > 1) cluster_sync(); else __syncthreads();
  wait_for_previous_kernel();
  const Waiter wait{&ring.dead, p.error, p.polls};
  const float k = p.inv_tau * kLog2e;
  Place<kSlots> slot;
  Place<kRowSlots> at;
  int label1 = first < p.rows ? p.labels[first] : -1, label2 = first + step < p.rows ? p.labels[first + step] : -1;
  const auto label_of = [&](int64_t r) {      // fetched two rows ahead
    const int y = label1;
    label1 = label2;
    if (r + 2 * (int64_t)step < p.rows) label2 = p.labels[r + 2 * (int64_t)step];
    return y >= 0 && y < p.vocab ? y : -1;
  };
  bool ok = true;
  if (warp < kRingWarps) {                    // the sums
    int turn = 0, sent = 1;
    for (int64_t r = first; r < p.rows; r += step) {
      const int label = label_of(r);
      if (label < 0) continue;
      const RingSlice<T> s(p, r, rank);
      // the label's logit comes from the block that has it, before any block may write this row's gradient to the same memory
      float mark = 0.0f;
      const int hot = (label + s.row.head) / Logit<T>::kPer, place = label - s.row.first(hot), whole = hot >= s.mid && hot < s.mid + s.n ? (int)(hot - s.mid) : -1;      // among the whole chunks
      if (warp == 0 && (hot == s.lo || hot == s.hi - 1)) mark = Logit<T>::load(s.row.z + label);
      PolicySum mine = {-INFINITY, 0.0f};
      s.edges(threadIdx.x, [&](int64_t c) {
        uint4 a = s.row.load(c);
        if (c == hot) a = without<T>(a, place);
        add_chunks<T, 1>(mine, &a, k);
      });
      __syncwarp();
      for (int i0 = 0; i0 < s.n; i0 += kSlotChunks, slot.next()) {
        // after a wait that ran out no more of them, but this row's barrier, where all warps learn of it
        if (ok) ok = __all_sync(0xffffffffu, wait(smem_addr(&ring.full[slot.i]), slot.parity));
        uint4 a[kSlotUnroll];
        const uint4* from = slots + slot.i * kSlotChunks + threadIdx.x;
#pragma unroll
        for (int u = 0; u < kSlotUnroll; ++u) a[u] = from[u * kRingGroup];
        if (i0 + kSlotChunks > s.n) {
#pragma unroll
          for (int u = 0; u < kSlotUnroll; ++u)
            if (i0 + (int)threadIdx.x + u * kRingGroup >= s.n) a[u] = Logit<T>::lowest();
        }
        if (whole >= i0 && whole < i0 + kSlotChunks) {
          if (warp == 0) mark = Logit<T>::load(reinterpret_cast<const T*>(slots + slot.i * kSlotChunks + whole - i0) + place);
          leave_out<T, kSlotUnroll>(a, i0 + (int)threadIdx.x, kRingGroup, whole, place);
        }
        add_chunks<T, kSlotUnroll>(mine, a, k);
      }
      mine = join_sums<32>(mine, k);
      if (lane == 0) ring.warp[turn][warp] = mine;
      uint32_t all_ok;
      __syncwarp();                           // lanes that took different ways meet before the barrier
      asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n barrier.cta.red.and.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
                   : "=r"(all_ok)
                   : "r"((uint32_t)ok), "n"(kRingGroup)
                   : "memory");
      if (!all_ok) break;                     // all of them, at the same barrier
      if (warp == 0) {
        mine = join_sums<16>(lane % 16 < kRingWarps ? ring.warp[turn][lane % 16] : PolicySum{-INFINITY, 0.0f}, k);
        const uint32_t bar = smem_addr(&ring.summed[at.i]);
        if (cluster == 1) {                   // asynchronous stores are for clusters: in a launch without them they are an illegal instruction
          if (lane == 0) {
            ring.part[at.i][0] = make_float4(mine.m, mine.s, mark, 0.0f);
            mbar_arrive(bar);
          }
        } else if (lane < cluster) {          // stores and an arrival that others see would wait 2500 cycles for the order between them
          const uint32_t to = peer_addr(smem_addr(&ring.part[at.i][rank]), lane), there = peer_addr(bar, lane);
          if (lane == 0) mbar_expect(bar, cluster * sizeof(float4));
          asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "f"(mine.m),
                       "f"(mine.s), "f"(mark), "f"(__int_as_float(sent)), "r"(there)
                       : "memory");
        }
        ++sent;
      }
      turn ^= 1;
      at.next();
    }
    if (warp == 0 && cluster > 1 && lane < cluster) {        // told to all, should one of them have given up
      const uint32_t to = peer_addr(smem_addr(&ring.sent[rank]), lane);
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(sent) : "memory");
    }
  } else if (warp < 2 * kRingWarps) {         // the gradients
    const int thread = threadIdx.x - kRingGroup;
    for (int64_t r = first; ok && r < p.rows; r += step) {
      const int label = label_of(r);
      const RingSlice<T> s(p, r, rank);
      T* dz = static_cast<T*>(p.dz) + r * p.dz_stride;
      const bool same_grid = on_same_grid<T>(s.row.z, dz);
      if (label < 0) {
        zero_chunks<T>(s.row, dz, same_grid, s.lo, s.hi, thread, kRingGroup);
        continue;
      }
      ok = __all_sync(0xffffffffu, wait(smem_addr(&ring.known[at.i]), at.parity));
      if (!ok) break;
      const RowTerms t = ring.row[at.i];
      const int label_chunk = (label + s.row.head) / Logit<T>::kPer;
      const PolicyGrad g = {k, t, label_chunk, label - s.row.first(label_chunk)};
      at.next();
      const bool zero = t.f == 0.0f, usual = same_grid && !t.far;
      if (zero) zero_chunks<T>(s.row, dz, same_grid, s.lo, s.hi, thread, kRingGroup);
      else s.edges(thread, [&](int64_t c) { policy_chunk<T>(s.row, dz, same_grid, c, s.row.load(c), g); });
      const int64_t hot = label_chunk - s.mid;
      uint4* out = reinterpret_cast<uint4*>(dz + s.row.first(s.mid)) + thread;     // used where it is aligned
      for (int i0 = 0; i0 < s.n; i0 += kSlotChunks, slot.next()) {
        // the slot is full: what is known of the row was known after its sums
        uint4 a[kSlotUnroll];
        const uint4* from = slots + slot.i * kSlotChunks + thread;
#pragma unroll
        for (int u = 0; u < kSlotUnroll; ++u) a[u] = from[u * kRingGroup];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&ring.empty[slot.i]));
        if (zero) continue;
        float v[Logit<T>::kPer];
        if (usual && i0 + kSlotChunks <= s.n && !(hot >= i0 && hot < i0 + kSlotChunks)) {
#pragma unroll
          for (int u = 0; u < kSlotUnroll; ++u) {
            policy_values<T>(a[u], g, v);
            st_stream(out + i0 + u * kRingGroup, Logit<T>::pack(v));
          }
        } else {
#pragma unroll
          for (int u = 0; u < kSlotUnroll; ++u)
            if (i0 + thread + u * kRingGroup < s.n) policy_chunk<T>(s.row, dz, same_grid, s.mid + i0 + thread + u * kRingGroup, a[u], g);
        }
      }
    }
  } else if (warp == 2 * kRingWarps) {        // the copies
    int64_t issued = 0;
    if (lane == 0) {
      for (int64_t r = first; ok && r < p.rows; r += step) {
        if (label_of(r) < 0) continue;
        const RingSlice<T> s(p, r, rank);
        const uint4* from = reinterpret_cast<const uint4*>(s.row.z + s.row.first(s.mid));
        for (int i0 = 0; ok && i0 < s.n; i0 += kSlotChunks, slot.next(), ++issued) {
          if (issued >= kSlots) ok = wait(smem_addr(&ring.empty[slot.i]), slot.parity ^ 1);
          if (!ok) break;
          const uint32_t bytes = (uint32_t)min(s.n - i0, kSlotChunks) * 16, bar = smem_addr(&ring.full[slot.i]);
          mbar_expect(bar, bytes);
          bulk_load(smem_addr(&slots[slot.i * kSlotChunks]), from + i0, bytes, bar);
        }
      }
      // none may be left under way, whoever gave up
      for (int64_t i = issued > kSlots ? issued - kSlots : 0; i < issued; ++i) drain(smem_addr(&ring.full[i % kSlots]), i / kSlots & 1);
    }
  } else {                                    // the rows: their sums to what the gradient needs
    for (int64_t r = first; ok && r < p.rows; r += step) {
      const int label = label_of(r);
      if (label < 0) {
        if (rank == 0 && lane == 0) {
          if (p.loss) p.loss[r] = 0.0f;
          p.logp[r] = 0.0f;
        }
        continue;
      }
      const RowInput in = row_input(p, r);
      ok = __all_sync(0xffffffffu, wait(smem_addr(&ring.summed[at.i]), at.parity));
      if (!ok) break;
      const float4 v = lane % kPolicyMaxCluster < cluster ? ring.part[at.i][lane % kPolicyMaxCluster] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
      const PolicySum all = join_sums<kPolicyMaxCluster>(PolicySum{v.x, v.y}, k);
      const int head = Row<T>(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab).head;
      const int owner = (int)((uint32_t)(label + head) / Logit<T>::kPer / (uint32_t)p.chunks_per_block);
      const RowTerms t = finish_sum(p, in, all, __shfl_sync(0xffffffffu, v.z, owner), k);
      if (lane == 0) {
        ring.row[at.i] = t;
        mbar_arrive(smem_addr(&ring.known[at.i]));
        if (rank == 0) write_loss(p, r, t);
      }
      at.next();
    }
  }
  __syncwarp();
  if (cluster == 1) return;
  cluster_sync();
  // Sums that were waited for have come. Where a wait ran out, nobody sends any more, but some may still be on their way here.
  if (ring.dead && warp == 0 && lane < cluster) {
    for (int n = max(1, ring.sent[lane] - kRowSlots); n < ring.sent[lane]; ++n) {
      const volatile float4* to = &ring.part[(n - 1) % kRowSlots][lane];
      for (uint32_t polls = 0; __float_as_int(to->w) != n && polls < (1u << 20); ++polls) __nanosleep(100);
    }
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

constexpr int kSms = 148;
constexpr int64_t kHeldChunks = 8 * 512;                 // rows up to 64 KB are held in registers
constexpr int64_t kMaxSliceChunks = 8704;                    // of the ring's 13312
constexpr int64_t kMinSliceChunks = 512;
constexpr int64_t kEnoughBlocks = kSms * 4, kRound = kSms * 5;

enum PolicyMode { kPolicyForward, kPolicyBackward, kPolicyStep };

// How many clusters of the ring's kernel run at once: blocks that stay must all be of the first round. Asked once per context, that is
// device, type and size.
template <typename K>
cudaError_t resident_clusters(slidedp_ctx* ctx, K kernel, bool f32, int cluster, size_t smem, int* out) {
  static_assert(sizeof(ctx->policy_clusters[0]) / sizeof(ctx->policy_clusters[0][0]) > kPolicyMaxCluster, "a place for each size");
  std::atomic<int>& known = ctx->policy_clusters[f32][cluster];
  *out = known;
  if (*out > 0) return cudaSuccess;
  if (cluster == 1) {
    *out = kSms;
  } else {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kSms / cluster * cluster);
    cfg.blockDim = dim3(kRingThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(out, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (*out < 1) return cudaErrorLaunchOutOfResources;
    if (*out > kSms / cluster) *out = kSms / cluster;
  }
  known = *out;
  return cudaSuccess;
}

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
  p.low = (float)(1.0 - a->clip_low);
  p.high = (float)(1.0 + a->clip_high);
  p.kl = (float)a->kl_weight;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t stream = st;
  const bool aligned = !odd(logits, 16) && (a->rows == 1 || a->logits_stride * elem % 16 == 0);
  const int64_t chunks = (a->vocab * elem + 15) / 16 + !aligned;   // an unaligned row touches one more
  p.error = ctx->kernel_error;
  p.polls = ctx->wait_polls;
  const bool f32 = a->dtype == SLIDEDP_F32;
  FAULT_POINT();
  cudaError_t failed = cudaSuccess;
  if (mode == kPolicyStep && chunks <= kHeldChunks) {
    const auto run = [&](auto kernel, int row) {
      const int64_t rows = row < 256 ? 256 / row : 1;
      launch_after(kernel, dim3((unsigned)((a->rows + rows - 1) / rows)), row < 256 ? 256 : row, 0, 1, stream, p);
    };
    const auto held = [&](auto type) {
      typedef decltype(type) T;
      if (chunks <= 4 * 32) run(policy_held_kernel<T, 4, 32>, 32);
      else if (chunks <= 8 * 32) run(policy_held_kernel<T, 8, 32>, 32);
      else if (chunks <= 16 * 32) run(policy_held_kernel<T, 16, 32>, 32);
      else if (chunks <= 3 * 256) run(policy_held_kernel<T, 3, 256>, 256);
      else if (chunks <= 4 * 256) run(policy_held_kernel<T, 4, 256>, 256);
      else if (chunks <= 6 * 256) run(policy_held_kernel<T, 6, 256>, 256);
      else if (chunks <= 8 * 256) run(policy_held_kernel<T, 8, 256>, 256);
      else if (chunks <= 6 * 512) run(policy_held_kernel<T, 6, 512>, 512);
      else run(policy_held_kernel<T, 8, 512>, 512);
    };
    f32 ? held(float()) : held(uint16_t());
  } else if (mode == kPolicyStep && chunks <= kPolicyMaxCluster * kMaxSliceChunks) {
    int cluster = 1;
    while (cluster < kPolicyMaxCluster && (chunks > cluster * kMaxSliceChunks || (a->rows * cluster < kSms && chunks > cluster * 1024))) cluster *= 2;
    p.chunks_per_block = (chunks + cluster - 1) / cluster;
    const size_t smem = kSlots * kSlotChunks * 16;
    const auto run = [&](auto kernel) {
      failed = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      int most = 0;
      if (failed == cudaSuccess) failed = resident_clusters(ctx, kernel, f32, cluster, smem, &most);
      const int64_t clusters = a->rows < most ? a->rows : most;
      if (failed == cudaSuccess) launch_after(kernel, dim3((unsigned)(clusters * cluster)), kRingThreads, smem, cluster, stream, p, cluster);
    };
    f32 ? run(policy_ring_kernel<float>) : run(policy_ring_kernel<uint16_t>);
  } else {
    int cluster = 1;
    while (cluster < kPolicyMaxCluster && a->rows * cluster < kEnoughBlocks && chunks >= 2 * kMinSliceChunks * cluster) cluster *= 2;
    // and where that saves a sixth of the rounds (1023 rows of 100003 FP32 logits: 1.4 rounds take as long as 2; forward 127 -> 106 us)
    const auto rounds = [&](int c) { return (double)((a->rows * c + kRound - 1) / kRound) / c; };
    while (cluster < kPolicyMaxCluster && rounds(2 * cluster) < 0.85 * rounds(cluster) && chunks >= 2 * kMinSliceChunks * cluster) cluster *= 2;
    p.chunks_per_block = (chunks + cluster - 1) / cluster;
    if (a->rows * cluster > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
    const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)(a->rows * cluster)), kPolicyThreads, 0, cluster, stream, p, cluster); };
    if (mode != kPolicyBackward) f32 ? run(policy_row_kernel<float, false>) : run(policy_row_kernel<uint16_t, false>);
    if (mode == kPolicyStep) {        // a row that no ring holds: one after the other
      ctx->launches += 1;
      CU_AFTER_LAUNCH();
      FAULT_POINT();
      p.saved_logp = logp;
    }
    if (mode != kPolicyForward) f32 ? run(policy_row_kernel<float, true>) : run(policy_row_kernel<uint16_t, true>);
  }
  if (failed != cudaSuccess) return cuda_fail(ctx, failed);
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
