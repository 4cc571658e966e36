// libslidedp: distillation from a teacher's top logits with hard labels beside it: loss, gradient, and
// both in one pass. See include/slidedp_ops.h for the contract.
//
// With c = 1 / temperature, m = max z, s = sum exp(c (z - m)):  lse = c m + log s,  log p = c z - lse and
//   dz = g (w_t tau (p - q) + w_l (p1 - onehot)),   p1 the softmax at temperature 1.
// Bound: HBM. The logits are all that is large: forward reads them once, backward reads them and writes the
// gradient. The step (both) reads a row twice in one kernel, the second time from L2, so that it moves what
// backward alone does. Measured on 4096 x 131072 BF16 logits: 445 us, 4.8 TB/s of one read and one write, 14
// instructions and two exponentials per logit. No unit is saturated there (issue 60 %, special functions 52 %, DRAM 51 % of the
// time): the warps wait for loads and for each other, as a block has no loads under way while its row starts and while the row's
// sums are exchanged. Keeping the row on chip instead, in the shared memory or the
// registers of a cluster of eight blocks, measured 481 to 860 us: the exchange of a row's sums costs each of the
// eight what 5000 of its own logits do, and too few rows fit to cover that.
#include "ops_internal.h"
#include "logit_rows.cuh"

namespace slidedp {

constexpr int kMaxEntries = 512;        // teacher entries per row
constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kDistillMaxCluster = 8;
// 16-byte chunks per thread and turn; the next turn's are on their way. A step's long slices of a row take four (70
// registers, three blocks per SM); short ones two, five blocks per SM, so that more rows cover each other's exchange of
// sums. Steps of BF16 logits with four / two: 8192 x 8000 135 / 105 us, 4096 x 32768 130 / 119, 4096 x 49152 180 / 173,
// 4096 x 65536 224 / 231, 4096 x 131072 446 / 473.
constexpr int kDistillUnroll = 4, kDistillUnrollShort = 2;
constexpr int64_t kShortSliceBytes = 112 * 1024;
constexpr int distill_min_blocks(int unroll) { return unroll == kDistillUnroll ? 0 : 5; }   // 0: as the compiler likes

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
  int* error;              // pinned host word that a wait which runs out sets
  uint32_t polls;          // and how long it polls
};

struct DistillShared {
  alignas(16) SoftSum warp[kDistillWarps];
  alignas(16) float4 part[kDistillMaxCluster];   // sums written by the blocks of the cluster
  uint64_t exchanged;
};

// The row's entries (and, last, its label) in shared memory: id (-1: absent), teacher probability, the student's
// logit there.
struct Entries {
  int* id;
  float* q;
  float* z;
  int count;   // stored entries; the label sits at [count], absent ones up to a multiple of four
  __device__ Entries(void* smem, int n) : id(static_cast<int*>(smem)), q(reinterpret_cast<float*>(id + padded(n))), z(q + padded(n)), count(n) {}
  static __host__ __device__ int padded(int n) { return (n + 4) & ~3; }
  static __host__ __device__ size_t bytes(int n) { return (size_t)padded(n) * 12; }
};

// Fetches the entries with all threads of a block. The logits are read here, before any block writes a
// gradient, which may go to the same memory. True when the thread saw an entry with some mass.
template <typename T>
__device__ __forceinline__ bool fetch_entries(const DistillParams& p, int64_t r, const T* z, const Entries& en) {
  bool some = false;
  for (int k = threadIdx.x; k < Entries::padded(en.count); k += kDistillThreads) {
    const bool stored = k < en.count;
    const int id = stored ? p.ids[r * en.count + k] : k == en.count && p.labels ? p.labels[r] : -1;
    const float t = stored ? p.t[r * en.count + k] : 0.0f;
    const bool ok = id >= 0 && id < p.vocab;
    en.id[k] = ok ? id : -1;
    en.z[k] = ok ? Logit<T>::load(z + id) : 0.0f;
    en.q[k] = stored && ok ? t : -INFINITY;
    some |= stored && ok && t != -INFINITY;
  }
  return some;
}

// One warp turns the teacher's logits into probabilities, in place. Adds the lane's share of
// sum q log q and of sum q; log q = (t - max) / tau - log sum.
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ void teacher_softmax(const DistillParams& p, const Entries& en, float* q_log_q, float* q_sum) {
  const int lane = threadIdx.x % 32;
  const float k0 = p.inv_tau * kLog2e;
  float top = -INFINITY;
  for (int k = lane; k < en.count; k += 32) top = en.q[k] != en.q[k] ? INFINITY : fmaxf(top, en.q[k]);   // NaN spoils the row
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float sum = 0.0f;
  for (int k = lane; k < en.count; k += 32) sum += en.q[k] == -INFINITY ? 0.0f : exp2_approx((en.q[k] - top) * k0);
  sum = warp_sum(sum);
  const float log_sum = top > -INFINITY ? logf(sum) : 0.0f;
  for (int k = lane; k < en.count; k += 32) {
    const float t = en.q[k];
    const float q = t == -INFINITY ? 0.0f : exp2_approx((t - top) * k0) / sum;
    if (q != 0.0f) {
      *q_log_q += q * ((t - top) * p.inv_tau - log_sum);
      *q_sum += q;
    }
    en.q[k] = q;
  }
  if (lane == 0) en.q[en.count] = 0.0f;
}
// The row's loss from sum q (z - m) / tau, the label's z - m, and the row's maximum m and log2 sums: log p =
// c (z - m) - log s, differences from the maximum, so that logits far from zero cost the loss no digits.
__device__ __forceinline__ void write_loss(const DistillParams& p, int64_t r, bool hard, float q_log_q, float q_sum, float cross, float label,
                                           float m, float l0, float l1) {
  const float kl = q_log_q - cross + q_sum * (l0 * kLn2);
  float loss = p.w_teacher != 0.0f && (q_sum > 0.0f || q_sum != q_sum) ? p.w_teacher * p.tau * p.tau * kl : 0.0f;
  if (hard) loss += p.w_label * (l1 * kLn2 - label);
  p.loss[r] = loss;
  p.lse[r] = m * p.inv_tau + l0 * kLn2;
  p.lse[p.rows + r] = p.labels ? m + l1 * kLn2 : 0.0f;
}

// All threads of a block; with _or, whether x holds for any of them.
__device__ __forceinline__ bool row_sync_or(bool x) { return __syncthreads_or(x); }
__device__ __forceinline__ void row_sync() { __syncthreads(); }

// Joins the block's threads; every thread gets the result, and whether `some` held for any.
template <bool kTwo>
__device__ __forceinline__ SoftSum join_block(SoftSum mine, SoftSum* warps, float k0, float k1, bool* some) {
  static_assert(kDistillMaxCluster == 8, "eight lanes join a cluster");
  mine = join_lanes<32, kTwo>(mine, k0, k1);
  if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = mine;
  *some = row_sync_or(*some);
  return join_lanes<kDistillWarps, kTwo>(warps[threadIdx.x % kDistillWarps], k0, k1);
}

// Sums travel between the blocks of a cluster as asynchronous stores into the receiver's `part`, which count
// towards its barrier: nobody waits for more than the sums.
__device__ __forceinline__ void send_sums(const SoftSum& v, DistillShared& sh, int rank, int size) {
  if (threadIdx.x == 0) mbar_expect(smem_addr(&sh.exchanged), size * sizeof(float4));
  if ((int)threadIdx.x >= size) return;
  const uint32_t to = peer_addr(smem_addr(&sh.part[rank]), threadIdx.x), at = peer_addr(smem_addr(&sh.exchanged), threadIdx.x);
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "f"(v.m),
               "f"(v.s0), "f"(v.s1), "f"(0.0f), "r"(at)
               : "memory");
}
// The cluster's sums in every thread; whether they came in time, which the block's warps may see differently. Where they did
// not they are NaN, and so is what follows from them: the warps go on to the same barriers without a branch on it, which cost
// 4 % of a step (1023 x 100003 FP32, two softmaxes: 187 us against 180).
template <bool kTwo>
__device__ __forceinline__ bool receive_sums(SoftSum* all, DistillShared& sh, int size, float k0, float k1, const Waiter& wait) {
  const int i = threadIdx.x % 8;
  const bool ok = __all_sync(0xffffffffu, wait(smem_addr(&sh.exchanged), 0));
  SoftSum one = {-INFINITY, 0.0f, 0.0f};
  if (i < size) {
    const float4 v = sh.part[i];
    one = SoftSum{v.x, v.y, v.z};
  }
  *all = join_lanes<8, kTwo>(one, k0, k1);
  if (!ok) all->s0 = all->s1 = __int_as_float(0x7fffffff);
  return ok;
}

// What a block needs of its place: the cluster's row and the block's 16-byte chunks [lo, hi) of it, of which
// [mid_lo, mid_lo + n) are whole; the row's first and last chunk may not be.
template <typename T>
struct Slice {
  int rank, size, n;
  int64_t r;
  Row<T> row;
  int64_t lo, hi, mid_lo;
  const uint4* mid;
  __device__ Slice(const DistillParams& p, int size_, int rank_, int64_t r_) : Slice(p, size_, rank_, r_, p.chunks_per_block) {}
  __device__ Slice(const DistillParams& p, int size_, int rank_, int64_t r_, int64_t per_block)
      : rank(rank_), size(size_), r(r_), row(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab) {
    const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
    lo = rank * per_block;
    hi = lo + per_block < chunks ? lo + per_block : chunks;
    if (lo > hi) lo = hi;
    mid_lo = lo < hi && !row.whole(lo) ? lo + 1 : lo;
    n = (int)((hi > mid_lo && !row.whole(hi - 1) ? hi - 1 : hi) - mid_lo);
    mid = reinterpret_cast<const uint4*>(row.z + row.first(mid_lo));
  }
  // f(which, chunk) for the partial chunks, each by one thread
  template <typename F>
  __device__ void edges(F f) const {
    if (threadIdx.x == 32 && mid_lo > lo) f(0, lo);
    if (threadIdx.x == 64 && mid_lo + n < hi) f(1, hi - 1);
  }
};

// Gradient of one value from its difference d to the row's maximum.
struct GradFactors {
  float k0, k1, l0, l1, f0, f1;   // f0 exp2(k0 d - l0) + f1 exp2(k1 d - l1)
};
template <typename T, bool kTwo>
__device__ __forceinline__ void gradients(uint4 a, float m, const GradFactors& f, float* g) {
  constexpr int P = Logit<T>::kPer;
  uint64_t v[P / 2];
  Logit<T>::unpack(a, v);
  const uint64_t minus = pair(-m, -m);
#pragma unroll
  for (int e = 0; e < P / 2; ++e) {
    const uint64_t d = add2(v[e], minus);
    uint64_t out = mul2(exp2_pair(fma2(d, pair(f.k0, f.k0), pair(-f.l0, -f.l0))), pair(f.f0, f.f0));
    if (kTwo) out = fma2(exp2_pair(fma2(d, pair(f.k1, f.k1), pair(-f.l1, -f.l1))), pair(f.f1, f.f1), out);
    split(out, &g[2 * e], &g[2 * e + 1]);
  }
}
// A chunk's gradient value by value: partial chunks, and rows whose gradient lies on another address grid.
template <typename T, bool kTwo>
__device__ __forceinline__ void write_values(const Row<T>& row, T* dz, int64_t c, uint4 a, float m, const GradFactors& f) {
  float g[Logit<T>::kPer];
  gradients<T, kTwo>(a, m, f, g);
  const int64_t first = row.first(c);
#pragma unroll
  for (int e = 0; e < Logit<T>::kPer; ++e)
    if (first + e >= 0 && first + e < row.vocab) Logit<T>::store(dz + first + e, g[e]);
}
// Walks a slice's whole chunks, U per thread and turn, with the next turn's loads issued before this
// turn's work: work(first chunk, chunks, how many of them exist); the others hold -inf.
template <typename T, int U, typename L, typename W>
__device__ __forceinline__ void stream_chunks(int n, L load, W work) {
  constexpr int kStep = kDistillThreads * U;
  uint4 a[U], b[U];
  const auto fetch = [&](int i0, uint4* to) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kDistillThreads;
      to[u] = i < n ? load(i) : Logit<T>::lowest();
    }
  };
  int i0 = threadIdx.x;
  if (i0 < n) fetch(i0, a);
  for (; i0 < n; i0 += kStep) {
    fetch(i0 + kStep, b);
    work(i0, a, n);
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = b[u];
  }
}
// The gradient of a slice's whole chunks.
template <typename T, bool kTwo, int U>
__device__ __forceinline__ void write_slice(const Slice<T>& s, T* dz, float m, const GradFactors& f) {
  const bool same_grid = (reinterpret_cast<uintptr_t>(dz) & 15u) == (reinterpret_cast<uintptr_t>(s.row.z) & 15u);
  uint4* out = reinterpret_cast<uint4*>(dz + s.row.first(s.mid_lo));
  const auto load = [&](int i) { return ld_stream(s.mid + i); };
  if (same_grid) {
    stream_chunks<T, U>(s.n, load, [&](int i0, const uint4* a, int n) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * kDistillThreads;
        if (i >= n) continue;
        float g[Logit<T>::kPer];
        gradients<T, kTwo>(a[u], m, f, g);
        st_stream(out + i, Logit<T>::pack(g));
      }
    });
  } else {
    for (int i = threadIdx.x; i < s.n; i += kDistillThreads) write_values<T, kTwo>(s.row, dz, s.mid_lo + i, load(i), m, f);
  }
}
// The values of the slice with a teacher entry or the label, after the block's other stores: the first
// entry of each id adds up its repeats.
template <typename T, bool kTwo>
__device__ __forceinline__ void write_entries(const Slice<T>& s, T* dz, const Entries& en, float m, const GradFactors& f, float a0, float a1) {
  const int64_t own_lo = s.row.first(s.lo), own_hi = s.row.first(s.hi);
  const int label = en.id[en.count];
  for (int k = threadIdx.x; k <= en.count; k += kDistillThreads) {
    const int id = en.id[k];
    if (id < 0 || id < own_lo || id >= own_hi) continue;
    float q = 0.0f;
    bool leader = true;
    for (int j4 = 0; j4 <= en.count; j4 += 4) {   // the list is padded with absent entries
      const int4 four = *reinterpret_cast<const int4*>(en.id + j4);
      if (four.x != id && four.y != id && four.z != id && four.w != id) continue;
      for (int j = j4; j < j4 + 4; ++j)
        if (en.id[j] == id) {
          leader &= j >= k;
          q += en.q[j];
        }
    }
    if (!leader) continue;
    const float d = en.z[k] - m;
    float v = f.f0 * exp2_approx(fmaf(d, f.k0, -f.l0)) + (kTwo ? f.f1 * exp2_approx(fmaf(d, f.k1, -f.l1)) : 0.0f);
    v -= a0 * q;
    if (id == label) v -= a1;
    Logit<T>::store(dz + id, v);
  }
}
// a0 and a1: the weights of the teacher's and the label's terms in this row's gradient. Without a second softmax
// the terms share p.
template <bool kTwo>
__device__ __forceinline__ GradFactors factors(const DistillParams& p, float g, bool some, bool hard, float l0, float l1, float* a0, float* a1) {
  *a0 = some ? g * p.w_teacher * p.tau : 0.0f;
  *a1 = hard ? g * p.w_label : 0.0f;
  return GradFactors{p.inv_tau * kLog2e, kLog2e, l0, l1, kTwo ? *a0 : *a0 + *a1, kTwo ? *a1 : 0.0f};
}

// Loss, and for a step the gradient in the same kernel: a row per block, or per cluster of blocks. kTwo: the softmax at
// temperature 1 is needed beside the one at tau (label term, tau != 1).
template <typename T, bool kTwo, bool kGradient, int U>
__global__ void __launch_bounds__(kDistillThreads, distill_min_blocks(U)) distill_row_kernel(const __grid_constant__ DistillParams p, int cluster) {
  extern __shared__ uint4 dynamic[];
  __shared__ DistillShared sh;
  __shared__ uint32_t dead;
  allow_next_kernel();
  if (cluster > 1) {
    if (threadIdx.x == 0) {
      mbar_init(smem_addr(&sh.exchanged), 1);
      dead = 0;
      mbar_init_fence();
    }
    cluster_sync();
  }
  wait_for_previous_kernel();
  const Slice<T> s(p, cluster, blockIdx.x % cluster, blockIdx.x / cluster);
  const Entries en(dynamic, p.entries);
  const float k0 = p.inv_tau * kLog2e, k1 = kLog2e;
  bool some = false;
  if (kGradient || s.rank == 0) some = fetch_entries<T>(p, s.r, s.row.z, en);
  SoftSum mine = {-INFINITY, 0.0f, 0.0f};
  stream_chunks<T, U>(s.n, [&](int i) { return kGradient ? s.mid[i] : ld_stream(s.mid + i); },
                   [&](int, const uint4* a, int) { accumulate<T, kTwo, U>(mine, a, k0, k1); });
  s.edges([&](int, int64_t c) {
    const uint4 a = s.row.load(c);
    accumulate<T, kTwo, 1>(mine, &a, k0, k1);
  });
  __syncwarp();
  mine = join_block<kTwo>(mine, sh.warp, k0, k1, &some);
  if (cluster > 1) send_sums(mine, sh, s.rank, s.size);
  float q_log_q = 0.0f, q_sum = 0.0f;
  if ((kGradient || s.rank == 0) && threadIdx.x < 32) teacher_softmax(p, en, &q_log_q, &q_sum);
  bool ok = true;
  if (cluster > 1) ok = receive_sums<kTwo>(&mine, sh, s.size, k0, k1, Waiter{&dead, p.error, p.polls});
  __syncwarp();
  const float m = finite_shift(mine.m), l0 = log2f(mine.s0), l1 = kTwo ? log2f(mine.s1) : l0;
  if (s.rank == 0 && threadIdx.x < 32) {
    float cross = 0.0f;
    for (int k = threadIdx.x; k < en.count; k += 32)
      if (en.q[k] != 0.0f) cross += en.q[k] * ((en.z[k] - m) * p.inv_tau);
    q_log_q = warp_sum(q_log_q);
    q_sum = warp_sum(q_sum);
    cross = warp_sum(cross);
    if (threadIdx.x == 0) write_loss(p, s.r, en.id[en.count] >= 0, q_log_q, q_sum, cross, en.z[en.count] - m, m, l0, l1);
  }
  if constexpr (kGradient) {
    float a0, a1;
    const GradFactors f = factors<kTwo>(p, p.row_grad ? p.row_grad[s.r] : 1.0f, some, en.id[en.count] >= 0, l0, l1, &a0, &a1);
    T* dz = static_cast<T*>(p.dz) + s.r * p.dz_stride;
    write_slice<T, kTwo, U>(s, dz, m, f);
    s.edges([&](int, int64_t c) { write_values<T, kTwo>(s.row, dz, c, s.row.load(c), m, f); });
    __syncthreads();   // the stores above come before those at the entries
    write_entries<T, kTwo>(s, dz, en, m, f, a0, a1);
  }
  if (cluster > 1) {   // nobody leaves while sums may still be sent to it
    cluster_sync();
    if (!ok) drain(smem_addr(&sh.exchanged), 0);
  }
}

// Sums of a whole row by one block, for rows whose saved lse is too far from zero.
template <typename T, bool kTwo>
static __device__ __noinline__ SoftSum row_sums(const DistillParams& p, int64_t r, SoftSum* warps) {
  const float k0 = p.inv_tau * kLog2e, k1 = kLog2e;
  const Slice<T> s(p, 1, 0, r, p.vocab);   // no row has more chunks than values
  SoftSum mine = {-INFINITY, 0.0f, 0.0f};
  stream_chunks<T, 1>(s.n, [&](int i) { return s.mid[i]; }, [&](int, const uint4* a, int) { accumulate<T, kTwo, 1>(mine, a, k0, k1); });
  s.edges([&](int, int64_t c) {
    const uint4 a = s.row.load(c);
    accumulate<T, kTwo, 1>(mine, &a, k0, k1);
  });
  __syncwarp();
  bool unused = false;
  return join_block<kTwo>(mine, warps, k0, k1, &unused);
}

// Gradient from the saved lse: blocks of a row share nothing. p = exp(z / tau - lse) has the relative error of lse's own
// rounding, |lse| 2^-25, and of differences of that size: (z - m) / tau - rest, with m where the exponent is zero, rounds no
// larger terms. Where that could be above 2 kFarLse 2^-25 = 8e-6, or lse has lost the sum altogether (a row of the type's
// lowest value: -3e38 + log vocab), or there is a NaN, the blocks of the row take its sums again instead.
constexpr float kFarLse = 128.0f;
template <typename T, bool kTwo>
__global__ void __launch_bounds__(kDistillThreads) distill_gradient_kernel(const __grid_constant__ DistillParams p, int parts) {
  start_after_previous_kernel();
  extern __shared__ uint4 dynamic[];
  __shared__ alignas(16) SoftSum warps[kDistillWarps];
  const Slice<T> s(p, parts, blockIdx.x % parts, blockIdx.x / parts);
  const Entries en(dynamic, p.entries);
  const float lse0 = p.lse[s.r], lse1 = kTwo ? p.lse[p.rows + s.r] : lse0;
  const bool some = __syncthreads_or(fetch_entries<T>(p, s.r, s.row.z, en));
  float m, l0, l1;
  if (fabsf(lse0) <= kFarLse && fabsf(lse1) <= kFarLse) {
    m = kTwo ? lse1 : lse0 * p.tau;
    l0 = fmaf(-m, p.inv_tau, lse0) * kLog2e;
    l1 = kTwo ? 0.0f : l0;
  } else {
    const SoftSum all = row_sums<T, kTwo>(p, s.r, warps);
    m = finite_shift(all.m);
    l0 = log2f(all.s0);
    l1 = kTwo ? log2f(all.s1) : l0;
    if (parts > 1) cluster_sync();   // the same lse, so all blocks of the row are here: nobody writes what another still reads
  }
  float a0, a1;
  const GradFactors f = factors<kTwo>(p, p.row_grad ? p.row_grad[s.r] : 1.0f, some, en.id[en.count] >= 0, l0, l1, &a0, &a1);
  T* dz = static_cast<T*>(p.dz) + s.r * p.dz_stride;
  write_slice<T, kTwo, kDistillUnroll>(s, dz, m, f);
  s.edges([&](int, int64_t c) { write_values<T, kTwo>(s.row, dz, c, s.row.load(c), m, f); });
  if (threadIdx.x < 32) {
    float unused = 0.0f;
    teacher_softmax(p, en, &unused, &unused);
  }
  __syncthreads();
  write_entries<T, kTwo>(s, dz, en, m, f, a0, a1);
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

int check_distill(const slidedp_distill_args* a) {
  if (!a || a->rows < 0 || a->rows > kMaxTokens || a->vocab < 1 || a->vocab > (1ll << 30) || a->entries < 0 ||
      a->entries > kMaxEntries || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) || a->logits_stride < 0)
    return SLIDEDP_ERR_INVALID_ARG;
  if (!positive_f32(a->temperature) || !positive_f32(1.0 / a->temperature) || !fits_f32(1.4426950408889634 / a->temperature) ||
      !fits_f32(a->w_teacher * a->temperature * a->temperature) || !fits_f32(a->w_teacher) || !fits_f32(a->w_label))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

// Blocks per row: one when the rows fill the device; when they do not, a row is cut, down to 8 KB. A step also cuts
// rows so that those being worked on (three blocks per SM) stay in L2 for their second reading: 4096 rows of
// 131072 BF16 logits, in 1 / 2 / 4 blocks each, 493 / 465 / 511 us (two blocks now 445).
constexpr int64_t kMinSliceBytes = 8 * 1024;
constexpr int64_t kEnoughBlocks = 148 * 4;
constexpr int64_t kWorkedOn = 148 * 3;
constexpr int64_t kResidentBytes = 96ll << 20;

unsigned blocks_per_row(int mode, int64_t rows, int64_t row_bytes) {
  unsigned n = 1;
  if (mode == kStep)
    while (n < (unsigned)kDistillMaxCluster && kWorkedOn * row_bytes > kResidentBytes * n) n *= 2;
  while (n < (unsigned)kDistillMaxCluster && rows * n < kEnoughBlocks && row_bytes >= 2 * kMinSliceBytes * n) n *= 2;
  return n;
}

int run_distill(slidedp_ctx* ctx, const slidedp_distill_args* a, int mode, const void* logits,
                const int32_t* ids, const float* t, const int32_t* labels, const float* row_grad, float* loss,
                float* lse, void* dz, cudaStream_t st) {
  if (!ctx || check_distill(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->rows == 0) return SLIDEDP_OK;
  const int64_t elem = a->dtype == SLIDEDP_F32 ? 4 : 2;
  const auto bad = [](const void* q, int64_t align) { return !q || reinterpret_cast<uintptr_t>(q) % (uintptr_t)align != 0; };
  if (bad(logits, elem) || bad(lse, 4) || (a->entries > 0 && (bad(ids, 4) || bad(t, 4)))) return SLIDEDP_ERR_INVALID_ARG;
  if (mode != kBackward && bad(loss, 4)) return SLIDEDP_ERR_INVALID_ARG;
  if (mode != kForward && (bad(dz, elem) || (a->rows > 1 && (a->d_logits_stride < a->vocab || (dz == logits && a->d_logits_stride != a->logits_stride))))) return SLIDEDP_ERR_INVALID_ARG;
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
  const unsigned cluster = blocks_per_row(mode, a->rows, chunks * 16);
  p.chunks_per_block = (chunks + cluster - 1) / cluster;
  p.error = ctx->kernel_error;
  p.polls = ctx->wait_polls;
  if ((int64_t)a->rows * cluster > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  const bool two = p.labels && a->temperature != 1.0;
  const bool f32 = a->dtype == SLIDEDP_F32;

  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  const size_t smem = Entries::bytes(a->entries);
  FAULT_POINT();
  const auto run = [&](auto kernel) {
    launch_after(kernel, (unsigned)(p.rows * cluster), kDistillThreads, smem, cluster, st, p, (int)cluster);
  };
#define SLIDEDP_KERNEL(KERNEL, ...) \
  (f32 ? (two ? run(KERNEL<float, true __VA_ARGS__>) : run(KERNEL<float, false __VA_ARGS__>)) \
       : (two ? run(KERNEL<uint16_t, true __VA_ARGS__>) : run(KERNEL<uint16_t, false __VA_ARGS__>)))
#define SLIDEDP_ALSO(x, u) , x, u
  const bool is_short = p.chunks_per_block * 16 <= kShortSliceBytes;
  if (mode == kForward) SLIDEDP_KERNEL(distill_row_kernel, SLIDEDP_ALSO(false, kDistillUnroll));
  else if (mode == kBackward) SLIDEDP_KERNEL(distill_gradient_kernel);
  else if (is_short) SLIDEDP_KERNEL(distill_row_kernel, SLIDEDP_ALSO(true, kDistillUnrollShort));
  else SLIDEDP_KERNEL(distill_row_kernel, SLIDEDP_ALSO(true, kDistillUnroll));
#undef SLIDEDP_ALSO
#undef SLIDEDP_KERNEL
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
