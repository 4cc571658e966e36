// libslidedp: distillation from a teacher's top logits with hard labels beside it: loss, gradient, and
// both in one pass. See include/slidedp_ops.h for the contract.
//
// With c = 1 / temperature, m = max z, s = sum exp(c (z - m)):  lse = c m + log s,  log p = c z - lse and
//   dz = g (w_t tau (p - q) + w_l (p1 - onehot)),   p1 the softmax at temperature 1.
// Bound: HBM. The logits are all that is large: forward reads them once, backward reads them and writes
// the gradient, and the step (both) reads and writes once because a row stays on chip between its two
// uses: a cluster of up to eight blocks holds it in shared memory (a row of 131072 BF16 logits is
// 256 KB, more than one SM has) and exchanges its maximum and sums through distributed shared memory.
#include "ops_internal.h"
#include "tcgen05.cuh"
#include "device_utils.cuh"

namespace slidedp {

constexpr int kMaxEntries = 512;        // teacher entries per row
constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kDistillMaxCluster = 8;
constexpr int kDistillUnroll = 8;       // 16-byte loads in flight per thread, from global memory
constexpr int kSmemUnroll = 4;          // and from shared memory
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
  int* error;              // pinned host word that a wait which runs out sets
};

template <typename T> struct Logit;
template <> struct Logit<uint16_t> {
  static constexpr int kPer = 8;   // values per 16 bytes
  static __device__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ void store(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
  // the four pairs of values of a chunk
  static __device__ uint64_t two(uint32_t a) { return pair(bf16_lo(a), bf16_hi(a)); }
  static __device__ void unpack(uint4 a, uint64_t* v) { v[0] = two(a.x); v[1] = two(a.y); v[2] = two(a.z); v[3] = two(a.w); }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
  static __device__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ float largest(uint4 a) {
    const uint32_t m = max2(max2(a.x, a.y), max2(a.z, a.w));
    return fmaxf(bf16_lo(m), bf16_hi(m));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
};
template <> struct Logit<float> {
  static constexpr int kPer = 4;
  static __device__ float load(const float* p) { return *p; }
  static __device__ void store(float* p, float v) { *p = v; }
  static __device__ void unpack(uint4 a, uint64_t* v) {
    v[0] = pair(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = pair(__uint_as_float(a.z), __uint_as_float(a.w));
  }
  static __device__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
  static __device__ float largest(uint4 a) {
    return fmaxf(fmaxf(__uint_as_float(a.x), __uint_as_float(a.y)), fmaxf(__uint_as_float(a.z), __uint_as_float(a.w)));
  }
  static __device__ uint4 lowest() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
};

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
  r.s0 = a.s0 * exp2_approx(shifted(a.m, r.m, k0)) + b.s0 * exp2_approx(shifted(b.m, r.m, k0));
  r.s1 = a.s1 * exp2_approx(shifted(a.m, r.m, k1)) + b.s1 * exp2_approx(shifted(b.m, r.m, k1));
  return r;
}
// Adds N chunks to a thread's sums. Differences are taken before they are scaled: the type's lowest value
// times a factor above one would be -inf.
template <typename T, bool kTwo, int N>
__device__ __forceinline__ void accumulate(SoftSum& mine, const uint4* a, float k0, float k1) {
  float top = mine.m;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, Logit<T>::largest(a[i]));
  const float shift = finite_shift(top);
  mine.s0 *= exp2_approx(shifted(mine.m, top, k0));
  if (kTwo) mine.s1 *= exp2_approx(shifted(mine.m, top, k1));
  mine.m = top;
  const uint64_t minus = pair(-shift, -shift), f0 = pair(k0, k0), f1 = pair(k1, k1);
  uint64_t s0 = 0, s1 = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint64_t v[Logit<T>::kPer / 2];
    Logit<T>::unpack(a[i], v);
#pragma unroll
    for (int e = 0; e < Logit<T>::kPer / 2; ++e) {
      const uint64_t d = add2(v[e], minus);
      float x, y;
      split(mul2(d, f0), &x, &y);
      s0 = add2(s0, pair(exp2_approx(x), exp2_approx(y)));
      if (kTwo) {
        split(mul2(d, f1), &x, &y);
        s1 = add2(s1, pair(exp2_approx(x), exp2_approx(y)));
      }
    }
  }
  float x, y;
  split(s0, &x, &y);
  mine.s0 += x + y;
  if (kTwo) {
    split(s1, &x, &y);
    mine.s1 += x + y;
  }
}

struct DistillShared {
  alignas(16) SoftSum warp[kDistillWarps];
  SoftSum part[kDistillMaxCluster];   // written by the blocks of the cluster
  alignas(8) uint64_t loaded;
  uint32_t dead;
  int some;                           // the row has a teacher term
};

// The row's entries (and, last, its label) in shared memory: id (-1: absent), teacher probability, the student's
// logit there.
struct Entries {
  int* id;
  float* q;
  float* z;
  int count;   // stored entries; the label sits at [count]
  __device__ Entries(void* smem, int n) : id(static_cast<int*>(smem)), q(reinterpret_cast<float*>(id + n + 1)), z(q + n + 1), count(n) {}
  static __host__ __device__ size_t bytes(int n) { return (size_t)(n + 1) * 12; }
};

// Fetches the entries with all threads of a block. The logits are read here, before any block writes a
// gradient, which may go to the same memory.
template <typename T>
__device__ __forceinline__ void fetch_entries(const DistillParams& p, int64_t r, const T* z, const Entries& en) {
  for (int k = threadIdx.x; k <= en.count; k += kDistillThreads) {
    const bool stored = k < en.count;
    int id = stored ? p.ids[r * en.count + k] : p.labels ? p.labels[r] : -1;
    const float t = stored ? p.t[r * en.count + k] : 0.0f;
    const bool ok = id >= 0 && id < p.vocab;
    en.id[k] = ok ? id : -1;
    en.z[k] = ok ? Logit<T>::load(z + id) : 0.0f;
    en.q[k] = stored && ok ? t : -INFINITY;
  }
}

// One warp turns the teacher's logits into probabilities, in place. Returns the lane's share of
// sum q log q and of sum q; log q = (t - max) / tau - log sum.
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ void teacher_softmax(const DistillParams& p, const Entries& en, float* q_log_q, float* q_sum, int* some) {
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
  if (lane == 0) {
    en.q[en.count] = 0.0f;
    *some = top > -INFINITY;
  }
}
// The same warp, once the row's maximum m and log2 sums are known: log p = c (z - m) - log s, differences
// from the maximum, so that logits far from zero cost the loss no digits.
__device__ __forceinline__ void write_loss(const DistillParams& p, int64_t r, const Entries& en, float q_log_q, float q_sum, float m,
                                           float l0, float l1) {
  const int lane = threadIdx.x % 32;
  float cross = 0.0f;
  for (int k = lane; k < en.count; k += 32)
    if (en.q[k] != 0.0f) cross += en.q[k] * ((en.z[k] - m) * p.inv_tau);
  const float total = warp_sum(q_sum), kl = warp_sum(q_log_q) - warp_sum(cross) + total * (l0 * kLn2);
  if (lane == 0) {
    float loss = p.w_teacher != 0.0f && (total > 0.0f || total != total) ? p.w_teacher * p.tau * p.tau * kl : 0.0f;
    if (en.id[en.count] >= 0) loss += p.w_label * (l1 * kLn2 - (en.z[en.count] - m));
    p.loss[r] = loss;
    p.lse[r] = m * p.inv_tau + l0 * kLn2;
    p.lse[p.rows + r] = p.labels ? m + l1 * kLn2 : 0.0f;
  }
}

// Joins the block's threads, leaving the result with every thread of warp 0.
__device__ __forceinline__ SoftSum join_block(SoftSum mine, SoftSum* warps, float k0, float k1) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    SoftSum other;
    other.m = __shfl_xor_sync(0xffffffffu, mine.m, o);
    other.s0 = __shfl_xor_sync(0xffffffffu, mine.s0, o);
    other.s1 = __shfl_xor_sync(0xffffffffu, mine.s1, o);
    mine = join(mine, other, k0, k1);
  }
  if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = mine;
  __syncthreads();
  if (threadIdx.x < 32) {
    mine = warps[0];
#pragma unroll
    for (int i = 1; i < kDistillWarps; ++i) mine = join(mine, warps[i], k0, k1);
  }
  return mine;
}

// The cluster's barrier in two halves, and a block's sums sent to the same place in another block.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void send(SoftSum* place, const SoftSum& v, int block) {
  uint32_t to;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(place)), "r"(block));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(v.m) : "memory");
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(v.s0) : "memory");
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 8), "f"(v.s1) : "memory");
}
// Exchanges the blocks' sums; cluster_arrive has been called once before, at the start of the kernel (a
// block's shared memory may be written once the block runs).
__device__ __forceinline__ SoftSum join_cluster(SoftSum mine, DistillShared& sh, int rank, int size, float k0, float k1) {
  cluster_wait();
  if ((int)threadIdx.x < size) send(&sh.part[rank], mine, threadIdx.x);   // threads of warp 0 hold the block's sums
  cluster_arrive();
  cluster_wait();
  SoftSum all = sh.part[0];
  for (int i = 1; i < size; ++i) all = join(all, sh.part[i], k0, k1);
  return all;
}

// What a block needs of its place: the cluster's row and the block's 16-byte chunks [lo, hi) of it.
template <typename T>
struct Slice {
  int rank, size;
  int64_t r;
  Row<T> row;
  int64_t lo, hi;
  __device__ Slice(const DistillParams& p, int size_)
      : rank((int)(blockIdx.x % size_)), size(size_), r(blockIdx.x / size_), row(static_cast<const T*>(p.z) + r * p.z_stride, p.vocab) {
    const int64_t chunks = (p.vocab + row.head + Logit<T>::kPer - 1) / Logit<T>::kPer;
    lo = rank * p.chunks_per_block;
    hi = lo + p.chunks_per_block < chunks ? lo + p.chunks_per_block : chunks;
    if (lo > hi) lo = hi;
  }
};

// Gradient of one value from its difference d to the row's maximum.
struct GradFactors {
  float k0, k1, l0, l1, f0, f1;   // f0 exp2(k0 d - l0) + f1 exp2(k1 d - l1)
};
template <typename T, bool kTwo>
__device__ __forceinline__ void write_chunk(const Row<T>& row, T* dz, bool same_grid, int64_t c, uint4 a, float m, const GradFactors& f) {
  constexpr int P = Logit<T>::kPer;
  uint64_t v[P / 2];
  float g[P];
  Logit<T>::unpack(a, v);
  const uint64_t minus = pair(-m, -m);
#pragma unroll
  for (int e = 0; e < P / 2; ++e) {
    const uint64_t d = add2(v[e], minus);
    float x, y;
    split(fma2(d, pair(f.k0, f.k0), pair(-f.l0, -f.l0)), &x, &y);
    uint64_t out = mul2(pair(exp2_approx(x), exp2_approx(y)), pair(f.f0, f.f0));
    if (kTwo) {
      split(fma2(d, pair(f.k1, f.k1), pair(-f.l1, -f.l1)), &x, &y);
      out = fma2(pair(exp2_approx(x), exp2_approx(y)), pair(f.f1, f.f1), out);
    }
    split(out, &g[2 * e], &g[2 * e + 1]);
  }
  const int64_t first = row.first(c);
  if (same_grid && first >= 0 && first + P <= row.vocab) {
    st_stream(dz + first, Logit<T>::pack(g));
  } else {
#pragma unroll
    for (int e = 0; e < P; ++e)
      if (first + e >= 0 && first + e < row.vocab) Logit<T>::store(dz + first + e, g[e]);
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
    for (int j = 0; j <= en.count; ++j) {
      const bool same = en.id[j] == id;
      if (same && j < k) leader = false;
      if (same) q += en.q[j];
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
__device__ __forceinline__ GradFactors factors(const DistillParams& p, int64_t r, bool some, bool hard, float l0, float l1, float* a0, float* a1) {
  const float g = p.row_grad ? p.row_grad[r] : 1.0f;
  *a0 = some ? g * p.w_teacher * p.tau : 0.0f;
  *a1 = hard ? g * p.w_label : 0.0f;
  return GradFactors{p.inv_tau * kLog2e, kLog2e, l0, l1, kTwo ? *a0 : *a0 + *a1, kTwo ? *a1 : 0.0f};
}

// Loss: a row per block, or per cluster of blocks when there are few rows. kTwo: the softmax at temperature 1
// is needed beside the one at tau (label term, tau != 1).
template <typename T, bool kTwo>
__global__ void __launch_bounds__(kDistillThreads) distill_loss_kernel(const __grid_constant__ DistillParams p, int cluster) {
  extern __shared__ uint4 dynamic[];
  __shared__ DistillShared sh;
  if (cluster > 1) cluster_arrive();
  const Slice<T> s(p, cluster);
  const Entries en(dynamic, p.entries);
  const float k0 = p.inv_tau * kLog2e, k1 = kLog2e;
  SoftSum mine = {-INFINITY, 0.0f, 0.0f};
  bool fetched = false;
  for (int64_t c0 = s.lo + threadIdx.x; c0 < s.hi; c0 += (int64_t)kDistillThreads * kDistillUnroll) {
    uint4 a[kDistillUnroll];
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i) {
      const int64_t c = c0 + (int64_t)i * kDistillThreads;
      a[i] = c < s.hi ? s.row.load(c) : Logit<T>::lowest();
    }
    if (!fetched && s.rank == 0) fetch_entries<T>(p, s.r, s.row.z, en);   // behind the first loads of the row
    fetched = true;
    accumulate<T, kTwo, kDistillUnroll>(mine, a, k0, k1);
  }
  if (!fetched && s.rank == 0) fetch_entries<T>(p, s.r, s.row.z, en);
  SoftSum all = join_block(mine, sh.warp, k0, k1);
  if (cluster > 1) all = join_cluster(all, sh, s.rank, s.size, k0, k1);
  if (s.rank == 0 && threadIdx.x < 32) {
    float q_log_q = 0.0f, q_sum = 0.0f;
    teacher_softmax(p, en, &q_log_q, &q_sum, &sh.some);
    __syncwarp();
    const float l0 = log2f(all.s0);
    write_loss(p, s.r, en, q_log_q, q_sum, finite_shift(all.m), l0, kTwo ? log2f(all.s1) : l0);
  }
}

// Gradient from the saved lse: blocks of a row share nothing.
template <typename T, bool kTwo>
__global__ void __launch_bounds__(kDistillThreads) distill_gradient_kernel(const __grid_constant__ DistillParams p, int parts) {
  extern __shared__ uint4 dynamic[];
  __shared__ DistillShared sh;
  const Slice<T> s(p, parts);
  const Entries en(dynamic, p.entries);
  fetch_entries<T>(p, s.r, s.row.z, en);
  const float l0 = p.lse[s.r] * kLog2e, l1 = p.labels ? p.lse[p.rows + s.r] * kLog2e : l0;
  __syncthreads();
  if (threadIdx.x < 32) {
    float unused = 0.0f;
    teacher_softmax(p, en, &unused, &unused, &sh.some);
  }
  __syncthreads();
  float a0, a1;
  const GradFactors f = factors<kTwo>(p, s.r, sh.some, en.id[en.count] >= 0, l0, l1, &a0, &a1);
  T* dz = static_cast<T*>(p.dz) + s.r * p.dz_stride;
  const bool same_grid = (reinterpret_cast<uintptr_t>(dz) & 15u) == (reinterpret_cast<uintptr_t>(s.row.z) & 15u);
  for (int64_t c0 = s.lo + threadIdx.x; c0 < s.hi; c0 += (int64_t)kDistillThreads * kSmemUnroll) {
    uint4 a[kSmemUnroll];
#pragma unroll
    for (int i = 0; i < kSmemUnroll; ++i) {
      const int64_t c = c0 + (int64_t)i * kDistillThreads;
      if (c < s.hi) a[i] = s.row.load(c);
    }
#pragma unroll
    for (int i = 0; i < kSmemUnroll; ++i) {
      const int64_t c = c0 + (int64_t)i * kDistillThreads;
      if (c < s.hi) write_chunk<T, kTwo>(s.row, dz, same_grid, c, a[i], 0.0f, f);
    }
  }
  __syncthreads();
  write_entries<T, kTwo>(s, dz, en, 0.0f, f, a0, a1);
}

// Loss and gradient in one pass: the block's slice is copied to shared memory by one bulk copy while the
// teacher's entries are worked on, summed from there, and used a second time for the gradient.
template <typename T, bool kTwo>
__global__ void __launch_bounds__(kDistillThreads, 5) distill_step_kernel(const __grid_constant__ DistillParams p, int cluster) {
  extern __shared__ uint4 dynamic[];
  __shared__ DistillShared sh;
  if (cluster > 1) cluster_arrive();
  const Slice<T> s(p, cluster);
  uint4* keep = dynamic;
  const Entries en(dynamic + p.chunks_per_block, p.entries);
  const float k0 = p.inv_tau * kLog2e, k1 = kLog2e;

  // the row's first and last chunk may be partial: those come by element
  const int64_t w_lo = s.lo < s.hi && !s.row.whole(s.lo) ? s.lo + 1 : s.lo;
  const int64_t w_hi = s.hi > w_lo && !s.row.whole(s.hi - 1) ? s.hi - 1 : s.hi;
  if (threadIdx.x == 0) {
    mbar_init(smem_addr(&sh.loaded), 1);
    sh.dead = 0;
    mbar_init_fence();
    if (w_lo < w_hi) {
      mbar_expect(smem_addr(&sh.loaded), (uint32_t)(w_hi - w_lo) * 16);
      bulk_load(smem_addr(keep + (w_lo - s.lo)), s.row.z + s.row.first(w_lo), (uint32_t)(w_hi - w_lo) * 16, smem_addr(&sh.loaded));
    }
  }
  if (threadIdx.x == 32 && w_lo > s.lo) keep[0] = s.row.load(s.lo);
  if (threadIdx.x == 64 && w_hi < s.hi) keep[w_hi - s.lo] = s.row.load(w_hi);
  fetch_entries<T>(p, s.r, s.row.z, en);
  __syncthreads();
  float q_log_q = 0.0f, q_sum = 0.0f;
  if (threadIdx.x < 32) teacher_softmax(p, en, &q_log_q, &q_sum, &sh.some);
  if (w_lo < w_hi) (void)Waiter{&sh.dead, p.error}(smem_addr(&sh.loaded), 0);

  SoftSum mine = {-INFINITY, 0.0f, 0.0f};
  for (int64_t c0 = s.lo + threadIdx.x; c0 < s.hi; c0 += kDistillThreads * kSmemUnroll) {
    uint4 a[kSmemUnroll];
#pragma unroll
    for (int i = 0; i < kSmemUnroll; ++i) {
      const int64_t c = c0 + i * kDistillThreads;
      a[i] = c < s.hi ? keep[c - s.lo] : Logit<T>::lowest();
    }
    accumulate<T, kTwo, kSmemUnroll>(mine, a, k0, k1);
  }
  SoftSum all = join_block(mine, sh.warp, k0, k1);
  if (cluster == 1) {
    if (threadIdx.x == 0) sh.part[0] = all;
    __syncthreads();
    all = sh.part[0];
  } else {
    all = join_cluster(all, sh, s.rank, s.size, k0, k1);
  }
  const float m = finite_shift(all.m), l0 = log2f(all.s0), l1 = kTwo ? log2f(all.s1) : l0;
  if (s.rank == 0 && threadIdx.x < 32) write_loss(p, s.r, en, q_log_q, q_sum, m, l0, l1);

  float a0, a1;
  const GradFactors f = factors<kTwo>(p, s.r, sh.some, en.id[en.count] >= 0, l0, l1, &a0, &a1);
  T* dz = static_cast<T*>(p.dz) + s.r * p.dz_stride;
  const bool same_grid = (reinterpret_cast<uintptr_t>(dz) & 15u) == (reinterpret_cast<uintptr_t>(s.row.z) & 15u);
  for (int64_t c = s.lo + threadIdx.x; c < s.hi; c += kDistillThreads)
    write_chunk<T, kTwo>(s.row, dz, same_grid, c, keep[c - s.lo], m, f);
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
  if (!(a->temperature > 0.0) || !is_finite(a->temperature) || !is_finite(1.0 / a->temperature) || !is_finite(a->w_teacher) ||
      !is_finite(a->w_label))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

template <typename K>
cudaError_t launch_distill(K kernel, const DistillParams& p, unsigned blocks_per_row, bool clustered, size_t smem, cudaStream_t st) {
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.rows * blocks_per_row);
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks_per_row;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = clustered && blocks_per_row > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p, (int)blocks_per_row);
}

// Blocks per row. A step holds its row in shared memory: as many blocks as leave each about 32 KB (five
// blocks per SM, so that one's loads run beside another's arithmetic and stores). Loss and gradient alone
// stream a row through one block when the rows fill the device, and cut it, down to 8 KB, when they do
// not.
constexpr int64_t kSliceBytes = 32 * 1024;
constexpr int64_t kMaxSliceBytes = 200 * 1024;
constexpr int64_t kMinSliceBytes = 8 * 1024;
constexpr int64_t kEnoughBlocks = 148 * 4;

unsigned blocks_per_row(int mode, int64_t rows, int64_t row_bytes) {
  unsigned n = 1;
  if (mode == kStep) {
    while (n < (unsigned)kDistillMaxCluster && row_bytes > kSliceBytes * n) n *= 2;
  }
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
  const unsigned cluster = blocks_per_row(mode, a->rows, chunks * 16);
  p.chunks_per_block = (chunks + cluster - 1) / cluster;
  p.error = ctx->kernel_error;
  if ((int64_t)a->rows * cluster > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  const bool two = p.labels && a->temperature != 1.0;
  const bool f32 = a->dtype == SLIDEDP_F32;

  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  // A row too long for a cluster's shared memory is read twice: forward, then backward.
  if (mode == kStep && p.chunks_per_block * 16 > kMaxSliceBytes) {
    const int first = run_distill(ctx, a, kForward, logits, ids, t, labels, nullptr, loss, lse, nullptr, st);
    return first != SLIDEDP_OK ? first : run_distill(ctx, a, kBackward, logits, ids, t, labels, row_grad, nullptr, lse, dz, st);
  }
  const size_t smem = (mode == kStep ? (size_t)p.chunks_per_block * 16 : 0) + Entries::bytes(a->entries);
  FAULT_POINT();
  cudaError_t e;
#define SLIDEDP_LAUNCH(KERNEL)                                                                           \
  e = f32 ? (two ? launch_distill(KERNEL<float, true>, p, cluster, mode != kBackward, smem, st)          \
                 : launch_distill(KERNEL<float, false>, p, cluster, mode != kBackward, smem, st))        \
          : (two ? launch_distill(KERNEL<uint16_t, true>, p, cluster, mode != kBackward, smem, st)       \
                 : launch_distill(KERNEL<uint16_t, false>, p, cluster, mode != kBackward, smem, st))
  switch (mode) {
    case kForward: SLIDEDP_LAUNCH(distill_loss_kernel); break;
    case kBackward: SLIDEDP_LAUNCH(distill_gradient_kernel); break;
    default: SLIDEDP_LAUNCH(distill_step_kernel); break;
  }
#undef SLIDEDP_LAUNCH
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
