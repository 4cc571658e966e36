// libslidedp: the norms before and after a block with its gate and residual. See include/slidedp_ops.h for the contract.
//
// n = y r w_post, x' = x + a g n, h = x' r' w_pre with r = rsqrt(mean y^2 + eps), r' = rsqrt(mean x'^2 + eps). Backward:
//   u = dh w_pre, d = dx' + r' (u - x' r'^2 mean(u x')), dx = d
//   v = a d g w_post, dy = r (v - y r mean(v y r)), dgate = a d n g', dw_pre = sum dh x' r', dw_post = sum a d g y r
// Bound: HBM; every tensor is read or written once, and x' is computed anew backward rather than kept. Blocks stay, one per SM, and take
// row after row, with the sums of the weights' gradients; each has one partial row of them, which a second kernel adds in
// a fixed order. Rows of up to 8192 columns are copied into shared memory ahead of their use, wider ones are read as they are needed.
#include "ops_internal.h"
#include "rows.cuh"
#include "tcgen05.cuh"

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

__device__ __forceinline__ float sigmoid(float x) { return rcp_approx(1.0f + __expf(-x)); }

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

// ---- wide rows ----------------------------------------------------------------------------------------------
// Rows that the rings below have no room for: more than 8192 columns, or FP32 ones close to that with a token's gate. A block of up to
// 1024 threads takes a row, 16 values per thread.

constexpr int kWideThreads = 1024, kWideValues = 16;

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

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
template <typename T, int V>
__device__ __forceinline__ void get_vector(const void* row, int64_t at, float* v) {
  to_floats<T, V>(*reinterpret_cast<const typename Raw<T, V>::type*>(static_cast<const T*>(row) + at), v);
}
// The factor a g w_post of y r of one vector, and the gate.
template <typename T, int V, bool kToken>
__device__ __forceinline__ void wide_factor(const BlockNormParams& p, int64_t row, int col, float* f, float* g) {
#pragma unroll
  for (int e = 0; e < V; ++e) f[e] = 1.0f;
  if (p.w_post) get_vector<T, V>(p.w_post, col, f);
#pragma unroll
  for (int e = 0; e < V; ++e) f[e] *= p.alpha;
  if (!kToken && !p.gate_kind) return;
  get_vector<T, V>(p.gate.p, kToken ? row * p.gate.stride + col : col, g);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (p.sigmoid) g[e] = sigmoid(g[e]);
    f[e] *= g[e];
  }
}
// What is read of a row, to L2.
template <typename T, bool kToken>
__device__ __forceinline__ void fetch_row(const BlockNormParams& p, int64_t row) {
  if (row >= p.tokens) return;
  const int step = 128 / (int)sizeof(T), last = p.hidden - 1;
  for (int c = threadIdx.x * step; c < p.hidden + step; c += blockDim.x * step) {
    const int col = c < last ? c : last;
    const auto line = [&](const NormView& v) {
      if (v.p) prefetch_l2(static_cast<const T*>(v.p) + row * v.stride + col);
    };
    line(p.x);
    line(p.y);
    line(p.dx_out);
    line(p.dh);
    if (kToken) line(p.gate);
  }
}

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

// kToken: the gate is [tokens, hidden]. Each thread has its columns to itself, with the weights in registers, so rows may be written
// where they were read. 2048 x 16384 BF16, both norms: 53 us (61 without fetching the next row to L2).
template <typename T, int V, bool kToken>
__global__ void __launch_bounds__(kWideThreads) block_norm_kernel(const __grid_constant__ BlockNormParams p) {
  start_after_previous_kernel();
  __shared__ BlockSums sh;
  constexpr int N = kWideValues;
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
    fetch_row<T, kToken>(p, row + gridDim.x);
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

// A row's values are read where a sum asks for them, by then from L2, into which each row is fetched while the one before it is
// computed: x' and y stay in registers, all of the row and the weights would not (64 for each of 1024 threads), and the sums of the
// weights' gradients lie in shared memory. 2048 x 16384 BF16, both norms: 170 us; with everything in registers, spilled, 934.
template <typename T, int V, bool kToken>
__global__ void __launch_bounds__(kWideThreads) block_norm_backward_kernel(const __grid_constant__ BlockNormParams p) {
  extern __shared__ uint4 dynamic[];
  start_after_previous_kernel();
  __shared__ BlockSums sh;
  constexpr int N = kWideValues, K = N / V;
  int turn = 0;
  const int n = blockDim.x, t = threadIdx.x;
  float *sum_post = reinterpret_cast<float*>(dynamic) + t, *sum_pre = sum_post + N * n;     // value i at i n
  if (p.partial) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum_post[i * n] = sum_pre[i * n] = 0.0f;
  }
  fetch_row<T, kToken>(p, blockIdx.x);
  for (int64_t row = blockIdx.x; row < p.tokens; row += gridDim.x) {
    fetch_row<T, kToken>(p, row + gridDim.x);
    Values<T, V, N> raw_y;
    float r = 1.0f, r2 = 0.0f, m = 0.0f, x[N];       // x', then v
    if (p.has_y) {
      raw_y.load(p.y.p, row * p.y.stride, p.hidden);
      if (p.post) {
        float s = 0.0f, y[N];
        raw_y.get(y);
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(y[i], y[i], s);
        r = rsqrtf(block_sums(s, 0.0f, sh, turn).x * p.inv_hidden + p.eps);
      }
    }
    if (p.pre) {
      float ss = 0.0f, ux = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int col = (k * n + t) * V;
        float *xk = x + k * V, f[V], g[V], y[V], h[V], w[V];
        if (col >= p.hidden) continue;
        get_vector<T, V>(p.x.p, row * p.x.stride + col, xk);
        if (p.has_y) {
          wide_factor<T, V, kToken>(p, row, col, f, g);
          to_floats<T, V>(raw_y.a[k], y);
#pragma unroll
          for (int e = 0; e < V; ++e) xk[e] = fmaf(f[e], y[e] * r, xk[e]);
        }
        get_vector<T, V>(p.dh.p, row * p.dh.stride + col, h);
        if (p.w_pre) get_vector<T, V>(p.w_pre, col, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ss = fmaf(xk[e], xk[e], ss);
          ux = fmaf(p.w_pre ? h[e] * w[e] : h[e], xk[e], ux);
        }
      }
      const float2 s = block_sums(ss, ux, sh, turn);
      r2 = rsqrtf(s.x * p.inv_hidden + p.eps);
      m = s.y * r2 * p.inv_hidden;
    }
    float dot = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * n + t) * V;
      if (col >= p.hidden) continue;
      float *v = x + k * V, d[V] = {}, f[V], g[V], y[V], h[V], w[V];
      if (p.dx_out.p) get_vector<T, V>(p.dx_out.p, row * p.dx_out.stride + col, d);
      if (p.pre) {
        get_vector<T, V>(p.dh.p, row * p.dh.stride + col, h);
        if (p.w_pre) get_vector<T, V>(p.w_pre, col, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float xh = v[e] * r2;
          if (p.partial) sum_pre[(k * V + e) * n] += h[e] * xh;
          d[e] = fmaf(r2, fmaf(-xh, m, p.w_pre ? h[e] * w[e] : h[e]), d[e]);
        }
      }
      if (p.has_y) {
        wide_factor<T, V, kToken>(p, row, col, f, g);                       // before this vector of dx or dgate may take its place
        if (kToken && p.dgate.p && p.w_post) get_vector<T, V>(p.w_post, col, w);
        to_floats<T, V>(raw_y.a[k], y);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          y[e] *= r;
          const float ad = p.alpha * d[e];
          if (p.partial) sum_post[(k * V + e) * n] += (kToken ? ad * g[e] : ad) * y[e];
          v[e] = f[e] * d[e];
          dot = fmaf(v[e], y[e], dot);
          if (kToken) g[e] = ad * y[e] * (p.w_post ? w[e] : 1.0f) * (p.sigmoid ? g[e] * (1.0f - g[e]) : 1.0f);   // a d n g'
        }
        if (kToken && p.dgate.p) store_values<V>(static_cast<T*>(p.dgate.p) + row * p.dgate.stride + col, g);
      }
      store_values<V>(static_cast<T*>(p.dx.p) + row * p.dx.stride + col, d);
    }
    if (!p.has_y) continue;
    if (p.post) m = block_sums(dot, 0.0f, sh, turn).x * p.inv_hidden;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * n + t) * V;
      if (col >= p.hidden) continue;
      float* v = x + k * V;
      if (p.post) {
        float y[V];
        to_floats<T, V>(raw_y.a[k], y);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = r * fmaf(-(y[e] * r), m, v[e]);
      }
      store_values<V>(static_cast<T*>(p.dy.p) + row * p.dy.stride + col, v);
    }
  }
  if (!p.partial) return;
  float* at = p.partial + (int64_t)blockIdx.x * 2 * p.hidden;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int col = (i / V * n + t) * V + i % V;
    if (col >= p.hidden) continue;
    at[col] = sum_post[i * n];
    at[p.hidden + col] = sum_pre[i * n];
  }
}

// ---- rows in shared memory ---------------------------------------------------------------------------------
// A block per SM, of several groups of warps that work on a row each. Rows are copied in bulk into each group's ring ahead of their use,
// so that what is under way costs no registers. A thread has 16 columns of every row: 16-byte vectors where rows are aligned to
// them, else pairs or single ones, neighbours with neighbouring threads (8192 x 4098 BF16, both norms, 89 and 248 us in pairs, 134 and 373
// one by one; 8192 x 4097 110 and 359). The factors of y r and of x' r' lie before the rings in FP32, for all
// groups. Two values per instruction. What bounds a group is the chain of its two or three sums over the row (700 cycles each);
// what a row needs is kept in registers from one sum to the next, which leaves room for two groups of 256 threads (three, with
// 80 registers and values read again from shared memory, took 150 us backward where two take 87).
// 8192 x 4096 BF16, both norms: forward 96 us with rows in registers and no copies ahead, 54 as blocks with a ring each, 47 now
// (268 MB at 5.7 TB/s); backward 166, 95, 85.

__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ float sum_of(uint64_t v) {
  float a, b;
  split(v, &a, &b);
  return a + b;
}
__device__ __forceinline__ uint64_t sigmoid2(uint64_t v) {
  float a, b;
  split(v, &a, &b);
  return pair(sigmoid(a), sigmoid(b));
}

constexpr int kCols = 16;              // per thread
constexpr int kPairs = kCols / 2;

// A thread's columns: its warp's are behind one another, K times 32 vectors of V, of which each lane has one, so that their distances
// are known when this is compiled (with the group's vectors behind one another they took 16 registers for single columns: 452 bytes spilled). Columns behind the row
// are zeros: whole vectors have zeros behind their rows in shared memory, for shorter ones it is asked.
template <typename T, int V_>
struct Columns {
  static constexpr int V = V_, K = kCols / V, kStep = 32 * V;
  static constexpr bool kVector = V * sizeof(T) == 16;
  int t, n;          // thread of the group, and how many it has
  __device__ __forceinline__ int first() const { return t / 32 * (32 * kCols) + t % 32 * V; }
  __device__ __forceinline__ void load(const char* row, int hidden, uint64_t* v) const {
    const char* at = row + first() * sizeof(T);
    const int left = hidden - first();
    float one[2];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const char* p = at + k * kStep * sizeof(T);
      if constexpr (kVector) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[k * 4 + e] = pair(bf16_lo(w[e]), bf16_hi(w[e]));
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) v[k * 2 + e] = pair(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
        }
      } else if constexpr (V == 2) {
        const uint32_t a = k * kStep < left ? *reinterpret_cast<const uint32_t*>(p) : 0;
        v[k] = pair(bf16_lo(a), bf16_hi(a));
      } else {
        one[k % 2] = 0.0f;
        if (k * kStep < left) {
          if constexpr (sizeof(T) == 2) one[k % 2] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
          else one[k % 2] = *reinterpret_cast<const float*>(p);
        }
        if (k % 2) v[k / 2] = pair(one[0], one[1]);
      }
    }
  }
  // Factors lie as threads read them: the fours of a thread's values 32 fours apart (behind one another in a thread's own order,
  // vectors of eight would meet in the same banks: 94.7 -> 87.5 us backward).
  __device__ __forceinline__ int place() const { return t / 32 * (32 * kCols) + t % 32 * 4; }
  __device__ __forceinline__ void load_factors(const float* w, uint64_t* v) const {
    const float* at = w + place();
#pragma unroll
    for (int j = 0; j < kCols / 4; ++j) {
      const float4 a = *reinterpret_cast<const float4*>(at + j * 128);
      v[2 * j] = pair(a.x, a.y);
      v[2 * j + 1] = pair(a.z, a.w);
    }
  }
  __device__ __forceinline__ void store_factors(float* w, const uint64_t* v) const {
    float* at = w + place();
#pragma unroll
    for (int j = 0; j < kCols / 4; ++j) {
      float4 a;
      split(v[2 * j], &a.x, &a.y);
      split(v[2 * j + 1], &a.z, &a.w);
      *reinterpret_cast<float4*>(at + j * 128) = a;
    }
  }
  // Vector number k.
  __device__ __forceinline__ void get(const uint64_t* v, int k, float* f) const {
    if constexpr (V > 1) {
#pragma unroll
      for (int e = 0; e < V / 2; ++e) split(v[k * V / 2 + e], &f[2 * e], &f[2 * e + 1]);
    } else {
      float lo, hi;
      split(v[k / 2], &lo, &hi);
      f[0] = k % 2 ? hi : lo;
    }
  }
  template <typename O>
  __device__ __forceinline__ void store(O* row, int hidden, const uint64_t* v) const {
    O* at = row + first();
    const int left = hidden - first();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[V];
      get(v, k, f);
      if (k * kStep < left) store_values<V>(at + k * kStep, f);
    }
  }
  __device__ __forceinline__ void store_f32(float* row, int hidden, const uint64_t* v) const {
    float* at = row + first();
    const int left = hidden - first();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[V];
      get(v, k, f);
      if (k * kStep >= left) continue;
#pragma unroll
      for (int e = 0; e < V; ++e) at[k * kStep + e] = f[e];
    }
  }
};

__device__ __forceinline__ void group_sync(int group, int n) {
  if (n == (int)blockDim.x) return __syncthreads();      // the only group: a barrier known when it is compiled
  __syncwarp();
  if (n > 32) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(n) : "memory");
}
// Sums of up to two values over a group; the second is folded onto the upper lanes of its warps, and every thread adds the warps' sums
// itself. Calls take the halves of `part` in turn, so that one barrier is enough.
template <int kWarps>
__device__ __forceinline__ float2 group_sums(float a, float b, float2 (*part)[kWarps], int& turn, int t, int n, int group) {
  const bool upper = t & 16;
  float v = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (n == 32) {
    __syncwarp();        // all lanes have read what is copied over next
    return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
  }
  turn ^= 1;
  if (t % 16 == 0) reinterpret_cast<float*>(&part[turn][t / 32])[t / 16 % 2] = v;
  group_sync(group, n);
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < kWarps; w += 2) {
    const float4 x = *reinterpret_cast<const float4*>(&part[turn][w]);
    s = add2(s, add2(pair(x.x, x.y), pair(x.z, x.w)));
  }
  float2 r;
  split(s, &r.x, &r.y);
  return r;
}

// A thread's share of a row's sum of squares.
template <typename T, int V>
__device__ __forceinline__ float sum_squares(const Columns<T, V>& cols, const char* row, int hidden) {
  uint64_t v[kPairs], s = 0;
  cols.load(row, hidden, v);
#pragma unroll
  for (int e = 0; e < kPairs; ++e) s = fma2(v[e], v[e], s);
  return sum_of(s);
}

constexpr int kMaxNormStages = 4, kMaxGroups = 15;
constexpr int kMaxNormInputs = 5;
enum NormInput { kInX, kInY, kInGate, kInDx, kInDh };

struct NormFeed {
  const char* src[kMaxNormInputs];
  int64_t stride[kMaxNormInputs];    // bytes
  int slot[kMaxNormInputs];          // the row's place in a stage
  int inputs, stages, groups, group_threads;
  uint32_t row_bytes, slot_bytes;    // a slot has room for the row wherever in its first 16 bytes it begins
};
struct NormRingParams {
  BlockNormParams n;
  NormFeed feed;
  int* error;
  uint32_t polls;
};
struct NormRings {
  uint64_t full[kMaxGroups][kMaxNormStages];
  uint32_t dead;
};

// A group's ring from the side of one thread; row number i of the group goes to stage i % stages. Its first thread copies. A wait that
// runs out makes it stop copying, and the group goes on with what there is to its end: the call has failed, and says so.
template <bool kVector>
struct NormRows {
  const NormRingParams& p;
  uint64_t* full;
  uint32_t* dead;
  char* smem;
  int64_t first, step, count;    // rows of this group
  int64_t issued = 0, ready = 0;
  int stage = 0;                 // of the present row
  uint32_t parity = 0;
  bool ok = true;
  __device__ NormRows(const NormRingParams& p_, NormRings& rings, float* factors, int group) : p(p_), full(rings.full[group]), dead(&rings.dead) {
    smem = reinterpret_cast<char*>(factors + 2 * kCols * p.feed.group_threads) + (size_t)group * p.feed.stages * p.feed.inputs * p.feed.slot_bytes;
    first = (int64_t)group * gridDim.x + blockIdx.x;
    step = (int64_t)gridDim.x * p.feed.groups;
    count = p.n.tokens > first ? (p.n.tokens - 1 - first) / step + 1 : 0;
  }
  __device__ __forceinline__ char* slot(int s, int input) const { return smem + (s * p.feed.inputs + p.feed.slot[input]) * p.feed.slot_bytes; }
  // Rows that are not aligned are copied from the 16 bytes that hold their first value to those that hold their last, and lie in
  // their slot as they lie in memory. What else those hold belongs to the rows next to them; before the first row and behind the last
  // nothing is read, but value by value up to the next 16 bytes.
  __device__ __forceinline__ void issue_next() {   // the first thread
    if (!ok || issued >= count) return;
    const int s = (int)(issued % p.feed.stages);
    const int64_t row = first + issued * step;
    const uint32_t bar = smem_addr(&full[s]);
    if constexpr (kVector) {
      mbar_expect(bar, p.feed.inputs * p.feed.row_bytes);
#pragma unroll
      for (int i = 0; i < kMaxNormInputs; ++i)
        if (p.feed.src[i]) bulk_load(smem_addr(slot(s, i)), p.feed.src[i] + row * p.feed.stride[i], p.feed.row_bytes, bar);
    } else {
      uint32_t bytes = 0;
#pragma unroll 1
      for (int turn = 0; turn < 2; ++turn) {       // how much it is, then the copies
        if (turn == 1) mbar_expect(bar, bytes);
#pragma unroll 1
        for (int i = 0; i < kMaxNormInputs; ++i) {
          if (!p.feed.src[i]) continue;
          const uintptr_t from = reinterpret_cast<uintptr_t>(p.feed.src[i] + row * p.feed.stride[i]), to = from + p.feed.row_bytes;
          const uintptr_t first = reinterpret_cast<uintptr_t>(p.feed.src[i]), last = first + (p.n.tokens - 1) * p.feed.stride[i] + p.feed.row_bytes;
          const uintptr_t grid = from & ~(uintptr_t)15, lo = grid < first ? (from + 15) & ~(uintptr_t)15 : grid;
          const uintptr_t hi = ((to + 15) & ~(uintptr_t)15) > last ? to & ~(uintptr_t)15 : (to + 15) & ~(uintptr_t)15;
          const bool some = hi > lo;
          if (turn == 1) {
            if (some) bulk_load(smem_addr(slot(s, i)) + (uint32_t)(lo - grid), reinterpret_cast<const void*>(lo), (uint32_t)(hi - lo), bar);
            continue;
          }
          if (some) bytes += (uint32_t)(hi - lo);
          const uintptr_t end = some ? lo : to, begin = some ? hi : to;      // what is left: [from, end) and [begin, to)
          for (uintptr_t a = from; a < end; a += 2) *reinterpret_cast<uint16_t*>(slot(s, i) + (a - grid)) = *reinterpret_cast<const uint16_t*>(a);
          for (uintptr_t a = begin; a < to; a += 2) *reinterpret_cast<uint16_t*>(slot(s, i) + (a - grid)) = *reinterpret_cast<const uint16_t*>(a);
        }
      }
    }
    ++issued;
  }
  __device__ __forceinline__ void wait(bool following = false) {      // for the present row, or the one after it
    const bool wraps = following && stage + 1 == p.feed.stages;
    ok &= Waiter{dead, p.error, p.polls}(smem_addr(&full[wraps ? 0 : stage + following]), parity ^ (uint32_t)wraps);
    if (ok) ++ready;
  }
  __device__ __forceinline__ void next() {
    if (++stage == p.feed.stages) stage = 0, parity ^= 1;
  }
  __device__ __forceinline__ const char* at(int input, int64_t row, bool following = false) const {
    const char* to = slot(following && stage + 1 == p.feed.stages ? 0 : stage + following, input);
    if constexpr (!kVector) to += reinterpret_cast<uintptr_t>(p.feed.src[input] + row * p.feed.stride[input]) & 15u;
    return to;
  }
  // Zeros behind the rows, once: copies do not reach them.
  __device__ __forceinline__ void clear_padding(int t) const {
    if (!kVector) return;
    const uint32_t words = (p.feed.slot_bytes - p.feed.row_bytes) / 4;
    for (int i = 0; i < p.feed.stages * p.feed.inputs; ++i)
      for (uint32_t w = t; w < words; w += p.feed.group_threads) reinterpret_cast<uint32_t*>(smem + i * p.feed.slot_bytes + p.feed.row_bytes)[w] = 0;
  }
  __device__ __forceinline__ void finish() {       // the first thread: no copy is left under way
    for (int64_t i = ready; i < issued; ++i) drain(smem_addr(&full[i % p.feed.stages]), i / p.feed.stages & 1);
  }
};

// The columns of a weight in global memory; ones without it.
template <typename T, int V>
__device__ __forceinline__ void load_weight(const Columns<T, V>& cols, const void* w, int hidden, uint64_t* v) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < kPairs; ++e) v[e] = both(1.0f);
    return;
  }
#pragma unroll
  for (int k = 0; k < cols.K; ++k) {
    const int c = cols.first() + k * cols.kStep;
    float f[V + 1] = {};
    if (c < hidden) {
      to_floats<T, V>(*reinterpret_cast<const typename Raw<T, V>::type*>(static_cast<const T*>(w) + c), f);
    }
    if constexpr (V > 1) {
#pragma unroll
      for (int e = 0; e < cols.V; e += 2) v[(k * cols.V + e) / 2] = pair(f[e], f[e + 1]);
    } else {
      float lo, hi;
      split(v[k / 2], &lo, &hi);
      v[k / 2] = k % 2 ? pair(lo, f[0]) : pair(f[0], 0.0f);
    }
  }
}
// The start that both kernels share: barriers, the first rows, the factors a g w_post (without a token's g) and w_pre, by the first group.
template <typename T, int V, bool kToken, int kWarps>
__device__ __forceinline__ void start_rings(const BlockNormParams& p, const Columns<T, V>& cols, NormRows<Columns<T, V>::kVector>& rows, NormRings& rings,
                                            float2 (*part)[kWarps], float* post, float* pre, int group) {
  if (cols.t == 0) {
    for (int s = 0; s < kMaxNormStages; ++s) mbar_init(smem_addr(&rows.full[s]), 1);
    if (group == 0) rings.dead = 0;
    mbar_init_fence();
  }
  rows.clear_padding(cols.t);
  for (int i = cols.t; i < 2 * kWarps; i += cols.n) part[i / kWarps][i % kWarps] = make_float2(0.0f, 0.0f);
  __syncthreads();
  wait_for_previous_kernel();
  if (cols.t == 0)
    for (int s = 0; s < rows.p.feed.stages; ++s) rows.issue_next();
  if (group == 0) {
    uint64_t f[kPairs], g[kPairs];
    load_weight(cols, p.w_post, p.hidden, f);
    if (!kToken && p.gate_kind) load_weight(cols, p.gate.p, p.hidden, g);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      f[e] = mul2(f[e], both(p.alpha));
      if (!kToken && p.gate_kind) f[e] = mul2(f[e], p.sigmoid ? sigmoid2(g[e]) : g[e]);
    }
    cols.store_factors(post, f);
    load_weight(cols, p.w_pre, p.hidden, f);
    cols.store_factors(pre, f);
  }
  __syncthreads();
}

// kToken: the gate is each token's. kForm: 1, there are a block's output, both norms and, backward, both gradients; 2, the same without the
// norm of the block's output; 0, anything. Known when it is compiled, they leave out the moves of values between branches (8192 x 4096,
// forward and backward: the first 53.6 + 108.5 us -> 51.6 + 94.7, the second backward 82 -> 77,
// with a token's gate 135 -> 95).
template <typename T, int V, bool kToken, int kForm, int kThreads, int kWarps>
__global__ void __launch_bounds__(kThreads, 1) block_norm_ring_kernel(const __grid_constant__ NormRingParams rp) {
  extern __shared__ uint4 dynamic[];
  __shared__ NormRings rings;
  __shared__ alignas(16) float2 parts[kMaxGroups][2][kWarps];
  allow_next_kernel();
  const BlockNormParams& p = rp.n;
  const int n = rp.feed.group_threads, group = threadIdx.x / n;
  constexpr bool kVector = Columns<T, V>::kVector;
  const Columns<T, V> cols = {(int)threadIdx.x - group * n, n};
  float *post = reinterpret_cast<float*>(dynamic), *pre = post + n * kCols;
  float2(*part)[kWarps] = parts[group];
  NormRows<kVector> rows(rp, rings, post, group);
  start_rings<T, V, kToken>(p, cols, rows, rings, part, post, pre, group);
  const bool leader = cols.t == 0;
  const bool has_y = kForm != 0 || p.has_y, norm_y = kForm == 1 || (kForm == 0 && p.post), norm_x = kForm != 0 || p.pre;
  int turn = 0;
  // A row's first sum is taken with the last one of the row before it, which makes the chain one sum shorter (8192 x 4096 BF16: 51.5
  // -> 45.9 us) but gives the row's place back later: with a token's gate, which leaves fewer rows under way, 79.9 -> 87.5 us for 5120.
  const bool ahead = !kToken && norm_y && norm_x && rp.feed.stages > 1;
  const auto squares = [&](int64_t row, bool following) { return sum_squares(cols, rows.at(kInY, row, following), p.hidden); };
  float r = 1.0f;
  if (ahead && rows.count > 0) {
    rows.wait();
    r = rsqrtf(group_sums<kWarps>(squares(rows.first, false), 0.0f, part, turn, cols.t, n, group).x * p.inv_hidden + p.eps);
  }
  for (int64_t i = 0; i < rows.count; ++i, rows.next()) {
    const int64_t row = rows.first + i * rows.step;
    if (!ahead) rows.wait();
    uint64_t x[kPairs], y[kPairs], f[kPairs];
    cols.load(rows.at(kInX, row), p.hidden, x);
    if (has_y) {
      cols.load(rows.at(kInY, row), p.hidden, y);
      cols.load_factors(post, f);
      if (kToken) {
        uint64_t g[kPairs];
        cols.load(rows.at(kInGate, row), p.hidden, g);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) f[e] = mul2(f[e], p.sigmoid ? sigmoid2(g[e]) : g[e]);
      }
      if (norm_y && !ahead) {
        uint64_t s = 0;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) s = fma2(y[e], y[e], s);
        r = rsqrtf(group_sums<kWarps>(sum_of(s), 0.0f, part, turn, cols.t, n, group).x * p.inv_hidden + p.eps);
        if (leader) rows.issue_next();      // all threads have the row
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) x[e] = fma2(mul2(f[e], both(r)), y[e], x[e]);
      cols.store(static_cast<T*>(p.x_out.p) + row * p.x_out.stride, p.hidden, x);
    }
    if (norm_x) {
      uint64_t s = 0;
#pragma unroll
      for (int e = 0; e < kPairs; ++e) s = fma2(x[e], x[e], s);
      float next = 0.0f;
      if (ahead && i + 1 < rows.count) {
        rows.wait(true);
        next = squares(row + rows.step, true);
      }
      const float2 both_sums = group_sums<kWarps>(sum_of(s), next, part, turn, cols.t, n, group);
      const float r2 = rsqrtf(both_sums.x * p.inv_hidden + p.eps);
      if (ahead) r = rsqrtf(both_sums.y * p.inv_hidden + p.eps);
      if ((ahead || !norm_y) && leader) rows.issue_next();
      cols.load_factors(pre, f);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) x[e] = mul2(mul2(f[e], both(r2)), x[e]);
      cols.store(static_cast<T*>(p.h_out.p) + row * p.h_out.stride, p.hidden, x);
    } else if (!norm_y) {
      group_sync(group, n);
      if (leader) rows.issue_next();
    }
  }
  if (leader) rows.finish();
}

template <typename T, int V, bool kToken, int kForm, int kThreads, int kWarps>
__global__ void __launch_bounds__(kThreads, 1) block_norm_backward_ring_kernel(const __grid_constant__ NormRingParams rp) {
  extern __shared__ uint4 dynamic[];
  __shared__ NormRings rings;
  __shared__ alignas(16) float2 parts[kMaxGroups][2][kWarps];
  allow_next_kernel();
  const BlockNormParams& p = rp.n;
  const int n = rp.feed.group_threads, group = threadIdx.x / n;
  constexpr bool kVector = Columns<T, V>::kVector;
  const Columns<T, V> cols = {(int)threadIdx.x - group * n, n};
  float *post = reinterpret_cast<float*>(dynamic), *pre = post + n * kCols;
  float2(*part)[kWarps] = parts[group];
  NormRows<kVector> rows(rp, rings, post, group);
  start_rings<T, V, kToken>(p, cols, rows, rings, part, post, pre, group);
  const bool leader = cols.t == 0;
  const bool has_y = kForm != 0 || p.has_y, norm_y = kForm == 1 || (kForm == 0 && p.post), norm_x = kForm != 0 || p.pre;
  // Whether a row stays in registers from one sum to the next, as far as there are any: a token's gate is 32 more, single columns take
  // more to address. Their rows are read again (8192 x 4096 BF16 with such a gate: 158 -> 124 us).
  constexpr bool kKeep = kVector && !kToken;
  uint64_t sum_post[kPairs] = {}, sum_pre[kPairs] = {};
  int turn = 0;
  // A row's first sum with the last one of the row before, as forward, where that was faster (us, without and with it). In vectors, one group of
  // up to ten warps: 8192 x 5120 BF16 128 -> 122, with a token's gate 204 -> 187, without the norm of x' 102 -> 97; 4096 x 5120 FP32
  // 87 -> 90, 4608 columns 77 -> 85, with a token's gate 160 -> 159, without the norm of x' 82 -> 78. In pairs: 6000 x 5002 BF16 192 -> 186,
  // with a token's gate 226 -> 246. In single columns: 6000 x 5001 BF16 208 -> 268, 3000 x 5001 FP32 99 -> 125. Two groups: 8192 x 4096
  // BF16 87 -> 96.
  constexpr bool kAhead = kThreads < 512 && (kVector || (V == 2 && !kToken));
  const bool ahead = kAhead && norm_y && (sizeof(T) == 2 || !norm_x) && rp.feed.stages > 1;
  const auto squares = [&](int64_t row, bool following) { return sum_squares(cols, rows.at(kInY, row, following), p.hidden); };
  float r = 1.0f;
  if (ahead && rows.count > 0) {
    rows.wait();
    r = rsqrtf(group_sums<kWarps>(squares(rows.first, false), 0.0f, part, turn, cols.t, n, group).x * p.inv_hidden + p.eps);
  }
  for (int64_t i = 0; i < rows.count; ++i, rows.next()) {
    const int64_t row = rows.first + i * rows.step;
    if (!ahead) rows.wait();
    uint64_t x[kPairs], y[kPairs], g[kPairs], h[kPairs], f[kPairs];     // y: times r
    float r2 = 0.0f, m = 0.0f;
    const auto load_y = [&] {
      cols.load(rows.at(kInY, row), p.hidden, y);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) y[e] = mul2(y[e], both(r));
    };
    const auto load_gate = [&] {
      cols.load(rows.at(kInGate, row), p.hidden, g);
      if (p.sigmoid) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) g[e] = sigmoid2(g[e]);
      }
    };
    if (has_y) {
      cols.load(rows.at(kInY, row), p.hidden, y);
      if (norm_y && !ahead) {
        uint64_t s = 0;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) s = fma2(y[e], y[e], s);
        r = rsqrtf(group_sums<kWarps>(sum_of(s), 0.0f, part, turn, cols.t, n, group).x * p.inv_hidden + p.eps);
      }
      if constexpr (kKeep) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) y[e] = mul2(y[e], both(r));
      } else {
        load_y();
      }
      if (kToken) load_gate();
    }
    if (norm_x) {
      cols.load(rows.at(kInX, row), p.hidden, x);
      if (has_y) {
        cols.load_factors(post, f);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) x[e] = fma2(kToken ? mul2(f[e], g[e]) : f[e], y[e], x[e]);
      }
      cols.load(rows.at(kInDh, row), p.hidden, h);
      cols.load_factors(pre, f);
      uint64_t ss = 0, ux = 0;
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        ss = fma2(x[e], x[e], ss);
        ux = fma2(mul2(h[e], f[e]), x[e], ux);
      }
      const float2 s = group_sums<kWarps>(sum_of(ss), sum_of(ux), part, turn, cols.t, n, group);
      r2 = rsqrtf(s.x * p.inv_hidden + p.eps);
      m = -s.y * r2 * p.inv_hidden;
    }
    uint64_t d[kPairs] = {};
    if (kForm != 0 || p.dx_out.p) cols.load(rows.at(kInDx, row), p.hidden, d);
    if (norm_x) {
      cols.load_factors(pre, f);
      if (!kKeep) cols.load(rows.at(kInDh, row), p.hidden, h);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const uint64_t xh = mul2(x[e], both(r2));
        sum_pre[e] = fma2(h[e], xh, sum_pre[e]);
        d[e] = fma2(both(r2), fma2(xh, both(m), mul2(h[e], f[e])), d[e]);
      }
    }
    cols.store(static_cast<T*>(p.dx.p) + row * p.dx.stride, p.hidden, d);
    uint64_t dot = 0;
    if (has_y) {
      cols.load_factors(post, f);
      if (!kKeep) {
        load_y();
        if (kToken) load_gate();
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        x[e] = mul2(f[e], d[e]);                   // v, or v / g
        d[e] = mul2(d[e], both(p.alpha));
        if (kToken) {
          const uint64_t v = mul2(x[e], g[e]);     // and x: dgate = v / g y r g'
          sum_post[e] = fma2(mul2(d[e], g[e]), y[e], sum_post[e]);
          dot = fma2(v, y[e], dot);
          f[e] = mul2(x[e], y[e]);
          if (p.sigmoid) f[e] = mul2(f[e], mul2(g[e], fma2(g[e], both(-1.0f), both(1.0f))));
          x[e] = v;
        } else {
          sum_post[e] = fma2(d[e], y[e], sum_post[e]);
          dot = fma2(x[e], y[e], dot);
        }
      }
      if (kToken && p.dgate.p) cols.store(static_cast<T*>(p.dgate.p) + row * p.dgate.stride, p.hidden, f);
    }
    if (norm_y) {
      float next = 0.0f;
      if (ahead && i + 1 < rows.count) {
        rows.wait(true);
        next = squares(row + rows.step, true);
      }
      const float2 both_sums = group_sums<kWarps>(sum_of(dot), next, part, turn, cols.t, n, group);
      m = -both_sums.x * p.inv_hidden;
      if (!kKeep) {
        load_y();
        group_sync(group, n);
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) x[e] = mul2(both(r), fma2(y[e], both(m), x[e]));
      if (ahead) r = rsqrtf(both_sums.y * p.inv_hidden + p.eps);
    } else {
      group_sync(group, n);
    }
    if (leader) rows.issue_next();       // all threads have read the row
    if (has_y) cols.store(static_cast<T*>(p.dy.p) + row * p.dy.stride, p.hidden, x);
  }
  if (leader) rows.finish();
  if (!p.partial) return;
  // the groups' sums, one after the other, where the factors were
  for (int g = 0; g < rp.feed.groups; ++g) {
    __syncthreads();
    if (g != group) continue;
    if (g > 0) {
      uint64_t s[kPairs];
      cols.load_factors(post, s);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) sum_post[e] = add2(s[e], sum_post[e]);
      cols.load_factors(pre, s);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) sum_pre[e] = add2(s[e], sum_pre[e]);
    }
    if (g + 1 < rp.feed.groups) {
      cols.store_factors(post, sum_post);
      cols.store_factors(pre, sum_pre);
    } else {
      float* at = p.partial + (int64_t)blockIdx.x * 2 * p.hidden;
      cols.store_f32(at, p.hidden, sum_post);
      cols.store_f32(at + p.hidden, p.hidden, sum_pre);
    }
  }
}

// ---- weights' gradients --------------------------------------------------------------------------------------

// Adds the blocks' partial rows: 32 columns per block, 32 parts of the blocks, joined in order. What the columns of the first
// sum stand for: sum a d y r, times g for w_post and times w_post g' for a gate for all tokens.
constexpr int kNormSumParts = 32;
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
  if (blocks == 0) {                  // no tokens: zeros, whatever the weight and the gate hold
    if (which == 1 && p.dw_pre) p.dw_pre[col] = 0.0f;
    if (which == 0 && p.dw_post) p.dw_post[col] = 0.0f;
    if (which == 0 && p.dgate_sum) p.dgate_sum[col] = 0.0f;
    return;
  }
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

unsigned wide_threads(const slidedp_block_norm_args* a) { return (unsigned)((a->hidden + kWideValues * 32 - 1) / (kWideValues * 32) * 32); }
// Blocks that stay, of which each has a row of partial sums: one per SM, or two wide rows' ones with up to half the threads (2048 x 8192
// FP32 with a token's gate, backward: 242 -> 174 us).
constexpr int kSms = 148;
int64_t norm_blocks(const slidedp_block_norm_args* a, int per_sm) { return a->tokens < kSms * per_sm ? a->tokens : kSms * per_sm; }
int wide_per_sm(const slidedp_block_norm_args* a) { return wide_threads(a) <= kWideThreads / 2 ? 2 : 1; }

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

// run(T, V) as template arguments
template <typename F>
void pick_wide_kernel(const slidedp_block_norm_args* a, int v, F run) {
  typedef std::integral_constant<int, 1> One;
  if (a->dtype == SLIDEDP_F32) v == 4 ? run(float(), std::integral_constant<int, 4>()) : run(float(), One());
  else if (v == 8) run(uint16_t(), std::integral_constant<int, 8>());
  else v == 2 ? run(uint16_t(), std::integral_constant<int, 2>()) : run(uint16_t(), One());
}

// A block per SM whose groups hold their rows in shared memory: threads of a group, groups, stages of a ring. The kernels are compiled for
// blocks of 512 threads, 128 registers each; forward two groups of up to 10 warps fit as well (5120 columns: 84 -> 59 us).
struct RingPlan {
  bool use, vector;
  int threads, groups, stages;
  size_t smem, slot;
};
constexpr int ring_class(bool backward, int group) { return group > 256 && group <= 320 ? (backward ? 320 : 640) : 512; }
// Of an SM's 227 KB, less what a block has besides. Kernels are allowed all of it: the limit belongs to the kernel, which calls with
// other plans launch from other threads at the same time.
constexpr int kNormSmem = 222 * 1024;

RingPlan ring_plan(const slidedp_block_norm_args* a, bool vector, int inputs, bool backward) {
  RingPlan r = {};
  if (a->hidden > 512 * kCols) return r;
  const int64_t row = a->hidden * elem_bytes(a->dtype);
  r.vector = vector;
  r.threads = (int)((a->hidden + kCols * 32 - 1) / (kCols * 32) * 32);
  r.slot = vector ? r.threads * kCols * elem_bytes(a->dtype) : (row + 15) / 16 * 16 + 16;
  const int most = ring_class(backward, r.threads) / r.threads;
  for (r.groups = most < kMaxGroups ? most : kMaxGroups; r.groups >= 1; --r.groups)
    for (r.stages = kMaxNormStages; r.stages >= (r.groups > 1 ? 2 : 1); --r.stages) {
      r.smem = r.groups * r.stages * inputs * r.slot + r.threads * kCols * 8;
      if (r.smem <= kNormSmem) {
        r.use = true;
        return r;
      }
    }
  return r;
}
NormRingParams ring_params(slidedp_ctx* ctx, const slidedp_block_norm_args* a, const BlockNormParams& n, const RingPlan& plan) {
  NormRingParams r = {};
  r.n = n;
  const NormView* in[kMaxNormInputs] = {&n.x, &n.y, &n.gate, &n.dx_out, &n.dh};
  const int elem = elem_bytes(a->dtype);
  for (int i = 0; i < kMaxNormInputs; ++i) {
    if (i == kInGate && a->gate_kind != 2) continue;
    r.feed.src[i] = static_cast<const char*>(in[i]->p);
    r.feed.stride[i] = in[i]->stride * elem;
    r.feed.slot[i] = r.feed.inputs;
    r.feed.inputs += in[i]->p != nullptr;
  }
  r.feed.stages = plan.stages;
  r.feed.groups = plan.groups;
  r.feed.group_threads = plan.threads;
  r.feed.row_bytes = (uint32_t)(a->hidden * elem);
  r.feed.slot_bytes = (uint32_t)plan.slot;
  r.error = ctx->kernel_error;
  r.polls = ctx->wait_polls;
  return r;
}
// run(T, V, token, form, threads, warps of a group) as template arguments.
template <bool kBackward, typename F>
void pick_ring_kernel(const slidedp_block_norm_args* a, const RingPlan& plan, int v, int form, F run) {
  typedef std::true_type Yes;
  typedef std::false_type No;
  const auto threads = [&](auto type, auto vector, auto token, auto whole) {
    typedef std::integral_constant<int, 512> Usual;
    if (plan.threads <= 256) return run(type, vector, token, whole, Usual(), std::integral_constant<int, 8>());
    if (plan.threads <= 320) return run(type, vector, token, whole, std::integral_constant<int, kBackward ? 320 : 640>(), std::integral_constant<int, 10>());
    run(type, vector, token, whole, Usual(), std::integral_constant<int, 16>());
  };
  const auto forms = [&](auto type, auto token) {
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 16 / (int)sizeof(type)> Whole;
    typedef std::integral_constant<int, 0> Any;
    typedef std::integral_constant<int, 2> Two;
    if (plan.vector) return form == 1 ? threads(type, Whole(), token, One()) : form == 2 ? threads(type, Whole(), token, Two()) : threads(type, Whole(), token, Any());
    if constexpr (sizeof(type) == 2)
      if (v == 2) return threads(type, Two(), token, Any());
    threads(type, One(), token, Any());
  };
  const auto gates = [&](auto type) { a->gate_kind == 2 ? forms(type, Yes()) : forms(type, No()); };
  a->dtype == SLIDEDP_BF16 ? gates(uint16_t()) : gates(float());
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
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const RingPlan plan = ring_plan(a, v * elem == 16, 1 + (y != nullptr) + (a->gate_kind == 2), false);
  cudaError_t attribute = cudaSuccess;
  const unsigned blocks = (unsigned)norm_blocks(a, plan.use ? 1 : wide_per_sm(a));      // rows go to groups block by block: all SMs have one before one has two
  FAULT_POINT();
  if (plan.use) {
    const NormRingParams r = ring_params(ctx, a, p, plan);
    pick_ring_kernel<false>(a, plan, v, y && a->pre_norm ? (a->post_norm ? 1 : 2) : 0, [&](auto type, auto vector, auto token, auto form, auto threads, auto warps) {
      typedef decltype(type) T_;
      const auto run = [&](auto kernel) {
        attribute = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSmem);
        if (attribute == cudaSuccess) launch_after(kernel, dim3(blocks), plan.threads * plan.groups, plan.smem, 1, st, r);
      };
      run(block_norm_ring_kernel<T_, vector, token, form, threads, warps>);
    });
  } else {
    pick_wide_kernel(a, v, [&](auto type, auto vec) {
      typedef decltype(type) T_;
      const auto run = [&](auto kernel) { launch_after(kernel, dim3(blocks), wide_threads(a), 0, 1, st, p); };
      a->gate_kind == 2 ? run(block_norm_kernel<T_, vec, true>) : run(block_norm_kernel<T_, vec, false>);
    });
  }
  if (attribute != cudaSuccess) return cuda_fail(ctx, attribute);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_block_norm_workspace(const slidedp_block_norm_args* a) {
  if (check_norm(a) != SLIDEDP_OK) return 0;
  return (size_t)(norm_blocks(a, 2) * 2 * a->hidden) * sizeof(float) + 16;
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
      (sums && (!workspace || (a->gate_kind == 1 && !rows_ok(gate, elem, 1, H, false)))))
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
  unsigned blocks = 0;
  if (T > 0) {
    const slidedp_rows wp = {const_cast<void*>(w_post), 0}, wq = {const_cast<void*>(w_pre), 0};
    const int v = vector_width(H, elem, {{x, elem}, {y, elem}, {gate, elem}, {dx_out, elem}, {dh_out, elem}, {dx, elem}, {dy, elem}, {dgate, elem},
                                         {&wp, elem}, {&wq, elem}});
    const RingPlan plan = ring_plan(a, v * elem == 16, 1 + (y != nullptr) + (a->gate_kind == 2) + (dx_out != nullptr) + a->pre_norm, true);
    cudaError_t attribute = cudaSuccess;
    blocks = (unsigned)norm_blocks(a, plan.use ? 1 : wide_per_sm(a));
    FAULT_POINT();
    if (plan.use) {
      const NormRingParams r = ring_params(ctx, a, p, plan);
      pick_ring_kernel<true>(a, plan, v, y && a->pre_norm && dx_out ? (a->post_norm ? 1 : 2) : 0, [&](auto type, auto vector, auto token, auto form, auto threads, auto warps) {
        typedef decltype(type) T_;
        const auto run = [&](auto kernel) {
          attribute = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSmem);
          if (attribute == cudaSuccess) launch_after(kernel, dim3(blocks), plan.threads * plan.groups, plan.smem, 1, st, r);
        };
        run(block_norm_backward_ring_kernel<T_, vector, token, form, threads, warps>);
      });
    } else {
      pick_wide_kernel(a, v, [&](auto type, auto vec) {
        typedef decltype(type) T_;
        const size_t smem = sums ? (size_t)wide_threads(a) * kWideValues * 2 * sizeof(float) : 0;
        const auto run = [&](auto kernel) {
          attribute = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWideThreads * kWideValues * 2 * (int)sizeof(float));
          if (attribute == cudaSuccess) launch_after(kernel, dim3(blocks), wide_threads(a), smem, 1, st, p);
        };
        a->gate_kind == 2 ? run(block_norm_backward_kernel<T_, vec, true>) : run(block_norm_backward_kernel<T_, vec, false>);
      });
    }
    if (attribute != cudaSuccess) return cuda_fail(ctx, attribute);
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
