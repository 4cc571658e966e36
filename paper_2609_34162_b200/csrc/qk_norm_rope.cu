// libslidedp: RMS norm of every query and key head with the position rotation in the same pass,
// forward and backward. See include/slidedp_ops.h for the contract.
//
// With r = rsqrt(mean(x^2) + eps), xh = x r, n = xh w and R the rotation of the token:
//   y  = R n
//   dz = R^T dy,  u = w dz,  dx = r (u - xh mean(u xh)),  dw = sum over rows of dz xh
// Bound: HBM. Forward reads x and writes y (4 bytes per BF16 value), backward reads x and dy and
// writes dx (6 bytes); the cos/sin row is read once per four heads, w once per block.
// Measured, 8192 tokens, 32 + 8 heads of 128, BF16: forward 28.8 us (5.8 TB/s), backward 43.9 + 3.1 us (5.7 TB/s);
// 16384 tokens, 40 + 8 heads: forward 65.6 us (6.1 TB/s).
#include "device_utils.cuh"
#include "ops_internal.h"

namespace slidedp {

constexpr int kQkThreads = 128;
// Heads of one token per task, which one cos/sin row serves. Eight: 31 and 75 us forward for the sizes above.
constexpr int kQkHeads = 4;
// Blocks that stay. Forward with five per SM: 31 and 72 us; backward with four (128 registers) spills: 50 us.
constexpr int kQkForwardPerSM = 4, kQkBackwardPerSM = 3, kQkBackwardBlocks = 148 * kQkBackwardPerSM;
constexpr int kQkPairs = 4;          // heads in single pairs: groups per lane, 32 * 4 * 2 = 256 values

struct QkSide {
  const void* x;
  const void* dy;   // backward
  void* out;        // y, or dx
  const void* w;
  int64_t x_t, x_h, dy_t, dy_h, out_t, out_h;
  int heads;
  int width, chunks;   // heads per task, tasks per token
};

struct QkParams {
  QkSide side[2];   // q, k
  const float* cos_sin;
  const int32_t* positions;
  int64_t table_rows;
  uint32_t tokens;
  int head_dim, rope_dim, interleaved;
  int chunks_q, chunks;   // single pairs forward: tasks of a token, the queries' first
  int blocks_q;           // otherwise: blocks that take queries
  double eps, inv_dim;
  float* partials;  // backward: [block][head_dim], null when no weight gradient is asked for
};

__device__ __forceinline__ void shared_16(uint32_t a, uint32_t* x, uint32_t* y, uint32_t* z, uint32_t* w) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(*x), "=r"(*y), "=r"(*z), "=r"(*w) : "r"(a) : "memory");
}

// A run of VW values of type T as they lie in memory.
template <typename T, int VW> struct Run;
template <> struct Run<uint16_t, 8> {
  uint4 r;
  __device__ void load(const uint16_t* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ void from_shared(uint32_t a) { shared_16(a, &r.x, &r.y, &r.z, &r.w); }
  __device__ void unpack(float* v) const {
    v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
    v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
  }
  static __device__ void store(uint16_t* p, const float* v) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7]));
  }
};
template <> struct Run<uint16_t, 4> {
  uint2 r;
  __device__ void load(const uint16_t* p) { r = *reinterpret_cast<const uint2*>(p); }
  __device__ void from_shared(uint32_t a) { asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory"); }
  __device__ void unpack(float* v) const { v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y); }
  static __device__ void store(uint16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
  }
};
template <> struct Run<uint16_t, 1> {
  uint16_t r;
  __device__ void load(const uint16_t* p) { r = *p; }
  __device__ void unpack(float* v) const { v[0] = __uint_as_float((uint32_t)r << 16); }
  static __device__ void store(uint16_t* p, const float* v) { *p = (uint16_t)f32_to_bf16_bits(v[0]); }
};
template <> struct Run<float, 4> {
  float4 r;
  __device__ void load(const float* p) { r = *reinterpret_cast<const float4*>(p); }
  __device__ void from_shared(uint32_t a) {
    uint32_t x, y, z, w;
    shared_16(a, &x, &y, &z, &w);
    r = make_float4(__uint_as_float(x), __uint_as_float(y), __uint_as_float(z), __uint_as_float(w));
  }
  __device__ void unpack(float* v) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ void store(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Run<float, 2> {   // half a group's cosines or sines
  float2 r;
  __device__ void load(const float* p) { r = *reinterpret_cast<const float2*>(p); }
  __device__ void unpack(float* v) const { v[0] = r.x; v[1] = r.y; }
};
template <> struct Run<float, 1> {
  float r;
  __device__ void load(const float* p) { r = *p; }
  __device__ void unpack(float* v) const { v[0] = r; }
  static __device__ void store(float* p, const float* v) { *p = v[0]; }
};

// A lane owns a group of VW pairs of its row (or several groups of one, L apart). A group is two runs of VW
// consecutive values at a0 and a1: the two members of its pairs (or, interleaved, VW / 2 whole pairs each; or, past
// rope_dim, two runs of values that are not rotated). So a row is loaded, rotated and stored without exchanging
// values between lanes, and neighbouring lanes have neighbouring runs. (Interleaved runs side by side in a lane make every
// request touch each sector twice: 8192 tokens, 40 heads of 128, 42 + 70 us against 29 + 45.)
struct Group {
  int a0, a1, pair, pair1;   // the first and the VW / 2-th pair's index in the cos/sin row
  bool on0, on1, rotated;
  __device__ Group(const QkParams& p, int g, int vw) {
    const int half = p.rope_dim / 2, first = g * vw;
    rotated = first < half;
    pair = p.interleaved && vw > 1 ? first / 2 : first;
    pair1 = p.interleaved ? pair + half / 2 : pair + vw / 2;
    if (rotated) {
      a0 = p.interleaved && vw == 1 ? 2 * first : first;
      a1 = p.interleaved && vw == 1 ? 2 * first + 1 : first + half;
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
struct Both {   // a group's two runs
  Run<T, VW> lo, hi;
  __device__ __forceinline__ void load(const T* row, const Group& g, bool live) {
    lo = Run<T, VW>();
    hi = Run<T, VW>();
    if (live && g.on0) lo.load(row + g.a0);
    if (live && g.on1) hi.load(row + g.a1);
  }
  __device__ __forceinline__ void from_shared(uint32_t a, uint32_t b) {
    lo.from_shared(a);
    hi.from_shared(b);
  }
  // INTER: first members of adjacent pairs before the second ones, so that v is always halves whose values pair up
  template <bool INTER = false>
  __device__ __forceinline__ void unpack(float* v) const {
    float y[2 * VW];
    lo.unpack(y);
    hi.unpack(y + VW);
#pragma unroll
    for (int e = 0; e < 2 * VW; ++e) v[order<INTER>(e)] = y[e];
  }
  template <bool INTER = false>
  static __device__ __forceinline__ void store(T* row, const Group& g, const float* v) {
    float y[2 * VW];
#pragma unroll
    for (int e = 0; e < 2 * VW; ++e) y[e] = v[order<INTER>(e)];
    if (g.on0) Run<T, VW>::store(row + g.a0, y);
    if (g.on1) Run<T, VW>::store(row + g.a1, y + VW);
  }
  template <bool INTER>
  static constexpr __device__ int order(int e) { return INTER ? e / 2 + e % 2 * VW : e; }
};

// (a, b) -> (a c - b s, b c + a s) for the pairs of a group; BACK: with s negated, which is the transpose.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = a, y = b;
  a = x * c - y * s;
  b = y * c + x * s;
}
template <int VW, bool BACK>
__device__ __forceinline__ void rotate(float* v, const float* c, const float* s) {
  if constexpr (VW == 1) {
    turn(v[0], v[1], c[0], BACK ? -s[0] : s[0]);
  } else {
#pragma unroll
    for (int i = 0; i < VW; i += 2) {   // neighbours two at a time, but for the half with the minus
      float *a = v + i, *b = v + VW + i;
      const uint64_t a2 = pair(a[0], a[1]), b2 = pair(b[0], b[1]), c2 = pair(c[i], c[i + 1]), s2 = pair(s[i], s[i + 1]);
      const uint64_t ac = mul2(a2, c2), bc = mul2(b2, c2);
      float t0, t1;
      if constexpr (BACK) {
        split(bc, &t0, &t1);
        b[0] = fmaf(-a[0], s[i], t0);
        b[1] = fmaf(-a[1], s[i + 1], t1);
        split(fma2(b2, s2, ac), &a[0], &a[1]);
      } else {
        split(ac, &t0, &t1);
        a[0] = fmaf(-b[0], s[i], t0);
        a[1] = fmaf(-b[1], s[i + 1], t1);
        split(fma2(a2, s2, bc), &b[0], &b[1]);
      }
    }
  }
}

// The cosines and sines of a position for a group; NaN when it is outside the table.
template <int VW>
__device__ __forceinline__ void load_angles(const QkParams& p, int64_t pos, const Group& g, float* c, float* s) {
  if (!g.rotated) return;
  if (pos < 0 || pos >= p.table_rows) {
#pragma unroll
    for (int i = 0; i < VW; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
    return;
  }
  const float* row = p.cos_sin + pos * p.rope_dim;
  const int half = p.rope_dim / 2;
  constexpr int R = VW == 1 ? 1 : VW / 2;
#pragma unroll
  for (int i = 0; i < VW; i += R) {
    Run<float, R> a, b;
    a.load(row + (i ? g.pair1 : g.pair));
    b.load(row + half + (i ? g.pair1 : g.pair));
    a.unpack(c + i);
    b.unpack(s + i);
  }
}

template <int L, typename A>
__device__ __forceinline__ A sum_lanes(A x) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// ---- heads in runs of several values ---------------------------------------------------------------------
//
// A fixed grid whose first blocks take queries, the others keys. One task = up to kQkHeads heads of one token for L
// lanes, head after head; the values of the next heads are on their way into a ring in shared memory, each lane copying
// what it will read itself, so nothing waits for another thread. The task's cosines and sines are fetched while
// the task before it is worked on, and serve all its heads. (Before: loads into registers, forward four heads of a task at
// once, backward one head ahead with its angles fetched in place: too few bytes in flight, 37, 95 and 62 us.) Four
// stages; three: 29, 68 and 45 us, eight forward: 29 and 69.

// N FP32 values as pairs of neighbours, for instructions that work on two.
template <int N>
struct Pairs {
  uint64_t v[N / 2];
  __device__ __forceinline__ void from(const float* f) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ void to(float* f) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) split(v[i], &f[2 * i], &f[2 * i + 1]);
  }
};
__device__ __forceinline__ float sum2(uint64_t v) {
  float a, b;
  split(v, &a, &b);
  return a + b;
}

// Copies B bytes (16 or 8) to shared memory in the background, or writes zeros if !live.
template <int B>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool live) {
  if constexpr (B == 16) {
    if (live) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
  } else {
    if (live) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(dst), "r"(0) : "memory");
  }
}

// A token and which of its tasks, walked in steps of a whole grid.
struct Spot {
  uint32_t t, c;
  __device__ __forceinline__ void advance(uint32_t by_t, uint32_t by_c, uint32_t chunks) {
    t += by_t;
    c += by_c;
    if (c >= chunks) {
      c -= chunks;
      ++t;
    }
  }
};

template <typename T, int VW, int L, bool BACK, bool INTER>
__global__ void __launch_bounds__(kQkThreads, BACK ? kQkBackwardPerSM : kQkForwardPerSM) qk_heads_kernel(const __grid_constant__ QkParams p) {
  constexpr int N = 2 * VW, B = VW * (int)sizeof(T), kRuns = BACK ? 4 : 2, kStages = 64 / B, kTasks = kQkThreads / L;
  constexpr int kRing = kStages * kRuns * kQkThreads * B, kPart = BACK ? kTasks * (L * N + 1) * 4 : 0;
  __shared__ __align__(16) uint8_t ring[kRing > kPart ? kRing : kPart];
  const bool is_k = (int)blockIdx.x >= p.blocks_q;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const uint32_t block = blockIdx.x - (is_k ? p.blocks_q : 0), blocks = is_k ? gridDim.x - p.blocks_q : p.blocks_q;
  const int lane = threadIdx.x % L;
  const Group g(p, lane, VW);
  const uint32_t chunks = sd.chunks, step = blocks * kTasks, by_t = step / chunks, by_c = step - by_t * chunks;
  const int width = sd.width;
  // every lane of a warp takes part in every round, so that the lane sums see whole warps
  const uint32_t mine = block * kTasks + threadIdx.x / L, tasks = p.tokens * chunks, rounds = (tasks + step - 1) / step;
  Spot now{mine / chunks, mine % chunks}, ahead = now;

  // the ring: stage k holds a head's runs, run r of thread t at [k][r][t]
  const uint32_t at = smem_addr(ring) + threadIdx.x * B;
  const auto slot = [&](int stage, int r) { return at + (stage * kRuns + r) * (kQkThreads * B); };
  int u_ahead = 0;
  const T *x = nullptr, *d = nullptr;
  const auto fetch = [&](int stage) {
    if (u_ahead == 0) {
      const int64_t t = ahead.t < p.tokens ? ahead.t : 0, h = ahead.c * width;
      x = static_cast<const T*>(sd.x) + t * sd.x_t + h * sd.x_h;
      if (BACK) d = static_cast<const T*>(sd.dy) + t * sd.dy_t + h * sd.dy_h;
    }
    const bool live = ahead.t < p.tokens && (int)ahead.c * width + u_ahead < sd.heads;
    copy_async<B>(slot(stage, 0), x + g.a0, live && g.on0);
    copy_async<B>(slot(stage, 1), x + g.a1, live && g.on1);
    if (BACK) {
      copy_async<B>(slot(stage, 2), d + g.a0, live && g.on0);
      copy_async<B>(slot(stage, 3), d + g.a1, live && g.on1);
      d += sd.dy_h;
    }
    x += sd.x_h;
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (++u_ahead == width) {
      u_ahead = 0;
      ahead.advance(by_t, by_c, chunks);
    }
  };
  start_after_previous_kernel();
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) fetch(k);

  Pairs<N> w, dw;
  {
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = 1.0f;
    if (sd.w) {
      Both<T, VW> rw;
      rw.load(static_cast<const T*>(sd.w), g, true);
      rw.template unpack<INTER>(f);
    }
    w.from(f);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) dw.v[e] = 0;
  }
  float c[VW], s[VW], next_c[VW], next_s[VW];
  const auto position = [&](const Spot& at) -> int64_t {
    if (p.rope_dim == 0 || at.t >= p.tokens) return 0;
    return p.positions ? (int64_t)p.positions[at.t] : at.t;
  };
  Spot later = now;
  load_angles<VW>(p, position(now), g, next_c, next_s);
  later.advance(by_t, by_c, chunks);
  int64_t next_position = position(later);

  int stage = 0;
  for (uint32_t k = 0; k < rounds; ++k) {
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      c[e] = next_c[e];
      s[e] = next_s[e];
    }
    if (k + 1 < rounds) load_angles<VW>(p, next_position, g, next_c, next_s);
    later.advance(by_t, by_c, chunks);
    next_position = position(later);
    const int h0 = (int)now.c * width;
    T* out = static_cast<T*>(sd.out) + (int64_t)now.t * sd.out_t + h0 * sd.out_h;
    const int heads = now.t < p.tokens ? min(width, sd.heads - h0) : 0;
    for (int u = 0; u < width; ++u, out += sd.out_h) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      float fx[N], fd[N];
      Both<T, VW> raw;
      raw.from_shared(slot(stage, 0), slot(stage, 1));
      raw.template unpack<INTER>(fx);
      if (BACK) {
        raw.from_shared(slot(stage, 2), slot(stage, 3));
        raw.template unpack<INTER>(fd);
      }
      // into the stage that was read last, a round ago: its values have been used
      fetch(stage == 0 ? kStages - 1 : stage - 1);
      if (++stage == kStages) stage = 0;
      Pairs<N> px;
      px.from(fx);
      uint64_t xx = mul2(px.v[0], px.v[0]);
#pragma unroll
      for (int e = 1; e < N / 2; ++e) xx = fma2(px.v[e], px.v[e], xx);
      if constexpr (!BACK) {
        const float r = rsqrtf(fmaf(sum_lanes<L>(sum2(xx)), (float)p.inv_dim, (float)p.eps));
        const uint64_t r2 = pair(r, r);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) px.v[e] = mul2(mul2(px.v[e], r2), w.v[e]);
        px.to(fx);
        if (g.rotated) rotate<VW, false>(fx, c, s);
        if (u < heads) Both<T, VW>::template store<INTER>(out, g, fx);
      } else {
        if (g.rotated) rotate<VW, true>(fd, c, s);
        Pairs<N> pd, pu;
        pd.from(fd);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) pu.v[e] = mul2(pd.v[e], w.v[e]);
        uint64_t xu = mul2(px.v[0], pu.v[0]);
#pragma unroll
        for (int e = 1; e < N / 2; ++e) xu = fma2(px.v[e], pu.v[e], xu);
        const float r = rsqrtf(fmaf(sum_lanes<L>(sum2(xx)), (float)p.inv_dim, (float)p.eps));
        const float mean = sum_lanes<L>(sum2(xu)) * r * (float)p.inv_dim;   // mean(u xh)
        if (u >= heads) continue;
        const uint64_t r2 = pair(r, r), less = pair(-mean, -mean);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          const uint64_t xh = mul2(px.v[e], r2);
          dw.v[e] = fma2(pd.v[e], xh, dw.v[e]);
          pu.v[e] = mul2(r2, fma2(xh, less, pu.v[e]));
        }
        pu.to(fd);
        Both<T, VW>::template store<INTER>(out, g, fd);
      }
    }
    now.advance(by_t, by_c, chunks);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  if (!BACK || !p.partials) return;
  // Every lane kept its values' share of dw over all its tasks; the block adds its lanes in a fixed order and writes one
  // row of partial sums, which qk_weight_grad_kernel adds in a fixed order. So dw has the same bits in every run.
  __syncthreads();
  float(*part)[L * N + 1] = reinterpret_cast<float(*)[L * N + 1]>(ring);
  float f[N];
  dw.to(f);
#pragma unroll
  for (int e = 0; e < N; ++e) part[threadIdx.x / L][lane * N + e] = f[Both<T, VW>::template order<INTER>(e)];
  __syncthreads();
  for (int k = threadIdx.x; k < L * N; k += kQkThreads) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kTasks; ++i) sum += part[i][k];
    const int e = k % N;
    const Group of(p, k / N, VW);
    if (e < VW ? of.on0 : of.on1) p.partials[(int64_t)blockIdx.x * p.head_dim + (e < VW ? of.a0 + e : of.a1 + e - VW)] = sum;
  }
}

// ---- heads in single pairs -------------------------------------------------------------------------------
//
// Odd lengths, unaligned tensors, heads of a few values: a lane owns kQkPairs groups of one pair, a value per access. 8192
// tokens, 32 + 8 heads of 128, one element off alignment: BF16 137 + 398 us against 31 + 47 aligned, FP32 101 + 403 against
// 64 + 91. Bound by its instructions, backward by FP64.

template <typename T>
__global__ void __launch_bounds__(kQkThreads) qk_pairs_kernel(const __grid_constant__ QkParams p) {
  start_after_previous_kernel();
  constexpr int U = kQkHeads, VW = 1, N = 2, L = 32, GPL = kQkPairs;
  const int lane = threadIdx.x % L;
  const uint32_t task = blockIdx.x * (kQkThreads / L) + threadIdx.x / L;
  uint32_t t = task / (uint32_t)p.chunks;
  int chunk = (int)(task - t * (uint32_t)p.chunks);
  const bool is_k = chunk >= p.chunks_q, live = t < p.tokens;
  if (!live) t = 0;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int h0 = (is_k ? chunk - p.chunks_q : chunk) * U;
  const int heads = live ? sd.heads - h0 : 0;
  const T* x = static_cast<const T*>(sd.x) + t * sd.x_t + h0 * sd.x_h;

  Both<T, VW> raw[GPL][U];
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[i][u].load(x + u * sd.x_h, g, u < heads);
  }
  float r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      float v[N];
      raw[i][u].unpack(v);
#pragma unroll
      for (int e = 0; e < N; ++e) sum = fmaf(v[e], v[e], sum);
    }
    r[u] = rsqrtf(fmaf(sum_lanes<L>(sum), (float)p.inv_dim, (float)p.eps));
  }
  T* y = static_cast<T*>(sd.out) + t * sd.out_t + h0 * sd.out_h;
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
    float w[N], c[VW], s[VW];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = 1.0f;
    if (sd.w) {
      Both<T, VW> rw;
      rw.load(static_cast<const T*>(sd.w), g, true);
      rw.unpack(w);
    }
    load_angles<VW>(p, p.positions ? (int64_t)p.positions[t] : t, g, c, s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      raw[i][u].unpack(v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= r[u] * w[e];
      if (g.rotated) rotate<VW, false>(v, c, s);
      if (u < heads) Both<T, VW>::store(y + u * sd.out_h, g, v);
    }
  }
}

// In FP64: it serves the heads of a few values, where dx is a small difference (one value: u (1 - xh^2), about eps of u).
template <typename T>
__global__ void __launch_bounds__(kQkThreads) qk_pairs_backward_kernel(const __grid_constant__ QkParams p) {
  start_after_previous_kernel();
  constexpr int VW = 1, N = 2, L = 32, GPL = kQkPairs, kTasks = kQkThreads / L;
  using A = double;
  __shared__ float part[kTasks][L * GPL * N + 1];
  const bool is_k = (int)blockIdx.x >= p.blocks_q;
  const QkSide& sd = p.side[is_k ? 1 : 0];
  const int block = (int)blockIdx.x - (is_k ? p.blocks_q : 0);
  const int blocks = is_k ? (int)gridDim.x - p.blocks_q : p.blocks_q;
  const int lane = threadIdx.x % L;
  const uint32_t heads = (uint32_t)sd.heads, tasks = p.tokens * heads, step = (uint32_t)blocks * kTasks;
  float w[GPL][N], dw[GPL][N];
#pragma unroll
  for (int i = 0; i < GPL; ++i) {
    const Group g(p, lane + i * L, VW);
#pragma unroll
    for (int e = 0; e < N; ++e) { w[i][e] = 1.0f; dw[i][e] = 0.0f; }
    if (sd.w) {
      Both<T, VW> rw;
      rw.load(static_cast<const T*>(sd.w), g, true);
      rw.unpack(w[i]);
    }
  }
  Both<T, VW> rx[GPL], rd[GPL];
  const auto fetch = [&](uint32_t task, bool live) {
    const uint32_t t = live ? task / heads : 0, h = live ? task - t * heads : 0;
    const T* x = static_cast<const T*>(sd.x) + t * sd.x_t + h * sd.x_h;
    const T* d = static_cast<const T*>(sd.dy) + t * sd.dy_t + h * sd.dy_h;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      rx[i].load(x, g, live);
      rd[i].load(d, g, live);
    }
  };
  // every lane of a warp takes part in every round, so that the lane sums see whole warps
  const uint32_t mine = (uint32_t)block * kTasks + threadIdx.x / L, rounds = (tasks + step - 1) / step;
  fetch(mine, mine < tasks);
  for (uint32_t k = 0; k < rounds; ++k) {
    const uint32_t task = mine + k * step;
    const bool live = task < tasks && task >= mine;
    const uint32_t t = live ? task / heads : 0, h = live ? task - t * heads : 0;
    float x[GPL][N], d[GPL][N];
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      rx[i].unpack(x[i]);
      rd[i].unpack(d[i]);
    }
    const uint32_t next = task + step;
    if (k + 1 < rounds) fetch(next, live && next < tasks && next > task);
    A xx = 0, xu = 0;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      if (g.rotated && live) {
        float c[VW], s[VW];
        load_angles<VW>(p, p.positions ? (int64_t)p.positions[t] : t, g, c, s);
        rotate<VW, true>(d[i], c, s);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        xx += (A)x[i][e] * (A)x[i][e];
        xu += (A)x[i][e] * ((A)d[i][e] * (A)w[i][e]);
      }
    }
    const A r = rsqrt(sum_lanes<L>(xx) * (A)p.inv_dim + (A)p.eps);
    const A mean = sum_lanes<L>(xu) * r * (A)p.inv_dim;   // mean(u xh)
    if (!live) continue;
    T* out = static_cast<T*>(sd.out) + t * sd.out_t + h * sd.out_h;
#pragma unroll
    for (int i = 0; i < GPL; ++i) {
      const Group g(p, lane + i * L, VW);
      float o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const A xh = (A)x[i][e] * r;
        dw[i][e] += (float)((A)d[i][e] * xh);
        o[e] = (float)(r * ((A)d[i][e] * (A)w[i][e] - xh * mean));
      }
      Both<T, VW>::store(out, g, o);
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
    const Group g(p, k / (N * GPL) + i * L, VW);
    if (e < VW ? g.on0 : g.on1)
      p.partials[(int64_t)blockIdx.x * p.head_dim + (e < VW ? g.a0 + e : g.a1 + e - VW)] = sum;
  }
}

// dw[d] = sum over the side's blocks of partials[block][d]: 32 columns per block, 32 threads per column,
// each adding every 32nd row, folded in a fixed order.
__global__ void __launch_bounds__(1024) qk_weight_grad_kernel(const float* partials, int head_dim, int blocks_q,
                                                              int blocks, float* dw_q, float* dw_k) {
  __shared__ float part[32][33];
  start_after_previous_kernel();
  const int column = threadIdx.x % 32, row = threadIdx.x / 32, side = blockIdx.y, d = blockIdx.x * 32 + column;
  float* dw = side ? dw_k : dw_q;
  const int lo = side ? blocks_q : 0, hi = side ? blocks : blocks_q;
  float s = 0.0f;
  if (d < head_dim)
    for (int b = lo + row; b < hi; b += 32) s += partials[(int64_t)b * head_dim + d];
  part[row][column] = s;
  __syncthreads();
  if (row == 0 && d < head_dim && dw) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += part[i][column];
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
  if (a->tokens * (a->heads_q > a->heads_k ? a->heads_q : a->heads_k) > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  if (a->rope_dim < 0 || a->rope_dim > a->head_dim || a->rope_dim % 2 != 0 || a->table_rows < 0 ||
      (a->interleaved != 0 && a->interleaved != 1) || (a->dtype != SLIDEDP_BF16 && a->dtype != SLIDEDP_F32) ||
      !(a->eps >= 0.0) || !fits_f32(a->eps) || (a->eps > 0.0 && !positive_f32(a->eps)))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

// What both directions need of their tensors; fills the common part of the parameters. vec: pairs per group, the
// widest that the lengths are multiples of and all tensors are aligned to (8 only for BF16: 16-byte runs).
struct QkPlan {
  QkParams p;
  int vec, lanes;
  unsigned grid;
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
  if (reinterpret_cast<uintptr_t>(positions) % 4 != 0) return SLIDEDP_ERR_INVALID_ARG;
  QkParams& p = plan->p;
  const auto fits = [&](int vec) {
    if (a->rope_dim % (2 * vec) != 0 || (a->head_dim - a->rope_dim) % (2 * vec) != 0) return false;
    if (a->rope_dim > 0 && (reinterpret_cast<uintptr_t>(cos_sin) % 16 != 0 || a->rope_dim % 8 != 0)) return false;
    for (int s = 0; s < 2; ++s) {
      if (heads[s] == 0) continue;
      if (!heads_aligned(in[s], elem, vec * elem, a->tokens, heads[s]) || !heads_aligned(out[s], elem, vec * elem, a->tokens, heads[s]) ||
          (dy && !heads_aligned(dy[s], elem, vec * elem, a->tokens, heads[s])) ||
          reinterpret_cast<uintptr_t>(w[s]) % (uintptr_t)(vec * elem) != 0)
        return false;
    }
    return true;
  };
  for (int s = 0; s < 2; ++s) {
    p.side[s] = QkSide{};
    p.side[s].heads = heads[s];
    if (heads[s] == 0) continue;
    if (!heads_ok(in[s], elem) || !heads_ok(out[s], elem) || (dy && !heads_ok(dy[s], elem)))
      return SLIDEDP_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(w[s]) % (uintptr_t)elem != 0) return SLIDEDP_ERR_INVALID_ARG;
    for (const slidedp_heads* over : {in[s], dy ? dy[s] : in[s]})   // in place, but not with other strides
      if (out[s]->data == over->data && ((a->tokens > 1 && out[s]->stride_token != over->stride_token) ||
                                         (heads[s] > 1 && out[s]->stride_head != over->stride_head)))
        return SLIDEDP_ERR_INVALID_ARG;
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
  }
  p.cos_sin = cos_sin;
  p.positions = positions;
  p.tokens = (uint32_t)a->tokens;
  p.table_rows = a->table_rows;
  p.head_dim = a->head_dim;
  p.rope_dim = a->rope_dim;
  p.interleaved = a->interleaved;
  p.eps = a->eps;
  p.inv_dim = 1.0 / a->head_dim;
  p.partials = nullptr;
  p.blocks_q = 0;
  p.chunks_q = (a->heads_q + kQkHeads - 1) / kQkHeads;
  p.chunks = p.chunks_q + (a->heads_k + kQkHeads - 1) / kQkHeads;
  plan->vec = elem == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
  plan->lanes = 32;
  if (plan->vec > 1)
    for (plan->lanes = 4; plan->lanes * 2 * plan->vec < a->head_dim;) plan->lanes *= 2;
  return SLIDEDP_OK;
}

// The fixed grid, split between queries and keys by their share of the heads: each side that has heads gets at
// least one block, and no more than it has work for.
void split_grid(const slidedp_qk_args* a, int64_t blocks, QkPlan* plan) {
  const int64_t per_block = kQkThreads / plan->lanes;
  int64_t need[2];
  for (int s = 0; s < 2; ++s) {
    QkSide& sd = plan->p.side[s];
    sd.width = sd.chunks = 1;
    need[s] = 0;
    if (sd.heads == 0) continue;
    if (plan->vec > 1) sd.chunks = (sd.heads + kQkHeads - 1) / kQkHeads;
    else sd.chunks = sd.heads;
    sd.width = (sd.heads + sd.chunks - 1) / sd.chunks;
    need[s] = (a->tokens * sd.chunks + per_block - 1) / per_block;
  }
  int64_t q = need[0], k = need[1];
  if (q + k > blocks) {
    q = (int64_t)blocks * a->heads_q / (a->heads_q + a->heads_k);
    if (a->heads_q > 0 && q < 1) q = 1;
    if (a->heads_k > 0 && q > blocks - 1) q = blocks - 1;
    k = blocks - q;
    if (q > need[0]) q = need[0];
    if (k > need[1]) k = need[1];
  }
  plan->p.blocks_q = (int)q;
  plan->grid = (unsigned)(q + k);
}

template <typename T, int VW, bool BACK, bool INTER>
void launch_heads(const QkPlan& plan, cudaStream_t st) {
  switch (plan.lanes) {
    case 4: launch_after(qk_heads_kernel<T, VW, 4, BACK, INTER>, plan.grid, kQkThreads, 0, 1, st, plan.p); break;
    case 8: launch_after(qk_heads_kernel<T, VW, 8, BACK, INTER>, plan.grid, kQkThreads, 0, 1, st, plan.p); break;
    case 16: launch_after(qk_heads_kernel<T, VW, 16, BACK, INTER>, plan.grid, kQkThreads, 0, 1, st, plan.p); break;
    default:   // 2 * VW * 32 values: more than a head has when VW is 8
      if constexpr (VW == 4) launch_after(qk_heads_kernel<T, VW, 32, BACK, INTER>, plan.grid, kQkThreads, 0, 1, st, plan.p);
  }
}
template <bool BACK, bool INTER>
void launch_heads(const slidedp_qk_args* a, const QkPlan& plan, cudaStream_t st) {
  if (a->dtype == SLIDEDP_F32) launch_heads<float, 4, BACK, INTER>(plan, st);
  else if (plan.vec == 8) launch_heads<uint16_t, 8, BACK, INTER>(plan, st);
  else launch_heads<uint16_t, 4, BACK, INTER>(plan, st);
}
template <bool BACK>
void launch_heads(const slidedp_qk_args* a, const QkPlan& plan, cudaStream_t st) {
  if (a->interleaved) launch_heads<BACK, true>(a, plan, st);
  else launch_heads<BACK, false>(a, plan, st);
}

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
  if (rc == SLIDEDP_OK) rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  split_grid(a, 148 * kQkForwardPerSM, &plan);
  FAULT_POINT();
  if (plan.vec > 1) {
    launch_heads<false>(a, plan, st);
  } else {
    const int64_t per_block = kQkThreads / 32;
    const unsigned grid = (unsigned)((a->tokens * plan.p.chunks + per_block - 1) / per_block);
    if (a->dtype == SLIDEDP_F32) launch_after(qk_pairs_kernel<float>, grid, kQkThreads, 0, 1, st, plan.p);
    else launch_after(qk_pairs_kernel<uint16_t>, grid, kQkThreads, 0, 1, st, plan.p);
  }
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
  if (rc == SLIDEDP_OK) rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // a side without rows: its weight gradient is zero
  const size_t dw_bytes = a->head_dim * sizeof(float);
  if (dw_q && (!work || a->heads_q == 0)) { CU(cudaMemsetAsync(dw_q, 0, dw_bytes, st)); dw_q = nullptr; }
  if (dw_k && (!work || a->heads_k == 0)) { CU(cudaMemsetAsync(dw_k, 0, dw_bytes, st)); dw_k = nullptr; }
  if (!work) return SLIDEDP_OK;
  split_grid(a, kQkBackwardBlocks, &plan);
  plan.p.partials = (dw_q || dw_k) ? static_cast<float*>(workspace) : nullptr;
  FAULT_POINT();
  if (plan.vec > 1) launch_heads<true>(a, plan, st);
  else if (a->dtype == SLIDEDP_F32) launch_after(qk_pairs_backward_kernel<float>, plan.grid, kQkThreads, 0, 1, st, plan.p);
  else launch_after(qk_pairs_backward_kernel<uint16_t>, plan.grid, kQkThreads, 0, 1, st, plan.p);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  if (plan.p.partials) {
    FAULT_POINT();
    launch_after(qk_weight_grad_kernel, dim3((a->head_dim + 31) / 32, 2), 1024, 0, 1, st, plan.p.partials, a->head_dim, plan.p.blocks_q,
                 (int)plan.grid, dw_q, dw_k);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  return SLIDEDP_OK;
}

}  // extern "C"
