// libslidedp: attention over packed documents on the tensor cores (tcgen05, TMA, TMEM), forward and
// backward, for head_dim a multiple of 8 up to 128. See include/slidedp_ops.h for the contract.
//
// Bound: the tensor cores, 4 head_dim flops per visible pair and query head forward, 10 backward (14 here,
// see the backward kernels). Everything else hides behind them: one block per SM, whose warps are an
// issuer of matrix products, a producer of TMA loads, and two warpgroups that turn scores into
// probabilities with one TMEM lane (row of the tile) per thread.
//
// BF16 roundings: probabilities and score gradients are BF16 operands of the second products (half an ulp,
// at most 2^-8 of each term, like the inputs they meet); scores, statistics and accumulators are FP32.
#include <atomic>
#include <type_traits>

#include "attention_rows.cuh"
#include "tcgen05.cuh"

namespace slidedp {

constexpr int kTile = 128;                 // rows of a tile: TMEM lanes, and keys or queries per step
constexpr int kHalfBytes = kTile * 128;    // 64 BF16 columns of a tile, as TMA writes them
// Eight warps of rows and a warpgroup with the issuer and the producer. Launched with 168 registers per
// thread (65536 / 384); the row warpgroups then take 216 and the third keeps 72: 2 * 216 + 72 = 3 * 168.
constexpr int kMmaThreads = 384;
constexpr int64_t kSMs = 148;
constexpr int kStageBytes = 4096;          // per warp of rows: 32 rows of 64 BF16 columns, on their way out
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 216;"); }
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 72;"); }
constexpr int kTmemColumns = 512;
constexpr uint32_t kKStep = 32 >> 4;       // descriptor step of 16 contracted values along a row
constexpr uint32_t kRowStep = 16 * 128 >> 4;   // and of 16 contracted rows
// Pairs of eight that take the polynomial exponential. 4096 tokens, 32 heads, forward with 0 / 2 / 4 of eight:
// heads of 64 (half the products per exponential) 118 / 108 / 124 us, of 128 in both directions 158 / 154 / - us.
constexpr int kPolyOfEight = 2;
constexpr float kRescaleAbove = 8.0f;      // log2: how far a row's maximum may run ahead of its scale

template <int HALVES>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int head, int row, uint32_t bar) {
#pragma unroll
  for (int c = 0; c < HALVES; ++c) tma_load_3d(dst + c * kHalfBytes, map, c * 64, head, row, bar);
}

// D = A B^T over the heads' values: A and B tiles in shared memory, both contracted along their rows.
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, int steps, uint32_t desc, bool leader) {
  const uint64_t da = smem_desc_k_major(a), db = smem_desc_k_major(b);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint64_t off = (k >> 2) * (kHalfBytes >> 4) + (k & 3) * kKStep;
    if (k < steps) mma_ss(d, da + off, db + off, desc, k > 0, leader);
  }
}
// D (+)= A B with A (BF16, 128 contracted columns) in TMEM and B a tile contracted over its rows. A's columns
// 64..127 start `second` TMEM columns after the first 64 (32 when all lie together). Steps FROM..TO - 1 of 16.
template <int FROM = 0, int TO = kTile / 16>
__device__ __forceinline__ void product_tmem(uint32_t d, uint32_t a, uint32_t second, uint32_t b, uint32_t desc, bool add, bool leader) {
  const uint64_t db = smem_desc_mn_major(b, kHalfBytes);
#pragma unroll
  for (int k = FROM; k < TO; ++k)
    mma_ts(d, a + (k >> 2) * second + (k & 3) * 8, db + k * kRowStep, desc, add || k > FROM, leader);
}

// How a product becomes a score, chosen per launch: the branches inside a tile's loops would keep the values' long
// chains of special functions from overlapping (9000 cycles a step where these take a third).
enum ScoreMode { kPlain = 0, kBias = 1, kCap = 2 };   // kBias also takes scales that are not positive; kCap has the bias as well

// Scores in units of log2 e, and the factor of d score / d (scale product), two neighbouring columns at a time.
template <int MODE>
struct ScoreMod {
  static constexpr float kSmall = 0.7f;   // where tanh is a polynomial
  float scale;   // of the product; with a cap, the product's scale over the cap
  float cap;     // cap log2 e
  float slope;   // log2 units per position
  __device__ ScoreMod(const AttnParams& p, int h) {
    scale = MODE == kCap ? p.scale / p.softcap : p.scale_log2;
    cap = p.softcap * kLog2e;
    slope = p.slopes ? -p.slopes[h] * kLog2e : 0.0f;
  }
  // Whether the polynomial serves the warp's columns: capped models keep most scores well below the cap.
  template <int N>
  __device__ __forceinline__ bool small(const uint32_t* x) const {
    if constexpr (MODE != kCap) return true;
    float top[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < N; ++c) top[c & 3] = fmaxf(top[c & 3], fabsf(__uint_as_float(x[c])));
    const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * fabsf(scale);
    return __all_sync(0xffffffffu, m <= kSmall);
  }
  // distance: query minus key of the first column; the second's is one less (columns are keys) or one more.
  template <bool SMALL>
  __device__ __forceinline__ void operator()(float r0, float r1, float distance0, float distance1, float* s, float* grad) const {
    grad[0] = grad[1] = 1.0f;
    float th[2];
    if constexpr (MODE == kCap) {
      uint64_t y = mul2(pair(r0, r1), pair(scale, scale)), t;
      if constexpr (SMALL) {
        // tanh y = y + y^3 q(y^2): the odd polynomial of degree 9 with the least greatest error for |y| <= 0.7 (1.4e-7, from
        // a linear program), on the multiply-add pipe: the special functions of the other form, three of them with the
        // exponential, would take longer than the tile's products
        const uint64_t z = mul2(y, y);
        const auto step = [&](uint64_t q, float c) { return fma2(q, z, pair(c, c)); };
        uint64_t q = step(pair(0.01359964907169342f, 0.01359964907169342f), -0.05067462846636772f);
        q = step(q, 0.1327691525220871f);
        q = step(q, -0.3333006501197815f);
        t = fma2(mul2(q, z), y, y);
        split(t, &th[0], &th[1]);
        split(fma2(mul2(t, t), pair(-1.0f, -1.0f), pair(1.0f, 1.0f)), &grad[0], &grad[1]);
      } else {
        // With r = 1 / (1 + exp 2|y|): tanh |y| = 1 - 2 r, absolute error near 2^-23, and 1 at the end; the derivative is
        // 4 r (1 - r), which keeps its digits there (1 - tanh^2 does not: a quarter of it is lost at y = 8)
        float e0, e1, y0, y1;
        split(mul2(y, pair(2.0f * kLog2e, 2.0f * kLog2e)), &e0, &e1);
        const float r0 = rcp_approx(1.0f + exp2_approx(fabsf(e0))), r1 = rcp_approx(1.0f + exp2_approx(fabsf(e1)));
        t = pair(r0, r1);
        split(y, &y0, &y1);
        split(fma2(t, pair(-2.0f, -2.0f), pair(1.0f, 1.0f)), &th[0], &th[1]);
        th[0] = copysignf(th[0], y0);
        th[1] = copysignf(th[1], y1);
        split(fma2(mul2(t, pair(-4.0f, -4.0f)), t, mul2(t, pair(4.0f, 4.0f))), &grad[0], &grad[1]);
      }
      s[0] = fmaf(cap, th[0], slope * fabsf(distance0));
      s[1] = fmaf(cap, th[1], slope * fabsf(distance1));
    } else {
      s[0] = fmaf(r0, scale, slope * fabsf(distance0));
      s[1] = fmaf(r1, scale, slope * fabsf(distance1));
    }
  }
};

// ---- work --------------------------------------------------------------------------------------------
//
// Blocks stay: when one has finished its tile it takes over a block of the grid that has not started yet
// (cluster launch control), so that a tile's loads and first products run while the rows of the tile before are
// stored, and tiles of very different lengths fill the SMs. A warp of the block asks for the next tile and works
// out its range of steps, one tile ahead of the others, who read it from a ring of two.
template <typename Plan>
struct WorkRing {
  alignas(16) uint4 answer;
  uint64_t answered, full[2], empty[2], ask;
  Plan plan[2];
  int item[2];   // -1: no more
  static constexpr uint32_t kNap = 100;
  __device__ void init(int readers) {   // one thread; readers: the warps that take items from the ring
    mbar_init(smem_addr(&answered), 1);
    mbar_init(smem_addr(&ask), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&full[i]), 1);
      mbar_init(smem_addr(&empty[i]), readers);
    }
  }
  // The n-th item, for all threads of a reading warp (or for the one thread `alone`).
  __device__ __forceinline__ bool next(int n, const Waiter& wait, int* it, Plan* pl, bool alone) {
    const int slot = n & 1;
    bool ok = wait(smem_addr(&full[slot]), n >> 1 & 1);
    if (!alone) ok = __all_sync(0xffffffffu, ok);
    if (!ok) return false;
    if (alone) {
      *it = item[slot];
      *pl = plan[slot];
    } else {
      // broadcast, so that all that follows from it is known to be the same for the whole warp
      *it = __shfl_sync(0xffffffffu, item[slot], 0);
      const int* from = reinterpret_cast<const int*>(&plan[slot]);
      int* to = reinterpret_cast<int*>(pl);
#pragma unroll
      for (int i = 0; i < (int)(sizeof(Plan) / sizeof(int)); ++i) to[i] = __shfl_sync(0xffffffffu, from[i], 0);
    }
    if (alone || threadIdx.x % 32 == 0) mbar_arrive(smem_addr(&empty[slot]));
    return *it >= 0;
  }
  // The producer, kAhead steps before it has sent for all of an item: only now is the next one taken, while the last steps
  // and the stores are still to come. (Taken a whole item ahead, the long items of a causal walk ended up two to a block:
  // keys' gradients of one document of 8192 tokens 1035 us.)
  __device__ __forceinline__ void take_next() { mbar_arrive(smem_addr(&ask)); }
  static constexpr int kAhead = 4;
  // The asking warp: make(item) returns the item's plan (in every lane).
  // single: the given item only.
  template <typename F>
  __device__ __forceinline__ void serve(const Waiter& wait, int now, bool single, F make) {
    const int lane = threadIdx.x % 32;
    for (int n = 0;; ++n) {
      const int slot = n & 1;
      if (n >= 2 && !__all_sync(0xffffffffu, wait(smem_addr(&empty[slot]), (n >> 1) + 1 & 1, kNap))) return;
      Plan pl = {};
      if (now >= 0) pl = make(now);
      if (lane == 0) {
        item[slot] = now;
        plan[slot] = pl;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_addr(&full[slot]));
      if (now < 0 || !__all_sync(0xffffffffu, wait(smem_addr(&ask), n & 1, kNap))) return;
      if (single) {
        now = -1;
        continue;
      }
      if (lane == 0) {
        mbar_expect(smem_addr(&answered), 16);
        take_over_next_block(smem_addr(&answer), smem_addr(&answered));
      }
      __syncwarp();
      if (!__all_sync(0xffffffffu, wait(smem_addr(&answered), n & 1))) {
        if (lane == 0) drain(smem_addr(&answered), n & 1);
        return;
      }
      now = taken_block(smem_addr(&answer));
      __syncwarp();
      fence_async_proxy();   // the answer has been read before the next one is written
    }
  }
};

// The document offsets, when there are not too many, in shared memory: every row looks its document up there.
constexpr int kDocCache = 64;
struct DocCache {
  int32_t cu[kDocCache + 1], prefix[kDocCache];
  __device__ void fill(const DocMask& m) {   // all threads of the block
    if (!m.cu || m.docs > kDocCache) return;
    for (int i = threadIdx.x; i <= m.docs; i += blockDim.x) cu[i] = __ldcg(m.cu + i);
    if (m.prefix)
      for (int i = threadIdx.x; i < m.docs; i += blockDim.x) prefix[i] = __ldcg(m.prefix + i);
  }
  __device__ DocMask mask(const DocMask& m) const {
    DocMask r = m;
    if (m.cu && m.docs <= kDocCache) {
      r.cu = cu;
      if (m.prefix) r.prefix = prefix;
    }
    return r;
  }
};

// The columns [a, b) that a row sees, as bits of the 32 columns from c0 on.
__device__ __forceinline__ uint32_t seen_bits(int a, int b, int c0) {
  const auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
  return below(b - c0) & ~below(a - c0);
}

// Stores 128 rows, a warp its own 32, of a tile whose row of FP32 values lies in the thread's TMEM lane, as BF16: 64 columns
// at a time through 4 KB of shared memory per warp, from where TMA writes them (16 bytes per thread straight to global
// memory touched 32 lines per instruction: 3000 cycles a tile). get(c, o) fetches columns 32 c .. of the 64. Returns whether
// the thread saw a NaN.
template <typename F>
__device__ __forceinline__ bool store_columns(uint32_t stage, const CUtensorMap* map, int head, int row0, int column, int head_dim, int tokens,
                                              float factor, F get) {
  const int lane = threadIdx.x % 32;
  if (lane == 0) tma_stores_read();   // the last 64 columns have left the stage
  __syncwarp();
  bool nan = false;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t o[32];
    get(c, o);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float v = __uint_as_float(o[e * 8 + 2 * k]) * factor, w = __uint_as_float(o[e * 8 + 2 * k + 1]) * factor;
        nan |= column + c * 32 + e * 8 < head_dim && !(v == v && w == w);   // columns past the head hold anything
        y[k] = pack_bf16(v, w);
      }
      const uint32_t at = stage + lane * 128 + (((c * 4 + e) ^ (lane & 7)) << 4);   // the 128-byte swizzle
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
    }
  }
  fence_async_proxy();
  __syncwarp();
  if (lane == 0 && row0 < tokens) tma_store_3d(map, stage, column, head, row0);
  return nan && row0 + lane < tokens;
}

// Columns from TMEM, or zeros where nothing was accumulated.
__device__ __forceinline__ void tmem_columns(uint32_t from, bool any, uint32_t* o) {
  if (any) {
    tmem_load32(from, o);
    tmem_wait_load();
    tmem_landed(o);
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e) o[e] = 0;
  }
}

template <int N>
__device__ __forceinline__ void load_floats(float* y, const float* from) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(from)[i];
    y[4 * i] = v.x;
    y[4 * i + 1] = v.y;
    y[4 * i + 2] = v.z;
    y[4 * i + 3] = v.w;
  }
}

// ---- forward -------------------------------------------------------------------------------------------
//
// An item is 256 queries of one head as two tiles of 128 (one per row warpgroup), for which the block walks the keys
// they see in steps of 128. TMEM: scores of the tiles (128 columns each, overwritten by their BF16
// probabilities) and their outputs. The issuer alternates between the tiles, so that one's products
// run while the other's warpgroup exponentiates. A row's accumulators are rescaled only when its
// maximum has grown by more than 2^8 since the last time.
// One causal document of 8192 tokens, 32 + 8 heads of 128: 437 us, 1.26 PFLOP/s of the visible pairs, tensor pipe 64 %
// active; what bounds it is the chain scores, softmax, products of a tile, of which two are in flight.

template <int HALVES> struct ForwardShape {
  static constexpr int kStages = HALVES == 2 ? 2 : 4;
  static constexpr int kTileBytes = HALVES * kHalfBytes;
  static constexpr int kSmem = (2 + 2 * kStages) * kTileBytes + 8 * kStageBytes;
};

struct ForwardPlan {
  int n_lo, steps;           // first key and steps of 128
  int first[2], last[2];     // the steps that concern each tile
  int above[2][2];           // each tile's first and last row in the document offsets
};

struct ForwardControl {
  WorkRing<ForwardPlan> work;
  DocCache docs;
  uint64_t q_full, q_empty, k_full[4], k_empty[4], v_full[4], v_empty[4], s_full[2], p_half[2], p_ready[2], o_full[2], done;
  uint32_t tmem, dead;
};

template <int HALVES, int MODE>
__global__ void __launch_bounds__(kMmaThreads, 1)
    attention_forward_mma_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map_q,
                                 const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                 const __grid_constant__ CUtensorMap map_o) {
  using Shape = ForwardShape<HALVES>;
  constexpr int S = Shape::kStages;
  extern __shared__ __align__(1024) uint8_t raw_smem[];
  __shared__ ForwardControl ctl;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  const int tiles = (p.tokens + 2 * kTile - 1) / (2 * kTile);
  // item -> head and first query: the last queries see the most keys when causal, so they come first
  const auto head_of = [&](int item) { return item % p.heads_q; };
  const auto row_of = [&](int item) { return (tiles - 1 - item / p.heads_q) * 2 * kTile; };
  const uint32_t base = smem_addr(raw_smem);
  const uint32_t smem_q = base, smem_k = base + 2 * Shape::kTileBytes, smem_v = smem_k + S * Shape::kTileBytes,
                 stages = smem_v + S * Shape::kTileBytes;
  const Waiter wait{&ctl.dead, p.error, p.polls};

  if (threadIdx.x == 0) {
    ctl.work.init(10);   // eight of rows, the issuer, the producer
    mbar_init(smem_addr(&ctl.q_full), 1);
    mbar_init(smem_addr(&ctl.q_empty), 1);
    for (int i = 0; i < S; ++i) {
      mbar_init(smem_addr(&ctl.k_full[i]), 1);
      mbar_init(smem_addr(&ctl.k_empty[i]), 1);
      mbar_init(smem_addr(&ctl.v_full[i]), 1);
      mbar_init(smem_addr(&ctl.v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&ctl.s_full[i]), 1);
      mbar_init(smem_addr(&ctl.p_half[i]), kTile);
      mbar_init(smem_addr(&ctl.p_ready[i]), kTile);
      mbar_init(smem_addr(&ctl.o_full[i]), 1);
    }
    mbar_init(smem_addr(&ctl.done), 1);
    ctl.dead = 0;
    mbar_init_fence();
  }
  wait_for_previous_kernel();   // (letting the next kernel in early cost more than it gave: prefixes and caps 67 -> 74 us)
  ctl.docs.fill(p.mask);
  if (warp == 8) tmem_alloc(smem_addr(&ctl.tmem), kTmemColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem;
  const DocMask mask = ctl.docs.mask(p.mask);

  if (warp >= 8) {
    fewer_registers();
    if (warp == 10) {   // ---- the next tiles
      ctl.work.serve(wait, (int)blockIdx.x, false, [&](int item) {
        // lanes 0..3: the keys of each tile's first and last row
        const int m0 = row_of(item), row = min(m0 + (lane >> 1) * kTile + (lane & 1 ? kTile - 1 : 0), p.tokens - 1);
        int lo = 0, hi = 0, index = 0;
        if (lane < 4) {
          index = mask.above(row);
          if (m0 + (lane >> 1) * kTile < p.tokens) mask.keys_of(row, index, &lo, &hi);
        }
        ForwardPlan pl = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) pl.above[i >> 1][i & 1] = __shfl_sync(0xffffffffu, index, i);
        const int lo0 = __shfl_sync(0xffffffffu, lo, 0), hi0 = __shfl_sync(0xffffffffu, hi, 1);
        const int lo1 = __shfl_sync(0xffffffffu, lo, 2), hi1 = __shfl_sync(0xffffffffu, hi, 3);
        const bool on0 = lo0 < hi0, on1 = lo1 < hi1;
        pl.n_lo = on0 && (!on1 || lo0 < lo1) ? lo0 : on1 ? lo1 : 0;
        pl.first[0] = on0 ? (lo0 - pl.n_lo) / kTile : 0;
        pl.last[0] = on0 ? (hi0 - pl.n_lo + kTile - 1) / kTile : 0;
        pl.first[1] = on1 ? (lo1 - pl.n_lo) / kTile : 0;
        pl.last[1] = on1 ? (hi1 - pl.n_lo + kTile - 1) / kTile : 0;
        pl.steps = pl.last[0] > pl.last[1] ? pl.last[0] : pl.last[1];
        return pl;
      });
    } else if (warp == 9 && lane == 0) {   // ---- producer
      int item, sent = 0, walks = 0, q_bytes = 0;   // sent: key and value tiles so far
      int k_sent = 0;
      bool ok = true;
      ForwardPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, true); ++n) {
        if (pl.steps == 0) {
          ctl.work.take_next();
          continue;
        }
        const int h = head_of(item), hk = h / p.group, m0 = row_of(item);
        if (walks > 0 && !(ok = wait(smem_addr(&ctl.q_empty), walks - 1 & 1))) break;
        q_bytes = ((pl.first[0] < pl.last[0]) + (pl.first[1] < pl.last[1])) * Shape::kTileBytes;
        mbar_expect(smem_addr(&ctl.q_full), q_bytes);
        for (int s = 0; s < 2; ++s)
          if (pl.first[s] < pl.last[s])
            load_tile<HALVES>(smem_q + s * Shape::kTileBytes, &map_q, h, m0 + s * kTile, smem_addr(&ctl.q_full));
        ++walks;
        for (int j = 0; j < pl.steps; ++j, ++sent) {
          if (j == max(pl.steps - ctl.work.kAhead, 0)) ctl.work.take_next();
          const int st = sent % S;
          const uint32_t turn = (uint32_t)(sent / S + 1) & 1;   // parity of the previous use's release
          if (sent >= S && !(ok = wait(smem_addr(&ctl.k_empty[st]), turn))) break;
          mbar_expect(smem_addr(&ctl.k_full[st]), Shape::kTileBytes);
          load_tile<HALVES>(smem_k + st * Shape::kTileBytes, &map_k, hk, pl.n_lo + j * kTile, smem_addr(&ctl.k_full[st]));
          ++k_sent;
          if (sent >= S && !(ok = wait(smem_addr(&ctl.v_empty[st]), turn))) break;
          mbar_expect(smem_addr(&ctl.v_full[st]), Shape::kTileBytes);
          load_tile<HALVES>(smem_v + st * Shape::kTileBytes, &map_v, hk, pl.n_lo + j * kTile, smem_addr(&ctl.v_full[st]));
        }
      }
      // leave no copy in flight (whatever `dead` says now: another warp may give up later, and then nobody waits for them)
      if (walks > 0) drain(smem_addr(&ctl.q_full), walks - 1 & 1);
      for (int j = k_sent > S ? k_sent - S : 0; j < k_sent; ++j) drain(smem_addr(&ctl.k_full[j % S]), (j / S) & 1);
      for (int j = sent > S ? sent - S : 0; j < sent; ++j) drain(smem_addr(&ctl.v_full[j % S]), (j / S) & 1);
    } else if (warp == 8) {   // ---- issuer
      const bool leader = elect_leader();
      const auto wait_all = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, wait(bar, parity)); };
      const int k_steps = (p.head_dim + 15) / 16;
      const uint32_t desc_s = mma_desc_bf16(kTile, false), desc_o = mma_desc_bf16(k_steps * 16, true);
      int item, done = 0, walks = 0, turns[2] = {0, 0};   // done: key tiles before this walk; turns: each tile's steps
      bool ok = true;
      ForwardPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
        if (pl.steps == 0) continue;
        if (!(ok = wait_all(smem_addr(&ctl.q_full), walks & 1))) break;
        ++walks;
        // Strictly in turn, so that the tiles stay half a period out of step, one on the tensor cores while the other is on
        // the special functions. (Serving whichever is ready first let the tiles fall into step: one document of 8192
        // tokens 540 us instead of 440.)
        for (int j = -1; j < pl.steps; ++j) {
          // products of step j's probabilities, and step j + 1's scores
          const int at = done + j, st = at % S, nx = (at + 1) % S;
          const bool more = j + 1 < pl.steps;
          bool have_k = false;
          if (j >= 0 && !(ok = wait_all(smem_addr(&ctl.v_full[st]), (at / S) & 1))) break;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (j >= pl.first[s] && j < pl.last[s]) {
              // the first 64 keys' products run while the row warps are on the other 64
              const uint32_t turn = turns[s]++ & 1, v = smem_v + st * Shape::kTileBytes;
              if (!(ok = wait_all(smem_addr(&ctl.p_half[s]), turn))) break;
              tc_fence_after();
              product_tmem<0, 4>(tmem + 256 + s * 128, tmem + s * 128, 32, v, desc_o, j > pl.first[s], leader);
              if (!(ok = wait_all(smem_addr(&ctl.p_ready[s]), turn))) break;
              tc_fence_after();
              product_tmem<4, 8>(tmem + 256 + s * 128, tmem + s * 128, 32, v, desc_o, true, leader);
              if (j == pl.last[s] - 1) mma_commit(smem_addr(&ctl.o_full[s]), leader);
            }
            if (j + 1 >= pl.first[s] && j + 1 < pl.last[s]) {
              if (!have_k) {
                if (!(ok = wait_all(smem_addr(&ctl.k_full[nx]), ((at + 1) / S) & 1))) break;
                have_k = true;
              }
              product_rows(tmem + s * 128, smem_q + s * Shape::kTileBytes, smem_k + nx * Shape::kTileBytes, k_steps, desc_s, leader);
              mma_commit(smem_addr(&ctl.s_full[s]), leader);
            }
          }
          if (!ok) break;
          if (j >= 0) mma_commit(smem_addr(&ctl.v_empty[st]), leader);
          if (more) {
            if (!have_k && !(ok = wait_all(smem_addr(&ctl.k_full[nx]), ((at + 1) / S) & 1))) break;
            mma_commit(smem_addr(&ctl.k_empty[nx]), leader);
            if (j + 2 == pl.steps) mma_commit(smem_addr(&ctl.q_empty), leader);
          }
        }
        done += pl.steps;
      }
      mma_commit(smem_addr(&ctl.done), leader);   // nor a product
      drain(smem_addr(&ctl.done), 0);
    }
  } else {   // ---- rows
    more_registers();
    const int s = warp / 4, r = (warp % 4) * 32;
    const uint32_t at = tmem + ((uint32_t)r << 16) + s * 128, at_o = at + 256;
    const float unit = MODE == kPlain ? p.scale_log2 : 1.0f;   // log2 per unit of the values compared
    int item, turns = 0, walks = 0;
    bool ok = true;
    ForwardPlan pl;
    for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
      const int h = head_of(item), i = row_of(item) + s * kTile + r + lane;
      const int from = s ? pl.first[1] : pl.first[0], to = s ? pl.last[1] : pl.last[0];
      const ScoreMod<MODE> mod(p, h);
      int lo = 0, hi = 0;
      if (i < p.tokens) mask.keys_of(i, mask.above(i, s ? pl.above[1][0] : pl.above[0][0], s ? pl.above[1][1] : pl.above[0][1]), &lo, &hi);
      float m = -INFINITY, l = 0.0f;
      for (int j = from; j < to; ++j, ++turns) {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.s_full[s]), turns & 1));
        if (!ok) break;
        tc_fence_after();
        uint32_t x[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_load32(at + c * 32, x + c * 32);
        tmem_wait_load();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_landed(x + c * 32);
        const int n0 = pl.n_lo + j * kTile;
        if constexpr (MODE != kPlain) {
          const float d0 = (float)(i - n0);
          const auto scores = [&](auto small) {
#pragma unroll
            for (int c = 0; c < 128; c += 2) {
              float y[2], g[2];
              mod.template operator()<decltype(small)::value>(__uint_as_float(x[c]), __uint_as_float(x[c + 1]), d0 - (float)c, d0 - (float)(c + 1), y, g);
              x[c] = __float_as_uint(y[0]);
              x[c + 1] = __float_as_uint(y[1]);
            }
          };
          if (mod.template small<128>(x)) scores(std::true_type()); else if constexpr (MODE == kCap) scores(std::false_type());
        }
        // Visible columns [a, b). Rows past the sequence are not stored: they need no mask.
        const int a = i < p.tokens ? lo - n0 : 0, b = i < p.tokens ? hi - n0 : kTile;
        if (!__all_sync(0xffffffffu, a <= 0 && b >= kTile)) {
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 32) {
            const uint32_t seen = seen_bits(a, b, c0);
#pragma unroll
            for (int c = 0; c < 32; ++c) x[c0 + c] = seen >> c & 1 ? x[c0 + c] : 0xff800000u;
          }
        }
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) top[c] = __uint_as_float(x[c]);
#pragma unroll
        for (int c = 4; c < 128; ++c) top[c & 3] = fmaxf(top[c & 3], __uint_as_float(x[c]));
        const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        const bool grow = mx > -INFINITY && (m == -INFINITY || (mx - m) * unit > kRescaleAbove);
        if (__any_sync(0xffffffffu, grow)) {
          const float keep = !grow ? 1.0f : m == -INFINITY ? 0.0f : exp2_approx((m - mx) * unit);
          if (grow) m = mx;
          l *= keep;
          if (j > from) {   // the products before these scores are complete: they were issued earlier
#pragma unroll
            for (int c = 0; c < HALVES * 2; ++c) {
              uint32_t o[32];
              tmem_load32(at_o + c * 32, o);
              tmem_wait_load();
              tmem_landed(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
              tmem_store32(at_o + c * 32, o);
            }
          }
        }
        const float shift = m == -INFINITY ? 0.0f : m * unit;
        const uint64_t unit2 = pair(unit, unit), shift2 = pair(-shift, -shift);
        uint64_t sum2[2] = {0, 0};
        const auto probabilities = [&](int half) {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const int e = half * 64 + 2 * c;
            const uint64_t y = fma2(pair(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), unit2, shift2);
            float e0, e1;
            if (c % 8 < kPolyOfEight) {
              exp2_pair_poly(y, &e0, &e1);
            } else {
              split(y, &e0, &e1);
              e0 = exp2_approx(e0);
              e1 = exp2_approx(e1);
            }
            sum2[c & 1] = add2(sum2[c & 1], pair(e0, e1));
            pk[c] = pack_bf16(e0, e1);
          }
          tmem_store32(at + half * 32, pk);
        };
        probabilities(0);
        tmem_wait_store();
        tc_fence_before();
        mbar_arrive(smem_addr(&ctl.p_half[s]));
        probabilities(1);
        float s0, s1;
        split(add2(sum2[0], sum2[1]), &s0, &s1);
        l += s0 + s1;
        tmem_wait_store();
        tc_fence_before();
        mbar_arrive(smem_addr(&ctl.p_ready[s]));
      }
      if (ok && from < to) {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.o_full[s]), walks++ & 1));
        tc_fence_after();
      }
      if (!ok) break;
      const bool live = i < p.tokens, some = lo < hi;
      const float inv = some ? 1.0f / l : 0.0f;
      const int row0 = i - lane;
      bool nan = false;
#pragma unroll
      for (int c = 0; c < HALVES; ++c)
        nan |= store_columns(stages + warp * kStageBytes, &map_o, h, row0, c * 64, p.head_dim, p.tokens, inv,
                             [&](int k, uint32_t* o) { tmem_columns(at_o + c * 64 + k * 32, from < to, o); });
      if (live) p.lse[(int64_t)h * p.tokens + i] = some ? (m * unit + log2f(l)) * (1.0f / kLog2e) : -INFINITY;
      // a row with a NaN among its own scores (l is NaN), or with nothing above -inf, is NaN
      uint32_t redo = __ballot_sync(0xffffffffu, nan && (l > 0.0f || !some));
      if (redo) {
        if (lane == 0) tma_stores_done();
        __syncwarp();
        redo = spoiled_out_rows(p, redo, row0, h, lo, hi);
        for (; redo; redo &= redo - 1) attention_out_row<true>(p, row0 + __ffs(redo) - 1, h, false);   // its lse is right: masked scores are dropped
      }
    }
    if (lane == 0) tma_stores_done();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_free(tmem, kTmemColumns);
}

// ---- backward -------------------------------------------------------------------------------------------
//
// With P = exp2(s - lse), dP = dO V^T and dS = P (dP - delta) (d score / d product):
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
// Two kernels, one walking the queries of a tile of keys and one the keys of a tile of queries, so that every
// sum is taken by one block in a fixed order. That costs the scores and dP twice (14 head_dim flops per
// pair instead of 10) and buys the same bits in every run without FP32 atomics on dQ.

// Keys: an item is 128 keys of one key head, for which the block walks all queries that see them, for every query head of
// the group. Rows of the tiles (TMEM lanes) are keys: S^T = K Q^T and dP^T = V dO^T, so that P^T and dS^T
// are, as they stand, the left operands of dV and dK. TMEM: S^T, dP^T (overwritten by P^T and dS^T, each
// warpgroup within its own 64 columns), dV, dK. When there are few tiles of keys, a cluster of blocks shares an item, each
// taking some of the group's query heads, and adds up through distributed shared memory.
// The same document: 868 us, 1.27 PFLOP/s of its 8 head_dim flops per pair, tensor pipe 60 % active: the rows' work on P and
// dS stands between the products of one step, and TMEM has no room for a second pair of S^T and dP^T.
template <int HALVES> struct KeysShape {
  static constexpr int kStages = 2;
  static constexpr int kTileBytes = HALVES * kHalfBytes;
  static constexpr int kSmem = (2 + 2 * kStages) * kTileBytes + 8 * kStageBytes;
};

struct KeysPlan {
  int q_lo, per_head;   // first tile of queries, tiles of queries per query head
  int above[2];         // the first and last key in the document offsets
};

struct KeysControl {
  WorkRing<KeysPlan> work;
  DocCache docs;
  alignas(16) float lse[2][kTile];
  alignas(16) float delta[2][kTile];
  uint64_t kv_full, kv_empty, q_full[2], q_empty[2], do_full[2], do_empty[2], s_full, dp_full, p_ready, ds_ready, acc_full, done;
  uint32_t tmem, dead;
};

template <int HALVES, int MODE>
__global__ void __launch_bounds__(kMmaThreads, 1)
    attention_dkv_mma_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map_q,
                             const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                             const __grid_constant__ CUtensorMap map_do, const __grid_constant__ CUtensorMap map_dk,
                             const __grid_constant__ CUtensorMap map_dv, int split) {
  using Shape = KeysShape<HALVES>;
  constexpr int S = Shape::kStages;
  extern __shared__ __align__(1024) uint8_t raw_smem[];
  __shared__ KeysControl ctl;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  // item -> key head and first key: the first keys are seen by the most queries when causal, so they come first
  const auto head_of = [&](int item) { return item % p.heads_kv; };
  const auto row_of = [&](int item) { return item / p.heads_kv * kTile; };
  // the block's share of the group's query heads
  const int rank = (int)(blockIdx.x % split), h_from = rank * p.group / split, heads = (rank + 1) * p.group / split - h_from;
  const uint32_t base = smem_addr(raw_smem);
  const uint32_t smem_k = base, smem_v = smem_k + Shape::kTileBytes, smem_q = smem_v + Shape::kTileBytes,
                 smem_do = smem_q + S * Shape::kTileBytes, stages = smem_do + S * Shape::kTileBytes;
  const Waiter wait{&ctl.dead, p.error, p.polls};

  if (threadIdx.x == 0) {
    ctl.work.init(10);   // eight of rows, the issuer, the producer
    mbar_init(smem_addr(&ctl.kv_full), 1);
    mbar_init(smem_addr(&ctl.kv_empty), 1);
    for (int i = 0; i < S; ++i) {
      mbar_init(smem_addr(&ctl.q_full[i]), 1);
      mbar_init(smem_addr(&ctl.q_empty[i]), 1);
      mbar_init(smem_addr(&ctl.do_full[i]), 1);
      mbar_init(smem_addr(&ctl.do_empty[i]), 1);
    }
    mbar_init(smem_addr(&ctl.s_full), 1);
    mbar_init(smem_addr(&ctl.dp_full), 1);
    mbar_init(smem_addr(&ctl.p_ready), 2 * kTile);
    mbar_init(smem_addr(&ctl.ds_ready), 2 * kTile);
    mbar_init(smem_addr(&ctl.acc_full), 1);
    mbar_init(smem_addr(&ctl.done), 1);
    ctl.dead = 0;
    mbar_init_fence();
  }
  wait_for_previous_kernel();
  allow_next_kernel();   // the queries' kernel, which needs what was there before this one
  ctl.docs.fill(p.mask);
  if (warp == 8) tmem_alloc(smem_addr(&ctl.tmem), kTmemColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem, at_s = tmem, at_dp = tmem + 128, at_dv = tmem + 256, at_dk = tmem + 384;
  const DocMask mask = ctl.docs.mask(p.mask);

  if (warp >= 8) {
    fewer_registers();
    if (warp == 10) {   // ---- the next tiles
      ctl.work.serve(wait, (int)(blockIdx.x / split), split > 1, [&](int item) {
        const int row = min(row_of(item) + (lane ? kTile - 1 : 0), p.tokens - 1);   // lanes 0 and 1: first and last key
        int lo = 0, hi = 0, index = 0;
        if (lane < 2) {
          index = mask.above(row);
          mask.queries_of(row, index, &lo, &hi);
        }
        lo = __shfl_sync(0xffffffffu, lo, 0);
        hi = __shfl_sync(0xffffffffu, hi, 1);
        return KeysPlan{lo / kTile, hi > lo ? (hi + kTile - 1) / kTile - lo / kTile : 0,
                        {__shfl_sync(0xffffffffu, index, 0), __shfl_sync(0xffffffffu, index, 1)}};
      });
    } else if (warp == 9 && lane == 0) {   // ---- producer
      int item, q_sent = 0, sent = 0, walks = 0;
      bool ok = true;
      KeysPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, true); ++n) {
        if (pl.per_head == 0) {
          ctl.work.take_next();
          continue;
        }
        const int hk = head_of(item), n0 = row_of(item);
        if (walks > 0 && !(ok = wait(smem_addr(&ctl.kv_empty), walks - 1 & 1))) break;
        mbar_expect(smem_addr(&ctl.kv_full), 2 * Shape::kTileBytes);
        load_tile<HALVES>(smem_k, &map_k, hk, n0, smem_addr(&ctl.kv_full));
        load_tile<HALVES>(smem_v, &map_v, hk, n0, smem_addr(&ctl.kv_full));
        ++walks;
        int left = pl.per_head * heads;
        for (int h = hk * p.group + h_from; left > 0 && ok; ++h)
          for (int tile = 0; tile < pl.per_head; ++tile, ++sent, --left) {
            if (left == min(pl.per_head * heads, ctl.work.kAhead)) ctl.work.take_next();
            const int st = sent % S, m0 = (pl.q_lo + tile) * kTile;
            const uint32_t turn = (uint32_t)(sent / S + 1) & 1;
            if (sent >= S && !(ok = wait(smem_addr(&ctl.q_empty[st]), turn))) break;
            mbar_expect(smem_addr(&ctl.q_full[st]), Shape::kTileBytes + 2 * kTile * sizeof(float));
            load_tile<HALVES>(smem_q + st * Shape::kTileBytes, &map_q, h, m0, smem_addr(&ctl.q_full[st]));
            bulk_load(smem_addr(ctl.lse[st]), p.row_lse + h * p.pitch + m0, kTile * sizeof(float), smem_addr(&ctl.q_full[st]));
            bulk_load(smem_addr(ctl.delta[st]), p.row_delta + h * p.pitch + m0, kTile * sizeof(float), smem_addr(&ctl.q_full[st]));
            ++q_sent;
            if (sent >= S && !(ok = wait(smem_addr(&ctl.do_empty[st]), turn))) break;
            mbar_expect(smem_addr(&ctl.do_full[st]), Shape::kTileBytes);
            load_tile<HALVES>(smem_do + st * Shape::kTileBytes, &map_do, h, m0, smem_addr(&ctl.do_full[st]));
          }
      }
      if (walks > 0) drain(smem_addr(&ctl.kv_full), walks - 1 & 1);
      for (int j = q_sent > S ? q_sent - S : 0; j < q_sent; ++j) drain(smem_addr(&ctl.q_full[j % S]), (j / S) & 1);
      for (int j = sent > S ? sent - S : 0; j < sent; ++j) drain(smem_addr(&ctl.do_full[j % S]), (j / S) & 1);
    } else if (warp == 8) {   // ---- issuer
      const bool leader = elect_leader();
      const auto wait_all = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, wait(bar, parity)); };
      const int k_steps = (p.head_dim + 15) / 16;
      const uint32_t desc_s = mma_desc_bf16(kTile, false), desc_acc = mma_desc_bf16(k_steps * 16, true);
      int item, done = 0, walks = 0;   // done: steps before this walk
      bool ok = true;
      KeysPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
        const int steps = pl.per_head * heads;
        if (steps == 0) continue;
        if (!(ok = wait_all(smem_addr(&ctl.kv_full), walks & 1))) break;
        ++walks;
        for (int it = -1; it < steps; ++it) {
          const int at = done + it, st = at % S, nx = (at + 1) % S;
          const bool more = it + 1 < steps;
          const uint32_t next_turn = ((at + 1) / S) & 1;
          if (it >= 0) {
            if (!(ok = wait_all(smem_addr(&ctl.p_ready), at & 1))) break;
            tc_fence_after();
            product_tmem(at_dv, at_s, 64, smem_do + st * Shape::kTileBytes, desc_acc, it > 0, leader);
            mma_commit(smem_addr(&ctl.do_empty[st]), leader);
          }
          if (more) {
            if (!(ok = wait_all(smem_addr(&ctl.q_full[nx]), next_turn))) break;
            product_rows(at_s, smem_k, smem_q + nx * Shape::kTileBytes, k_steps, desc_s, leader);
            mma_commit(smem_addr(&ctl.s_full), leader);
          }
          if (it >= 0) {
            if (!(ok = wait_all(smem_addr(&ctl.ds_ready), at & 1))) break;
            tc_fence_after();
            product_tmem(at_dk, at_dp, 64, smem_q + st * Shape::kTileBytes, desc_acc, it > 0, leader);
            mma_commit(smem_addr(&ctl.q_empty[st]), leader);
          }
          if (more) {
            if (!(ok = wait_all(smem_addr(&ctl.do_full[nx]), next_turn))) break;
            product_rows(at_dp, smem_v, smem_do + nx * Shape::kTileBytes, k_steps, desc_s, leader);
            mma_commit(smem_addr(&ctl.dp_full), leader);
            if (it + 2 == steps) mma_commit(smem_addr(&ctl.kv_empty), leader);
          }
        }
        done += steps;
        if (ok) mma_commit(smem_addr(&ctl.acc_full), leader);
      }
      mma_commit(smem_addr(&ctl.done), leader);   // nor a product
      drain(smem_addr(&ctl.done), 0);
    }
    if (split > 1) {   // as below
      __syncwarp();
      cluster_sync();
      cluster_sync();
    }
  } else {   // ---- rows: keys; the warpgroups take 64 of a step's queries each
    more_registers();
    const int g = warp / 4, r = (warp % 4) * 32;
    const uint32_t at = ((uint32_t)r << 16) + g * 64;
    int item, turns = 0, walks = 0;
    bool ok = true, joined = false;
    KeysPlan pl;
    for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
      const int hk = head_of(item), n0 = row_of(item), j = n0 + r + lane, steps = pl.per_head * heads;
      int lo = 0, hi = 0;
      if (j < p.tokens) mask.queries_of(j, mask.above(j, pl.above[0], pl.above[1]), &lo, &hi);
      int h = hk * p.group + h_from, tile = 0;
      ScoreMod<MODE> mod(p, h);
      for (int it = 0; it < steps; ++it, ++tile, ++turns) {
        if (tile == pl.per_head) {
          tile = 0;
          mod = ScoreMod<MODE>(p, ++h);
        }
        const int st = turns % S, m0 = (pl.q_lo + tile) * kTile + g * 64;
        // The queries' statistics come from shared memory, which the tensor cores keep busy: they are
        // fetched in blocks ahead of the waits (one at a time, each use waited 200 cycles).
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.q_full[st]), (turns / S) & 1));
        if (!ok) break;
        float y[64];
        load_floats<64>(y, &ctl.lse[st][g * 64]);
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.s_full), turns & 1));
        if (!ok) break;
        tc_fence_after();
        uint32_t x[64];
        tmem_load32(at_s + at, x);
        tmem_load32(at_s + at + 32, x + 32);
        tmem_wait_load();
        tmem_landed(x);
        tmem_landed(x + 32);
        const int a = j < p.tokens ? lo - m0 : 0, b = j < p.tokens ? hi - m0 : 64;   // visible columns [a, b)
        const bool whole = __all_sync(0xffffffffu, a <= 0 && b >= 64);
        const uint32_t seen[2] = {seen_bits(a, b, 0), seen_bits(a, b, 32)};
        float pr[64];   // P (d score / d product)
        {
          uint32_t pk[32];
          const float d0 = (float)(j - m0);
          const auto probabilities = [&](auto masked, auto small) {
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
              float e[2], grad[2] = {1.0f, 1.0f};
              if constexpr (MODE != kPlain)
                mod.template operator()<decltype(small)::value>(__uint_as_float(x[c]), __uint_as_float(x[c + 1]), d0 - (float)c, d0 - (float)(c + 1), e, grad);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                e[k] = exp2_approx(MODE != kPlain ? e[k] - y[c + k] : fmaf(__uint_as_float(x[c + k]), p.scale_log2, -y[c + k]));
                if (decltype(masked)::value) e[k] = seen[c / 32] >> (c % 32 + k) & 1 ? e[k] : 0.0f;
                pr[c + k] = MODE == kCap ? e[k] * grad[k] : e[k];
              }
              pk[c / 2] = pack_bf16(e[0], e[1]);
            }
          };
          if (mod.template small<64>(x)) {
            if (whole) probabilities(std::false_type(), std::true_type()); else probabilities(std::true_type(), std::true_type());
          } else if constexpr (MODE == kCap) {
            probabilities(std::true_type(), std::false_type());
          }
          tmem_store32(at_s + at, pk);
        }
        tmem_wait_store();
        tc_fence_before();
        mbar_arrive(smem_addr(&ctl.p_ready));

        load_floats<64>(y, &ctl.delta[st][g * 64]);
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.dp_full), turns & 1));
        if (!ok) break;
        tc_fence_after();
        {
          uint32_t pk[32];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t d[32];
            tmem_load32(at_dp + at + half * 32, d);
            tmem_wait_load();
            tmem_landed(d);
            const auto gradients = [&](auto masked) {
#pragma unroll
              for (int c = 0; c < 32; c += 2) {
                const int n = half * 32 + c;
                float e0 = pr[n] * (__uint_as_float(d[c]) - y[n]), e1 = pr[n + 1] * (__uint_as_float(d[c + 1]) - y[n + 1]);
                if (decltype(masked)::value) {   // not zero times what a masked pair holds
                  e0 = seen[half] >> c & 1 ? e0 : 0.0f;
                  e1 = seen[half] >> (c + 1) & 1 ? e1 : 0.0f;
                }
                pk[n / 2] = pack_bf16(e0, e1);
              }
            };
            if (whole) gradients(std::false_type()); else gradients(std::true_type());
          }
          tmem_store32(at_dp + at, pk);
        }
        tmem_wait_store();
        tc_fence_before();
        mbar_arrive(smem_addr(&ctl.ds_ready));
      }
      if (ok && steps > 0) {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.acc_full), walks++ & 1));
        tc_fence_after();
      }
      if (!ok) break;
      const int row0 = j - lane;
      const uint32_t lanes = (uint32_t)r << 16;
      if (split > 1) {
        // The blocks of the cluster hold the sums over their heads of both outputs, side by side as 2 HALVES 64 columns. Each
        // block adds up its share of the columns, in the order of the blocks: the others write theirs into its rings, which
        // are free once everyone's products are done.
        constexpr int kColumns = 2 * HALVES * 64;
        const int width = kColumns / split;
        const auto column = [&](int c) { return (c < HALVES * 64 ? at_dv + c : at_dk + c - HALVES * 64) + lanes; };
        const auto slot = [&](int from, int c) { return smem_q + (from * width + c) * (kTile * 4) + (r + lane) * 16; };   // [column / 4][row]
        cluster_sync();
        for (int to = 0; to < split; ++to) {
          if (to == rank) continue;
          const uint32_t there = peer_addr(slot(rank, 0), to);
          for (int c = g * 32; c < width; c += 64) {
            uint32_t o[32];
            tmem_columns(column(to * width + c), steps > 0, o);
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there + (c + e) * (kTile * 4)), "r"(o[e]), "r"(o[e + 1]),
                           "r"(o[e + 2]), "r"(o[e + 3])
                           : "memory");
          }
        }
        cluster_sync();
        if (g * 64 < width) {
          const int first = rank * width + g * 64, d0 = first % (HALVES * 64);
          const bool is_k = first >= HALVES * 64;
          const bool nan = store_columns(stages + warp * kStageBytes, is_k ? &map_dk : &map_dv, hk, row0, d0, p.head_dim, p.tokens,
                                         is_k ? p.scale : 1.0f, [&](int k, uint32_t* o) {
            float sum[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) sum[e] = 0.0f;
            for (int from = 0; from < split; ++from) {
              if (from == rank) {
                tmem_columns(column(first + k * 32), steps > 0, o);
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[e] += __uint_as_float(o[e]);
              } else {
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  float v[4];
                  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                               : "r"(slot(from, g * 64 + k * 32 + e)) : "memory");
#pragma unroll
                  for (int i = 0; i < 4; ++i) sum[e + i] += v[i];
                }
              }
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(sum[e]);
          });
          uint32_t redo = __ballot_sync(0xffffffffu, nan);
          if (redo) {
            if (lane == 0) tma_stores_done();
            __syncwarp();
            const int d1 = min(d0 + 64, p.head_dim);
            redo = spoiled_key_rows(p, redo, row0, hk, lo, hi, !is_k, d0, d1);
            for (; redo; redo &= redo - 1) attention_dkv_row<true>(p, row0 + __ffs(redo) - 1, hk, is_k, !is_k, d0, d1);
          }
        }
        joined = true;
      } else {
        // warpgroup 0 stores dV, warpgroup 1 dK
        bool nan = false;
#pragma unroll
        for (int c = 0; c < HALVES; ++c)
          nan |= store_columns(stages + warp * kStageBytes, g ? &map_dk : &map_dv, hk, row0, c * 64, p.head_dim, p.tokens, g ? p.scale : 1.0f,
                               [&](int k, uint32_t* o) { tmem_columns((g ? at_dk : at_dv) + lanes + c * 64 + k * 32, steps > 0, o); });
        uint32_t redo = __ballot_sync(0xffffffffu, nan);
        if (redo) {
          if (lane == 0) tma_stores_done();
          __syncwarp();
          redo = spoiled_key_rows(p, redo, row0, hk, lo, hi, g == 0, 0, p.head_dim);
          for (; redo; redo &= redo - 1) attention_dkv_row<true>(p, row0 + __ffs(redo) - 1, hk, g == 1, g == 0, 0, p.head_dim);
        }
      }
    }
    if (split > 1 && !joined) {   // gave up: the others still come to the barriers
      __syncwarp();
      cluster_sync();
      cluster_sync();
    }
    if (lane == 0) tma_stores_done();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_free(tmem, kTmemColumns);
}

// Queries: an item is 128 queries of one head, for which the block walks the keys that they see. Rows are queries; dS goes
// where its scores were. TMEM: two buffers of scores (the next step's are made while this one's are
// worked on), dP, dQ. The same document: 567 us, 1.46 PFLOP/s of its 6 head_dim flops per pair, tensor pipe 72 % active.
//
// It starts without a wait of its own, beside the keys' kernel. All that it reads was there before that kernel: a block of that
// lets it start only after its own wait has returned, that is when the kernels before it are complete and their writes are in
// L2, and from L2 this one reads, by TMA or with loads that pass L1 by (the statistics, offsets that fit the cache; of a longer
// list of offsets L1 holds nothing older than this kernel's start). It writes dQ only, which no kernel reads that may still
// run, as no output may lie over an input; and its blocks end after the keys' kernel has.
template <int HALVES> struct QueriesShape {
  static constexpr int kKStages = 3;   // the next step's scores need K beside this step's dS K
  static constexpr int kVStages = HALVES == 2 ? 1 : 2;   // the stores' room; V comes back while the rows work on dP
  static constexpr int kTileBytes = HALVES * kHalfBytes;
  static constexpr int kSmem = (2 + kKStages + kVStages) * kTileBytes + 8 * kStageBytes;
};

struct QueriesPlan {
  int n_lo, steps;   // first key and steps of 128
  int above[2];      // the first and last query in the document offsets
};

struct QueriesControl {
  WorkRing<QueriesPlan> work;
  DocCache docs;
  uint64_t q_full, q_empty, k_full[3], k_empty[3], v_full[2], v_empty[2], s_full[2], dp_full, ds_ready, acc_full, done;
  uint32_t tmem, dead;
};

template <int HALVES, int MODE>
__global__ void __launch_bounds__(kMmaThreads, 1)
    attention_dq_mma_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map_q,
                            const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                            const __grid_constant__ CUtensorMap map_do, const __grid_constant__ CUtensorMap map_dq) {
  using Shape = QueriesShape<HALVES>;
  constexpr int SK = Shape::kKStages, SV = Shape::kVStages;
  extern __shared__ __align__(1024) uint8_t raw_smem[];
  __shared__ QueriesControl ctl;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  const int tiles = (p.tokens + kTile - 1) / kTile;
  const auto head_of = [&](int item) { return item % p.heads_q; };
  const auto row_of = [&](int item) { return (tiles - 1 - item / p.heads_q) * kTile; };
  const uint32_t base = smem_addr(raw_smem);
  const uint32_t smem_q = base, smem_do = smem_q + Shape::kTileBytes, smem_k = smem_do + Shape::kTileBytes,
                 smem_v = smem_k + SK * Shape::kTileBytes, stages = smem_v + SV * Shape::kTileBytes;
  const Waiter wait{&ctl.dead, p.error, p.polls};

  if (threadIdx.x == 0) {
    ctl.work.init(10);
    mbar_init(smem_addr(&ctl.q_full), 1);
    mbar_init(smem_addr(&ctl.q_empty), 1);
    for (int i = 0; i < SK; ++i) {
      mbar_init(smem_addr(&ctl.k_full[i]), 1);
      mbar_init(smem_addr(&ctl.k_empty[i]), 1);
    }
    for (int i = 0; i < SV; ++i) {
      mbar_init(smem_addr(&ctl.v_full[i]), 1);
      mbar_init(smem_addr(&ctl.v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(smem_addr(&ctl.s_full[i]), 1);
    mbar_init(smem_addr(&ctl.dp_full), 1);
    mbar_init(smem_addr(&ctl.ds_ready), 2 * kTile);
    mbar_init(smem_addr(&ctl.acc_full), 1);
    mbar_init(smem_addr(&ctl.done), 1);
    ctl.dead = 0;
    mbar_init_fence();
  }
  ctl.docs.fill(p.mask);
  if (warp == 8) tmem_alloc(smem_addr(&ctl.tmem), kTmemColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem, at_s = tmem, at_dp = tmem + 256, at_dq = tmem + 384;   // at_s: two buffers
  const DocMask mask = ctl.docs.mask(p.mask);

  if (warp >= 8) {
    fewer_registers();
    if (warp == 10) {   // ---- the next tiles
      ctl.work.serve(wait, (int)blockIdx.x, false, [&](int item) {
        const int row = min(row_of(item) + (lane ? kTile - 1 : 0), p.tokens - 1);   // lanes 0 and 1: first and last query
        int lo = 0, hi = 0, index = 0;
        if (lane < 2) {
          index = mask.above(row);
          mask.keys_of(row, index, &lo, &hi);
        }
        lo = __shfl_sync(0xffffffffu, lo, 0);
        hi = __shfl_sync(0xffffffffu, hi, 1);
        return QueriesPlan{lo, hi > lo ? (hi - lo + kTile - 1) / kTile : 0,
                           {__shfl_sync(0xffffffffu, index, 0), __shfl_sync(0xffffffffu, index, 1)}};
      });
    } else if (warp == 9 && lane == 0) {   // ---- producer
      int item, k_sent = 0, sent = 0, walks = 0;
      bool ok = true;
      QueriesPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, true); ++n) {
        if (pl.steps == 0) {
          ctl.work.take_next();
          continue;
        }
        const int h = head_of(item), hk = h / p.group, m0 = row_of(item);
        if (walks > 0 && !(ok = wait(smem_addr(&ctl.q_empty), walks - 1 & 1))) break;
        mbar_expect(smem_addr(&ctl.q_full), 2 * Shape::kTileBytes);
        load_tile<HALVES>(smem_q, &map_q, h, m0, smem_addr(&ctl.q_full));
        load_tile<HALVES>(smem_do, &map_do, h, m0, smem_addr(&ctl.q_full));
        ++walks;
        for (int j = 0; j < pl.steps; ++j, ++sent) {
          if (j == max(pl.steps - ctl.work.kAhead, 0)) ctl.work.take_next();
          const int sk = sent % SK, sv = sent % SV;
          if (sent >= SK && !(ok = wait(smem_addr(&ctl.k_empty[sk]), (uint32_t)(sent / SK + 1) & 1))) break;
          mbar_expect(smem_addr(&ctl.k_full[sk]), Shape::kTileBytes);
          load_tile<HALVES>(smem_k + sk * Shape::kTileBytes, &map_k, hk, pl.n_lo + j * kTile, smem_addr(&ctl.k_full[sk]));
          ++k_sent;
          if (sent >= SV && !(ok = wait(smem_addr(&ctl.v_empty[sv]), (uint32_t)(sent / SV + 1) & 1))) break;
          mbar_expect(smem_addr(&ctl.v_full[sv]), Shape::kTileBytes);
          load_tile<HALVES>(smem_v + sv * Shape::kTileBytes, &map_v, hk, pl.n_lo + j * kTile, smem_addr(&ctl.v_full[sv]));
        }
      }
      if (walks > 0) drain(smem_addr(&ctl.q_full), walks - 1 & 1);
      for (int j = k_sent > SK ? k_sent - SK : 0; j < k_sent; ++j) drain(smem_addr(&ctl.k_full[j % SK]), (j / SK) & 1);
      for (int j = sent > SV ? sent - SV : 0; j < sent; ++j) drain(smem_addr(&ctl.v_full[j % SV]), (j / SV) & 1);
    } else if (warp == 8) {   // ---- issuer
      const bool leader = elect_leader();
      const auto wait_all = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, wait(bar, parity)); };
      const int k_steps = (p.head_dim + 15) / 16;
      const uint32_t desc_s = mma_desc_bf16(kTile, false), desc_acc = mma_desc_bf16(k_steps * 16, true);
      int item, done = 0, walks = 0;   // done: steps before this walk
      bool ok = true;
      QueriesPlan pl;
      for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
        if (pl.steps == 0) continue;
        if (!(ok = wait_all(smem_addr(&ctl.q_full), walks & 1))) break;
        ++walks;
        for (int j = -1; j < pl.steps; ++j) {
          const int at = done + j, nk = (at + 1) % SK, nv = (at + 1) % SV;
          const bool more = j + 1 < pl.steps;
          if (more) {
            if (!(ok = wait_all(smem_addr(&ctl.k_full[nk]), ((at + 1) / SK) & 1))) break;
            product_rows(at_s + (at + 1 & 1) * 128, smem_q, smem_k + nk * Shape::kTileBytes, k_steps, desc_s, leader);
            mma_commit(smem_addr(&ctl.s_full[at + 1 & 1]), leader);
          }
          if (j >= 0) {
            if (!(ok = wait_all(smem_addr(&ctl.ds_ready), at & 1))) break;
            tc_fence_after();
          }
          if (more) {
            if (!(ok = wait_all(smem_addr(&ctl.v_full[nv]), ((at + 1) / SV) & 1))) break;
            product_rows(at_dp, smem_do, smem_v + nv * Shape::kTileBytes, k_steps, desc_s, leader);
            mma_commit(smem_addr(&ctl.dp_full), leader);
            mma_commit(smem_addr(&ctl.v_empty[nv]), leader);
            if (j + 2 == pl.steps) mma_commit(smem_addr(&ctl.q_empty), leader);
          }
          if (j >= 0) {
            product_tmem(at_dq, at_s + (at & 1) * 128, 64, smem_k + (at % SK) * Shape::kTileBytes, desc_acc, j > 0, leader);
            mma_commit(smem_addr(&ctl.k_empty[at % SK]), leader);
          }
        }
        done += pl.steps;
        if (ok) mma_commit(smem_addr(&ctl.acc_full), leader);
      }
      mma_commit(smem_addr(&ctl.done), leader);   // nor a product
      drain(smem_addr(&ctl.done), 0);
    }
  } else {   // ---- rows: queries; the warpgroups take 64 of a step's keys each
    more_registers();
    const int g = warp / 4, r = (warp % 4) * 32;
    const uint32_t at = ((uint32_t)r << 16) + g * 64;
    int item, turns = 0, walks = 0;
    bool ok = true;
    QueriesPlan pl;
    for (int n = 0; ok && ctl.work.next(n, wait, &item, &pl, false); ++n) {
      const int h = head_of(item), m0 = row_of(item), i = m0 + r + lane, steps = pl.steps;
      const ScoreMod<MODE> mod(p, h);
      int lo = 0, hi = 0;
      float lse = 0.0f, delta = 0.0f;
      if (i < p.tokens) {
        mask.keys_of(i, mask.above(i, pl.above[0], pl.above[1]), &lo, &hi);
        lse = __ldcg(p.row_lse + h * p.pitch + i);
        delta = __ldcg(p.row_delta + h * p.pitch + i);
      }
      for (int j = 0; j < steps; ++j, ++turns) {
        const uint32_t buf = at_s + (turns & 1) * 128 + at;
        const int c0 = pl.n_lo + j * kTile + g * 64;
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.s_full[turns & 1]), (turns >> 1) & 1));
        if (!ok) break;
        tc_fence_after();
        uint32_t x[64];
        tmem_load32(buf, x);
        tmem_load32(buf + 32, x + 32);
        tmem_wait_load();
        tmem_landed(x);
        tmem_landed(x + 32);
        const int a = i < p.tokens ? lo - c0 : 0, b = i < p.tokens ? hi - c0 : 64;   // visible columns [a, b)
        const bool whole = __all_sync(0xffffffffu, a <= 0 && b >= 64);
        const uint32_t seen[2] = {seen_bits(a, b, 0), seen_bits(a, b, 32)};
        float pr[64];
        const float d0 = (float)(i - c0);
        const auto probabilities = [&](auto small) {
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            float e[2], grad[2] = {1.0f, 1.0f};
            if constexpr (MODE != kPlain)
              mod.template operator()<decltype(small)::value>(__uint_as_float(x[c]), __uint_as_float(x[c + 1]), d0 - (float)c, d0 - (float)(c + 1), e, grad);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              pr[c + k] = exp2_approx(MODE != kPlain ? e[k] - lse : fmaf(__uint_as_float(x[c + k]), p.scale_log2, -lse));
              if (MODE == kCap) pr[c + k] *= grad[k];
            }
          }
        };
        if (mod.template small<64>(x)) probabilities(std::true_type()); else if constexpr (MODE == kCap) probabilities(std::false_type());
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.dp_full), turns & 1));
        if (!ok) break;
        tc_fence_after();
        tmem_load32(at_dp + at, x);
        tmem_load32(at_dp + at + 32, x + 32);
        tmem_wait_load();
        tmem_landed(x);
        tmem_landed(x + 32);
        uint32_t pk[32];
        const auto gradients = [&](auto masked) {
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            float e0 = pr[c] * (__uint_as_float(x[c]) - delta), e1 = pr[c + 1] * (__uint_as_float(x[c + 1]) - delta);
            if (decltype(masked)::value) {   // not zero times what a masked pair holds
              e0 = seen[c / 32] >> (c % 32) & 1 ? e0 : 0.0f;
              e1 = seen[c / 32] >> (c % 32 + 1) & 1 ? e1 : 0.0f;
            }
            pk[c / 2] = pack_bf16(e0, e1);
          }
        };
        if (whole) gradients(std::false_type()); else gradients(std::true_type());
        tmem_store32(buf, pk);
        tmem_wait_store();
        tc_fence_before();
        mbar_arrive(smem_addr(&ctl.ds_ready));
      }
      if (ok && steps > 0) {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&ctl.acc_full), walks++ & 1));
        tc_fence_after();
      }
      if (!ok) break;
      if (g < HALVES) {   // a warpgroup stores 64 columns
        const int row0 = i - lane;
        const bool nan = store_columns(stages + warp * kStageBytes, &map_dq, h, row0, g * 64, p.head_dim, p.tokens, p.scale, [&](int k, uint32_t* o) {
          tmem_columns(at_dq + ((uint32_t)r << 16) + g * 64 + k * 32, steps > 0, o);
        });
        // a NaN among the row's scores shows in lse, one in dout or in the values it sees in delta: then the row is NaN
        uint32_t redo = __ballot_sync(0xffffffffu, nan && ((finite(lse) && finite(delta)) || lo >= hi));
        if (redo) {
          if (lane == 0) tma_stores_done();
          __syncwarp();
          for (; redo; redo &= redo - 1) attention_dq_row<true>(p, row0 + __ffs(redo) - 1, h, g * 64, min(g * 64 + 64, p.head_dim));
        }
      }
    }
    if (lane == 0) tma_stores_done();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_free(tmem, kTmemColumns);
  wait_for_previous_kernel();   // so that what is queued after this kernel also finds the keys' gradients
}

// ---- host -------------------------------------------------------------------------------------------------

namespace host {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled() {
  static std::atomic<void*> cached{nullptr};
  void* f = cached.load();
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return nullptr;
    cached.store(f);
  }
  return reinterpret_cast<EncodeTiled>(f);
}

// A view as (value, head, token) with boxes of 64 values of `rows` tokens of one head; zeros are read outside.
static bool make_map(CUtensorMap* map, const AttnView& v, const AttnParams& p, int heads, int rows = kTile) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)p.head_dim, (cuuint64_t)heads, (cuuint64_t)p.tokens};
  // the stride of an axis of one entry is not used, but must be valid
  const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? v.h * 2 : p.head_dim * 2), (cuuint64_t)(p.tokens > 1 ? v.t * 2 : p.head_dim * 2)};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)rows}, ones[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, v.p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The shared memory that a kernel needs beyond the default is asked for once per device and kernel.
template <typename K>
static cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>* done, int device) {
  const uint64_t bit = 1ull << (device & 63);
  if (done->load() & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done->fetch_or(bit);
  return e;
}

// Blocks that share a tile of keys, by query heads: two below two tiles per SM, four where all of those then
// take a quarter of the SMs (a tile's columns can be cut no finer than into 64). Backward pass in us, by 1 / 2 / 4 blocks: 6
// tiles - / 28 / 24, 64 (1024 tokens, causal) - / 45 / 60, 160 (2500) 220 / 194 / -, 256 (4096) 454 / 465 / -, not causal
// 564 / 585 / -, 264 (4099 in seven documents, capped) 311 / 243 / -, 512 (8192) 191 / 224 / - for the keys alone. What decides
// between one and two near 256 tiles is how uneven the tiles' walks are, which the host does not know (the offsets are on the
// device): the rule gives 2 to 4 % to even walks in order not to lose 22 % to uneven ones.
static int key_split(int64_t tiles, int group, int halves) {
  int n = 1;
  while (n < 2 * halves && n * 2 <= group && tiles * n < (n == 1 ? 2 * kSMs : kSMs / 4)) n *= 2;
  return n;
}

static int score_mode(const AttnParams& p) { return p.softcap > 0.0f ? kCap : p.slopes || !(p.scale_log2 > 0.0f) ? kBias : kPlain; }

template <int HALVES, int MODE>
static int forward(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};
  CUtensorMap q, k, v, o;
  if (!make_map(&q, p.q, p, p.heads_q) || !make_map(&k, p.k, p, p.heads_kv) || !make_map(&v, p.v, p, p.heads_kv) ||
      !make_map(&o, p.o, p, p.heads_q, 32))
    return SLIDEDP_ERR_CUDA;
  CU(allow_smem(attention_forward_mma_kernel<HALVES, MODE>, ForwardShape<HALVES>::kSmem, &ready, ctx->device));
  const int64_t blocks = (int64_t)((p.tokens + 2 * kTile - 1) / (2 * kTile)) * p.heads_q;
  if (blocks > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  launch_after(attention_forward_mma_kernel<HALVES, MODE>, (unsigned)blocks, kMmaThreads, ForwardShape<HALVES>::kSmem, 1, st, p, q, k, v, o);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

template <int HALVES, int MODE>
static int backward(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready_q{0}, ready_k{0};
  CUtensorMap q, k, v, d, dq, dk, dv;
  if (!make_map(&q, p.q, p, p.heads_q) || !make_map(&k, p.k, p, p.heads_kv) || !make_map(&v, p.v, p, p.heads_kv) ||
      !make_map(&d, p.dout, p, p.heads_q) || !make_map(&dq, p.dq, p, p.heads_q, 32) || !make_map(&dk, p.dk, p, p.heads_kv, 32) ||
      !make_map(&dv, p.dv, p, p.heads_kv, 32))
    return SLIDEDP_ERR_CUDA;
  CU(allow_smem(attention_dkv_mma_kernel<HALVES, MODE>, KeysShape<HALVES>::kSmem, &ready_k, ctx->device));
  CU(allow_smem(attention_dq_mma_kernel<HALVES, MODE>, QueriesShape<HALVES>::kSmem, &ready_q, ctx->device));
  const int64_t tiles = (p.tokens + kTile - 1) / kTile;
  if (tiles * p.heads_q > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  const int split = key_split(tiles * p.heads_kv, p.group, HALVES);
  // The queries' kernel needs nothing of the keys' kernel and may start once all blocks of that have passed their wait, on SMs
  // that run out of tiles; its blocks end after it. Backward pass of 4099 tokens with prefixes 148 -> 121 us, of 1000
  // tokens, 8 heads 43 -> 29.
  FAULT_POINT();
  launch_after(attention_dkv_mma_kernel<HALVES, MODE>, (unsigned)(tiles * p.heads_kv * split), kMmaThreads, KeysShape<HALVES>::kSmem, split, st,
               p, q, k, v, d, dk, dv, split);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  FAULT_POINT();
  launch_after(attention_dq_mma_kernel<HALVES, MODE>, (unsigned)(tiles * p.heads_q), kMmaThreads, QueriesShape<HALVES>::kSmem, 1, st, p, q, k, v, d,
               dq);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

int attention_forward_mma(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st) {
  const bool narrow = p.head_dim <= 64;
  switch (score_mode(p)) {
    case kPlain: return narrow ? forward<1, kPlain>(ctx, p, st) : forward<2, kPlain>(ctx, p, st);
    case kBias: return narrow ? forward<1, kBias>(ctx, p, st) : forward<2, kBias>(ctx, p, st);
    default: return narrow ? forward<1, kCap>(ctx, p, st) : forward<2, kCap>(ctx, p, st);
  }
}

int attention_backward_mma(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st) {
  const bool narrow = p.head_dim <= 64;
  switch (score_mode(p)) {
    case kPlain: return narrow ? backward<1, kPlain>(ctx, p, st) : backward<2, kPlain>(ctx, p, st);
    case kBias: return narrow ? backward<1, kBias>(ctx, p, st) : backward<2, kBias>(ctx, p, st);
    default: return narrow ? backward<1, kCap>(ctx, p, st) : backward<2, kCap>(ctx, p, st);
  }
}

}  // namespace host
}  // namespace slidedp
