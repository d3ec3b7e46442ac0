// The norms around a block, fused with its gate and the scaled residual, forward and backward.
//
// A group of threads takes one row at a time; a thread keeps its 16 elements of the row in registers from the load
// to the store, so every array crosses HBM once, which is what bounds it.  The group is part of a warp, a CTA or, for rows that
// one CTA cannot hold often enough on an SM, the CTAs of a cluster: several small CTAs hide each other's waits.  The CTAs
// of a cluster exchange a row's sums by asynchronous stores into each other's shared memory that count themselves on an
// mbarrier; a cluster barrier instead would hold every row until its stores to global memory are done (gradient at
// d = 8192: 814 us against 740 at the same grid).  No more clusters than the device holds at once: a second round of them
// nearly doubles the time (501 us then).
//
// Measured on 65,536 rows of 2048, bf16: 208 us for the forward pass (6.45 TB/s); 32,768 rows of 2048, float32 residual, bf16
// activations: 238 us for the gradient, 6.2 TB/s, and about 15 us more until the weights' sums are done.  Rows of 8192 bf16
// are bound by the exchange (255 us for the bytes of 205); narrow rows of odd width by the latency of a few rows a group.
//
// Rows whose width is no multiple of 8 start at eight different places of a 16-byte-aligned grid of pieces.  The rows of a CTA
// are then taken `period` apart (the smallest number of rows whose elements are a multiple of 8), so that all of them start
// at the same place: a thread's columns, its weights and its sums stay the same from row to row, and only the pieces
// that hold a row's two ends go element by element.
#include "sl_inner.cuh"
#include "sl_norm_rows.cuh"

namespace sl {
namespace {

constexpr int kMaxThreads = 320;   // of a CTA
constexpr int kMaxWarps = 40;       // of a row: a CTA of 10, or 8 CTAs of 5 warps
enum Group { kLanes, kCta, kCluster };     // what shares a row

// What a thread holds of a row, as it is stored; a piece that it does not have holds something else.  Nothing here looks at
// what it loaded before mask(), so that the loads of a row's arrays are all on their way together.
template <class T, int E, int K>
struct Piece {
  static constexpr int W = E == 1 ? 1 : E * (int)sizeof(T) / 4;
  uint32_t w[K][W];

  __device__ __forceinline__ static uint32_t bits(const T* p) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(__ldcs(reinterpret_cast<const float*>(p)));
    else return (uint32_t)__ldcs(reinterpret_cast<const uint16_t*>(p));
  }
  // near_end: too little comes behind this row for a vector that reaches past its end
  template <bool SHIFT>
  __device__ __forceinline__ void load(const T* row, const Columns<E, K, SHIFT>& c, bool near_end) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const T* p = row + c.safe(k);
      if constexpr (E == 1) {
        w[k][0] = bits(p);
      } else if (!c.by_vector(k, near_end)) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[k][i] = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c.any(k) && c.has(k, e)) w[k][e * (int)sizeof(T) / 4] |= bits(p + e) << (sizeof(T) == 4 ? 0 : 16 * (e & 1));
      } else {
        // a piece with one of the row's ends also reads elements of the rows beside it, which mask() takes out
        Raw<T, E> r;
        r.load(p);
#pragma unroll
        for (int i = 0; i < W; ++i) w[k][i] = r.w[i];
      }
    }
  }
  template <bool SHIFT>
  __device__ __forceinline__ void mask(const Columns<E, K, SHIFT>& c) {
    if constexpr (SHIFT) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (!c.whole(k)) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (!c.has(k, e)) w[k][e * (int)sizeof(T) / 4] &= sizeof(T) == 4 ? 0u : (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
        }
    }
  }
  __device__ __forceinline__ float get(int k, int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k][e]);
    else if constexpr (E == 1) return __uint_as_float(w[k][0] << 16);
    else return __uint_as_float((e & 1) ? (w[k][e / 2] & 0xFFFF0000u) : (w[k][e / 2] << 16));
  }
  // the compiler may not keep what was computed from the piece before this point: registers hold the piece itself
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < W; ++i) asm volatile("" : "+r"(w[k][i]));
  }
};

// elements of a k-th piece that are not the row's, as mask() does, for a value that several arrays enter
template <int E, int K, bool SHIFT>
__device__ __forceinline__ void zero_outside(const Columns<E, K, SHIFT>& c, int k, float (&f)[E]) {
  if constexpr (SHIFT)
    if (!c.whole(k)) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (!c.has(k, e)) f[e] = 0.0f;
    }
}

template <class T, int E, int K, bool SHIFT>
__device__ __forceinline__ void store_part(T* row, const Columns<E, K, SHIFT>& c, int k, const float (&f)[E]) {
  T* p = row + c.col(k);
  if constexpr (E == 1) {
    *p = from_f32<T>(f[0]);
  } else if (c.whole(k)) {
    Raw<T, E> r;
    r.set(f);
    r.store(p);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (c.has(k, e)) p[e] = from_f32<T>(f[e]);
  }
}

// A weight times `factor` in shared memory as float32, zero outside the row: every thread keeps its own pieces there (a CTA's
// rows of lanes share the first one's).  E = 8: the first and the second four elements of the pieces lie apart, so that
// a warp's 16-byte reads are consecutive.
template <int E, int K, bool SHIFT>
__device__ __forceinline__ void stage_weight(float* to, const void* w, int w_bf16, float factor, uint32_t my, uint32_t own,
                                             const Columns<E, K, SHIFT>& c) {
  float v[K][E];
  auto load = [&](auto get) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = c.any(k) && c.has(k, e) ? get(c.col(k) + e) : 0.0f;
  };
  if (w_bf16) load([&](int i) { return to_f32(static_cast<const Bf16*>(w)[i]); });
  else load([&](int i) { return __ldg(static_cast<const float*>(w) + i); });
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t slot = my + k * own;
    if constexpr (E == 1) {
      to[slot] = factor * v[k][0];
    } else {
      reinterpret_cast<float4*>(to)[slot] = make_float4(factor * v[k][0], factor * v[k][1], factor * v[k][2], factor * v[k][3]);
      reinterpret_cast<float4*>(to)[K * own + slot] = make_float4(factor * v[k][4], factor * v[k][5], factor * v[k][6], factor * v[k][7]);
    }
  }
}
// piece `slot` of `count`
template <int E>
__device__ __forceinline__ void read_weight(const float* w, uint32_t slot, uint32_t count, float (&f)[E]) {
  if constexpr (E == 1) {
    f[0] = w[slot];
  } else {
    const float4 a = reinterpret_cast<const float4*>(w)[slot], b = reinterpret_cast<const float4*>(w)[count + slot];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// all threads of the CTA or cluster, everything before it visible
template <Group G>
__device__ __forceinline__ void group_barrier() {
  if constexpr (G == kCluster) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
}

// Sums over the threads of a row, the same in all of them and in a fixed order.  kLanes: a row has `width` lanes of a
// warp (a power of two).  kCta, kCluster: every warp leaves its sums in a buffer of all the row's CTAs.  There are two
// buffers, used in turn: one is written again only after all threads have met over the other, so have read it.
struct Exchange {
  float4 sums[2][kMaxWarps];       // of every warp of the row
  uint64_t full[2];                // kCluster: completes when all of them have arrived
};
constexpr long long kWaitClocks = 2000000000ll;            // bound of a wait, about a second

template <Group G>
struct RowSum {
  Exchange& x;
  uint32_t* flags;
  uint32_t polls, calls = 0, warps, rank = 0;              // polls: bound of a wait if not 0 (~0: none at all)
  bool dead = false;                                       // a wait ran out: nothing is waited for any more

  __device__ __forceinline__ RowSum(Exchange& x_, uint32_t* flags_, uint32_t polls_) : x(x_), flags(flags_), polls(polls_) {
    warps = blockDim.x >> 5;
    if constexpr (G == kCluster) rank = cluster_rank();
    for (int i = threadIdx.x; i < 8 * kMaxWarps; i += blockDim.x) reinterpret_cast<float*>(x.sums)[i] = 0.0f;
    if (G == kCluster && threadIdx.x == 0) {
      for (int i = 0; i < 2; ++i)
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"((uint32_t)__cvta_generic_to_shared(&x.full[i])));
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  __device__ __forceinline__ void send(float4* slot, uint64_t* bar, uint32_t to, float4 v) {
    uint32_t at = (uint32_t)__cvta_generic_to_shared(slot), b = (uint32_t)__cvta_generic_to_shared(bar);
    asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(to));
    asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(b) : "r"(to));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(b) : "memory");
  }
  // the whole warp; false: given up, now or before
  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    const uint32_t b = (uint32_t)__cvta_generic_to_shared(bar);
    const long long start = clock64();
    uint32_t done = 0, n = 0;
    while (polls != ~0u) {
      asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                   : "=r"(done) : "r"(b), "r"(parity) : "memory");
      if (done || (polls ? ++n >= polls : clock64() - start > kWaitClocks)) break;
    }
    return __all_sync(0xFFFFFFFFu, done);
  }
  template <int N>
  __device__ __forceinline__ void operator()(float (&s)[N], int width) {
    if constexpr (G == kLanes) {
      for (int o = width / 2; o > 0; o >>= 1) add_lanes(s, o);
    } else {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) add_lanes(s, o);
      const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, turn = calls & 1;
      if constexpr (G == kCta) {
        float(*sums)[kMaxWarps] = reinterpret_cast<float(*)[kMaxWarps]>(x.sums[turn]);     // [N][warps]
        if (lane == 0)
#pragma unroll
          for (int i = 0; i < N; ++i) sums[i][warp] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = quad(&sums[i][0]);
        if (warps > 4)
#pragma unroll
          for (int i = 0; i < N; ++i) s[i] += quad(&sums[i][4]);
        if (warps > 8)
#pragma unroll
          for (int i = 0; i < N; ++i) s[i] += quad(&sums[i][8]);
      } else {
        float4* sums = x.sums[turn];
        const float4 v = make_float4(s[0], N > 1 ? s[N > 1] : 0.0f, N > 2 ? s[N > 2 ? 2 : 0] : 0.0f, 0.0f);
        const uint32_t ctas = cluster_size(), all = ctas * warps;
        if (!dead) {
          if (threadIdx.x == 0)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                         ::"r"((uint32_t)__cvta_generic_to_shared(&x.full[turn])), "r"(all * 16) : "memory");
          if (lane < ctas) send(&sums[rank * warps + warp], &x.full[turn], lane, v);
          dead = !wait(&x.full[turn], (calls >> 1) & 1);
          if (dead && lane == 0 && flags) atomicOr(flags, (uint32_t)SL_FLAG_TIMEOUT);
        }
        float4 t = sums[lane];                             // zero where nobody writes
        if (lane + 32 < all) {
          const float4 u = sums[lane + 32];
          t.x += u.x;
          t.y += u.y;
          t.z += u.z;
        }
        s[0] = t.x;
        if (N > 1) s[N > 1] = t.y;
        if (N > 2) s[N > 2 ? 2 : 0] = t.z;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) add_lanes(s, o);
      }
      ++calls;
    }
  }
  template <int N>
  __device__ __forceinline__ static void add_lanes(float (&s)[N], int o) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], o);
  }
  __device__ __forceinline__ static float quad(const float* p) {      // four warps' sums; zero where there is none
    const float4 v = *reinterpret_cast<const float4*>(p);
    return (v.x + v.y) + (v.z + v.w);
  }
  // a CTA stays until nobody writes to its shared memory any more
  __device__ __forceinline__ void leave() {
    if constexpr (G == kCluster) {
      group_barrier<G>();                                  // all stores have been issued; what was waited for has arrived
      if (dead)
        for (const long long start = clock64(); clock64() - start < 200000;) {}
    }
  }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.44269504f;

// Fast, also for float32 activations: the product -log2e g is rounded (1.3 |g| units of 2^-24 in the exponential), the
// exponential is off by at most 4 such units and the reciprocal by 2, so sigmoid by (8 + 1.3 |g|) 2^-24 of itself for g < 0 and
// less above.  expf and a division instead: 65,536 rows of 2048 bf16 210 -> 263 us, the gradient of 32,768 203 -> 308 us.
__device__ __forceinline__ float sigmoid(float g) { return rcp_fast(1.0f + exp2_fast(-kLog2e * g)); }
// sigmoid s and its complement: with e = exp(-g), s = 1 / (1 + e) and 1 - s = e s, so that neither loses digits at either end
// (e is kept at 2^127, where s is flushed to 0 and 1 - s has nothing left to multiply); a NaN stays one
__device__ __forceinline__ void gate(float g, float& s, float& one_minus_s) {
  float t;
  asm("min.NaN.f32 %0, %1, 0f42FE0000;" : "=f"(t) : "f"(-kLog2e * g));      // 127
  const float e = exp2_fast(t);
  s = rcp_fast(1.0f + e);
  one_minus_s = e * s;
}

// Rows of a launch.  kLanes: `width` threads share a row and a CTA holds blockDim.x / width rows at a time; otherwise the
// groups are CTAs or clusters.  Group q (CTA or cluster) has rows q % period, + period, ..., every
// (groups / period)-th bunch of them.
struct Launch {
  int width;
  uint32_t period;
  uint32_t busy;                   // groups that have a row: the first ones
  uint32_t near;                   // rows_near_end()
};
template <Group G>
struct Rows {
  uint64_t row, base, step;        // this thread's row, its group's first row, distance to the next ones
  uint32_t lane, lanes;            // the thread's place among those of its row
  __device__ __forceinline__ Rows(const Launch& l) {
    const uint32_t ctas = G == kCluster ? cluster_size() : 1, per = G == kLanes ? blockDim.x / l.width : 1;
    const uint32_t mine = G == kLanes ? threadIdx.x / l.width : 0, q = blockIdx.x / ctas, groups = gridDim.x / ctas;
    lane = G == kLanes ? threadIdx.x % l.width : G == kCluster ? cluster_rank() * blockDim.x + threadIdx.x : threadIdx.x;
    lanes = G == kLanes ? l.width : ctas * blockDim.x;
    base = q % l.period + (uint64_t)(q / l.period) * per * l.period;
    row = base + (uint64_t)mine * l.period;
    step = (uint64_t)(groups / l.period) * per * l.period;
  }
};
template <class RT, class AT, int E, int K, Group G, bool SHIFT>
__global__ void __launch_bounds__(kMaxThreads) norm_block_kernel(const NormArgs a, const Launch l) {
  extern __shared__ __align__(16) float weights[];
  __shared__ __align__(16) Exchange exchange;
  const float inv_d = 1.0f / (float)a.d;
  Rows<G> rw(l);
  const auto c = columns_of<E, K, SHIFT>(rw.row, rw.lane, rw.lanes, a.d);
  const uint32_t own = G == kLanes ? l.width : blockDim.x, my = G == kLanes ? rw.lane : threadIdx.x;
  Piece<RT, E, K> x;
  Piece<AT, E, K> b, g;
  auto load = [&](uint64_t r) {
    if (r >= a.n) return;
    const bool near_end = SHIFT && near_array_end(r, a.n, l.near);
    x.load(static_cast<const RT*>(a.x) + r * a.d, c, near_end);
    if (a.b) b.load(static_cast<const AT*>(a.b) + r * a.ldb, c, near_end);
    if (a.g) g.load(static_cast<const AT*>(a.g) + r * a.ldg, c, near_end);
  };
  uint64_t r = rw.row;
  load(r);
  float *w_post = weights, *w_pre = weights + (a.w_post ? own * K * E : 0);
  if (G != kLanes || threadIdx.x < own) {
    if (a.w_post) stage_weight(w_post, a.w_post, a.w_bf16, a.alpha, my, own, c);
    if (a.y) stage_weight(w_pre, a.w_pre, a.w_bf16, 1.0f, my, own, c);
  }
  RowSum<G> row_sum(exchange, a.flags, a.wait_polls);
  group_barrier<G>();
  for (; rw.base < a.n; rw.base += rw.step, r += rw.step) {
    const bool in = r < a.n;
    if (a.w_post) b.mask(c);
    float h[K][E];
    float rp = a.alpha;                                    // factor of u: rms(b), with alpha in w_post, or alpha
    if (a.w_post) {
      float s[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (c.any(k))
#pragma unroll
          for (int e = 0; e < E; ++e) s[0] = __fmaf_rn(b.get(k, e), b.get(k, e), s[0]);
      row_sum(s, l.width);
      rp = 1.0f / sqrtf(s[0] * inv_d + a.eps);
      if (a.r_post && in && rw.lane == 0) a.r_post[r] = rp;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] = x.get(k, e);
      if (a.b && c.any(k)) {
        float u[E], w[E];
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = b.get(k, e);
        if (a.w_post) {
          read_weight(w_post, my + k * own, own * K, w);
#pragma unroll
          for (int e = 0; e < E; ++e) u[e] = u[e] * w[e];
        }
        if (a.g)
#pragma unroll
          for (int e = 0; e < E; ++e) u[e] = u[e] * sigmoid(g.get(k, e));
#pragma unroll
        for (int e = 0; e < E; ++e) h[k][e] = __fmaf_rn(rp, u[e], h[k][e]);
      }
      if (a.y) zero_outside(c, k, h[k]);                   // x and g beside the row may hold anything, NaN too
    }
    load(r + rw.step);                                     // the next row is on its way while this one is finished
    if (a.b && in) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (c.any(k)) store_part(static_cast<RT*>(a.h) + r * a.d, c, k, h[k]);
    }
    if (a.y) {
      float s[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (c.any(k))
#pragma unroll
          for (int e = 0; e < E; ++e) s[0] = __fmaf_rn(h[k][e], h[k][e], s[0]);
      row_sum(s, l.width);
      const float rh = 1.0f / sqrtf(s[0] * inv_d + a.eps);
      if (a.r_pre && in && rw.lane == 0) a.r_pre[r] = rh;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (in && c.any(k)) {
          float w[E];
          read_weight(w_pre, my + k * own, own * K, w);
#pragma unroll
          for (int e = 0; e < E; ++e) h[k][e] = h[k][e] * rh * w[e];
          store_part(static_cast<AT*>(a.y) + r * a.d, c, k, h[k]);
        }
      }
    }
  }
  row_sum.leave();
}

// words of a row of partial sums: a piece more than the row where rows are shifted
__host__ __device__ __forceinline__ uint32_t partial_width(uint32_t d) { return d % 8 == 0 ? d : (d + 14) / 8 * 8; }

// With k = alpha s w_post b and z = dh + rms(h) dn, the second norm's sum is linear in the first's:
//     sum q b = sum k dx = sum k z - (rms(h)^3 / d) (sum dn h) (sum k h),
// so all three sums of a row go through one exchange.  Across it a thread keeps z and, as they are stored, h, b and g: what
// else is needed is computed again, which lets more threads fit an SM.
template <class RT, class AT, int E, int K, Group G, bool SHIFT>
__global__ void __maxnreg__(128) norm_block_grad_kernel(const NormGradArgs a, const Launch l) {
  extern __shared__ __align__(16) float weights[];
  __shared__ __align__(16) Exchange exchange;
  let_next_start();
  const float inv_d = 1.0f / (float)a.d;
  Rows<G> rw(l);
  const auto c = columns_of<E, K, SHIFT>(rw.row, rw.lane, rw.lanes, a.d);
  const uint32_t own = G == kLanes ? l.width : blockDim.x, my = G == kLanes ? rw.lane : threadIdx.x;
  Piece<RT, E, K> h, dh;
  Piece<AT, E, K> dy, b, g;
  float rh = 0.0f, rp = 1.0f;
  auto load = [&](uint64_t r) {
    if (r >= a.n) return;
    const bool near_end = SHIFT && near_array_end(r, a.n, l.near);
    h.load(static_cast<const RT*>(a.h) + r * a.d, c, near_end);
    if (a.dh) dh.load(static_cast<const RT*>(a.dh) + r * a.d, c, near_end);
    if (a.dy) {
      dy.load(static_cast<const AT*>(a.dy) + r * a.d, c, near_end);
      rh = __ldg(a.r_pre + r);
    }
    if (a.b) b.load(static_cast<const AT*>(a.b) + r * a.ldb, c, near_end);
    if (a.g) g.load(static_cast<const AT*>(a.g) + r * a.ldg, c, near_end);
    if (a.w_post) rp = __ldg(a.r_post + r);
  };
  uint64_t r = rw.row;
  load(r);
  float *w_post = weights, *w_pre = weights + (a.w_post ? own * K * E : 0);
  if (G != kLanes || threadIdx.x < own) {
    if (a.w_post) stage_weight(w_post, a.w_post, a.w_bf16, a.alpha, my, own, c);
    if (a.dy) stage_weight(w_pre, a.w_pre, a.w_bf16, 1.0f, my, own, c);
  }
  RowSum<G> row_sum(exchange, a.flags, a.wait_polls);
  group_barrier<G>();
  float dpre[K][E] = {}, dpost[K][E] = {};
  for (; rw.base < a.n; rw.base += rw.step, r += rw.step) {
    const bool in = r < a.n;
    h.mask(c);
    if (a.dh) dh.mask(c);
    if (a.dy) dy.mask(c);
    float z[K][E];
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && c.any(k)) {
        float w[E];
        if (a.dh) {
#pragma unroll
          for (int e = 0; e < E; ++e) z[k][e] = dh.get(k, e);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) z[k][e] = 0.0f;
        }
        if (a.dy) {
          read_weight(w_pre, my + k * own, own * K, w);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float dn = dy.get(k, e) * w[e], hv = h.get(k, e);
            s[0] = __fmaf_rn(dn, hv, s[0]);
            dpre[k][e] = __fmaf_rn(dy.get(k, e) * hv, rh, dpre[k][e]);
            z[k][e] = __fmaf_rn(rh, dn, z[k][e]);
          }
        }
        if (a.w_post) {
          read_weight(w_post, my + k * own, own * K, w);
#pragma unroll
          for (int e = 0; e < E; ++e) w[e] = w[e] * b.get(k, e);
          if (a.g)
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = w[e] * sigmoid(g.get(k, e));
          zero_outside(c, k, w);                           // b and g beside the row may hold anything, NaN too
#pragma unroll
          for (int e = 0; e < E; ++e) {
            s[1] = __fmaf_rn(w[e], z[k][e], s[1]);
            s[2] = __fmaf_rn(w[e], h.get(k, e), s[2]);
          }
        }
      }
    }
    row_sum(s, l.width);
    // rms(h)^3 alone leaves float32 where rms(h)^2 and the products with the sums do not
    const float ch = rh * ((rh * inv_d) * (rh * s[0]));              // dx = z - ch h
    const float cb = rp * (inv_d * (rp * (s[1] - ch * s[2])));      // db = rp (q - cb b)
    h.forget();
    if (a.b) b.forget();
    if (a.g) g.forget();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && c.any(k)) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[k][e] = __fmaf_rn(-ch, h.get(k, e), z[k][e]);
        store_part(static_cast<RT*>(a.dx) + r * a.d, c, k, z[k]);
        if (a.b) {
          float w[E], dg[E] = {};
          if (a.g)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              float sg;
              gate(g.get(k, e), sg, dg[e]);
              z[k][e] = z[k][e] * sg;                                // s dx
            }
          if (a.w_post) {
            read_weight(w_post, my + k * own, own * K, w);             // alpha w_post
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float n0 = b.get(k, e) * rp, q = z[k][e] * w[e];
              dg[e] = n0 * q * dg[e];
              dpost[k][e] = __fmaf_rn(z[k][e], n0, dpost[k][e]);
              z[k][e] = rp * __fmaf_rn(-cb, b.get(k, e), q);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              z[k][e] = a.alpha * z[k][e];
              dg[e] = z[k][e] * b.get(k, e) * dg[e];
            }
          }
          store_part(static_cast<AT*>(a.db) + r * a.ldb, c, k, z[k]);
          if (a.g) store_part(static_cast<AT*>(a.dg) + r * a.ldg, c, k, dg);
        }
      }
    }
    load(r + rw.step);
  }
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) dpost[k][e] *= a.alpha;
  row_sum.leave();
  // one row of partial sums a weight and CTA or cluster; the rows of a warp and then the warps of a CTA are added first
  const uint32_t q = blockIdx.x / (G == kCluster ? cluster_size() : 1);
  if (q >= l.busy) return;
  const uint32_t wide = partial_width(a.d);                // a row begins where its group's rows do on the grid of vectors
  float* out = a.ws + (uint64_t)q * wide + c.lead;
  const uint64_t other = (uint64_t)l.busy * wide;          // from a row of w_pre's to the same of w_post's
  if constexpr (G == kLanes) {
    __syncthreads();                                       // the weights are not needed any more
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int o = l.width; o < 32; o <<= 1) {
          dpre[k][e] += __shfl_xor_sync(0xFFFFFFFFu, dpre[k][e], o);
          dpost[k][e] += __shfl_xor_sync(0xFFFFFFFFu, dpost[k][e], o);
        }
    const uint32_t warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float* part = weights;                                 // [2][width K E]
    for (uint32_t w = 0; w < warps; ++w) {
      if (w == warp && (threadIdx.x & 31) < l.width)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float* p = part + (k * E + e) * l.width + rw.lane;
            float* q = p + l.width * K * E;
            *p = dpre[k][e] = w ? *p + dpre[k][e] : dpre[k][e];
            *q = dpost[k][e] = w ? *q + dpost[k][e] : dpost[k][e];
          }
      __syncthreads();
    }
    if (warp != warps - 1 || (threadIdx.x & 31) >= l.width) return;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (!c.any(k)) continue;
    auto put = [&](float* p, const float(&f)[E]) {
      if constexpr (E == 8) {                              // what lies outside the row is never read
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
      } else {
        p[0] = f[0];
      }
    };
    if (a.dw_pre) put(out + c.col(k), dpre[k]);
    if (a.dw_post) put(out + other + c.col(k), dpost[k]);
  }
}

// Sums the partial rows of both weights; 32 columns to a CTA, 32 threads to a column.  Row p begins `lead` words behind its
// place, which depends on the group's first row (p mod period).
__global__ void __launch_bounds__(1024) norm_weight_grad_kernel(const NormGradArgs a, uint32_t rows, uint32_t period) {
  __shared__ float part[32][33];
  wait_for_previous();
  void* out = blockIdx.y ? a.dw_post : a.dw_pre;
  if (!out) return;
  const uint32_t c = blockIdx.x * 32 + threadIdx.x, wide = partial_width(a.d);
  const float* from = a.ws + (uint64_t)blockIdx.y * rows * wide + c;
  float s = 0.0f;
  if (c < a.d)
#pragma unroll 8
    for (uint32_t p = threadIdx.y; p < rows; p += 32) s += from[(uint64_t)p * wide + ((p & (period - 1)) * a.d & 7)];
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = part[threadIdx.x][threadIdx.y];                      // warp y: column y
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  const uint32_t col = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && col < a.d) {
    if (a.w_bf16) {
      Bf16* w = static_cast<Bf16*>(out) + col;
      *w = from_f32<Bf16>(a.acc ? to_f32(*w) + s : s);
    } else {
      float* w = static_cast<float*>(out) + col;
      *w = a.acc ? *w + s : s;
    }
  }
}

// How rows are dealt out.  A thread has 16 elements: two vectors of 8 (rows aligned, or `period` rows apart), or 16
// single ones a row's threads apart where the arrays' rows do not share a place on the grid of vectors.
struct Shape {
  int threads, vec, ctas;         // vec: elements of a piece, 8 or 1; ctas: of a cluster
  bool shift;
  Group group;
  Launch l;
  uint32_t rows() const { return group == kLanes ? threads / l.width : 1; }
  uint32_t lanes() const { return group == kLanes ? l.width : threads; }
};

// places[]: elements between the rows of every array; `aligned`: every array starts where vectors of 8 may; single: threads
// that one CTA has for a row at most
inline Shape shape_of(uint32_t d, bool aligned, const uint64_t* places, int n, uint32_t single) {
  Shape s;
  for (int i = 0; i < n; ++i) aligned = aligned && places[i] % 8 == d % 8;
  s.vec = aligned ? 8 : 1;
  s.shift = aligned && d % 8 != 0;
  s.l.period = 1;
  s.l.near = rows_near_end(d);
  if (s.shift)
    while ((uint64_t)s.l.period * d % 8 != 0) s.l.period *= 2;
  const uint32_t parts = s.vec == 8 ? (d + (s.shift ? 7 : 0) + 7) / 8 : d, per_thread = s.vec == 8 ? 2 : 16;
  const uint32_t lanes = (parts + per_thread - 1) / per_thread;
  s.ctas = 1;
  if (lanes <= 32) {
    s.group = kLanes;
    s.threads = 128;
    s.l.width = 1;
    while ((uint32_t)s.l.width < lanes) s.l.width *= 2;
  } else {
    if (s.vec == 1) single = 160;                          // more registers: a CTA as wide as the row would have an SM to itself
    if (lanes > single) s.ctas = lanes <= 320 ? 2 : (int)((lanes + 127) / 128 < 8 ? (lanes + 127) / 128 : 8);
    s.group = s.ctas > 1 ? kCluster : kCta;
    s.threads = (int)(((lanes + s.ctas - 1) / s.ctas + 31) / 32 * 32);
    s.l.width = s.threads;
  }
  return s;
}

// partial rows of a weight gradient at most
constexpr uint32_t kMaxPartials = 1184;

template <class F>
cudaError_t with_types(int res_type, int act_type, F&& f) {
  if (res_type == SL_BF16) return f(Bf16{}, Bf16{});
  if (act_type == SL_BF16) return f(float{}, Bf16{});
  return f(float{}, float{});
}

// launches `kernel` with enough groups for its rows, no more than fit the device at once or than `cap`; a multiple of
// the period
template <class Args>
cudaError_t launch_rows(void (*kernel)(const Args, const Launch), const Args& a, const Shape& s, size_t smem, uint32_t cap, uint32_t* busy,
                        cudaStream_t st) {
  cudaError_t e;
  const int sms = sm_count(&e);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = s.ctas;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(s.ctas);
  cfg.blockDim = dim3(s.threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = s.ctas > 1 ? 1 : 0;
  const uint32_t per_class = (a.n + s.l.period - 1) / s.l.period;
  uint64_t want = (uint64_t)((per_class + s.rows() - 1) / s.rows()) * s.l.period;
  if (want * s.ctas > (uint32_t)sms) {
    int fit = 0;                  // groups the device holds at once; a second round of rows would double the time
    if (s.ctas > 1) e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg);
    else e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, kernel, s.threads, smem), fit *= sms;
    if (e != cudaSuccess) return e;
    const uint32_t most = (fit < 1 ? 1u : (uint32_t)fit) / s.l.period * s.l.period;
    if (want > most) want = most < s.l.period ? s.l.period : most;
  }
  cap = cap < s.l.period ? s.l.period : cap / s.l.period * s.l.period;
  const uint32_t groups = (uint32_t)(want > cap ? cap : want);
  // all bunches of `period` groups but the last have rows throughout
  const uint64_t before = (uint64_t)(groups / s.l.period - 1) * s.rows() * s.l.period, left = a.n - before;
  Launch l = s.l;
  *busy = l.busy = groups - s.l.period + (uint32_t)(left < s.l.period ? left : s.l.period);
  cfg.gridDim = dim3(groups * s.ctas);
  return cudaLaunchKernelEx(&cfg, kernel, a, l);
}

inline size_t weights_smem(int weights, const Shape& s) { return (size_t)weights * s.lanes() * 16 * sizeof(float); }

}  // namespace

#define SL_PICK(KERNEL)                                                      \
  if (s.vec == 1) {                                                          \
    if (s.group == kLanes) return go(KERNEL<RT, AT, 1, 16, kLanes, false>);  \
    if (s.group == kCta) return go(KERNEL<RT, AT, 1, 16, kCta, false>);      \
    return go(KERNEL<RT, AT, 1, 16, kCluster, false>);                       \
  }                                                                          \
  if (s.shift) {                                                             \
    if (s.group == kLanes) return go(KERNEL<RT, AT, 8, 2, kLanes, true>);    \
    if (s.group == kCta) return go(KERNEL<RT, AT, 8, 2, kCta, true>);        \
    return go(KERNEL<RT, AT, 8, 2, kCluster, true>);                         \
  }                                                                          \
  if (s.group == kLanes) return go(KERNEL<RT, AT, 8, 2, kLanes, false>);     \
  if (s.group == kCta) return go(KERNEL<RT, AT, 8, 2, kCta, false>);         \
  return go(KERNEL<RT, AT, 8, 2, kCluster, false>)

cudaError_t launch_norm_block(const NormArgs& a, int res_type, int act_type, cudaStream_t st) {
  auto ok = [](const void* p, int type) { return vector_aligned(p, type); };
  const bool aligned = ok(a.x, res_type) && ok(a.h, res_type) && ok(a.b, act_type) && ok(a.g, act_type) && ok(a.y, act_type);
  const uint64_t places[3] = {a.d, a.b ? a.ldb : a.d, a.g ? a.ldg : a.d};
  // One CTA up to 4,608 elements, two up to 5,120: 134 M elements bf16 in rows of 4096: 213 us, 242 with two CTAs; of 5120: 249
  // with two, 286 with three.  One CTA for these too would take less (5120: 235 us, float32 238 -> 231): a boundary still to be
  // moved.  float32 residuals beside bf16 activations fill an SM less well: 4096: 305 us with one, 289 with two (without gate
  // and post-norm 255 and 274).
  const bool less = res_type == SL_F32 && act_type == SL_BF16 && a.d % 8 == 0 && a.d <= 4096;
  const Shape s = shape_of(a.d, aligned, places, 3, less ? 160 : 288);
  const size_t smem = weights_smem((a.w_post ? 1 : 0) + (a.y ? 1 : 0), s);
  uint32_t busy;
  return with_types(res_type, act_type, [&](auto rt, auto act) {
    using RT = decltype(rt);
    using AT = decltype(act);
    auto go = [&](void (*kernel)(const NormArgs, const Launch)) { return launch_rows(kernel, a, s, smem, 0x7FFFFFFFu, &busy, st); };
    SL_PICK(norm_block_kernel);
  });
}

uint64_t norm_block_grad_workspace(uint64_t n, uint32_t d) {
  const uint32_t rows = n < kMaxPartials ? (uint32_t)n : kMaxPartials;
  return 2ull * rows * partial_width(d) * sizeof(float);
}

cudaError_t launch_norm_block_grad(const NormGradArgs& a, int res_type, int act_type, cudaStream_t st) {
  auto ok = [](const void* p, int type) { return vector_aligned(p, type); };
  const bool aligned = ok(a.dh, res_type) && ok(a.h, res_type) && ok(a.dx, res_type) && ok(a.dy, act_type) && ok(a.b, act_type) &&
                       ok(a.g, act_type) && ok(a.db, act_type) && ok(a.dg, act_type);
  const uint64_t places[3] = {a.d, a.b ? a.ldb : a.d, a.g ? a.ldg : a.d};
  // One CTA up to 4,096 elements, two up to 5,120: 67 M elements bf16 in rows of 4096: 214 us, 224 with two CTAs; of 5120: 248
  // with two, 308 with one (of which an SM holds one), 282 with three.
  const Shape s = shape_of(a.d, aligned, places, 3, 256);
  const size_t smem = weights_smem(2, s);                  // the partial sums take their place at the end
  uint32_t busy = 0;
  cudaError_t e = cudaSuccess;
  if (a.n > 0)
    e = with_types(res_type, act_type, [&](auto rt, auto act) {
      using RT = decltype(rt);
      using AT = decltype(act);
      auto go = [&](void (*kernel)(const NormGradArgs, const Launch)) {
        return launch_rows(kernel, a, s, smem, kMaxPartials, &busy, st);
      };
      SL_PICK(norm_block_grad_kernel);
    });
  if (e != cudaSuccess || (!a.dw_pre && !a.dw_post)) return e;
  return launch_behind(norm_weight_grad_kernel, dim3((a.d + 31) / 32, 2), dim3(32, 32), 0, st, a, busy, s.l.period);
}
#undef SL_PICK

}  // namespace sl
