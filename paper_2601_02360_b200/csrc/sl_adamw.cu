// AdamW over every tensor of an arena (Eq. 1's inner optimiser), moments in 32 or in 8 bits.
//
// Pure streaming: nothing is used twice, so both forms are bound by HBM and the work is in keeping enough
// bytes in flight and the arithmetic under the memory's pace.  990 M elements, 32-bit states: 4.47 ms for 27.7 GB (6.2 TB/s).
// 187 M elements, 8-bit states, bf16 gradient: 598 us for 2.99 GB (5.0 TB/s); there the encoding's instructions
// bound it (550 us without them), and reading the states out takes 317 us, the time of its 1.5 GB of writes.
#include "sl_inner.cuh"

namespace sl {
namespace {

struct Seg {
  uint64_t base;     // first element of the block in the arena
  uint32_t len;
  float keep;
};

// Walks the blocks of an arena in ascending order; the tensor of the last one is kept in registers.
// SHIFT: blocks begin on a grid; the 8-bit form's begin at their tensor (634 -> 598 us for 187 M elements without the shift)
template <int T, bool SHIFT>
struct Walk {
  const BlockTable<T>& tb;
  uint32_t block, first = 0, behind = 0;     // blocks of the tensor: [first, behind)
  uint64_t start = 0, base = 0, end = 0;
  float keep = 1.0f;
  __device__ __forceinline__ Walk(const BlockTable<T>& tb_, uint32_t block_) : tb(tb_), block(block_) {}
  __device__ __forceinline__ Seg at(uint32_t g) {
    if (g >= behind) {
      uint32_t lo = 0, hi = tb.n_tensors;              // first_block[lo] <= g < first_block[hi]
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (tb.first_block[mid] <= g) lo = mid; else hi = mid;
      }
      first = tb.first_block[lo];
      behind = tb.first_block[lo + 1];
      start = tb.offset[lo];
      base = SHIFT ? start & ~(uint64_t)(tb.align - 1) : start;
      end = tb.offset[lo + 1];
      keep = tb.keep[lo];
    }
    Seg s;
    s.base = base + (uint64_t)(g - first) * block;
    const uint64_t left = end - s.base;
    s.len = left < block ? (uint32_t)left : block;
    if (SHIFT && s.base < start) {                              // the tensor's first block, cut short in front
      s.len -= (uint32_t)(start - s.base);
      s.base = start;
    }
    s.keep = keep;
    return s;
  }
};

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

__device__ __forceinline__ float sqrt_fast(float x) {      // relative error at most 2^-23
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {       // 1 ulp
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// One element; `g` is the scaled gradient.  The file is compiled without contraction: each operation rounds once.
// FAST: the root (2^-23) and the quotient by a reciprocal (2^-23) leave the move within 2^-20 of the exact form's, which saves a
// fifth of the 8-bit form's instructions (they and not bytes set its pace); the moments are the same to the bit.  Both flush
// subnormal numbers, so not every eps allows it.
template <bool FAST>
__device__ __forceinline__ void adamw_element(const AdamwHyper& h, float keep, float g, float& m, float& v, float& theta) {
  m = h.beta1 * m + h.omb1 * g;
  v = h.beta2 * v + h.omb2 * (g * g);
  if constexpr (FAST) {
    const float denom = sqrt_fast(v) * h.a + h.eps;
    theta = theta * keep - h.c * (m * rcp_fast(denom));
  } else {
    const float denom = __fsqrt_rn(v) * h.a + h.eps;
    theta = theta * keep - h.c * __fdiv_rn(m, denom);
  }
}

// Whether FAST keeps its bound: a flushed v < 2^-126 takes less than 2^-63 a from denom, at most 2^-22 of it from this eps on
// (1.4e-11 for a = 31.6, the first step at beta2 = 0.999; below, an eps that is subnormal itself would even give 0 * inf where
// v = 0); and 1 / denom must not be subnormal.  The exact form takes 700 us for the 187 M elements that take 587.
inline bool fast_move(const AdamwHyper& h) { return h.eps >= h.a * 0x1p-41f && h.eps <= 0x1p100f; }

// the gradient's factor; false (with the flag raised): skip the step
__device__ __forceinline__ bool gradient_scale(const float* p, uint32_t* flags, float& s) {
  s = p ? __ldg(p) : 1.0f;
  if (finite(s)) return true;
  if (flags && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(flags, (uint32_t)SL_FLAG_NONFINITE);
  return false;
}

__device__ __forceinline__ void raise_nonfinite(bool bad, uint32_t* flags) {
  if (__any_sync(0xFFFFFFFFu, bad) && flags && (threadIdx.x & 31) == 0) atomicOr(flags, (uint32_t)SL_FLAG_NONFINITE);
}

// ---------------------------------------------------------------------------
// 32-bit moments
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;

template <class TH, class GR, int T>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamwArgs<T> a) {
  float s;
  if (!gradient_scale(a.grad_scale, a.flags, s)) return;
  TH* theta = static_cast<TH*>(a.theta);
  const GR* grad = static_cast<const GR*>(a.grad);
  const AdamwHyper hy = a.hy;
  bool bad = false;
  Walk<T, true> walk(a.tb, a.block);
  for (uint32_t g = blockIdx.x; g < a.tb.n_blocks; g += gridDim.x) {
    const Seg sg = walk.at(g);
    // elements before the first multiple of 4 and behind the last one go one by one
    uint32_t head = a.aligned ? (uint32_t)(-(int64_t)sg.base & 3) : sg.len;
    if (head > sg.len) head = sg.len;
    const uint32_t quads = (sg.len - head) / 4;
#pragma unroll 2
    for (uint32_t q = threadIdx.x; q < quads; q += kThreads) {
      const uint64_t i = sg.base + head + 4u * q;
      Raw<TH, 4> rt;
      Raw<GR, 4> rg;
      Raw<float, 4> rm, rv;
      rt.load(theta + i);
      rg.load(grad + i);
      rm.load(a.m + i);
      rv.load(a.v + i);
      float th[4], m[4], v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float gr = s * rg.get(e);
        bad |= !finite(gr);
        th[e] = rt.get(e); m[e] = rm.get(e); v[e] = rv.get(e);
        adamw_element<false>(hy, sg.keep, gr, m[e], v[e], th[e]);
      }
      rt.set(th);
      rm.set(m);
      rv.set(v);
      rt.store(theta + i);
      rm.store(a.m + i);
      rv.store(a.v + i);
      if (a.copy) {
        Raw<Bf16, 4> rc;
        rc.set(th);
        rc.store(reinterpret_cast<Bf16*>(a.copy) + i);
      }
    }
    const uint32_t rest = sg.len - 4 * quads;
    for (uint32_t r = threadIdx.x; r < rest; r += kThreads) {
      const uint64_t i = sg.base + (r < head ? r : 4 * quads + r);
      const float gr = s * to_f32(grad[i]);
      bad |= !finite(gr);
      float th = to_f32(theta[i]), m = a.m[i], v = a.v[i];
      adamw_element<false>(hy, sg.keep, gr, m, v, th);
      theta[i] = from_f32<TH>(th);
      a.m[i] = m;
      a.v[i] = v;
      if (a.copy) a.copy[i] = from_f32<Bf16>(th).bits;
    }
  }
  raise_nonfinite(bad, a.flags);
}

// ---------------------------------------------------------------------------
// 8-bit moments: one warp per block of 256, eight elements to a lane
// ---------------------------------------------------------------------------
constexpr uint32_t kTiny = 0x00800000u, kInf = 0x7F800000u;   // patterns: smallest normal number, infinity

// byte e of a word as a float: the byte becomes the low mantissa bits of 2^23, which a subtraction takes off again
template <int E>
__device__ __forceinline__ float byte_float(uint2 c, float off) {
  return __uint_as_float(__byte_perm(E < 4 ? c.x : c.y, 0x4B000000u, 0x7440 + (E & 3))) - off;
}
// the values that codes stand for; the code of m is signed
__device__ __forceinline__ void decode(uint2 cm, uint2 cv, float tm, float tv, float (&m)[8], float (&v)[8]) {
  cm.x ^= 0x80808080u;                                     // int8 -> int8 + 128
  cm.y ^= 0x80808080u;
  const float om = 8388608.0f + 128.0f, ov = 8388608.0f;
  m[0] = byte_float<0>(cm, om); m[1] = byte_float<1>(cm, om); m[2] = byte_float<2>(cm, om); m[3] = byte_float<3>(cm, om);
  m[4] = byte_float<4>(cm, om); m[5] = byte_float<5>(cm, om); m[6] = byte_float<6>(cm, om); m[7] = byte_float<7>(cm, om);
  v[0] = byte_float<0>(cv, ov); v[1] = byte_float<1>(cv, ov); v[2] = byte_float<2>(cv, ov); v[3] = byte_float<3>(cv, ov);
  v[4] = byte_float<4>(cv, ov); v[5] = byte_float<5>(cv, ov); v[6] = byte_float<6>(cv, ov); v[7] = byte_float<7>(cv, ov);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    m[e] = tm * ((m[e] * fabsf(m[e])) * (1.0f / 16129.0f));
    const float r = (v[e] * v[e]) * (1.0f / 65025.0f);
    v[e] = tv * (r * r);
  }
}

// the scale that is stored and its reciprocal (0 for a block of zeros), from the largest magnitude's pattern
__device__ __forceinline__ void block_scale(uint32_t top_bits, float& top, float& inv) {
  if (top_bits >= kInf) { top = __uint_as_float(0x7FC00000u); inv = 0.0f; return; }
  const bool zero = top_bits < kTiny;
  top = zero ? 0.0f : __uint_as_float(top_bits);
  inv = zero ? 0.0f : __fdiv_rn(1.0f, top);
}
__device__ __forceinline__ int encode_m(float m, float inv) {
  const int q = __float2int_rn(__fsqrt_rn(fabsf(m) * inv) * 127.0f);
  return m < 0.0f ? -q : q;
}
__device__ __forceinline__ uint32_t encode_v(float v, float inv) {
  const uint32_t q = (uint32_t)__float2int_rn(__fsqrt_rn(__fsqrt_rn(v * inv)) * 255.0f);
  return (v > 0.0f && inv > 0.0f && q == 0) ? 1u : q;
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// The codes of a lane's eight elements.  The roots are taken fast and rounded by adding 1.5 * 2^23, whose sum's low byte is the
// code.  A fast root is off by 2^-23, so 127 sqrt(x) by at most 2.3e-5 and 255 x^(1/4) by at most 6.1e-5; the exactly rounded
// operations that define the code are off by 2.3e-5 and 4.6e-5 themselves.  So where no value comes within 5e-5 (1.2e-4)
// of the middle of two codes the codes are the defined ones; otherwise, for one lane in 360, the lane takes exact roots.
__device__ __forceinline__ void encode(const float (&m)[8], const float (&v)[8], float im, float iv, uint2& cm, uint2& cv) {
  constexpr float kRound = 12582912.0f, kNearM = 5e-5f, kNearV = 1.2e-4f;
  const float least = iv > 0.0f ? 1.0f : 0.0f;             // v > 0 keeps a code of at least 1
  float off = 0.0f;                                        // largest distance from a code, v's with what its bound is wider
  uint32_t bm[8], bv[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = copysignf(sqrt_fast(fabsf(m[e]) * im) * 127.0f, m[e]), t = y + kRound;
    float z = sqrt_fast(sqrt_fast(v[e] * iv)) * 255.0f;
    z = v[e] > 0.0f ? fmaxf(z, least) : z;
    const float u = z + kRound;
    off = fmaxf(off, fabsf(y - (t - kRound)));
    off = fmaxf(off, fabsf(z - (u - kRound)) + (kNearV - kNearM));
    bm[e] = __float_as_uint(t);
    bv[e] = __float_as_uint(u);
  }
  cm = make_uint2(low_bytes(bm[0], bm[1], bm[2], bm[3]), low_bytes(bm[4], bm[5], bm[6], bm[7]));
  cv = make_uint2(low_bytes(bv[0], bv[1], bv[2], bv[3]), low_bytes(bv[4], bv[5], bv[6], bv[7]));
  if (off > 0.5f - kNearM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bm[e] = (uint32_t)encode_m(m[e], im);
      bv[e] = encode_v(v[e], iv);
    }
    cm = make_uint2(low_bytes(bm[0], bm[1], bm[2], bm[3]), low_bytes(bm[4], bm[5], bm[6], bm[7]));
    cv = make_uint2(low_bytes(bv[0], bv[1], bv[2], bv[3]), low_bytes(bv[4], bv[5], bv[6], bv[7]));
  }
}

// The eight elements of a lane.
//   kWhole    a whole block that starts on a multiple of 8: eight consecutive elements to a lane
//   kShifted  any other whole block: it spreads over 33 aligned groups of 8.  Lanes 1..31 have the groups inside it, lane 0 the
//             two ends, which are one group together: slot j of the first group where that lies in the block, of the last
//             group otherwise.  Lane 0 reads both groups whole and writes element by element.
//   kSingle   short blocks and arrays whose start is not aligned: a lane's elements are 32 apart
// Nothing is done with what was loaded before take(), so that all loads of a block are on their way together.
enum Lanes { kWhole, kShifted, kSingle };

template <Lanes M>
struct Lane {
  uint64_t base;              // kWhole, kShifted: the lane's group; kSingle: the block
  uint32_t len, lane, before; // before: elements of the first group in front of the block

  __device__ __forceinline__ Lane(const Seg& s, uint32_t lane_) : base(s.base), len(s.len), lane(lane_), before(0) {
    if constexpr (M == kShifted) before = (uint32_t)s.base & 7;
    if constexpr (M != kSingle) base = s.base - before + 8u * lane;
  }
  __device__ __forceinline__ bool ends() const { return M == kShifted && lane == 0; }
  // where element e lies
  __device__ __forceinline__ uint64_t at(int e) const {
    if constexpr (M == kSingle) return base + lane + 32u * e;
    return base + e + (ends() && (uint32_t)e < before ? SL_STATE_BLOCK : 0);
  }
  __device__ __forceinline__ bool has(int e) const { return M != kSingle || lane + 32u * e < len; }

  template <class T>
  struct Held {
    Raw<T, 8> r, last;
    uint32_t one[8];
  };
  struct HeldCodes {
    uint2 c, last;
    uint32_t one[8];
  };
  template <class T>
  __device__ __forceinline__ void load(const T* p, Held<T>& h) const {
    if constexpr (M != kSingle) {
      h.r.load(p + base);
      if (ends()) h.last.load(p + base + SL_STATE_BLOCK);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h.one[e] = 0;
        if (has(e)) {
          if constexpr (sizeof(T) == 4) h.one[e] = __float_as_uint(p[at(e)]);
          else h.one[e] = p[at(e)].bits;
        }
      }
    }
  }
  template <class T>
  __device__ __forceinline__ void take(const Held<T>& h, float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (M == kSingle) f[e] = __uint_as_float(sizeof(T) == 4 ? h.one[e] : h.one[e] << 16);
      else f[e] = h.r.get(e);
    }
    if (ends())
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((uint32_t)e < before) f[e] = h.last.get(e);
  }
  __device__ __forceinline__ void load(const void* q, HeldCodes& h) const {
    const uint8_t* p = static_cast<const uint8_t*>(q);
    if constexpr (M != kSingle) {
      h.c = __ldcs(reinterpret_cast<const uint2*>(p + base));
      if (ends()) h.last = __ldcs(reinterpret_cast<const uint2*>(p + base + SL_STATE_BLOCK));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) h.one[e] = has(e) ? p[at(e)] : 0u;
    }
  }
  __device__ __forceinline__ uint2 take(const HeldCodes& h) const {
    if constexpr (M == kSingle)
      return make_uint2(low_bytes(h.one[0], h.one[1], h.one[2], h.one[3]), low_bytes(h.one[4], h.one[5], h.one[6], h.one[7]));
    if (!ends()) return h.c;
    const uint64_t mask = (1ull << (8 * before)) - 1;      // the slots of the last group
    const uint64_t c = ((uint64_t)h.c.y << 32 | h.c.x) & ~mask, l = ((uint64_t)h.last.y << 32 | h.last.x) & mask;
    return make_uint2((uint32_t)(c | l), (uint32_t)((c | l) >> 32));
  }
  template <class T>
  __device__ __forceinline__ void store(T* p, const float (&f)[8]) const {
    if (M != kSingle && !ends()) {
      Raw<T, 8> r;
      r.set(f);
      r.store(p + base);
    } else if constexpr (M != kWhole) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (has(e)) p[at(e)] = from_f32<T>(f[e]);
    }
  }
  __device__ __forceinline__ void store_codes(void* q, uint2 c) const {
    uint8_t* p = static_cast<uint8_t*>(q);
    if (M != kSingle && !ends()) {
      __stcs(reinterpret_cast<uint2*>(p + base), c);
    } else if constexpr (M != kWhole) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (has(e)) p[at(e)] = (uint8_t)((e < 4 ? c.x >> (8 * e) : c.y >> (8 * e - 32)) & 0xFFu);
    }
  }
};

// how a block's elements are dealt to the lanes; n_total: elements of the arena, which a group may not reach past
__device__ __forceinline__ Lanes lanes_of(const Seg& s, bool aligned, uint64_t n_total) {
  if (!aligned || s.len != SL_STATE_BLOCK) return kSingle;
  if ((s.base & 7) == 0) return kWhole;
  return (s.base & ~7ull) + SL_STATE_BLOCK + 8 <= n_total ? kShifted : kSingle;
}

// scales and codes of a block from its lanes' moments; false: some moment is Inf or NaN (all codes are 0, the scale is NaN)
__device__ __forceinline__ bool quantise(const float (&m)[8], const float (&v)[8], uint2& cm, uint2& cv, float& tm, float& tv) {
  float fm = 0.0f, fv = 0.0f;                              // NaN if one of them is
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(fm) : "f"(fabsf(m[e])));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(fv) : "f"(v[e]));
  }
  const uint32_t um = __reduce_max_sync(0xFFFFFFFFu, key_of(fm)), uv = __reduce_max_sync(0xFFFFFFFFu, key_of(fv));
  float im, iv;
  block_scale(um, tm, im);
  block_scale(uv, tv, iv);
  encode(m, v, im, iv, cm, cv);
  if (um >= kInf) cm = make_uint2(0, 0);
  if (uv >= kInf) cv = make_uint2(0, 0);
  return um < kInf && uv < kInf;
}

// one block of the step, by a warp; false: some new moment is Inf or NaN
template <class TH, class GR, bool FAST, Lanes M, int T>
__device__ __forceinline__ bool step_block(const AdamwArgs<T>& a, const Seg& sg, uint32_t g, uint32_t lane, float s) {
  const Lane<M> le(sg, lane);
  typename Lane<M>::template Held<TH> ht;
  typename Lane<M>::template Held<GR> hg;
  typename Lane<M>::HeldCodes hm, hv;
  le.load(static_cast<const TH*>(a.theta), ht);
  le.load(static_cast<const GR*>(a.grad), hg);
  le.load(a.m8, hm);
  le.load(a.v8, hv);
  float tm = a.m_scale[g], tv = a.v_scale[g];
  float th[8], gr[8], m[8], v[8];
  decode(le.take(hm), le.take(hv), tm, tv, m, v);
  le.take(ht, th);
  le.take(hg, gr);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    adamw_element<FAST>(a.hy, sg.keep, s * gr[e], m[e], v[e], th[e]);
    if (!le.has(e)) m[e] = v[e] = 0.0f;                    // behind the end of a short block
  }
  le.store(static_cast<TH*>(a.theta), th);
  if (a.copy) le.store(reinterpret_cast<Bf16*>(a.copy), th);
  uint2 cm, cv;
  const bool good = quantise(m, v, cm, cv, tm, tv);
  le.store_codes(a.m8, cm);
  le.store_codes(a.v8, cv);
  if (lane == 0) {
    a.m_scale[g] = tm;
    a.v_scale[g] = tv;
  }
  return good;
}
// the same out of line, so that the blocks that need more registers do not take them from the others (187 M elements: 679 us
// with all three forms in line, 586 us with the whole blocks alone)
template <class TH, class GR, bool FAST, Lanes M, int T>
__device__ __noinline__ bool step_block_apart(const AdamwArgs<T>& a, const Seg& sg, uint32_t g, uint32_t lane, float s) {
  return step_block<TH, GR, FAST, M, T>(a, sg, g, lane, s);
}

// 64 registers, so that four CTAs fit an SM
template <class TH, class GR, bool FAST, int T>
__global__ void __maxnreg__(64) adamw8_kernel(const __grid_constant__ AdamwArgs<T> a) {
  float s;
  if (!gradient_scale(a.grad_scale, a.flags, s)) return;
  const uint32_t lane = threadIdx.x & 31, warps = gridDim.x * (kThreads / 32);
  bool bad = false;
  Walk<T, false> walk(a.tb, SL_STATE_BLOCK);
  const uint64_t n_total = a.tb.offset[a.tb.n_tensors];
  for (uint32_t g = blockIdx.x * (kThreads / 32) + threadIdx.x / 32; g < a.tb.n_blocks; g += warps) {
    const Seg sg = walk.at(g);
    const Lanes how = lanes_of(sg, a.aligned, n_total);
    if (how == kWhole) bad |= !step_block<TH, GR, FAST, kWhole>(a, sg, g, lane, s);
    else if (how == kShifted) bad |= !step_block_apart<TH, GR, FAST, kShifted>(a, sg, g, lane, s);
    else bad |= !step_block_apart<TH, GR, FAST, kSingle>(a, sg, g, lane, s);
  }
  raise_nonfinite(bad, a.flags);
}

template <bool PACK, Lanes M, int T>
__device__ __forceinline__ void convert_block(const AdamwArgs<T>& a, const Seg& sg, uint32_t g, uint32_t lane) {
  const Lane<M> le(sg, lane);
  float m[8], v[8];
  if constexpr (PACK) {
    typename Lane<M>::template Held<float> hm, hv;
    le.load(a.m, hm);
    le.load(a.v, hv);
    le.take(hm, m);
    le.take(hv, v);
    uint2 cm, cv;
    float tm, tv;
    quantise(m, v, cm, cv, tm, tv);
    le.store_codes(a.m8, cm);
    le.store_codes(a.v8, cv);
    if (lane == 0) {
      a.m_scale[g] = tm;
      a.v_scale[g] = tv;
    }
  } else {
    typename Lane<M>::HeldCodes hm, hv;
    le.load(a.m8, hm);
    le.load(a.v8, hv);
    decode(le.take(hm), le.take(hv), a.m_scale[g], a.v_scale[g], m, v);
    le.store(a.m, m);
    le.store(a.v, v);
  }
}

template <bool PACK, int T>
__global__ void __launch_bounds__(kThreads) adamw8_convert_kernel(const __grid_constant__ AdamwArgs<T> a) {
  const uint32_t lane = threadIdx.x & 31, warps = gridDim.x * (kThreads / 32);
  Walk<T, false> walk(a.tb, SL_STATE_BLOCK);
  const uint64_t n_total = a.tb.offset[a.tb.n_tensors];
  for (uint32_t g = blockIdx.x * (kThreads / 32) + threadIdx.x / 32; g < a.tb.n_blocks; g += warps) {
    const Seg sg = walk.at(g);
    const Lanes how = lanes_of(sg, a.aligned, n_total);
    if (how == kWhole) convert_block<PACK, kWhole>(a, sg, g, lane);
    else if (how == kShifted) convert_block<PACK, kShifted>(a, sg, g, lane);
    else convert_block<PACK, kSingle>(a, sg, g, lane);
  }
}

// CTAs of a grid-stride launch: what fits the device at once, or fewer when there is less work
inline cudaError_t stride_grid(uint64_t want, int per_sm, uint32_t* grid) {
  cudaError_t e;
  const int sms = sm_count(&e);
  if (sms <= 0) return e == cudaSuccess ? cudaErrorInvalidDevice : e;
  const uint64_t most = (uint64_t)sms * per_sm;
  *grid = (uint32_t)(want < most ? want : most);
  return cudaSuccess;
}

}  // namespace

template <int T>
cudaError_t launch_adamw(const AdamwArgs<T>& a, int theta_type, int grad_type, cudaStream_t st) {
  uint32_t grid;
  cudaError_t e = stride_grid(a.tb.n_blocks, 8, &grid);
  if (e != cudaSuccess) return e;
  return with_type(theta_type, [&](auto th) {
    return with_type(grad_type, [&](auto gr) {
      adamw_kernel<decltype(th), decltype(gr), T><<<grid, kThreads, 0, st>>>(a);
      return cudaPeekAtLastError();
    });
  });
}

template <int T>
cudaError_t launch_adamw8(const AdamwArgs<T>& a, int theta_type, int grad_type, cudaStream_t st) {
  uint32_t grid;
  cudaError_t e = stride_grid((a.tb.n_blocks + kThreads / 32 - 1) / (kThreads / 32), 8, &grid);
  if (e != cudaSuccess) return e;
  return with_type(theta_type, [&](auto th) {
    return with_type(grad_type, [&](auto gr) {
      if (fast_move(a.hy)) adamw8_kernel<decltype(th), decltype(gr), true, T><<<grid, kThreads, 0, st>>>(a);
      else adamw8_kernel<decltype(th), decltype(gr), false, T><<<grid, kThreads, 0, st>>>(a);
      return cudaPeekAtLastError();
    });
  });
}

template <bool PACK, int T>
static cudaError_t launch_convert(const AdamwArgs<T>& a, cudaStream_t st) {
  uint32_t grid;
  cudaError_t e = stride_grid((a.tb.n_blocks + kThreads / 32 - 1) / (kThreads / 32), 8, &grid);
  if (e != cudaSuccess) return e;
  adamw8_convert_kernel<PACK, T><<<grid, kThreads, 0, st>>>(a);
  return cudaPeekAtLastError();
}
template <int T>
cudaError_t launch_adamw8_pack(const AdamwArgs<T>& a, cudaStream_t st) { return launch_convert<true, T>(a, st); }
template <int T>
cudaError_t launch_adamw8_unpack(const AdamwArgs<T>& a, cudaStream_t st) { return launch_convert<false, T>(a, st); }

#define SL_INSTANTIATE(T)                                                                        \
  template cudaError_t launch_adamw<T>(const AdamwArgs<T>&, int, int, cudaStream_t);            \
  template cudaError_t launch_adamw8<T>(const AdamwArgs<T>&, int, int, cudaStream_t);           \
  template cudaError_t launch_adamw8_pack<T>(const AdamwArgs<T>&, cudaStream_t);                \
  template cudaError_t launch_adamw8_unpack<T>(const AdamwArgs<T>&, cudaStream_t);
SL_INSTANTIATE(32)
SL_INSTANTIATE(256)
SL_INSTANTIATE(SL_MAX_TENSORS)
#undef SL_INSTANTIATE

}  // namespace sl
