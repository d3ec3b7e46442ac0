// Shared pieces of the inner-step kernels (Eq. 1): element types, vector loads, host-side helpers.
#pragma once
#include <type_traits>

#include "sl_common.cuh"

namespace sl {

// bfloat16 as it is stored; a type of its own so that templates can tell it from an integer
struct Bf16 {
  uint16_t bits;
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(Bf16 v) { return bf16_widen(v.bits); }
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ Bf16 from_f32<Bf16>(float v) {     // to nearest, ties to even, NaN to NaN
  uint16_t r;
  asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(v));
  return Bf16{r};
}

// two floats -> two bfloat16 in one instruction (lo in the low half): to nearest, ties to even, NaN to NaN
__device__ __forceinline__ uint32_t bf16x2_round(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// E consecutive elements held as they are stored, moved by accesses of up to 32 bytes: a warp whose lanes hold eight floats
// each would touch every 32-byte sector twice with 16-byte accesses.  The address is a multiple of min(32, E * sizeof(T)).
template <class T, int E>
struct Raw {
  static constexpr int W = E * (int)sizeof(T) / 4;      // 32-bit words
  static_assert(W == 1 || W == 2 || W == 4 || W == 8, "one access");
  uint32_t w[W];

  __device__ __forceinline__ void load(const T* p) {     // streamed once: not kept in L1
    if constexpr (W == 8) {
      asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p));
    } else if constexpr (W == 4) {
      const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (W == 2) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
      w[0] = v.x; w[1] = v.y;
    } else {
      w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
    }
  }
  __device__ __forceinline__ void load_kept(const T* p) {       // others read it too
    static_assert(W >= 4, "vectors");
    if constexpr (W == 8) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p));
    } else {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (W == 8) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else if constexpr (W == 4) {
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else if constexpr (W == 2) {
      __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
    } else {
      __stcs(reinterpret_cast<uint32_t*>(p), w[0]);
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (std::is_same_v<T, float>) return __uint_as_float(w[e]);
    else return __uint_as_float((e & 1) ? (w[e / 2] & 0xFFFF0000u) : (w[e / 2] << 16));
  }
  __device__ __forceinline__ void set(const float (&f)[E]) {
    if constexpr (std::is_same_v<T, float>) {
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = __float_as_uint(f[e]);
    } else {
#pragma unroll
      for (int e = 0; e < E / 2; ++e) w[e] = bf16x2_round(f[2 * e], f[2 * e + 1]);
    }
  }
};

// Programmatic dependent launch: a kernel that is launched with launch_behind() may start while the one before it in the
// stream still runs, once all of that one's CTAs have called let_next_start() or ended; wait_for_previous() returns when
// it has ended and its writes are visible.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... P, class... A>
inline cudaError_t launch_behind(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

inline bool is_aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
inline bool vector_aligned(const void* p, int type) { return is_aligned(p, type == SL_BF16 ? 16 : 32); }   // of eight elements
inline size_t type_size(int type) { return type == SL_BF16 ? 2 : 4; }

// calls f with a value of the element type that `type` names
template <class F>
inline cudaError_t with_type(int type, F&& f) {
  return type == SL_BF16 ? f(Bf16{}) : f(float{});
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
struct AdamwHyper {
  float beta1, omb1, beta2, omb2, eps, a, c;
};

// The arena cut into blocks of consecutive elements that do not straddle tensors.  Blocks begin at a tensor's first
// element rounded down to a multiple of `align`; what lies before the tensor is not part of its first block.
template <int T>
struct BlockTable {
  uint32_t n_tensors, n_blocks, align;
  uint32_t first_block[T + 1];
  float keep[T];              // 1 - lr * decay
  uint64_t offset[T + 1];
};

template <int T>
struct AdamwArgs {
  BlockTable<T> tb;
  AdamwHyper hy;
  void* theta;
  const void* grad;
  float *m, *v;               // 32-bit states
  int8_t* m8;                 // 8-bit states
  uint8_t* v8;
  float *m_scale, *v_scale;
  uint16_t* copy;
  const float* grad_scale;
  uint32_t* flags;
  uint32_t block;             // elements of a block of the 32-bit form
  bool aligned;               // every array starts on the boundary its vector accesses need
};

// Elements of one tensor that a CTA of the 32-bit form takes at a time: 4096, or 1024 where that would leave SMs without
// work (262,656 elements: 4.4 -> 2.8 us)
constexpr uint32_t adamw_block(uint64_t n_total) { return n_total < 148ull * 8 * 4096 ? 1024 : 4096; }

template <int T> cudaError_t launch_adamw(const AdamwArgs<T>& a, int theta_type, int grad_type, cudaStream_t st);
template <int T> cudaError_t launch_adamw8(const AdamwArgs<T>& a, int theta_type, int grad_type, cudaStream_t st);
template <int T> cudaError_t launch_adamw8_pack(const AdamwArgs<T>& a, cudaStream_t st);
template <int T> cudaError_t launch_adamw8_unpack(const AdamwArgs<T>& a, cudaStream_t st);

// ---------------------------------------------------------------------------
// embedding lookup and its gradient
// ---------------------------------------------------------------------------
struct LookupArgs {
  const int32_t* ids;
  const void *T_S, *T_perp, *pos;
  void* X;
  uint32_t* flags;
  float scale;
  uint32_t n_tok, L, V, d;
};
struct EmbedGradArgs {
  const int32_t* ids;
  const void* dX;
  void *dT, *dpos;
  void* ws;
  uint32_t* flags;
  float scale;
  uint32_t n_tok, L, V, d;
  int acc;
};
cudaError_t launch_embed_lookup(const LookupArgs& a, int table_type, int x_type, cudaStream_t st);
cudaError_t launch_embed_grad(const EmbedGradArgs& a, int dx_type, int dt_type, cudaStream_t st);
uint64_t embed_grad_workspace(uint64_t n_tok, uint64_t V, uint32_t d);
bool embed_grad_fits(const EmbedGradArgs& a, int dx_type, int dt_type);      // a grid holds its columns

// ---------------------------------------------------------------------------
// norm block
// ---------------------------------------------------------------------------
struct NormArgs {
  const void *x, *b, *g, *w_post, *w_pre;
  void *h, *y;
  float *r_post, *r_pre;
  uint64_t ldb, ldg;
  uint32_t n, d;
  float alpha, eps;
  int w_bf16;
  uint32_t* flags;
  uint32_t wait_polls;       // as in CompressArgs
};
struct NormGradArgs {
  const void *dh, *dy, *h, *b, *g, *w_post, *w_pre;
  const float *r_post, *r_pre;
  void *dx, *db, *dg, *dw_post, *dw_pre;
  float* ws;
  uint64_t ldb, ldg;
  uint32_t n, d;
  float alpha;
  int w_bf16, acc;
  uint32_t* flags;
  uint32_t wait_polls;
};
cudaError_t launch_norm_block(const NormArgs& a, int res_type, int act_type, cudaStream_t st);
cudaError_t launch_norm_block_grad(const NormGradArgs& a, int res_type, int act_type, cudaStream_t st);
uint64_t norm_block_grad_workspace(uint64_t n, uint32_t d);

}  // namespace sl
