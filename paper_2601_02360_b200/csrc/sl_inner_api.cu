// Host side of the inner-step calls of include/sparseloco.h: argument checks, the by-value arena table, dispatch.
// No allocation, no state, no synchronisation.
#include <cfloat>
#include <cmath>

#include "sl_inner.cuh"

namespace {

using namespace sl;

inline bool type_ok(int t) { return t == SL_F32 || t == SL_BF16; }
inline bool typed_aligned(const void* p, int type) { return is_aligned(p, type_size(type)); }
inline int status(cudaError_t e) { return e == cudaSuccess ? SL_OK : SL_ERR_CUDA; }

// blocks of tensor t that begin at its start rounded down to a multiple of `align`
uint64_t blocks_in(const sl_layout* L, uint32_t t, uint32_t block, uint32_t align) {
  if (L->offset[t + 1] == L->offset[t]) return 0;
  return (L->offset[t + 1] - (L->offset[t] & ~(uint64_t)(align - 1)) + block - 1) / block;
}

int check_layout(const sl_layout* L, uint32_t block, uint32_t align) {
  if (!L || !L->offset || L->n_tensors < 1) return SL_ERR_INVALID_ARG;
  if (L->n_tensors > SL_MAX_TENSORS) return SL_ERR_UNSUPPORTED;
  if (L->offset[0] != 0 || L->offset[L->n_tensors] != L->n_total) return SL_ERR_INVALID_ARG;
  uint64_t n = 0;
  for (uint32_t t = 0; t < L->n_tensors; ++t) {
    if (L->offset[t + 1] < L->offset[t]) return SL_ERR_INVALID_ARG;
    n += blocks_in(L, t, block, align);
  }
  return n > 0x7FFFFFFFull ? SL_ERR_UNSUPPORTED : SL_OK;
}

template <int T>
void fill_blocks(BlockTable<T>& tb, const sl_layout* L, uint32_t block, uint32_t align, const float* decay, double lr) {
  tb.align = align;
  tb.n_tensors = L->n_tensors;
  uint32_t n = 0;
  for (uint32_t t = 0; t < L->n_tensors; ++t) {
    tb.first_block[t] = n;
    tb.offset[t] = L->offset[t];
    tb.keep[t] = (float)(1.0 - lr * (decay ? (double)decay[t] : 0.0));
    n += (uint32_t)blocks_in(L, t, block, align);
  }
  tb.first_block[L->n_tensors] = n;
  tb.offset[L->n_tensors] = L->n_total;
  tb.n_blocks = n;
}

// the kernels' argument block, built on the caller's stack; `go` launches it
template <int T, class F>
int with_args_of(AdamwArgs<T>& a, const AdamwArgs<1>& common, const sl_layout* L, uint32_t block, uint32_t align, const float* decay,
                 double lr, F&& go) {
  fill_blocks(a.tb, L, block, align, decay, lr);
  a.hy = common.hy;
  a.theta = common.theta;
  a.grad = common.grad;
  a.m = common.m;
  a.v = common.v;
  a.m8 = common.m8;
  a.v8 = common.v8;
  a.m_scale = common.m_scale;
  a.v_scale = common.v_scale;
  a.copy = common.copy;
  a.grad_scale = common.grad_scale;
  a.flags = common.flags;
  a.block = block;
  a.aligned = common.aligned;
  return a.tb.n_blocks == 0 ? SL_OK : status(go(a));
}
template <class F>
int with_args(const AdamwArgs<1>& common, const sl_layout* L, uint32_t block, uint32_t align, const float* decay, double lr, F&& go) {
  if (L->n_tensors <= 32) {
    AdamwArgs<32> a;
    return with_args_of(a, common, L, block, align, decay, lr, go);
  }
  if (L->n_tensors <= 256) {
    AdamwArgs<256> a;
    return with_args_of(a, common, L, block, align, decay, lr, go);
  }
  AdamwArgs<SL_MAX_TENSORS> a;
  return with_args_of(a, common, L, block, align, decay, lr, go);
}

// what both forms of the step check of their arguments, and the constants of the step; vec: elements of a vector access
int adamw_common(AdamwArgs<1>& a, void* theta, int theta_type, const void* grad, int grad_type, uint16_t* copy, const sl_layout* L,
                 uint32_t block, uint32_t vec, const float* decay, double lr, double beta1, double beta2, double eps, uint64_t step,
                 const float* grad_scale, uint32_t* flags) {
  if (!type_ok(theta_type) || !type_ok(grad_type) || (copy && theta_type != SL_F32)) return SL_ERR_INVALID_ARG;
  if (!L || (L->n_total > 0 && (!theta || !grad))) return SL_ERR_INVALID_ARG;
  if (!std::isfinite(lr) || lr < 0 || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps > 0) || !(eps <= FLT_MAX) ||
      (float)eps == 0.0f || step < 1)
    return SL_ERR_INVALID_ARG;
  const int rc = check_layout(L, block, block == SL_STATE_BLOCK ? 1 : vec);
  if (rc != SL_OK) return rc;
  if (decay)
    for (uint32_t t = 0; t < L->n_tensors; ++t)
      if (!std::isfinite(decay[t]) || decay[t] < 0) return SL_ERR_INVALID_ARG;
  if (!typed_aligned(theta, theta_type) || !typed_aligned(grad, grad_type) || !is_aligned(copy, 2) || !is_aligned(grad_scale, 4) ||
      !is_aligned(flags, 4))
    return SL_ERR_ALIGNMENT;
  a.theta = theta;
  a.grad = grad;
  a.m = a.v = nullptr;
  a.m8 = nullptr;
  a.v8 = nullptr;
  a.m_scale = a.v_scale = nullptr;
  a.copy = copy;
  a.grad_scale = grad_scale;
  a.flags = flags;
  a.hy.beta1 = (float)beta1;
  a.hy.omb1 = (float)(1.0 - beta1);
  a.hy.beta2 = (float)beta2;
  a.hy.omb2 = (float)(1.0 - beta2);
  a.hy.eps = (float)eps;
  a.hy.a = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  a.hy.c = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  a.aligned = is_aligned(theta, vec * type_size(theta_type)) && is_aligned(grad, vec * type_size(grad_type)) && is_aligned(copy, vec * 2);
  return SL_OK;
}

int states8_check(const sl_layout* L, const int8_t* m8, const uint8_t* v8, const float* m_scale, const float* v_scale) {
  if (!L || (L->n_total > 0 && (!m8 || !v8 || !m_scale || !v_scale))) return SL_ERR_INVALID_ARG;
  return is_aligned(m_scale, 4) && is_aligned(v_scale, 4) ? SL_OK : SL_ERR_ALIGNMENT;
}

AdamwArgs<1> convert_args(float* m, float* v, int8_t* m8, uint8_t* v8, float* m_scale, float* v_scale) {
  AdamwArgs<1> a{};
  a.m = m;
  a.v = v;
  a.m8 = m8;
  a.v8 = v8;
  a.m_scale = m_scale;
  a.v_scale = v_scale;
  a.aligned = vector_aligned(m, SL_F32) && vector_aligned(v, SL_F32) && is_aligned(m8, 8) && is_aligned(v8, 8);
  return a;
}

int convert_check(const float* m, const float* v, const sl_layout* L, const int8_t* m8, const uint8_t* v8, const float* m_scale,
                  const float* v_scale) {
  int rc = states8_check(L, m8, v8, m_scale, v_scale);
  if (rc != SL_OK) return rc;
  if (L->n_total > 0 && (!m || !v)) return SL_ERR_INVALID_ARG;
  if ((rc = check_layout(L, SL_STATE_BLOCK, 1)) != SL_OK) return rc;
  return is_aligned(m, 4) && is_aligned(v, 4) ? SL_OK : SL_ERR_ALIGNMENT;
}

int norm_types_check(int res_type, int act_type, int w_type) {
  if (!type_ok(res_type) || !type_ok(act_type) || !type_ok(w_type)) return SL_ERR_INVALID_ARG;
  return res_type == SL_BF16 && act_type == SL_F32 ? SL_ERR_UNSUPPORTED : SL_OK;
}

}  // namespace

extern "C" {

int sl_adamw(void* theta, int theta_type, const void* grad, int grad_type, float* m, float* v, uint16_t* copy, const sl_layout* L,
             const float* decay, double lr, double beta1, double beta2, double eps, uint64_t step, const float* grad_scale,
             uint32_t* flags, void* stream) {
  AdamwArgs<1> a;
  if (!L || (L->n_total > 0 && (!m || !v))) return SL_ERR_INVALID_ARG;
  const uint32_t block = adamw_block(L->n_total);
  const int rc = adamw_common(a, theta, theta_type, grad, grad_type, copy, L, block, 4, decay, lr, beta1, beta2, eps, step,
                              grad_scale, flags);
  if (rc != SL_OK) return rc;
  if (!is_aligned(m, 4) || !is_aligned(v, 4)) return SL_ERR_ALIGNMENT;
  a.m = m;
  a.v = v;
  a.aligned = a.aligned && is_aligned(m, 16) && is_aligned(v, 16);
  return with_args(a, L, block, 4, decay, lr,
                   [&](const auto& args) { return launch_adamw(args, theta_type, grad_type, (cudaStream_t)stream); });
}

uint64_t sl_adamw8_blocks(const sl_layout* L) {
  if (check_layout(L, SL_STATE_BLOCK, 1) != SL_OK) return 0;
  uint64_t n = 0;
  for (uint32_t t = 0; t < L->n_tensors; ++t) n += blocks_in(L, t, SL_STATE_BLOCK, 1);
  return n;
}

int sl_adamw8(void* theta, int theta_type, const void* grad, int grad_type, int8_t* m8, uint8_t* v8, float* m_scale, float* v_scale,
              uint16_t* copy, const sl_layout* L, const float* decay, double lr, double beta1, double beta2, double eps,
              uint64_t step, const float* grad_scale, uint32_t* flags, void* stream) {
  AdamwArgs<1> a;
  int rc = states8_check(L, m8, v8, m_scale, v_scale);
  if (rc != SL_OK) return rc;
  rc = adamw_common(a, theta, theta_type, grad, grad_type, copy, L, SL_STATE_BLOCK, 8, decay, lr, beta1, beta2, eps, step, grad_scale,
                    flags);
  if (rc != SL_OK) return rc;
  a.m8 = m8;
  a.v8 = v8;
  a.m_scale = m_scale;
  a.v_scale = v_scale;
  a.aligned = a.aligned && is_aligned(m8, 8) && is_aligned(v8, 8);
  return with_args(a, L, SL_STATE_BLOCK, 1, decay, lr,
                   [&](const auto& args) { return launch_adamw8(args, theta_type, grad_type, (cudaStream_t)stream); });
}

int sl_adamw8_pack(const float* m, const float* v, const sl_layout* L, int8_t* m8, uint8_t* v8, float* m_scale, float* v_scale,
                   void* stream) {
  const int rc = convert_check(m, v, L, m8, v8, m_scale, v_scale);
  if (rc != SL_OK) return rc;
  return with_args(convert_args(const_cast<float*>(m), const_cast<float*>(v), m8, v8, m_scale, v_scale), L, SL_STATE_BLOCK, 1, nullptr, 0.0,
                   [&](const auto& args) { return launch_adamw8_pack(args, (cudaStream_t)stream); });
}

int sl_adamw8_unpack(const int8_t* m8, const uint8_t* v8, const float* m_scale, const float* v_scale, const sl_layout* L, float* m,
                     float* v, void* stream) {
  const int rc = convert_check(m, v, L, m8, v8, m_scale, v_scale);
  if (rc != SL_OK) return rc;
  return with_args(convert_args(m, v, const_cast<int8_t*>(m8), const_cast<uint8_t*>(v8), const_cast<float*>(m_scale),
                                const_cast<float*>(v_scale)), L, SL_STATE_BLOCK, 1, nullptr, 0.0,
                   [&](const auto& args) { return launch_adamw8_unpack(args, (cudaStream_t)stream); });
}

int sl_embed_lookup(const int32_t* ids, const void* T_S, const void* T_perp, const void* pos, int table_type, float scale,
                    uint64_t n_tok, uint32_t L, uint64_t V, uint32_t d, void* X, int x_type, uint32_t* flags, void* stream) {
  if (!T_S || (n_tok > 0 && (!ids || !X)) || !type_ok(table_type) || !type_ok(x_type) || d < 1 || V < 1 || (pos && L < 1) || !std::isfinite(scale))
    return SL_ERR_INVALID_ARG;
  if (!is_aligned(ids, 4) || !typed_aligned(T_S, table_type) || !typed_aligned(T_perp, table_type) || !typed_aligned(pos, table_type) ||
      !typed_aligned(X, x_type) || !is_aligned(flags, 4))
    return SL_ERR_ALIGNMENT;
  if (n_tok > 0x7FFFFFFFull || V > 0x7FFFFFFFull || d > 0x7FFFFFFFu) return SL_ERR_UNSUPPORTED;
  if (n_tok == 0) return SL_OK;
  // positions behind the last token are nobody's: the kernel walks L places a sequence (one token of 131,072 positions: 12.8 us, 2.1 without
  // them)
  const uint32_t positions = L < 1 ? 1u : L < n_tok ? L : (uint32_t)n_tok;
  LookupArgs a{ids, T_S, T_perp, pos, X, flags, scale, (uint32_t)n_tok, positions, (uint32_t)V, d};
  return status(launch_embed_lookup(a, table_type, x_type, (cudaStream_t)stream));
}

uint64_t sl_embed_grad_workspace(uint64_t n_tok, uint64_t V, uint32_t d) {
  if (d < 1 || d > 0x7FFFFFFFu || n_tok > 0x7FFFFFFFull) return 0;         // sizes that the call refuses
  return embed_grad_workspace(n_tok, V, d);
}

int sl_embed_grad(const int32_t* ids, const void* dX, int dx_type, float scale, uint64_t n_tok, uint32_t L, uint64_t V, uint32_t d,
                  void* dT, void* dpos, int dt_type, int acc, void* ws, uint32_t* flags, void* stream) {
  if (!dT || !type_ok(dx_type) || !type_ok(dt_type) || d < 1 || V < 1 || (dpos && L < 1) || !std::isfinite(scale) ||
      (n_tok > 0 && (!ids || !dX || !ws)))
    return SL_ERR_INVALID_ARG;
  if (!is_aligned(ids, 4) || !typed_aligned(dX, dx_type) || !typed_aligned(dT, dt_type) || !typed_aligned(dpos, dt_type) ||
      !is_aligned(ws, 32) || !is_aligned(flags, 4))
    return SL_ERR_ALIGNMENT;
  if (n_tok > 0x7FFFFFFFull || V > 0x7FFFFFFFull || d > 0x7FFFFFFFu) return SL_ERR_UNSUPPORTED;
  if (n_tok == 0 && acc) return SL_OK;
  EmbedGradArgs a{ids, dX, dT, dpos, ws, flags, scale, (uint32_t)n_tok, L < 1 ? 1u : L, (uint32_t)V, d, acc ? 1 : 0};
  if (!embed_grad_fits(a, dx_type, dt_type)) return SL_ERR_UNSUPPORTED;
  return status(launch_embed_grad(a, dx_type, dt_type, (cudaStream_t)stream));
}

int sl_norm_block(const void* x, const void* b, const void* g, int res_type, int act_type, const void* w_post, const void* w_pre,
                  int w_type, uint64_t n, uint32_t d, uint64_t ldb, uint64_t ldg, float alpha, float eps, void* h, void* y,
                  float* r_post, float* r_pre, uint32_t* flags, void* stream) {
  int rc = norm_types_check(res_type, act_type, w_type);
  if (rc != SL_OK) return rc;
  if (d < 1 || !std::isfinite(alpha) || !(eps >= 0) || !std::isfinite(eps)) return SL_ERR_INVALID_ARG;
  if (n == 0) return d > SL_MAX_WIDTH ? SL_ERR_UNSUPPORTED : SL_OK;        // no pointer tells what is there: empty arrays may have none
  if (!x) return SL_ERR_INVALID_ARG;
  if (b ? (!h || ldb < d || (g && ldg < d)) : (g || w_post || h || !y)) return SL_ERR_INVALID_ARG;
  if ((y && !w_pre) || (!y && (w_pre || r_pre))) return SL_ERR_INVALID_ARG;
  if (!typed_aligned(x, res_type) || !typed_aligned(h, res_type) || !typed_aligned(b, act_type) || !typed_aligned(g, act_type) ||
      !typed_aligned(y, act_type) || !typed_aligned(w_post, w_type) || !typed_aligned(w_pre, w_type) || !is_aligned(r_post, 4) ||
      !is_aligned(r_pre, 4) || !is_aligned(flags, 4))
    return SL_ERR_ALIGNMENT;
  if (n > 0x7FFFFFFFull || d > SL_MAX_WIDTH) return SL_ERR_UNSUPPORTED;
  NormArgs a{x, b, g, w_post, w_pre, h, y, r_post, r_pre, b ? ldb : 0, g ? ldg : 0, (uint32_t)n, d, alpha, eps, w_type == SL_BF16, flags,
             debug_wait_polls()};
  return status(launch_norm_block(a, res_type, act_type, (cudaStream_t)stream));
}

uint64_t sl_norm_block_grad_workspace(uint64_t n, uint32_t d) { return norm_block_grad_workspace(n, d); }

int sl_norm_block_grad(const void* dh, const void* dy, const void* h, const void* b, const void* g, int res_type, int act_type,
                       const void* w_post, const void* w_pre, int w_type, const float* r_post, const float* r_pre, uint64_t n,
                       uint32_t d, uint64_t ldb, uint64_t ldg, float alpha, void* dx, void* db, void* dg, void* dw_post, void* dw_pre,
                       int acc, void* ws, uint32_t* flags, void* stream) {
  int rc = norm_types_check(res_type, act_type, w_type);
  if (rc != SL_OK) return rc;
  if (d < 1 || !std::isfinite(alpha)) return SL_ERR_INVALID_ARG;
  if (n > 0) {                                             // of no rows only the weights' gradients (zeros) are looked at
    if (!h || !dx || (!dh && !dy)) return SL_ERR_INVALID_ARG;
    if (b ? (!db || ldb < d || (g && ldg < d)) : (g || w_post || db)) return SL_ERR_INVALID_ARG;
    if ((g != nullptr) != (dg != nullptr) || (w_post && !r_post) || (w_post != nullptr) != (dw_post != nullptr)) return SL_ERR_INVALID_ARG;
    if ((dy != nullptr) != (w_pre != nullptr) || (dy != nullptr) != (r_pre != nullptr) || (dy != nullptr) != (dw_pre != nullptr))
      return SL_ERR_INVALID_ARG;
    if ((dw_post || dw_pre) && !ws) return SL_ERR_INVALID_ARG;
  }
  if (!typed_aligned(dh, res_type) || !typed_aligned(h, res_type) || !typed_aligned(dx, res_type) || !typed_aligned(dy, act_type) ||
      !typed_aligned(b, act_type) || !typed_aligned(g, act_type) || !typed_aligned(db, act_type) || !typed_aligned(dg, act_type) ||
      !typed_aligned(w_post, w_type) || !typed_aligned(w_pre, w_type) || !typed_aligned(dw_post, w_type) ||
      !typed_aligned(dw_pre, w_type) || !is_aligned(r_post, 4) || !is_aligned(r_pre, 4) || !is_aligned(ws, 16) || !is_aligned(flags, 4))
    return SL_ERR_ALIGNMENT;
  if (n > 0x7FFFFFFFull || d > SL_MAX_WIDTH) return SL_ERR_UNSUPPORTED;
  if (n == 0 && acc) return SL_OK;
  NormGradArgs a{dh, dy, h, b, g, w_post, w_pre, r_post, r_pre, dx, db, dg, dw_post, dw_pre, static_cast<float*>(ws), b ? ldb : 0,
                 g ? ldg : 0, (uint32_t)n, d, alpha, w_type == SL_BF16, acc ? 1 : 0, flags, debug_wait_polls()};
  return status(launch_norm_block_grad(a, res_type, act_type, (cudaStream_t)stream));
}

}  // extern "C"
