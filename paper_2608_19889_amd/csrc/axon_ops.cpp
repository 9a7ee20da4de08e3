// C ABI of the row operators on a caller's tensors: layer norm forward and
// backward, log-probabilities of tokens and the losses over them.  Argument checks
// only; the kernels are in k_layernorm.hip and k_loss.hip.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kernels.h"
#include "op_checks.h"

using namespace axon;

namespace {

int check_ln(int64_t rows, int32_t cols, float eps) {
  if (rows < 0 || rows > (int64_t)1 << 40) return fail(AXON_E_INVALID, "rows must be in [0, 2^40], got " + num(rows));
  if (cols < 1 || cols > LN_MAX_COLS)
    return fail(AXON_E_INVALID, "cols must be in [1, " + num(LN_MAX_COLS) + "], got " + num(cols));
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(AXON_E_INVALID, "eps must be finite and > 0");
  return AXON_OK;
}

// f(x type, y type, parameter type) as pointers of those types
template <typename F>
void by_types(int32_t x, int32_t y, int32_t p, F&& f) {
  auto third = [&](auto* a, auto* b) {
    if (p == AXON_BF16) f(a, b, (bf16*)nullptr);
    else f(a, b, (float*)nullptr);
  };
  auto second = [&](auto* a) {
    if (y == AXON_BF16) third(a, (bf16*)nullptr);
    else third(a, (float*)nullptr);
  };
  if (x == AXON_BF16) second((bf16*)nullptr);
  else second((float*)nullptr);
}

int check_logits(int64_t tokens, int32_t vocab, const void* logits, int32_t dtype, int64_t ld, const int32_t* targets) {
  if (tokens < 0 || tokens > MAX_TOKENS) return fail(AXON_E_INVALID, "tokens must be in [0, 2^30], got " + num(tokens));
  if (vocab < 1 || vocab > MAX_TOKENS) return fail(AXON_E_INVALID, "vocab must be in [1, 2^30], got " + num(vocab));
  if (int r = check_rows("logits", logits, dtype, ld, tokens, vocab)) return r;
  return tokens > 0 ? check_array("d_targets", targets, 4) : AXON_OK;
}

// the gradient's rows: none, the logits' own, or another buffer
int check_grad(const void* dz, int32_t dtype, int64_t ld, int64_t tokens, int32_t vocab, const void* z, int32_t z_dtype,
               int64_t z_ld) {
  if (int r = check_rows("dlogits", dz, dtype, ld, tokens, vocab)) return r;
  if (dz == z && (dtype != z_dtype || ld != z_ld))
    return fail(AXON_E_INVALID, "dlogits in the logits' buffer needs their dtype and row stride");
  return AXON_OK;
}

LogitRows rows_of(const void* z, int32_t dtype, int64_t ld, int64_t tokens, int32_t vocab, const int32_t* targets,
                  void* dz, int32_t dz_dtype, int64_t lddz) {
  return LogitRows{z, dtype == AXON_BF16, ld, tokens, vocab, targets, dz, dz_dtype == AXON_BF16, lddz};
}

}  // namespace

extern "C" int axon_layernorm(int64_t rows, int32_t cols, const void* x, int32_t x_dtype, int64_t ldx, const void* gain,
                              const void* bias, int32_t param_dtype, float eps, void* y, int32_t y_dtype, int64_t ldy,
                              void* stream) {
  return entry([&]() -> int {
    if (int r = check_ln(rows, cols, eps)) return r;
    if (int r = check_rows("x", x, x_dtype, ldx, rows, cols)) return r;
    if (int r = check_rows("y", y, y_dtype, ldy, rows, cols)) return r;
    if (int r = check_type("gain and bias", param_dtype)) return r;
    if (int r = check_array("gain", gain, size_of(param_dtype))) return r;
    if (bias)
      if (int r = check_array("bias", bias, size_of(param_dtype))) return r;
    if (x == y && (x_dtype != y_dtype || ldx != ldy))
      return fail(AXON_E_INVALID, "y in x's buffer needs its dtype and row stride");
    by_types(x_dtype, y_dtype, param_dtype, [&](auto* tx, auto* ty, auto* tp) {
      launch_ln_fwd((decltype(tx))x, ldx, (const std::remove_pointer_t<decltype(tp)>*)gain,
                    (const std::remove_pointer_t<decltype(tp)>*)bias, eps, (decltype(ty))y, ldy, rows, cols,
                    (hipStream_t)stream);
    });
    return check_launch("layer norm");
  });
}

extern "C" int64_t axon_layernorm_backward_workspace(int64_t rows, int32_t cols) {
  if (rows <= 0 || cols < 1 || cols > LN_MAX_COLS) return 0;
  return ln_bwd_part_floats(rows, cols) * 4;
}

extern "C" int axon_layernorm_backward(int64_t rows, int32_t cols, const void* x, int32_t x_dtype, int64_t ldx,
                                       const void* dy, int32_t dy_dtype, int64_t lddy, const void* gain,
                                       int32_t param_dtype, float eps, void* dx, int64_t lddx, float* dgain,
                                       float* dbias, void* workspace, int64_t workspace_bytes, void* stream) {
  return entry([&]() -> int {
    if (int r = check_ln(rows, cols, eps)) return r;
    if (int r = check_rows("x", x, x_dtype, ldx, rows, cols)) return r;
    if (int r = check_rows("dy", dy, dy_dtype, lddy, rows, cols)) return r;
    if (int r = check_rows("dx", dx, x_dtype, lddx, rows, cols)) return r;
    if (int r = check_type("gain", param_dtype)) return r;
    if (int r = check_array("gain", gain, size_of(param_dtype))) return r;
    if (int r = check_array("dgain", dgain, 4)) return r;
    if (dbias)
      if (int r = check_array("dbias", dbias, 4)) return r;
    if ((dx == x && lddx != ldx) || (dx == dy && (lddx != lddy || x_dtype != dy_dtype)))
      return fail(AXON_E_INVALID, "dx in the buffer of x or dy needs its dtype and row stride");
    if (int r = check_workspace(workspace, workspace_bytes, axon_layernorm_backward_workspace(rows, cols))) return r;
    by_types(x_dtype, dy_dtype, param_dtype, [&](auto* tx, auto* td, auto* tp) {
      launch_ln_bwd((const std::remove_pointer_t<decltype(tx)>*)x, ldx, (const std::remove_pointer_t<decltype(td)>*)dy,
                    lddy, (const std::remove_pointer_t<decltype(tp)>*)gain, eps, (decltype(tx))dx, lddx, dgain, dbias,
                    (float*)workspace, rows, cols, (hipStream_t)stream);
    });
    return check_launch("layer norm backward");
  });
}

extern "C" int64_t axon_token_loss_workspace(int64_t tokens, int32_t vocab, int32_t seqs) {
  if (tokens < 0 || tokens > MAX_TOKENS || vocab < 1 || vocab > MAX_TOKENS || seqs < 0) return 0;
  return (int64_t)loss_workspace_bytes(tokens, vocab, seqs);
}

extern "C" int axon_token_logprobs(int64_t tokens, int32_t vocab, const void* logits, int32_t dtype, int64_t ld,
                                   const int32_t* d_targets, float* d_logps, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
  return entry([&]() -> int {
    if (int r = check_logits(tokens, vocab, logits, dtype, ld, d_targets)) return r;
    if (tokens == 0) return AXON_OK;
    if (int r = check_array("d_logps", d_logps, 4)) return r;
    if (int r = check_workspace(workspace, workspace_bytes, axon_token_loss_workspace(tokens, vocab, 0))) return r;
    launch_token_logps(rows_of(logits, dtype, ld, tokens, vocab, d_targets, nullptr, 0, 0), d_logps, workspace,
                       (hipStream_t)stream);
    return check_launch("token log-probabilities");
  });
}

extern "C" int axon_token_logprobs_backward(int64_t tokens, int32_t vocab, const void* logits, int32_t dtype,
                                            int64_t ld, const int32_t* d_targets, const float* d_dlogps, void* dlogits,
                                            int32_t grad_dtype, int64_t ldg, void* stream) {
  return entry([&]() -> int {
    if (int r = check_logits(tokens, vocab, logits, dtype, ld, d_targets)) return r;
    if (int r = check_grad(dlogits, grad_dtype, ldg, tokens, vocab, logits, dtype, ld)) return r;
    if (tokens == 0) return AXON_OK;
    if (int r = check_array("d_dlogps", d_dlogps, 4)) return r;
    launch_token_logps_bwd(rows_of(logits, dtype, ld, tokens, vocab, d_targets, dlogits, grad_dtype, ldg), d_dlogps,
                           (hipStream_t)stream);
    return check_launch("token log-probabilities backward");
  });
}

namespace axon {

int check_preference(int32_t pairs, float beta, float label_smoothing) {
  if (pairs < 1 || pairs > 1 << 29) return fail(AXON_E_INVALID, "pairs must be >= 1, got " + num(pairs));
  if (!(beta > 0.f) || !std::isfinite(beta)) return fail(AXON_E_INVALID, "beta must be finite and > 0");
  if (!(label_smoothing >= 0.f && label_smoothing < 0.5f))
    return fail(AXON_E_INVALID, "label_smoothing must be in [0, 0.5)");
  return AXON_OK;
}

int check_policy(float clip_low, float clip_high, float kl_coef, int32_t per_sequence) {
  if (!(clip_low >= 0.f && clip_low <= 1.f)) return fail(AXON_E_INVALID, "clip_low must be in [0, 1]");
  if (!(clip_high >= 0.f) || !std::isfinite(clip_high)) return fail(AXON_E_INVALID, "clip_high must be finite and >= 0");
  if (!(kl_coef >= 0.f) || !std::isfinite(kl_coef)) return fail(AXON_E_INVALID, "kl_coef must be finite and >= 0");
  if (per_sequence != 0 && per_sequence != 1) return fail(AXON_E_INVALID, "per_sequence must be 0 or 1");
  return AXON_OK;
}

}  // namespace axon

extern "C" int axon_preference_loss(int64_t tokens, int32_t vocab, const void* logits, int32_t dtype, int64_t ld,
                                    const int32_t* d_targets, int32_t pairs, const int32_t* d_cu_seqlens,
                                    const int32_t* h_cu_seqlens, const float* d_ref_logps, float beta,
                                    float label_smoothing, float* d_loss, float* d_seq_logps, float* d_margins,
                                    void* dlogits, int32_t grad_dtype, int64_t ldg, void* workspace,
                                    int64_t workspace_bytes, void* stream) {
  return entry([&]() -> int {
    if (int r = check_logits(tokens, vocab, logits, dtype, ld, d_targets)) return r;
    if (int r = check_preference(pairs, beta, label_smoothing)) return r;
    if (int r = check_cu(d_cu_seqlens, h_cu_seqlens, 2 * pairs, tokens)) return r;
    if (dlogits)
      if (int r = check_grad(dlogits, grad_dtype, ldg, tokens, vocab, logits, dtype, ld)) return r;
    if (d_ref_logps)
      if (int r = check_array("d_ref_logps", d_ref_logps, 4)) return r;
    if (int r = check_array("d_loss", d_loss, 4)) return r;
    if (int r = check_array("d_seq_logps", d_seq_logps, 4)) return r;
    if (int r = check_array("d_margins", d_margins, 4)) return r;
    if (int r = check_workspace(workspace, workspace_bytes, axon_token_loss_workspace(tokens, vocab, 2 * pairs)))
      return r;
    launch_preference_loss(rows_of(logits, dtype, ld, tokens, vocab, d_targets, dlogits, grad_dtype, ldg),
                           PreferenceArgs{d_cu_seqlens, 2 * pairs, d_ref_logps, beta, label_smoothing, d_loss,
                                          d_seq_logps, d_margins},
                           workspace, (hipStream_t)stream);
    return check_launch("preference loss");
  });
}

extern "C" int axon_policy_loss(int64_t tokens, int32_t vocab, const void* logits, int32_t dtype, int64_t ld,
                                const int32_t* d_targets, int32_t batch, const int32_t* d_cu_seqlens,
                                const int32_t* h_cu_seqlens, const float* d_old_logps, const float* d_ref_logps,
                                const float* d_advantages, float clip_low, float clip_high, float kl_coef,
                                int32_t per_sequence, float* d_loss, float* d_stats, float* d_logps, void* dlogits,
                                int32_t grad_dtype, int64_t ldg, void* workspace, int64_t workspace_bytes,
                                void* stream) {
  return entry([&]() -> int {
    if (int r = check_logits(tokens, vocab, logits, dtype, ld, d_targets)) return r;
    if (int r = check_policy(clip_low, clip_high, kl_coef, per_sequence)) return r;
    if (batch < 1) return fail(AXON_E_INVALID, "batch must be >= 1, got " + num(batch));
    if (int r = check_cu(d_cu_seqlens, h_cu_seqlens, batch, tokens)) return r;
    if (dlogits)
      if (int r = check_grad(dlogits, grad_dtype, ldg, tokens, vocab, logits, dtype, ld)) return r;
    if (tokens > 0) {
      if (int r = check_array("d_old_logps", d_old_logps, 4)) return r;
      if (int r = check_array("d_advantages", d_advantages, 4)) return r;
      if (int r = check_array("d_logps", d_logps, 4)) return r;
    }
    if (d_ref_logps)
      if (int r = check_array("d_ref_logps", d_ref_logps, 4)) return r;
    if (kl_coef > 0.f && !d_ref_logps) return fail(AXON_E_INVALID, "kl_coef > 0 needs d_ref_logps");
    if (int r = check_array("d_loss", d_loss, 4)) return r;
    if (int r = check_array("d_stats", d_stats, 4)) return r;
    if (int r = check_workspace(workspace, workspace_bytes, axon_token_loss_workspace(tokens, vocab, batch))) return r;
    launch_policy_loss(rows_of(logits, dtype, ld, tokens, vocab, d_targets, dlogits, grad_dtype, ldg),
                       PolicyArgs{per_sequence ? d_cu_seqlens : nullptr, batch, d_old_logps, d_ref_logps, d_advantages,
                                  clip_low, clip_high, kl_coef, d_loss, d_stats, d_logps},
                       workspace, (hipStream_t)stream);
    return check_launch("policy loss");
  });
}
