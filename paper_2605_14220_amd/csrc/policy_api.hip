// C-ABI entry points of tim_policy.h: argument checks and launches.

#include <hip/hip_runtime.h>

#include "policy.h"
#include "tim_policy.h"

namespace {

inline tim_status hip_status(hipError_t e) { return e == hipSuccess ? TIM_OK : TIM_ERR_HIP; }

tim::RuleArgs rule_args(const void* logits, int64_t T, int32_t V, int64_t ld, const tim_logit_rules* rules,
                        float temperature) {
  tim::RuleArgs a = {};
  a.logits = logits;
  a.T = T;
  a.ld = ld;
  a.V = V;
  a.inv_tau = (float)(1.0 / (double)temperature);
  if (rules) a.r = *rules;
  // without tokens to count, or penalties to apply, there is no history; an empty bias list or mask set is none
  if (a.r.history_len == 0 || (!a.r.repetition && !a.r.frequency && !a.r.presence)) a.r.history = nullptr;
  if (a.r.bias_len == 0) a.r.bias_ids = nullptr;
  if (a.r.n_masks == 0) a.r.mask = nullptr;
  return a;
}

}  // namespace

extern "C" {

tim_status tim_mxfp4_quantize(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld, uint8_t* codes,
                              uint8_t* scales, hipStream_t stream) {
  const tim_status st = tim::validate_mxfp4_quantize(x, dtype, rows, d, ld, codes, scales);
  if (st != TIM_OK || rows == 0) return st;
  return hip_status(tim::launch_mxfp4_quantize(x, dtype, rows, d, ld, codes, scales, stream));
}

tim_status tim_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d, void* out,
                                int32_t dtype, hipStream_t stream) {
  const tim_status st = tim::validate_mxfp4_dequantize(codes, scales, rows, d, out, dtype);
  if (st != TIM_OK || rows == 0) return st;
  return hip_status(tim::launch_mxfp4_dequantize(codes, scales, rows, d, out, dtype, stream));
}

tim_status tim_mxfp4_logits(const uint8_t* h_codes, const uint8_t* h_scales, const uint8_t* w_codes,
                            const uint8_t* w_scales, int64_t T, int32_t d, int32_t V, float temperature, void* logits,
                            int32_t dtype, int64_t ld, hipStream_t stream) {
  const tim_status st =
      tim::validate_mxfp4_logits(h_codes, h_scales, w_codes, w_scales, T, d, V, temperature, logits, dtype, ld);
  if (st != TIM_OK || T == 0) return st;
  const tim::Mxfp4LogitsArgs a = {h_codes, h_scales, w_codes, w_scales, T, d, V, (float)(1.0 / (double)temperature),
                                  logits, ld};
  return hip_status(tim::launch_mxfp4_logits(a, dtype, stream));
}

tim_status tim_logits_adjust(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                             const tim_logit_rules* rules, float temperature, void* out, int64_t out_ld,
                             hipStream_t stream) {
  const tim_status st = tim::validate_logits_adjust(logits, dtype, T, V, ld, rules, temperature, out, out_ld);
  if (st != TIM_OK || T == 0) return st;
  tim::RuleArgs a = rule_args(logits, T, V, ld, rules, temperature);
  a.out = out;
  a.out_ld = out_ld;
  return hip_status(tim::launch_logits_adjust(a, dtype, stream));
}

size_t tim_logits_logprobs_workspace_size(int64_t T, int32_t V) {
  return (T <= 0 || V < 1 || V > TIM_MAX_VOCAB) ? 0 : tim::logits_logprobs_workspace(T, V);
}

tim_status tim_logits_logprobs(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                               const int32_t* tokens, const tim_logit_rules* rules, float temperature, float* logp,
                               float* entropy, float* lse, void* workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  const tim_status st = tim::validate_logits_logprobs(logits, dtype, T, V, ld, tokens, rules, temperature, logp,
                                                      workspace, workspace_bytes);
  if (st != TIM_OK || T == 0) return st;
  tim::RuleArgs a = rule_args(logits, T, V, ld, rules, temperature);
  a.tokens = tokens;
  a.part = workspace;
  return hip_status(tim::launch_logits_logprobs(a, dtype, logp, entropy, lse, stream));
}

tim_status tim_logits_logprobs_backward(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                        const int32_t* tokens, const tim_logit_rules* rules, float temperature,
                                        const float* lse, const float* entropy, const float* grad_logp,
                                        const float* grad_entropy, void* grad, int32_t grad_dtype, int64_t grad_ld,
                                        hipStream_t stream) {
  const tim_status st =
      tim::validate_logits_logprobs_backward(logits, dtype, T, V, ld, tokens, rules, temperature, lse, entropy,
                                             grad_logp, grad_entropy, grad, grad_dtype, grad_ld);
  if (st != TIM_OK || T == 0) return st;
  tim::RuleArgs a = rule_args(logits, T, V, ld, rules, temperature);
  a.tokens = tokens;
  a.out = grad;
  a.out_ld = grad_ld;
  a.lse = lse;
  a.entropy = entropy;
  a.grad_logp = grad_logp;
  a.grad_entropy = grad_entropy;
  return hip_status(tim::launch_logits_logprobs_backward(a, dtype, grad_dtype, stream));
}

}  // extern "C"
