// Internal launch interface and host-side checks of the tim_policy.h entry
// points. The checks are pure C++, so every error path runs without a GPU.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "tim_policy.h"
#include "validate.h"

namespace tim {

inline bool valid_dtype(int32_t t) { return t == TIM_F32 || t == TIM_BF16 || t == TIM_F16; }
inline int dtype_bytes(int32_t t) { return t == TIM_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % (unsigned)n == 0; }
inline int rule_chunks_of(int32_t V) { return (V + TIM_RULE_CHUNK - 1) / TIM_RULE_CHUNK; }

inline tim_status validate_mxfp4_quantize(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld,
                                          const uint8_t* codes, const uint8_t* scales) {
  if (rows < 0 || d <= 0 || d % TIM_MXFP4_BLOCK != 0 || ld < d) return TIM_ERR_SHAPE;
  if (!valid_dtype(dtype)) return TIM_ERR_VALUE;
  if (rows == 0) return TIM_OK;
  if (!x || !codes || !scales) return TIM_ERR_NULL;
  if (!aligned_to(x, dtype_bytes(dtype))) return TIM_ERR_VALUE;
  return TIM_OK;
}

inline tim_status validate_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d,
                                            const void* out, int32_t dtype) {
  if (rows < 0 || d <= 0 || d % TIM_MXFP4_BLOCK != 0) return TIM_ERR_SHAPE;
  if (dtype != TIM_F32 && dtype != TIM_BF16) return TIM_ERR_VALUE;
  if (rows == 0) return TIM_OK;
  if (!codes || !scales || !out) return TIM_ERR_NULL;
  if (!aligned_to(out, dtype_bytes(dtype))) return TIM_ERR_VALUE;
  return TIM_OK;
}

inline tim_status validate_mxfp4_logits(const uint8_t* h_codes, const uint8_t* h_scales, const uint8_t* w_codes,
                                        const uint8_t* w_scales, int64_t T, int32_t d, int32_t V, float temperature,
                                        const void* logits, int32_t dtype, int64_t ld) {
  if (T < 0) return TIM_ERR_SHAPE;
  if (T == 0) return TIM_OK;
  if (!h_codes || !h_scales || !w_codes || !w_scales || !logits) return TIM_ERR_NULL;
  const tim_status s = check_shape(T, d, V, TIM_ORDER_INVARIANT);
  if (s != TIM_OK) return s;
  if (d > TIM_MXFP4_MAX_D || ld < V) return TIM_ERR_SHAPE;
  if (!positive_finite(temperature) || !valid_dtype(dtype)) return TIM_ERR_VALUE;
  if (!aligned16(h_codes) || !aligned16(w_codes) || !aligned_to(h_scales, 4) || !aligned_to(w_scales, 4) ||
      !aligned_to(logits, dtype_bytes(dtype)))
    return TIM_ERR_VALUE;
  return TIM_OK;
}

inline tim_status validate_rules(const tim_logit_rules* r, int32_t V) {
  if (!r) return TIM_OK;
  if (r->history) {
    if (r->history_len < 0) return TIM_ERR_SHAPE;
    if (!r->hist_begin || !r->hist_end) return TIM_ERR_NULL;
    if (!aligned_to(r->history, 4)) return TIM_ERR_VALUE;
  }
  if (r->bias_ids) {
    if (r->bias_len < 0 || r->bias_len > INT32_MAX - 1) return TIM_ERR_SHAPE;
    if (!r->bias_values || !r->bias_begin || !r->bias_end) return TIM_ERR_NULL;
  }
  if (r->mask) {
    if (r->n_masks < 0 || r->mask_ld < ((int64_t)V + 31) / 32) return TIM_ERR_SHAPE;
    if (!aligned_to(r->mask, 4)) return TIM_ERR_VALUE;
  }
  return TIM_OK;
}

// The logits argument of the three operators on changed logits, and their rules.
inline tim_status validate_changed(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                   const tim_logit_rules* rules, float temperature) {
  if (!logits) return TIM_ERR_NULL;
  if (V < 1 || V > TIM_MAX_VOCAB || ld < V) return TIM_ERR_SHAPE;
  if (!positive_finite(temperature) || !valid_dtype(dtype)) return TIM_ERR_VALUE;
  if (!aligned_to(logits, dtype_bytes(dtype))) return TIM_ERR_VALUE;
  return validate_rules(rules, V);
}

inline tim_status validate_logits_adjust(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                         const tim_logit_rules* rules, float temperature, const void* out,
                                         int64_t out_ld) {
  if (T < 0) return TIM_ERR_SHAPE;
  if (T == 0) return TIM_OK;
  if (!out) return TIM_ERR_NULL;
  const tim_status s = validate_changed(logits, dtype, T, V, ld, rules, temperature);
  if (s != TIM_OK) return s;
  if (out_ld < V || (out == logits && out_ld != ld)) return TIM_ERR_SHAPE;
  return aligned_to(out, dtype_bytes(dtype)) ? TIM_OK : TIM_ERR_VALUE;
}

inline size_t logits_logprobs_workspace(int64_t T, int32_t V) { return (size_t)T * (size_t)rule_chunks_of(V) * 16u; }

inline tim_status validate_logits_logprobs(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                           const int32_t* tokens, const tim_logit_rules* rules, float temperature,
                                           const float* logp, const void* ws, size_t ws_bytes) {
  if (T < 0) return TIM_ERR_SHAPE;
  if (T == 0) return TIM_OK;
  if (!tokens || !logp) return TIM_ERR_NULL;
  const tim_status s = validate_changed(logits, dtype, T, V, ld, rules, temperature);
  if (s != TIM_OK) return s;
  if (!ws || !aligned16(ws) || ws_bytes < logits_logprobs_workspace(T, V)) return TIM_ERR_WORKSPACE;
  return TIM_OK;
}

inline tim_status validate_logits_logprobs_backward(const void* logits, int32_t dtype, int64_t T, int32_t V,
                                                    int64_t ld, const int32_t* tokens, const tim_logit_rules* rules,
                                                    float temperature, const float* lse, const float* entropy,
                                                    const float* grad_logp, const float* grad_entropy,
                                                    const void* grad, int32_t grad_dtype, int64_t grad_ld) {
  if (T < 0) return TIM_ERR_SHAPE;
  if (T == 0) return TIM_OK;
  if (!tokens || !lse || !grad_logp || !grad || (grad_entropy && !entropy)) return TIM_ERR_NULL;
  const tim_status s = validate_changed(logits, dtype, T, V, ld, rules, temperature);
  if (s != TIM_OK) return s;
  if (!valid_dtype(grad_dtype) || !aligned_to(grad, dtype_bytes(grad_dtype))) return TIM_ERR_VALUE;
  if (grad_ld < V) return TIM_ERR_SHAPE;
  if (grad == logits && (grad_ld != ld || grad_dtype != dtype)) return TIM_ERR_SHAPE;
  return TIM_OK;
}

// Arguments of the three operators on changed logits, rules resolved: a
// missing history or bias list has its pointer NULL here too.
struct RuleArgs {
  const void* logits;
  int64_t T, ld;
  int32_t V;
  float inv_tau;
  tim_logit_rules r;
  const int32_t* tokens;  // logprobs, backward
  void* part;             // logprobs: Partial [T, chunks]
  void* out;              // adjust, backward: [T, out_ld]
  int64_t out_ld;
  const float *lse, *entropy, *grad_logp, *grad_entropy;  // backward
  int32_t past_caches;    // out is larger than the caches
};

// An fp32 value rounded once to T. To fp16 the compiler would merge a multiply
// before it into one mixed-precision instruction that rounds the exact product
// to fp16, other bits than the fp32 product's; the empty asm keeps the two
// apart.
template <class T>
__device__ __forceinline__ T narrow(float x) {
  return (T)x;
}
template <>
__device__ __forceinline__ _Float16 narrow<_Float16>(float x) {
  asm volatile("" : "+v"(x));
  return (_Float16)x;
}

hipError_t launch_mxfp4_quantize(const void* x, int dtype, int64_t rows, int d, int64_t ld, uint8_t* codes,
                                 uint8_t* scales, hipStream_t s);
hipError_t launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* out,
                                   int dtype, hipStream_t s);

struct Mxfp4LogitsArgs {
  const uint8_t *h_codes, *h_scales, *w_codes, *w_scales;
  int64_t T;
  int32_t d, V;
  float inv_tau;
  void* logits;
  int64_t ld;
};
hipError_t launch_mxfp4_logits(const Mxfp4LogitsArgs& a, int dtype, hipStream_t s);

hipError_t launch_logits_adjust(const RuleArgs& a, int dtype, hipStream_t s);
// Per-chunk partials into a.part, then their merge in chunk order.
hipError_t launch_logits_logprobs(const RuleArgs& a, int dtype, float* logp, float* entropy, float* lse,
                                  hipStream_t s);
hipError_t launch_logits_logprobs_backward(const RuleArgs& a, int dtype, int grad_dtype, hipStream_t s);

}  // namespace tim
