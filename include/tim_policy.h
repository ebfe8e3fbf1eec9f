/*
 * tim_policy.h -- the distribution a rollout engine samples from, on AMD
 * MI355X (gfx950): logits of an LM head held in 4-bit microscaled floating
 * point, logits changed by penalties, biases and grammar masks, and the
 * log-probabilities of sampled tokens under the changed logits with their
 * gradient.
 *
 * tim.h scores tokens under softmax(h W^T / temperature). A rollout engine
 * whose head is quantised, or that samples from changed logits, draws from
 * another distribution; the trainer's log pi (Section 2, Eq. 1) has to be
 * taken under that same one, or the two differ before any rounding does.
 *
 * Conventions as in tim.h: array arguments are device pointers owned by the
 * caller, nothing is allocated or kept, every kernel is enqueued on `stream`,
 * argument errors are found on the host before anything is enqueued, and a row
 * count of 0 is a successful no-op. Device arrays of indices are only read on
 * the device: values out of range are clamped or ignored as stated, never
 * followed outside their arrays. A row's outputs are bitwise independent of
 * the other rows, of T and of the row's position.
 */
#ifndef TIM_POLICY_H
#define TIM_POLICY_H

#include "tim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of a matrix argument (passed as int32_t). */
typedef enum {
  TIM_F32 = 0,
  TIM_BF16 = 1,
  TIM_F16 = 2
} tim_dtype;

/* ------------------------------------------------------ 4-bit microscaling
 *
 * MXFP4 (the OCP microscaling formats): a row is cut into blocks of 32
 * elements along d; element k of a block stands for c_k * 2^(s - 127) with one
 * scale byte s per block (E8M0; 255 = NaN) and 4-bit codes c_k (E2M1: 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 and their negatives, the sign in bit 3).
 *   codes  uint8 [rows, d / 2] row-major, element 2j in the low half of byte j
 *   scales uint8 [rows, d / 32] row-major
 */
#define TIM_MXFP4_BLOCK 32
/* Largest d of tim_mxfp4_logits. */
#define TIM_MXFP4_MAX_D (1 << 20)

/* Quantises rows of d elements (d a positive multiple of 32). Per block, with
 * top = max |x|:
 *   E      = max(floor(log2 top) - 2, -127)    (-127 for a block of zeros)
 *   scale  = E + 127
 *   c_k    = x_k / 2^E to the nearest E2M1 value, ties to the even code,
 *            magnitudes above 6 to 6; the sign is kept, of zeros too
 * A block that holds a NaN or an infinity gets scale 255 and stands for NaN.
 *
 * x       dtype [rows, d], row r at x + r * ld elements, ld >= d; aligned to
 *         its element.
 * codes, scales  outputs, any alignment.
 * Errors: TIM_ERR_SHAPE for rows < 0, a bad d, ld < d; TIM_ERR_VALUE for an
 * unknown dtype or a misaligned x; TIM_ERR_NULL for a NULL pointer. */
tim_status tim_mxfp4_quantize(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld,
                              uint8_t* codes, uint8_t* scales, hipStream_t stream);

/* The values the codes stand for, dtype TIM_BF16 or TIM_F32 [rows, d]
 * row-major; exact in both (TIM_F16 cannot hold them and is TIM_ERR_VALUE),
 * values past the type's range infinite. Errors as tim_mxfp4_quantize. */
tim_status tim_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d,
                                void* out, int32_t dtype, hipStream_t stream);

/* Logits of a quantised head, as tim_logits forms them for a bf16 one:
 *   logits[t, v] = (sum_k h[t, k] w[v, k]) * (float)(1 / temperature)
 * for MXFP4 h [T, d] and w [V, d] (d a positive multiple of 128, at most
 * TIM_MXFP4_MAX_D), written as dtype [T, V], row t at logits + t * ld elements, ld >= V.
 *
 * Arithmetic: the products of 4-bit codes with their scales on the matrix
 * cores, accumulated in fp32 with one chain per logit in an order that depends
 * on d alone; one rounding to dtype after the temperature. A block of scale
 * 255 makes the logits it enters NaN. Codes 16-byte and scales 4-byte aligned,
 * logits aligned to their element. Errors: TIM_ERR_SHAPE (T < 0, d, V outside
 * [1, TIM_MAX_VOCAB], ld < V), TIM_ERR_VALUE (temperature not finite or <= 0,
 * unknown dtype, alignment), TIM_ERR_NULL. */
tim_status tim_mxfp4_logits(const uint8_t* h_codes, const uint8_t* h_scales, const uint8_t* w_codes,
                            const uint8_t* w_scales, int64_t T, int32_t d, int32_t V, float temperature,
                            void* logits, int32_t dtype, int64_t ld, hipStream_t stream);

/* ---------------------------------------------------------- changed logits
 *
 * Rules that change the logits of T rows before sampling. Row i, with token
 * history history[hist_begin[i] .. hist_end[i]) of which the part from
 * hist_split[i] on was generated (the output) and the part before it given
 * (the prompt), changes logit z of vocabulary entry v to
 *   x = z
 *   x = x > 0 ? x / repetition[i] : x * repetition[i]   if v is in the history
 *   x = x - frequency[i] * c                            c = count of v in the output
 *   x = x - presence[i]                                 if c > 0
 *   x = x + bias_values[k]                              k = last entry of the row's bias list with bias_ids[k] = v
 *   x = x * (float)(1 / temperature)
 *   x = -inf                                            if the row's mask has bit v clear
 * each step one fp32 operation. A masked entry is excluded whatever its logit
 * holds (NaN and infinities too).
 *
 * Engines differ in where the bias enters; this order, the bias on the logits
 * that the penalties leave, is the library's choice, and with a repetition
 * penalty the other one is another distribution. An engine that adds its biases
 * first is had by two calls: tim_logits_adjust with the bias list alone, at
 * temperature 1 and in fp32, and then any call of this section with the other
 * rules on its output. The gradient with respect to that output is the one with
 * respect to the logits.
 *
 * Histories may overlap and share a stream: decode rows point at their
 * requests' tokens, the rows of a packed training stream each at the tokens
 * before their own. Consecutive rows of the same begin and split whose end
 * grows share the work of counting.
 *
 * Every pointer may be NULL: no history (then the penalties are not applied),
 * no bias, no mask; of the penalties, NULL leaves its step out. Offsets are
 * clamped into their arrays and put in order (split to at least begin, end to
 * at least split); tokens and bias ids outside [0, V) are ignored. A token may
 * occur up to 2^31 - 1 times in a row's output. */
typedef struct {
  const int32_t* history;     /* [history_len] tokens */
  int64_t history_len;
  const int64_t* hist_begin;  /* [T], required with history */
  const int64_t* hist_split;  /* [T], NULL: no prompt (split = begin) */
  const int64_t* hist_end;    /* [T], required with history */
  const float* repetition;    /* [T], > 0 */
  const float* frequency;     /* [T] */
  const float* presence;      /* [T] */
  const int32_t* bias_ids;    /* [bias_len] */
  const float* bias_values;   /* [bias_len], required with bias_ids */
  int64_t bias_len;           /* at most 2^31 - 2 */
  const int64_t* bias_begin;  /* [T], required with bias_ids; lists may be shared */
  const int64_t* bias_end;    /* [T], required with bias_ids */
  const uint32_t* mask;       /* [n_masks] rows of mask_ld words; bit v % 32 of word v / 32 set: v is allowed */
  int64_t n_masks;
  int64_t mask_ld;            /* >= ceil(V / 32) words */
  const int32_t* mask_rows;   /* [T] mask of each row, outside [0, n_masks): none; NULL: row i takes mask i */
} tim_logit_rules;

/* Writes the changed logits (each rounded once to dtype): out and logits are
 * dtype [T, V] with row strides out_ld and ld >= V elements. out may be logits
 * itself with the same stride; otherwise the two must not overlap. rules NULL:
 * the temperature alone. Errors: TIM_ERR_SHAPE (T < 0, V outside
 * [1, TIM_MAX_VOCAB], strides, negative lengths, mask_ld), TIM_ERR_VALUE
 * (temperature, dtype, alignment to the element), TIM_ERR_NULL (a required
 * pointer). */
tim_status tim_logits_adjust(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                             const tim_logit_rules* rules, float temperature, void* out, int64_t out_ld,
                             hipStream_t stream);

/* Bytes of device workspace tim_logits_logprobs needs:
 * T * ceil(V / TIM_RULE_CHUNK) * 16; 0 for invalid arguments or T == 0. */
#define TIM_RULE_CHUNK 8192
size_t tim_logits_logprobs_workspace_size(int64_t T, int32_t V);

/* Log-probabilities, entropies and log-normalisers of T tokens under the
 * changed logits x: the quantities of tim_logprobs with x in the place of z.
 *   logp[i] = x_{tokens[i]} - lse[i], entropy[i] = -sum_v p_v log p_v,
 *   lse[i] = log sum_v exp(x_v),      p_v = exp(x_v - lse[i])
 * An entry at -inf (masked, or of a logit or bias of -inf) has p = 0 and adds
 * nothing to the entropy. Where nothing is left (every x is -inf) lse = -inf,
 * entropy = 0 and logp = -inf. A token outside [0, V) yields logp = NaN. NaN
 * or +inf in an entry that is not masked propagates to the row's outputs. lse is
 * infinite where its value lies past fp32's range (entries near the largest or
 * lowest number over a temperature below 1); logp and entropy are not touched.
 *
 * logits, dtype, ld, rules, temperature as tim_logits_adjust; tokens int32
 * [T]; logp fp32 [T] (required), entropy, lse fp32 [T] or NULL. x is not
 * rounded to dtype, and the temperature is applied to differences from the
 * row's maximum. Statistics are fp32 over chunks of TIM_RULE_CHUNK entries
 * merged in a fixed order. workspace 16-byte aligned; also TIM_ERR_WORKSPACE. */
tim_status tim_logits_logprobs(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                               const int32_t* tokens, const tim_logit_rules* rules, float temperature,
                               float* logp, float* entropy, float* lse, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/* Gradient with respect to the logits z of sum_i grad_logp[i] logp[i] +
 * grad_entropy[i] entropy[i], the changes included:
 *   grad[i, v] = slope_v (g ([v == tokens[i]] - p_v) - e p_v (log p_v + H))
 * with g = grad_logp[i] (0 for a token outside [0, V)), e = grad_entropy[i]
 * (or 0), H = entropy[i], p_v = exp(x_v - lse[i]), p_v log p_v = 0 where
 * p_v = 0, and slope_v = dx_v / dz_v: (float)(1 / temperature), times
 * 1 / repetition (z > 0) or repetition (z <= 0) for entries in the history, 0
 * for masked ones. A row with g = e = 0 (padding) and a row with nothing allowed
 * get zeros.
 *
 * p_v goes by lse where |lse| < 1024 and carries its error, relatively 2^-14 or
 * little more. Rows beyond, whose lse says too little of them (at fp32's lowest
 * number it holds no log V, and it may be infinite), have their maximum and sum
 * formed anew from the logits, in one workgroup each: right, but slower.
 *
 * lse, entropy  fp32 [T] from tim_logits_logprobs for the same inputs
 *         (entropy may be NULL when grad_entropy is).
 * grad    grad_dtype [T, V], row stride grad_ld >= V elements; may be logits
 *         itself with the same type and stride, otherwise no overlap.
 * Errors as tim_logits_adjust; TIM_ERR_NULL for a missing lse, grad_logp, or
 * entropy with grad_entropy. */
tim_status tim_logits_logprobs_backward(const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                        const int32_t* tokens, const tim_logit_rules* rules, float temperature,
                                        const float* lse, const float* entropy, const float* grad_logp,
                                        const float* grad_entropy, void* grad, int32_t grad_dtype, int64_t grad_ld,
                                        hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* TIM_POLICY_H */
