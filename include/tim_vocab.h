/*
 * tim_vocab.h -- what stands beside the LM head on AMD MI355X (gfx950): the
 * vocabulary's matrix at the model's other end (token embedding and its
 * gradient), and low-rank adapters of many requests beside a shared projection,
 * the head's among them, with their gradients.
 *
 * A tied model uses one matrix for both ends: the embedding's gradient is then
 * added to the grad_w of tim_logprobs_backward. An engine that serves several
 * policies as adapters of one model adds each row's own adapter to the logits
 * of tim_logits or tim_mxfp4_logits before it scores them (tim_policy.h); the
 * trainer takes the adapters' gradients from the gradient of those logits
 * (tim_logits_logprobs_backward).
 *
 * Conventions as in tim.h and tim_policy.h: array arguments are device pointers
 * owned by the caller, nothing is allocated or kept, every kernel is enqueued on
 * `stream`, argument errors are found on the host before anything is enqueued,
 * and a row count of 0 enqueues nothing but zeros of the gradients that are not
 * accumulated. Tokens and adapter indices are only read on the device; values
 * out of range mean "none" as stated, never an access outside the arrays. No
 * result depends on the order in which threads run. A row's outputs are bitwise
 * independent of the other rows, of T and of the row's position.
 */
#ifndef TIM_VOCAB_H
#define TIM_VOCAB_H

#include "tim_policy.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest T of the calls that group rows by token or adapter. */
#define TIM_MAX_GROUPED_ROWS (1 << 23)
/* Largest width of an embedding or a projection. */
#define TIM_MAX_WIDTH (1 << 20)
/* Largest rank of an adapter. */
#define TIM_MAX_RANK 256

/* -------------------------------------------------------------- embedding */

/* out[t, :] = scale * table[tokens[t], :], formed in fp32 and rounded once to
 * out_dtype; a row of zeros for a token outside [0, V) (padding).
 *
 * table   dtype [V, d], row v at table + v * ld elements, ld >= d; V in
 *         [1, TIM_MAX_VOCAB], d in [1, TIM_MAX_WIDTH].
 * tokens  int32 [T].
 * out     out_dtype [T, d], row stride out_ld >= d elements, no overlap with
 *         the inputs.
 * scale   any finite fp32 value.
 * Errors: TIM_ERR_SHAPE (T < 0, V, d, strides), TIM_ERR_VALUE (dtypes, scale,
 * alignment to the element, overlap), TIM_ERR_NULL. */
tim_status tim_embedding(const void* table, int32_t dtype, int32_t V, int32_t d, int64_t ld, const int32_t* tokens,
                         int64_t T, float scale, void* out, int32_t out_dtype, int64_t out_ld, hipStream_t stream);

/* Gradient of the table from the gradients of its looked-up rows:
 *   grad_table[v, :] (+)= scale * sum_{t: tokens[t] = v} grad_out[t, :]
 * in fp32. A token's rows are summed in runs of TIM_EMBED_RUN by ascending t,
 * one chain each, and the runs' sums by a chain over the runs, so its bits
 * depend on its own rows only. Tokens outside [0, V) add nothing.
 *
 * grad_out    dtype [T, d], row stride ld >= d elements; T at most
 *             TIM_MAX_GROUPED_ROWS.
 * grad_table  fp32 [V, d], row stride grad_ld >= d elements. With accumulate =
 *             1 the sums are added to the rows of the tokens that occur and no
 *             other row is touched; with 0 every row is written, zeros where a
 *             token does not occur (elements d .. grad_ld - 1 stay untouched).
 *             No overlap with the inputs.
 * workspace   tim_embedding_backward_workspace_size(T, V, d) bytes, 16-byte
 *             aligned; 0 for invalid arguments or T == 0.
 * Errors as tim_embedding; TIM_ERR_VALUE also for accumulate not 0 or 1;
 * TIM_ERR_WORKSPACE. T == 0 writes zeros unless accumulating. */
#define TIM_EMBED_RUN 64
size_t tim_embedding_backward_workspace_size(int64_t T, int32_t V, int32_t d);
tim_status tim_embedding_backward(const void* grad_out, int32_t dtype, int64_t T, int32_t d, int64_t ld,
                                  const int32_t* tokens, int32_t V, float scale, float* grad_table, int64_t grad_ld,
                                  int32_t accumulate, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------- adapters
 *
 * n adapters of rank r (r in [1, TIM_MAX_RANK]; one of a lower rank has rows or
 * columns of zeros) of a projection from d to N elements (both in
 * [1, TIM_MAX_WIDTH]):
 *   a       dtype [n, r, d], contiguous
 *   b       dtype [n, N, r], contiguous
 *   scales  fp32 [n] (alpha / r, say), NULL for ones
 * dtype is TIM_BF16 or TIM_F16, the same for a, b and the rows x. rows is int32
 * [T]: the adapter of each row; outside [0, n) the row has none. */
typedef struct {
  const void* a;
  const void* b;
  const float* scales;
  int32_t dtype;
  int32_t n; /* in [1, TIM_MAX_VOCAB] */
  int32_t r;
  int32_t d;
  int32_t N;
} tim_adapters;

/* out[t, :] = base[t, :] + scales[k] (x[t, :] a_k^T) b_k^T,   k = rows[t]
 * (base[t, :] itself where the row has no adapter).
 *
 * x       dtype of the adapters [T, d], row stride x_ld >= d elements; T at
 *         most TIM_MAX_GROUPED_ROWS.
 * base    out_dtype [T, N], row stride base_ld >= N elements; the shared
 *         projection's output (logits of tim_logits with their temperature of
 *         1, say). NULL: zeros.
 * out     out_dtype [T, N], row stride out_ld >= N; may be base itself with the
 *         same stride, and x may lie there, otherwise no overlap with the inputs.
 * Arithmetic: x a^T is accumulated in fp32 in an order that depends on d alone
 * and kept in fp32; its product with b^T is accumulated in fp32 over ascending
 * groups of 16 ranks (bf16 adapters: with the fp32 number as the sum of three bf16
 * ones, which hold its 24 bits; beyond bf16's largest number it becomes infinite).
 * One rounding of the sum with base to out_dtype. Infinities and NaN give what the
 * formula gives; those in a row or its adapter reach that row only.
 * workspace  tim_adapters_add_workspace_size(T, d, N, n, r) bytes, 16-byte
 *         aligned.
 * Errors: TIM_ERR_SHAPE (T, n, r, d, N, strides), TIM_ERR_VALUE (dtypes,
 * alignment to the element, overlap), TIM_ERR_NULL, TIM_ERR_WORKSPACE. */
size_t tim_adapters_add_workspace_size(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r);
tim_status tim_adapters_add(const tim_adapters* adapters, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                            const void* base, int64_t base_ld, void* out, int32_t out_dtype, int64_t out_ld,
                            void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Gradients of a loss L through tim_adapters_add, grad = dL/dout:
 *   u_t = scales[k] x_t a_k^T,   v_t = scales[k] grad_t b_k        k = rows[t]
 *   grad_x[t, :]   (+)= v_t a_k
 *   grad_a[k, j, :] (+)= sum_{t: rows[t] = k} v_tj x[t, :]          fp32 [n, r, d]
 *   grad_b[k, :, j] (+)= sum_{t: rows[t] = k} u_tj grad[t, :]       fp32 [n, N, r]
 * (the gradient of base is grad itself; scales are held fixed).
 *
 * x, rows  as given to tim_adapters_add.
 * grad     grad_dtype [T, N], row stride grad_ld >= N elements.
 * grad_x   gx_dtype [T, d], row stride gx_ld >= d; NULL: not computed. With
 *          accumulate_x = 1 it is added to (one rounding of the sum), else
 *          written, zeros for a row without an adapter.
 * grad_a, grad_b  contiguous; either may be NULL. With accumulate_ab = 1 both are
 *          added to, else written, zeros for an adapter without rows.
 * The gradients written overlap neither each other nor an input, but grad_x may lie
 * over grad (over x it may not: in the same buffer's columns beside it).
 * workspace  tim_adapters_backward_workspace_size(T, d, N, n, r) bytes, 16-byte
 *          aligned.
 * Arithmetic: u and v are accumulated and kept in fp32 (in products with bf16 as
 * in tim_adapters_add); grad_a and grad_b are fp32 chains over runs of an adapter's
 * rows by ascending t, of 128, 256 or 512 rows as T, n, the width, r and the types
 * say, the runs' sums joined by a chain; no atomics on them. A row's grad_x is
 * bitwise independent of the other rows, of T and of n; for given T and n an
 * adapter's grad_a and grad_b are bitwise independent of the other adapters and
 * their rows. Errors as tim_adapters_add; TIM_ERR_VALUE also for accumulate_x or
 * accumulate_ab not 0 or 1. T == 0 writes zeros to grad_a and grad_b unless
 * accumulating. */
size_t tim_adapters_backward_workspace_size(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r);
tim_status tim_adapters_backward(const tim_adapters* adapters, const void* x, int64_t x_ld, const int32_t* rows,
                                 int64_t T, const void* grad, int32_t grad_dtype, int64_t grad_ld, void* grad_x,
                                 int32_t gx_dtype, int64_t gx_ld, int32_t accumulate_x, float* grad_a, float* grad_b,
                                 int32_t accumulate_ab, void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* TIM_VOCAB_H */
