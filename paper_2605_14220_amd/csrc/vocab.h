// Internal launch interface and host-side checks of the tim_vocab.h entry
// points. The checks are pure C++, so every error path runs without a GPU.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "adapters_plan.h"
#include "grouping.h"
#include "overlap.h"
#include "policy.h"
#include "tim_vocab.h"

namespace tim {

inline bool valid_width(int64_t d) { return d >= 1 && d <= TIM_MAX_WIDTH; }
inline bool valid_keys(int64_t V) { return V >= 1 && V <= TIM_MAX_VOCAB; }
inline bool grouped_rows(int64_t T) { return T >= 0 && T <= TIM_MAX_GROUPED_ROWS; }
inline bool valid_flag(int32_t f) { return f == 0 || f == 1; }

inline tim_status validate_embedding(const void* table, int32_t dtype, int32_t V, int32_t d, int64_t ld,
                                     const int32_t* tokens, int64_t T, float scale, const void* out, int32_t out_dtype,
                                     int64_t out_ld) {
  if (T < 0 || !valid_keys(V) || !valid_width(d) || ld < d || out_ld < d) return TIM_ERR_SHAPE;
  if (!valid_dtype(dtype) || !valid_dtype(out_dtype) || !std::isfinite(scale)) return TIM_ERR_VALUE;
  if (T == 0) return TIM_OK;
  if (!table || !tokens || !out) return TIM_ERR_NULL;
  if (!aligned_to(table, dtype_bytes(dtype)) || !aligned_to(tokens, 4) || !aligned_to(out, dtype_bytes(out_dtype)))
    return TIM_ERR_VALUE;
  const Rows o = rows_of(out, T, d, out_ld, dtype_bytes(out_dtype));
  if (share_bytes(o, rows_of(table, V, d, ld, dtype_bytes(dtype))) || share_bytes(o, flat(tokens, T, 4)))
    return TIM_ERR_VALUE;
  return TIM_OK;
}

// The embedding gradient's workspace: the grouping, a byte per token that
// occurs, the partial sums of tokens with several runs.
constexpr int kLogEmbedRun = 6;
static_assert(TIM_EMBED_RUN == 1 << kLogEmbedRun, "the documented run");
struct EmbedPlan {
  Grouping g;
  size_t seen, part, bytes;
};
inline EmbedPlan plan_embedding_backward(int64_t T, int32_t V, int32_t d) {
  const int log_C[1] = {kLogEmbedRun};
  EmbedPlan p = {plan_grouping(T, V, 1, log_C), 0, 0, 0};
  size_t at = p.g.bytes;
  p.seen = at, at += group_align((size_t)V);
  p.part = at, at += T > TIM_EMBED_RUN ? group_align((size_t)run_slots(T, kLogEmbedRun) * d * 4) : 0;
  p.bytes = at;
  return p;
}

inline tim_status validate_embedding_backward(const void* grad_out, int32_t dtype, int64_t T, int32_t d, int64_t ld,
                                              const int32_t* tokens, int32_t V, float scale, const float* grad_table,
                                              int64_t grad_ld, int32_t accumulate, const void* ws, size_t ws_bytes) {
  if (!grouped_rows(T) || !valid_keys(V) || !valid_width(d) || ld < d || grad_ld < d) return TIM_ERR_SHAPE;
  if (!valid_dtype(dtype) || !std::isfinite(scale) || !valid_flag(accumulate)) return TIM_ERR_VALUE;
  if (!grad_table) return TIM_ERR_NULL;
  if (!aligned_to(grad_table, 4)) return TIM_ERR_VALUE;
  if (T == 0) return TIM_OK;
  if (!grad_out || !tokens) return TIM_ERR_NULL;
  if (!aligned_to(grad_out, dtype_bytes(dtype)) || !aligned_to(tokens, 4)) return TIM_ERR_VALUE;
  if (!ws || !aligned16(ws) || ws_bytes < plan_embedding_backward(T, V, d).bytes) return TIM_ERR_WORKSPACE;
  const Rows o = rows_of(grad_table, V, d, grad_ld, 4);
  if (share_bytes(o, rows_of(grad_out, T, d, ld, dtype_bytes(dtype))) || share_bytes(o, flat(tokens, T, 4)))
    return TIM_ERR_VALUE;
  return TIM_OK;
}

struct EmbedArgs {
  const void* table;
  int32_t V, d;
  int64_t ld;
  const int32_t* tokens;
  int64_t T;
  float scale;
  void* out;
  int64_t out_ld;
};
hipError_t launch_embedding(const EmbedArgs& a, int dtype, int out_dtype, hipStream_t s);

struct EmbedGradArgs {
  const void* grad_out;
  int64_t T, ld;
  int32_t V, d;
  const int32_t* tokens;
  float scale;
  float* grad_table;
  int64_t grad_ld;
  int32_t accumulate;
};
hipError_t launch_embedding_backward(const EmbedGradArgs& a, int dtype, void* ws, hipStream_t s);

// ------------------------------------------------------------------ adapters

inline bool valid_adapter_shape(int64_t T, int64_t d, int64_t N, int64_t n, int64_t r) {
  return grouped_rows(T) && valid_width(d) && valid_width(N) && valid_keys(n) && r >= 1 && r <= TIM_MAX_RANK;
}

// The adapters and the rows they apply to.
inline tim_status validate_adapters(const tim_adapters* ad, const void* x, int64_t x_ld, const int32_t* rows,
                                    int64_t T) {
  if (!ad) return TIM_ERR_NULL;
  if (!valid_adapter_shape(T, ad->d, ad->N, ad->n, ad->r) || x_ld < ad->d) return TIM_ERR_SHAPE;
  if (ad->dtype != TIM_BF16 && ad->dtype != TIM_F16) return TIM_ERR_VALUE;
  if (T == 0) return TIM_OK;
  if (!ad->a || !ad->b || !x || !rows) return TIM_ERR_NULL;
  if (!aligned_to(ad->a, 2) || !aligned_to(ad->b, 2) || !aligned_to(ad->scales, 4) || !aligned_to(x, 2) ||
      !aligned_to(rows, 4))
    return TIM_ERR_VALUE;
  return TIM_OK;
}

// Whether `out` has a byte in common with the adapters or the rows' indices.
inline bool shares_adapters(const Rows& out, const tim_adapters& ad, const int32_t* rows, int64_t T) {
  return share_bytes(out, flat(rows, T, 4)) || share_bytes(out, flat(ad.a, ad.n, (int64_t)ad.r * ad.d * 2)) ||
         share_bytes(out, flat(ad.b, ad.n, (int64_t)ad.r * ad.N * 2)) || share_bytes(out, flat(ad.scales, ad.n, 4));
}

inline tim_status validate_adapters_add(const tim_adapters* ad, const void* x, int64_t x_ld, const int32_t* rows,
                                        int64_t T, const void* base, int64_t base_ld, const void* out,
                                        int32_t out_dtype, int64_t out_ld, const void* ws, size_t ws_bytes) {
  const tim_status s = validate_adapters(ad, x, x_ld, rows, T);
  if (s != TIM_OK) return s;
  if ((base && base_ld < ad->N) || out_ld < ad->N) return TIM_ERR_SHAPE;
  if (!valid_dtype(out_dtype)) return TIM_ERR_VALUE;
  if (T == 0) return TIM_OK;
  if (!out) return TIM_ERR_NULL;
  if (base == out && base_ld != out_ld) return TIM_ERR_SHAPE;
  if (!aligned_to(base, dtype_bytes(out_dtype)) || !aligned_to(out, dtype_bytes(out_dtype))) return TIM_ERR_VALUE;
  if (!ws || !aligned16(ws) || ws_bytes < plan_adapters(T, ad->d, ad->N, ad->n, ad->r, 0).bytes)
    return TIM_ERR_WORKSPACE;
  // x may lie under out: launch_adapters_add reads all of it first
  const int bytes = dtype_bytes(out_dtype);
  const Rows o = rows_of(out, T, ad->N, out_ld, bytes);
  if (shares_adapters(o, *ad, rows, T) || (base != out && share_bytes(o, rows_of(base, T, ad->N, base_ld, bytes))))
    return TIM_ERR_VALUE;
  return TIM_OK;
}

inline tim_status validate_adapters_backward(const tim_adapters* ad, const void* x, int64_t x_ld, const int32_t* rows,
                                             int64_t T, const void* grad, int32_t grad_dtype, int64_t grad_ld,
                                             const void* grad_x, int32_t gx_dtype, int64_t gx_ld, int32_t accumulate_x,
                                             const float* grad_a, const float* grad_b, int32_t accumulate_ab,
                                             const void* ws, size_t ws_bytes) {
  const tim_status s = validate_adapters(ad, x, x_ld, rows, T);
  if (s != TIM_OK) return s;
  if (grad_ld < ad->N || (grad_x && gx_ld < ad->d)) return TIM_ERR_SHAPE;
  if (!valid_dtype(grad_dtype) || !valid_flag(accumulate_x) || !valid_flag(accumulate_ab)) return TIM_ERR_VALUE;
  if (grad_x && (!valid_dtype(gx_dtype) || !aligned_to(grad_x, dtype_bytes(gx_dtype)))) return TIM_ERR_VALUE;
  if (!aligned_to(grad_a, 4) || !aligned_to(grad_b, 4)) return TIM_ERR_VALUE;
  if (T == 0) return TIM_OK;
  if (!grad) return TIM_ERR_NULL;
  if (!aligned_to(grad, dtype_bytes(grad_dtype))) return TIM_ERR_VALUE;
  if (!ws || !aligned16(ws) || ws_bytes < adapters_backward_workspace(T, ad->d, ad->N, ad->n, ad->r))
    return TIM_ERR_WORKSPACE;
  const Rows outs[3] = {rows_of(grad_x, T, ad->d, gx_ld, grad_x ? dtype_bytes(gx_dtype) : 0),
                        flat(grad_a, ad->n, (int64_t)ad->r * ad->d * 4), flat(grad_b, ad->n, (int64_t)ad->r * ad->N * 4)};
  // grad may lie under grad_x: launch_adapters_backward reads all of it before it writes there, but x after
  const Rows of_x = rows_of(x, T, ad->d, x_ld, 2), of_grad = rows_of(grad, T, ad->N, grad_ld, dtype_bytes(grad_dtype));
  for (int i = 0; i < 3; ++i)
    if (shares_adapters(outs[i], *ad, rows, T) || share_bytes(outs[i], of_x) || (i > 0 && share_bytes(outs[i], of_grad)) ||
        share_bytes(outs[i], outs[(i + 1) % 3]))
      return TIM_ERR_VALUE;
  return TIM_OK;
}

hipError_t launch_adapters_add(const tim_adapters& ad, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                               const void* base, int64_t base_ld, void* out, int out_dtype, int64_t out_ld, void* ws,
                               hipStream_t s);

struct AdapterGradArgs {
  const void* x;
  int64_t x_ld;
  const int32_t* rows;
  int64_t T;
  const void* grad;
  int64_t grad_ld;
  void* grad_x;
  int64_t gx_ld;
  int32_t accumulate_x;
  float *grad_a, *grad_b;
  int32_t accumulate_ab;
};
hipError_t launch_adapters_backward(const tim_adapters& ad, const AdapterGradArgs& a, int grad_dtype, int gx_dtype,
                                    void* ws, hipStream_t s);
// p[r * ld + c] = 0 for r < rows, c < d.
hipError_t launch_zero_rows(float* p, int64_t rows, int64_t d, int64_t ld, hipStream_t s);

}  // namespace tim
