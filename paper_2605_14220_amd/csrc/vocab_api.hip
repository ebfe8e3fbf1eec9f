// C-ABI entry points of tim_vocab.h: argument checks and launches.

#include <hip/hip_runtime.h>

#include "tim_vocab.h"
#include "vocab.h"

namespace {

inline tim_status hip_status(hipError_t e) { return e == hipSuccess ? TIM_OK : TIM_ERR_HIP; }

}  // namespace

extern "C" {

tim_status tim_embedding(const void* table, int32_t dtype, int32_t V, int32_t d, int64_t ld, const int32_t* tokens,
                         int64_t T, float scale, void* out, int32_t out_dtype, int64_t out_ld, hipStream_t stream) {
  const tim_status st = tim::validate_embedding(table, dtype, V, d, ld, tokens, T, scale, out, out_dtype, out_ld);
  if (st != TIM_OK || T == 0) return st;
  const tim::EmbedArgs a = {table, V, d, ld, tokens, T, scale, out, out_ld};
  return hip_status(tim::launch_embedding(a, dtype, out_dtype, stream));
}

size_t tim_embedding_backward_workspace_size(int64_t T, int32_t V, int32_t d) {
  if (T <= 0 || !tim::grouped_rows(T) || !tim::valid_keys(V) || !tim::valid_width(d)) return 0;
  return tim::plan_embedding_backward(T, V, d).bytes;
}

tim_status tim_embedding_backward(const void* grad_out, int32_t dtype, int64_t T, int32_t d, int64_t ld,
                                  const int32_t* tokens, int32_t V, float scale, float* grad_table, int64_t grad_ld,
                                  int32_t accumulate, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const tim_status st = tim::validate_embedding_backward(grad_out, dtype, T, d, ld, tokens, V, scale, grad_table,
                                                         grad_ld, accumulate, workspace, workspace_bytes);
  if (st != TIM_OK) return st;
  if (T == 0) return accumulate ? TIM_OK : hip_status(tim::launch_zero_rows(grad_table, V, d, grad_ld, stream));
  const tim::EmbedGradArgs a = {grad_out, T, ld, V, d, tokens, scale, grad_table, grad_ld, accumulate};
  return hip_status(tim::launch_embedding_backward(a, dtype, workspace, stream));
}

size_t tim_adapters_add_workspace_size(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r) {
  if (T <= 0 || !tim::valid_adapter_shape(T, d, N, n, r)) return 0;
  return tim::plan_adapters(T, d, N, n, r, 0).bytes;
}

tim_status tim_adapters_add(const tim_adapters* adapters, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                            const void* base, int64_t base_ld, void* out, int32_t out_dtype, int64_t out_ld,
                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const tim_status st = tim::validate_adapters_add(adapters, x, x_ld, rows, T, base, base_ld, out, out_dtype, out_ld,
                                                   workspace, workspace_bytes);
  if (st != TIM_OK || T == 0) return st;
  return hip_status(tim::launch_adapters_add(*adapters, x, x_ld, rows, T, base, base_ld, out, out_dtype, out_ld,
                                             workspace, stream));
}

size_t tim_adapters_backward_workspace_size(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r) {
  if (T <= 0 || !tim::valid_adapter_shape(T, d, N, n, r)) return 0;
  return tim::adapters_backward_workspace(T, d, N, n, r);
}

tim_status tim_adapters_backward(const tim_adapters* adapters, const void* x, int64_t x_ld, const int32_t* rows,
                                 int64_t T, const void* grad, int32_t grad_dtype, int64_t grad_ld, void* grad_x,
                                 int32_t gx_dtype, int64_t gx_ld, int32_t accumulate_x, float* grad_a, float* grad_b,
                                 int32_t accumulate_ab, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const tim_status st =
      tim::validate_adapters_backward(adapters, x, x_ld, rows, T, grad, grad_dtype, grad_ld, grad_x, gx_dtype, gx_ld,
                                      accumulate_x, grad_a, grad_b, accumulate_ab, workspace, workspace_bytes);
  if (st != TIM_OK) return st;
  if (T == 0) {
    hipError_t e = hipSuccess;
    const int64_t n = (int64_t)adapters->n * adapters->r;
    if (grad_a && !accumulate_ab) e = tim::launch_zero_rows(grad_a, n, adapters->d, adapters->d, stream);
    if (e == hipSuccess && grad_b && !accumulate_ab)
      e = tim::launch_zero_rows(grad_b, n, adapters->N, adapters->N, stream);
    return hip_status(e);
  }
  if (!grad_x && !grad_a && !grad_b) return TIM_OK;
  const tim::AdapterGradArgs a = {x,      x_ld,         rows,   T,      grad,          grad_ld, grad_x,
                                  gx_ld,  accumulate_x, grad_a, grad_b, accumulate_ab};
  return hip_status(tim::launch_adapters_backward(*adapters, a, grad_dtype, gx_dtype, workspace, stream));
}

}  // extern "C"
