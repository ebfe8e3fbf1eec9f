// Token embedding and its gradient on gfx950. Both move bytes: the lookup reads
// the rows that occur and writes T rows; the gradient reads T rows and writes
// the table (or the touched rows of it).

#include <hip/hip_runtime.h>

#include <type_traits>

#include "group_rows.h"
#include "vocab.h"

namespace tim {
namespace {

constexpr int kThreads = 256;

// N consecutive elements at p, aligned to their element only.
template <class T, int N>
struct Pack {
  T v[N];
};
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  Pack<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}
// Past the caches: what the table's zeros leave there, nobody reads (two
// micro-batches of 301 rows, V 50257, d 1536: 73 us against 80).
__device__ __forceinline__ void store_zeros(float* p) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  typedef f4 f4_by4 __attribute__((aligned(4)));
  __builtin_nontemporal_store(f4{}, (f4_by4*)p);
}

// A row is taken by `lanes` threads (a power of two up to 256), N elements at a
// time; blockIdx.y walks slices of lanes * N elements. A thread takes kEmbedRows
// rows, whose loads are in flight together (16384 rows of 4096 bf16 elements 36-42
// us, 4.9 TB/s; one row a thread 64).
constexpr int kEmbedRows = 4;
template <class T, class O, int N>
__global__ __launch_bounds__(kThreads) void embed(EmbedArgs a, int64_t row0, int lanes) {
  const int down = kThreads / lanes;
  const int64_t t0 = row0 + (int64_t)blockIdx.x * down * kEmbedRows + threadIdx.x / lanes;
  const int c = (blockIdx.y * lanes + threadIdx.x % lanes) * N;
  if (c >= a.d) return;
  uint32_t v[kEmbedRows];
#pragma unroll
  for (int k = 0; k < kEmbedRows; ++k) v[k] = t0 + k * down < a.T ? (uint32_t)a.tokens[t0 + k * down] : ~0u;
  const T* table = (const T*)a.table + c;
  O* out = (O*)a.out + c;
  if (c + N <= a.d) {
    Pack<T, N> x[kEmbedRows];
#pragma unroll
    for (int k = 0; k < kEmbedRows; ++k)
      x[k] = load_pack<T, N>(table + (v[k] < (uint32_t)a.V ? (int64_t)v[k] : 0) * a.ld);
#pragma unroll
    for (int k = 0; k < kEmbedRows; ++k) {
      if (t0 + k * down >= a.T) break;
      const bool there = v[k] < (uint32_t)a.V;
      Pack<O, N> y;
#pragma unroll
      for (int e = 0; e < N; ++e) y.v[e] = there ? narrow<O>((float)x[k].v[e] * a.scale) : (O)0.f;
      store_pack(out + (t0 + k * down) * a.out_ld, y);
    }
  } else {
    for (int k = 0; k < kEmbedRows; ++k)
      for (int e = 0; c + e < a.d && t0 + k * down < a.T; ++e)
        out[(t0 + k * down) * a.out_ld + e] =
            v[k] < (uint32_t)a.V ? narrow<O>((float)table[v[k] * a.ld + e] * a.scale) : (O)0.f;
  }
}

template <class T, class O>
hipError_t embed_typed(const EmbedArgs& a, hipStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  int lanes = 1;
  while (lanes < kThreads && (int64_t)lanes * N < a.d) lanes *= 2;
  const int rows = kThreads / lanes * kEmbedRows;
  const unsigned slices = (unsigned)((a.d + (int64_t)lanes * N - 1) / ((int64_t)lanes * N));
  // fewer than 2^32 threads a launch and direction
  const int64_t per = (int64_t)1 << 23;
  for (int64_t t = 0; t < a.T; t += per * rows) {
    const int64_t left = (a.T - t + rows - 1) / rows;
    embed<T, O, N><<<dim3((unsigned)(left < per ? left : per), slices), kThreads, 0, s>>>(a, t, lanes);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class T>
hipError_t embed_out(const EmbedArgs& a, int out_dtype, hipStream_t s) {
  switch (out_dtype) {
    case TIM_F32: return embed_typed<T, float>(a, s);
    case TIM_BF16: return embed_typed<T, __bf16>(a, s);
    default: return embed_typed<T, _Float16>(a, s);
  }
}

// ------------------------------------------------------------------ gradient

// Zeros in a row, by kThreads threads.
__device__ __forceinline__ void zero_row(float* q, int64_t d) {
  int64_t c = (int64_t)(threadIdx.x % kThreads) * 4;
  for (; c + 4 <= d; c += kThreads * 4) store_zeros(q + c);
  for (int e = 0; c + e < d && e < 4; ++e) q[c + e] = 0.f;
}
__global__ __launch_bounds__(kThreads) void zero_all(float* p, int64_t d, int64_t ld) {
  zero_row(p + (int64_t)blockIdx.x * ld, d);
}
// The grouping of few rows (the first workgroup) beside zeros in the whole table:
// the few rows of tokens that occur are written again, but neither waits for the
// other (two micro-batches of 301 rows, V 50257, d 1536: 82 us against 93).
constexpr int kZeroRows = kSmallThreads / kThreads;
__global__ __launch_bounds__(kSmallThreads) void group_and_zero(GroupArgs ga, float* p, int64_t rows, int64_t d,
                                                                int64_t ld) {
  if (blockIdx.x == 0) {
    group_rows<12>(ga);
    return;
  }
  const int64_t r = (int64_t)(blockIdx.x - 1) * kZeroRows + threadIdx.x / kThreads;
  if (r < rows) zero_row(p + r * ld, d);
}

// The sum of a run's rows, a chain by ascending t, for one slice of columns. A
// token's only run is scaled and stored (or added to the table's row), one of
// several is left in its slot. The workgroups past the runs' clear the rows of
// the tokens that do not occur: the runs' chains then hide behind the stores.
template <class T, int N>
__global__ __launch_bounds__(kThreads) void sum_runs(EmbedGradArgs a, RunList l, float* part,
                                                         const uint8_t* seen) {
  if (blockIdx.x >= l.max_runs) {
    const int64_t r = (blockIdx.x - l.max_runs) * gridDim.y + blockIdx.y;
    if (r < a.V && !seen[r]) zero_row(a.grad_table + r * a.grad_ld, a.d);
    return;
  }
  const Run run = run_of(l, blockIdx.x);
  if (run.count == 0) return;
  const int c = (blockIdx.y * kThreads + threadIdx.x) * N;
  if (c >= a.d) return;
  const int n = a.d - c < N ? a.d - c : N;
  const int32_t* order = l.order + run.first;
  float sum[N] = {};
  const T* g = (const T*)a.grad_out + c;
  constexpr int kAhead = 4;
  int k = 0;
  if (n == N) {
    for (; k + kAhead <= run.count; k += kAhead) {
      Pack<T, N> x[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) x[q] = load_pack<T, N>(g + order[k + q] * a.ld);
#pragma unroll
      for (int q = 0; q < kAhead; ++q)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += (float)x[q].v[e];
    }
    for (; k < run.count; ++k) {
      const Pack<T, N> x = load_pack<T, N>(g + order[k] * a.ld);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += (float)x.v[e];
    }
  } else {
    for (; k < run.count; ++k)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < n) sum[e] += (float)g[order[k] * a.ld + e];
  }
  const bool only = run.slot < 0;
  float* dst = only ? a.grad_table + run.key * a.grad_ld + c : part + (int64_t)run.slot * a.d + c;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (only) sum[e] *= a.scale;
  if (n == N) {
    if (only && a.accumulate) {
      const Pack<float, N> old = load_pack<float, N>(dst);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += old.v[e];
    }
    Pack<float, N> y;
#pragma unroll
    for (int e = 0; e < N; ++e) y.v[e] = sum[e];
    store_pack(dst, y);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) dst[e] = only && a.accumulate ? dst[e] + sum[e] : sum[e];
  }
}

// Tokens of several runs: the runs' sums in order, scaled once.
__global__ __launch_bounds__(kThreads) void join_runs(EmbedGradArgs a, RunList l, const float* part) {
  const int64_t item = blockIdx.x;
  if (item >= *l.n_joins) return;
  const Join j = l.joins[item];
  const int c = blockIdx.y * kThreads + threadIdx.x;
  if (c >= a.d) return;
  float sum = 0.f;
#pragma unroll 4
  for (int p = j.first; p < j.end; p += TIM_EMBED_RUN)
    sum += part[(int64_t)run_slot(p, kLogEmbedRun, p + TIM_EMBED_RUN >= j.end) * a.d + c];
  sum *= a.scale;
  float* dst = a.grad_table + j.key * a.grad_ld + c;
  *dst = a.accumulate ? *dst + sum : sum;
}

template <class T>
hipError_t grad_typed(const EmbedGradArgs& a, const EmbedPlan& p, char* ws, hipStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  const RunList l = run_list(p.g, ws, 0);
  float* part = (float*)(ws + p.part);
  const int slices = (a.d + kThreads * N - 1) / (kThreads * N);
  hipError_t e;
  uint8_t* seen = nullptr;
  int64_t zero_blocks = 0;
  if (!a.accumulate && p.g.small && a.T <= 4096) {
    group_and_zero<<<1 + (unsigned)((a.V + kZeroRows - 1) / kZeroRows), kSmallThreads, 0, s>>>(
        group_args(p.g, a.tokens, false, nullptr, ws), a.grad_table, a.V, a.d, a.grad_ld);
    e = hipGetLastError();
  } else {
    if (!a.accumulate) {
      seen = (uint8_t*)(ws + p.seen);
      zero_blocks = (a.V + slices - 1) / slices;
    }
    e = launch_grouping(p.g, a.tokens, false, seen, ws, s);
  }
  if (e != hipSuccess) return e;
  sum_runs<T, N><<<dim3((unsigned)(l.max_runs + zero_blocks), slices), kThreads, 0, s>>>(a, l, part, seen);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (l.max_joins > 0) {
    const int js = (a.d + kThreads - 1) / kThreads;
    join_runs<<<dim3((unsigned)l.max_joins, js), kThreads, 0, s>>>(a, l, part);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_zero_rows(float* p, int64_t rows, int64_t d, int64_t ld, hipStream_t s) {
  constexpr int64_t kRows = (int64_t)1 << 23;  // fewer than 2^32 threads a launch
  for (int64_t r = 0; r < rows; r += kRows) {
    zero_all<<<(unsigned)(rows - r < kRows ? rows - r : kRows), kThreads, 0, s>>>(p + r * ld, d, ld);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_embedding(const EmbedArgs& a, int dtype, int out_dtype, hipStream_t s) {
  switch (dtype) {
    case TIM_F32: return embed_out<float>(a, out_dtype, s);
    case TIM_BF16: return embed_out<__bf16>(a, out_dtype, s);
    default: return embed_out<_Float16>(a, out_dtype, s);
  }
}

hipError_t launch_embedding_backward(const EmbedGradArgs& a, int dtype, void* ws, hipStream_t s) {
  const EmbedPlan p = plan_embedding_backward(a.T, a.V, a.d);
  switch (dtype) {
    case TIM_F32: return grad_typed<float>(a, p, (char*)ws, s);
    case TIM_BF16: return grad_typed<__bf16>(a, p, (char*)ws, s);
    default: return grad_typed<_Float16>(a, p, (char*)ws, s);
  }
}

}  // namespace tim
