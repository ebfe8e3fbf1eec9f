// Adapters: the product that begins with rows of d elements, u = x a^T, the
// sums of partial products, and the order of the launches.

#include <hip/hip_runtime.h>

#include "adapters.h"
#include "group_rows.h"

namespace tim {
namespace {

struct ShrinkArgs {
  const void* x;
  int64_t x_ld, T;
  const void* w;  // [n, r, d]
  int32_t n, r, rp, d;
  float* part;    // [chunks, T, rp]
};

// part[chunk][row][j] = sum over the chunk's elements of x[row][k] a[j][k] for RB
// blocks of 16 rows of one adapter (row[rb]: this lane's) and JB blocks of 16
// ranks from j0 on, zeros for the ranks from r on. Four waves take a quarter of
// the chunk each; their sums are added in order through lds. `rows` of the rows
// are stored.
template <class T, int JB, int RB>
__device__ __forceinline__ void shrink_rows(const ShrinkArgs& a, int key, const int32_t (&row)[RB], int rows, int chunk,
                                            int j0, int wave, f32x4 (*lds)[JB][RB][64]) {
  const int lane = threadIdx.x & 63, m = lane % 16, g = lane / 16, blocks = (rows + 15) / 16;
  const T* w = (const T*)a.w + (int64_t)key * a.r * a.d;
  const T *wr[JB], *xr[RB];
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int j = j0 + jb * 16 + m;
    wr[jb] = w + (int64_t)(j < a.r ? j : a.r - 1) * a.d;
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) xr[rb] = (const T*)a.x + row[rb] * a.x_ld;
  f32x4 acc[JB][RB] = {};
  constexpr int kEach = kShrinkChunk / kWaves;
  const int from = chunk * kShrinkChunk + wave * kEach;
  auto step = [&](auto whole, int k0) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int k = k0 + g * 8, n = a.d - k;
    x8<T> wf[JB], xf[RB];
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) wf[jb] = load_n<WHOLE, x8<T>, 8>(wr[jb] + k, n);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (rb < blocks) xf[rb] = load_n<WHOLE, x8<T>, 8>(xr[rb] + k, n);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      if (rb < blocks)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[jb][rb] = mfma(wf[jb], xf[rb], acc[jb][rb]);
  };
  if (from + kEach <= a.d) {
#pragma unroll
    for (int k0 = 0; k0 < kEach; k0 += 32) step(std::true_type{}, from + k0);
  } else {
    for (int k0 = from; k0 < a.d && k0 < from + kEach; k0 += 32) step(std::false_type{}, k0);
  }
  if (wave > 0) {
#pragma unroll
    for (int jb = 0; jb < JB; ++jb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) lds[wave - 1][jb][rb][lane] = acc[jb][rb];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int jb = 0; jb < JB; ++jb)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      f32x4 s = acc[jb][rb];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) s += lds[w][jb][rb][lane];
      const int j = j0 + jb * 16 + g * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e >= a.r) s[e] = 0.f;
      if (rb * 16 + m < rows && j < a.rp) *(f32x4*)(a.part + ((int64_t)chunk * a.T + row[rb]) * a.rp + j) = s;
    }
}

// A run a workgroup and chunk: 8192 rows of 4096 and adapters of rank 32 in 24 us
// (2.8 TB/s of x; chunks of 1024 elements 28), 4096 rows and rank 16 in 13.
template <class T, int JB>
__global__ __launch_bounds__(kThreads) void shrink(ShrinkArgs a, RunList l) {
  __shared__ f32x4 lds[kWaves - 1][JB][4][64];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0 || run.key >= a.n) return;
  int32_t row[4];
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) {
    const int t = rb * 16 + (int)threadIdx.x % 16;
    row[rb] = l.order[run.first + (t < run.count ? t : run.count - 1)];
  }
  shrink_rows<T, JB, 4>(a, run.key, row, run.count, at.tile, blockIdx.z * JB * 16, threadIdx.x >> 6, lds);
}

// The same with each row by itself, which needs no grouping, beside the grouping
// of the rows (the first workgroup): a row costs a whole block of 16 in the
// matrix instructions and its adapter's weights from the caches, but one launch
// less stands between the call and its result. Four rows a workgroup, the same
// arithmetic, so the same bits.
template <class T, int JB>
__global__ __launch_bounds__(kSmallThreads) void group_and_shrink(GroupArgs ga, ShrinkArgs a, int chunks) {
  if (blockIdx.x == 0) {
    if (blockIdx.z == 0) group_rows<12>(ga);
    return;
  }
  __shared__ f32x4 lds[4][kWaves - 1][JB][1][64];
  const int id = blockIdx.x - 1, part = threadIdx.x / kThreads;
  const int t = id / chunks * 4 + part;
  const int32_t row[1] = {t < a.T ? t : 0};
  const uint32_t key = key_of(ga.keys, row[0], a.n);
  const bool there = t < a.T && key < (uint32_t)a.n;
  // rows without an adapter go along, to the barrier, with the first one's weights
  shrink_rows<T, JB, 1>(a, there ? key : 0, row, there ? 1 : 0, id % chunks, blockIdx.z * JB * 16,
                        (threadIdx.x % kThreads) >> 6, lds[part]);
}

// out[row][j] = scale of the row's adapter * the sum of its chunks: in order over
// `inner` chunks (1 or 2), then a sixteenth of these sums a group of 16 lanes, each
// in order, then the groups in order. 64 consecutive elements a workgroup. terms
// (may be null): the same as three bf16 numbers each, [row][3][j].
__global__ __launch_bounds__(kThreads) void sum_chunks(const float* part, const int32_t* rows, int64_t T, int r, int rp,
                                                       int chunks, int inner, int n, const float* scales, float* out,
                                                       __bf16* terms) {
  __shared__ f32x4 lds[16][16];
  const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64, i = at + threadIdx.x % 16 * 4;
  if (at >= T * rp) return;
  const int group = threadIdx.x / 16;
  const uint32_t key = i < T * rp ? key_of(rows, i / rp, n) : n;
  const bool there = key < (uint32_t)n;
  const int outer = (chunks + inner - 1) / inner, per = (outer + 15) / 16 * inner;
  const int from = group * per, to = from + per < chunks ? from + per : chunks;
  const float* p = part + i;
  const int64_t step = T * rp;
  f32x4 s = {};
  if (there) {
    if (inner == 1) {
#pragma unroll 8
      for (int c = from; c < to; ++c) s += *(const f32x4*)(p + c * step);
    } else {
#pragma unroll 4
      for (int c = from; c < to; c += 2) {
        f32x4 q = *(const f32x4*)(p + c * step);
        if (c + 1 < to) q += *(const f32x4*)(p + (c + 1) * step);
        s += q;
      }
    }
  }
  lds[group][threadIdx.x % 16] = s;
  __syncthreads();
  if (group > 0 || !there) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x];
  s *= scales ? scales[key] : 1.f;
  const int j = (int)(i % rp);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e >= r) s[e] = 0.f;  // whatever the rows hold
  *(f32x4*)(out + i) = s;
  if (terms) {
    x4<__bf16> q[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      __bf16 t[3];
      split3(s[e], t);
#pragma unroll
      for (int k = 0; k < 3; ++k) q[k][e] = t[k];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *(x4<__bf16>*)(terms + (i / rp * 3 + k) * rp + j) = q[k];
  }
}

// What follows the passes: of adapters with several runs of rows the runs' sums
// in order, and zeros for the adapters without rows. blockIdx.z: of grad_a, of grad_b.
struct FinishArgs {
  const float* part[2];
  float* out[2];
  int64_t size[2];  // r * d, r * N
  int32_t log_C[2];
  RunList l[2];
  int32_t n, joins, accumulate;
  const uint8_t* seen;
};
__global__ __launch_bounds__(kThreads) void finish(FinishArgs a) {
  const Place at = place_of();
  const int z = blockIdx.z;
  const int64_t size = a.size[z], step = (int64_t)gridDim.y * kThreads;
  float* out = a.out[z];
  if (!out) return;
  if ((int)at.item >= a.joins) {
    for (int k = (int)at.item - a.joins; k < a.n; k += gridDim.x - a.joins) {
      if (a.seen[k]) continue;
      for (int64_t i = (int64_t)at.tile * kThreads + threadIdx.x; i < size; i += step) out[k * size + i] = 0.f;
    }
    return;
  }
  if ((int)at.item >= *a.l[z].n_joins) return;
  const Join j = a.l[z].joins[at.item];
  if (j.key >= a.n) return;
  const int C = 1 << a.log_C[z], runs = (j.end - j.first + C - 1) / C;
  // the key's runs are two slots apart, the last one's is the odd one
  const float* part = a.part[z] + (int64_t)run_slot(j.first, a.log_C[z], false) * size;
  for (int64_t i = (int64_t)at.tile * kThreads + threadIdx.x; i < size; i += step) {
    float s = 0.f;
    constexpr int kAhead = 8;  // loads in flight, added in order
    for (int k0 = 0; k0 < runs; k0 += kAhead) {
      float x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int q = k0 + k < runs ? k0 + k : runs - 1;
        x[k] = part[(int64_t)(2 * q + (q == runs - 1)) * size + i];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) s += k0 + k < runs ? x[k] : 0.f;
    }
    float* q = out + j.key * size + i;
    *q = a.accumulate ? *q + s : s;
  }
}

template <class T>
hipError_t run_shrink(const ShrinkArgs& a, const RunList& l, int chunks, hipStream_t s) {
  const unsigned runs = (unsigned)l.max_runs;
  if (a.rp <= 16)
    TIM_LAUNCH((shrink<T, 1><<<dim3(runs, chunks), kThreads, 0, s>>>(a, l)));
  else if (a.rp <= 32)
    TIM_LAUNCH((shrink<T, 2><<<dim3(runs, chunks), kThreads, 0, s>>>(a, l)));
  else
    TIM_LAUNCH((shrink<T, 4><<<dim3(runs, chunks, (a.rp + 63) / 64), kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class T>
hipError_t run_group_and_shrink(const GroupArgs& ga, const ShrinkArgs& a, int chunks, hipStream_t s) {
  const unsigned blocks = 1 + (unsigned)((a.T + 3) / 4) * chunks;
  if (a.rp <= 16)
    TIM_LAUNCH((group_and_shrink<T, 1><<<blocks, kSmallThreads, 0, s>>>(ga, a, chunks)));
  else if (a.rp <= 32)
    TIM_LAUNCH((group_and_shrink<T, 2><<<blocks, kSmallThreads, 0, s>>>(ga, a, chunks)));
  else
    TIM_LAUNCH((group_and_shrink<T, 4><<<dim3(blocks, 1, (a.rp + 63) / 64), kSmallThreads, 0, s>>>(ga, a, chunks)));
  return hipSuccess;
}

// The grouping of the rows, and u = x a^T as partial sums of its chunks.
hipError_t group_and_shrink_rows(const tim_adapters& ad, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                                 bool shrink_too, uint8_t* seen, const AdapterPlan& p, void* ws, hipStream_t s) {
  const ShrinkArgs a = {x, x_ld, T, ad.a, ad.n, ad.r, p.rp, ad.d, (float*)((char*)ws + p.u_part)};
  if (shrink_too && p.rows_alone) {
    const GroupArgs ga = group_args(p.g, rows, true, seen, ws);
    return ad.dtype == TIM_BF16 ? run_group_and_shrink<__bf16>(ga, a, p.x_chunks, s)
                                : run_group_and_shrink<_Float16>(ga, a, p.x_chunks, s);
  }
  const hipError_t e = launch_grouping(p.g, rows, true, seen, ws, s);
  if (e != hipSuccess || !shrink_too) return e;
  const RunList l = run_list(p.g, ws, 0);
  return ad.dtype == TIM_BF16 ? run_shrink<__bf16>(a, l, p.x_chunks, s) : run_shrink<_Float16>(a, l, p.x_chunks, s);
}

hipError_t launch_sum_chunks(const float* part, const int32_t* rows, int64_t T, int r, int rp, int chunks, int inner, int n,
                             const float* scales, float* out, void* terms, hipStream_t s) {
  const int64_t blocks = (T * rp + 63) / 64, across = blocks < 1 << 20 ? blocks : 1 << 20;
  TIM_LAUNCH((sum_chunks<<<dim3((unsigned)across, (unsigned)((blocks + across - 1) / across)), kThreads, 0, s>>>(
      part, rows, T, r, rp, chunks, inner, n, scales, out, (__bf16*)terms)));
  return hipSuccess;
}

}  // namespace

hipError_t launch_adapters_add(const tim_adapters& ad, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                               const void* base, int64_t base_ld, void* out, int out_dtype, int64_t out_ld, void* ws,
                               hipStream_t s) {
  const AdapterPlan p = plan_adapters(T, ad.d, ad.N, ad.n, ad.r, 0);
  const hipError_t e = group_and_shrink_rows(ad, x, x_ld, rows, T, true, nullptr, p, ws, s);
  if (e != hipSuccess) return e;
  const ExpandArgs ea = {(const float*)((char*)ws + p.u_part), nullptr, T, p.x_chunks, ad.n, ad.r, p.rp, ad.N, ad.scales, ad.b,
                         base, base_ld, out, out_ld};
  return launch_expand(ea, ad.dtype, out_dtype, false, run_list(p.g, ws, 0), s);
}

hipError_t launch_adapters_backward(const tim_adapters& ad, const AdapterGradArgs& a, int grad_dtype, int gx_dtype,
                                    void* workspace, hipStream_t s) {
  const AdapterPlan p = plan_adapters(a.T, ad.d, ad.N, ad.n, ad.r, pass_cols(grad_dtype, ad.dtype));
  char* ws = (char*)workspace;
  uint8_t* seen = (uint8_t*)(ws + p.seen);
  hipError_t e = group_and_shrink_rows(ad, a.x, a.x_ld, a.rows, a.T, a.grad_b != nullptr, seen, p, ws, s);
  if (e != hipSuccess) return e;
  const RunList l = run_list(p.g, ws, 0), la = run_list(p.g, ws, 1), lb = run_list(p.g, ws, 2);
  float *u = nullptr, *v = (float*)(ws + p.v), *a_part = (float*)(ws + p.a_part), *b_part = (float*)(ws + p.b_part);
  if (a.grad_b) {
    u = (float*)(ws + p.u);
    e = launch_sum_chunks((const float*)(ws + p.u_part), a.rows, a.T, ad.r, p.rp, p.x_chunks, 1, ad.n, ad.scales, u, nullptr, s);
    if (e != hipSuccess) return e;
  }
  const PassArgs pb = {a.grad, a.grad_ld, a.T,      u,        ad.b,   (float*)(ws + p.v_part), ad.n, ad.r, p.rp,
                       ad.N,   a.grad_b,  b_part, a.accumulate_ab};
  e = launch_pass(pb, grad_dtype, ad.dtype, true, p.of_grad.tiles, lb, s);
  if (e != hipSuccess) return e;
  // for the bf16 instructions of grad_x's product
  void* terms = a.grad_x && ad.dtype == TIM_BF16 && p.rp <= 64 ? ws + p.v_terms : nullptr;
  if (a.grad_x || a.grad_a) {
    e = launch_sum_chunks(pb.part, a.rows, a.T, ad.r, p.rp, p.g_chunks, kTilePair / p.of_grad.tiles, ad.n, ad.scales, v, terms, s);
    if (e != hipSuccess) return e;
  }
  if (a.grad_x) {
    const ExpandArgs ea = {v, terms, a.T, 1, ad.n, ad.r, p.rp, ad.d, nullptr, ad.a, a.accumulate_x ? a.grad_x : nullptr,
                           a.gx_ld, a.grad_x, a.gx_ld};
    e = launch_expand(ea, ad.dtype, gx_dtype, true, l, s);
    if (e != hipSuccess) return e;
  }
  if (a.grad_a) {
    const PassArgs pa = {a.x,  a.x_ld,   a.T,    v, nullptr, nullptr, ad.n, ad.r, p.rp,
                         ad.d, a.grad_a, a_part, a.accumulate_ab};
    e = launch_pass(pa, ad.dtype, ad.dtype, false, 1, la, s);
    if (e != hipSuccess) return e;
  }
  if (!a.grad_a && !a.grad_b) return hipSuccess;
  FinishArgs f = {{a_part, b_part},
                  {a.grad_a, a.grad_b},
                  {(int64_t)ad.r * ad.d, (int64_t)ad.r * ad.N},
                  {p.of_x.log_rows, p.of_grad.log_rows},
                  {la, lb},
                  ad.n,
                  (int32_t)(la.max_joins > lb.max_joins ? la.max_joins : lb.max_joins),
                  a.accumulate_ab,
                  seen};
  const int zeros = a.accumulate_ab ? 0 : ad.n < 1024 ? ad.n : 1024;
  const int64_t most = f.size[0] > f.size[1] ? f.size[0] : f.size[1];
  const unsigned across = (unsigned)(most < 512 * kThreads ? (most + kThreads - 1) / kThreads : 512);
  if (f.joins + zeros > 0) TIM_LAUNCH((finish<<<dim3(f.joins + zeros, across, 2), kThreads, 0, s>>>(f)));
  return hipSuccess;
}

}  // namespace tim
