// Low-rank adapters of many requests beside a shared projection, and their
// gradients, on gfx950. Rows are grouped by adapter (grouping.h); a workgroup
// takes a run of up to 64 rows of one adapter:
//
//   shrink   u = x a^T          contraction over d, 1024 elements a workgroup
//   expand   out = base + u b^T 256 columns a workgroup (backward: v a)
//   contract v = grad b         contraction over N, 1024 elements a workgroup
//   outer    sum_t src[t] w[t]  up to 512 rows of one adapter, 256 columns a workgroup
//
// x, a and b are 16 bits wide; their products with each other run on the 16-bit
// matrix instructions. u and v stay in fp32, and so do the products that they
// enter (16x16x4 fp32 MFMA): what a call moves, not what it computes, bounds it.

#include <hip/hip_runtime.h>

#include <type_traits>

#include "vocab.h"

namespace tim {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}
__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}
template <class T>
using x8 = std::conditional_t<std::is_same_v<T, __bf16>, bf16x8, f16x8>;

// N elements from p, the first n of them (the others zero); aligned to their
// element only.
template <class V, int N, class T>
__device__ __forceinline__ V load_some(const T* p, int n) {
  V r = {};
  if (n >= N) {
    __builtin_memcpy(&r, p, N * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) r[e] = p[e];
  }
  return r;
}
template <class T>
using x4 = T __attribute__((ext_vector_type(4)));
template <class T>
__device__ __forceinline__ f32x4 load4(const T* p, int n) {
  const x4<T> r = load_some<x4<T>, 4>(p, n);
  return f32x4{(float)r[0], (float)r[1], (float)r[2], (float)r[3]};
}

// A wave's results of JB blocks of 16 ranks for RB blocks of 16 rows, summed
// over the workgroup's waves in wave order and stored as part[place][rank].
template <int JB>
__device__ __forceinline__ void store_sums(f32x4 (&acc)[JB][4], f32x4 (*lds)[JB][4][64], float* part, int rp, int j0,
                                           int count, int lane, int wave) {
  if (wave > 0) {
#pragma unroll
    for (int jb = 0; jb < JB; ++jb)
#pragma unroll
      for (int rb = 0; rb < 4; ++rb) lds[wave - 1][jb][rb][lane] = acc[jb][rb];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int jb = 0; jb < JB; ++jb)
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      f32x4 s = acc[jb][rb];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) s += lds[w][jb][rb][lane];
      const int t = rb * 16 + lane % 16, j = j0 + jb * 16 + lane / 16 * 4;
      if (t < count && j < rp) *(f32x4*)(part + (int64_t)t * rp + j) = s;
    }
}

struct ShrinkArgs {
  const void* x;
  int64_t x_ld, T;
  const void* w;  // [n, r, d]
  int32_t n, r, rp, d;
  float* part;    // [chunks, T, rp]
};

// u_part[chunk][place][j] = sum over the chunk's elements of x[row][k] a[j][k].
template <class T, int JB>
__global__ __launch_bounds__(kThreads) void shrink(ShrinkArgs a, RunList l) {
  __shared__ f32x4 lds[kWaves - 1][JB][4][64];
  if ((int)blockIdx.x >= *l.n_runs) return;
  const Run run = l.runs[blockIdx.x];
  if (run.key >= a.n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int j0 = blockIdx.z * JB * 16;
  const T* w = (const T*)a.w + (int64_t)run.key * a.r * a.d;
  const T* xr[4];
  const int blocks = (run.count + 15) / 16;
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) {
    const int t = rb * 16 + m;
    xr[rb] = (const T*)a.x + l.order[run.first + (t < run.count ? t : run.count - 1)] * a.x_ld;
  }
  f32x4 acc[JB][4] = {};
  const int from = blockIdx.y * kShrinkChunk + wave * (kShrinkChunk / kWaves);
  const int to = from + kShrinkChunk / kWaves < a.d ? from + kShrinkChunk / kWaves : a.d;
  for (int k0 = from; k0 < to; k0 += 32) {
    const int k = k0 + g * 8, n = a.d - k;
    x8<T> wf[JB];
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) {
      const int j = j0 + jb * 16 + m;
      wf[jb] = j < a.r ? load_some<x8<T>, 8>(w + (int64_t)j * a.d + k, n) : x8<T>{};
    }
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks) {
        const x8<T> xf = load_some<x8<T>, 8>(xr[rb] + k, n);
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[jb][rb] = mfma(wf[jb], xf, acc[jb][rb]);
      }
  }
  store_sums<JB>(acc, lds, a.part + ((int64_t)blockIdx.y * a.T + run.first) * a.rp, a.rp, j0, run.count, lane, wave);
}

struct ContractArgs {
  const void* grad;
  int64_t ld, T;
  const void* w;  // [n, N, r]
  int32_t n, r, rp, N;
  float* part;    // [chunks, T, rp]
};

// v_part[chunk][place][j] = sum over the chunk's columns of grad[row][c] b[c][j].
template <class T, class G, int JB>
__global__ __launch_bounds__(kThreads) void contract(ContractArgs a, RunList l) {
  __shared__ f32x4 lds[kWaves - 1][JB][4][64];
  if ((int)blockIdx.x >= *l.n_runs) return;
  const Run run = l.runs[blockIdx.x];
  if (run.key >= a.n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int j0 = blockIdx.z * JB * 16;
  const T* w = (const T*)a.w + (int64_t)run.key * a.N * a.r;
  const G* row[4];
  const int blocks = (run.count + 15) / 16;
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) {
    const int t = rb * 16 + m;
    row[rb] = (const G*)a.grad + l.order[run.first + (t < run.count ? t : run.count - 1)] * a.ld;
  }
  f32x4 acc[JB][4] = {};
  const int from = blockIdx.y * kGradChunk + wave * (kGradChunk / kWaves);
  const int to = from + kGradChunk / kWaves < a.N ? from + kGradChunk / kWaves : a.N;
  for (int c0 = from; c0 < to; c0 += 16) {
    const int c = c0 + g * 4, n = a.N - c;
    f32x4 wf[JB];
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) {
      const int j = j0 + jb * 16 + m;
#pragma unroll
      for (int s = 0; s < 4; ++s) wf[jb][s] = j < a.r && s < n ? (float)w[(int64_t)(c + s) * a.r + j] : 0.f;
    }
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks) {
        const f32x4 gf = load4(row[rb] + c, n);
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
          for (int s = 0; s < 4; ++s) acc[jb][rb] = mfma(wf[jb][s], gf[s], acc[jb][rb]);
      }
  }
  store_sums<JB>(acc, lds, a.part + ((int64_t)blockIdx.y * a.T + run.first) * a.rp, a.rp, j0, run.count, lane, wave);
}

// out[place][j] = scale of the place's adapter * the sum of its chunks in order.
__global__ __launch_bounds__(kThreads) void sum_chunks(const float* part, int64_t T, int rp, int chunks, int n,
                                                       const float* scales, float* out, RunList l) {
  if ((int)blockIdx.x >= *l.n_runs) return;
  const Run run = l.runs[blockIdx.x];
  if (run.key >= n) return;
  const float scale = scales ? scales[run.key] : 1.f;
  const int64_t at = (int64_t)run.first * rp;
  for (int i = threadIdx.x; i < run.count * rp; i += kThreads) {
    float s = 0.f;
#pragma unroll 8
    for (int c = 0; c < chunks; ++c) s += part[(int64_t)c * T * rp + at + i];
    out[at + i] = scale * s;
  }
}

struct ExpandArgs {
  const float* u;  // [chunks, T, rp], summed and scaled here
  int64_t T;
  int32_t chunks, n, r, rp, N;
  const float* scales;
  const void* w;   // [n, N, r], or [n, r, N] where FLAT
  const void* base;
  int64_t base_ld;
  void* out;
  int64_t out_ld;
};

// out[row][c] = base[row][c] + sum_j u[place][j] w[c][j] for 256 columns of a
// run. The matrix instructions' results pass through LDS, so that rows are read
// and written 256 bytes at a time.
template <class T, class O, bool FLAT, int JB>
__global__ __launch_bounds__(kThreads) void expand(ExpandArgs a, RunList l) {
  constexpr int kU = JB * 16 + 4;    // a row of u, apart in the banks
  constexpr int kTile = 64 + 4;      // a row of a wave's 16 x 64 results
  constexpr bool kHold = JB <= 4;    // the columns' weights stay in registers for all rows
  __shared__ float u[64 * kU];
  __shared__ float tile[kWaves][16 * kTile];
  if ((int)blockIdx.x >= *l.n_runs) return;
  const Run run = l.runs[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c0 = (blockIdx.y * kWaves + wave) * 64;
  const int32_t* order = l.order + run.first;
  if (run.key >= a.n) {  // no adapter
    for (int t = wave; t < run.count; t += kWaves) {
      const int64_t row = order[t];
      for (int c = (int)blockIdx.y * kWaves * 64 + lane; c < a.N && c < ((int)blockIdx.y + 1) * kWaves * 64; c += 64)
        ((O*)a.out)[row * a.out_ld + c] = a.base ? ((const O*)a.base)[row * a.base_ld + c] : (O)0.f;
    }
    return;
  }
  const float scale = a.scales ? a.scales[run.key] : 1.f;
  for (int i = threadIdx.x; i < 64 * a.rp / 4; i += kThreads) {
    const int t = i / (a.rp / 4), j = i % (a.rp / 4) * 4;
    f32x4 s = {};
    if (t < run.count) {
      for (int c = 0; c < a.chunks; ++c) s += *(const f32x4*)(a.u + ((int64_t)c * a.T + run.first + t) * a.rp + j);
      s *= scale;
    }
    *(f32x4*)(u + t * kU + j) = s;
  }
  __syncthreads();
  if (c0 >= a.N) return;
  const T* w = (const T*)a.w + (int64_t)run.key * a.r * a.N;
  // wf[nb][s]: the weight of rank jb * 16 + 4 g + s in column c0 + 16 nb + m, or (FLAT) c0 + 4 m + nb
  auto weights = [&](int jb, f32x4(&wf)[4]) {
    const int j = jb * 16 + g * 4;
    if constexpr (FLAT) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const f32x4 x = j + s < a.r ? load4(w + (int64_t)(j + s) * a.N + c0 + 4 * m, a.N - c0 - 4 * m) : f32x4{};
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) wf[nb][s] = x[nb];
      }
    } else {
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        const int c = c0 + nb * 16 + m;
        wf[nb] = c < a.N ? load4(w + (int64_t)c * a.r + j, a.r - j) : f32x4{};
      }
    }
  };
  f32x4 held[kHold ? JB : 1][4];
  if constexpr (kHold)
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) weights(jb, held[jb]);
  float* const my = tile[wave];
  const int blocks = (run.count + 15) / 16;
  for (int rb = 0; rb < blocks; ++rb) {
    f32x4 acc[4] = {};
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) {
      if (jb * 16 >= a.rp) break;
      if constexpr (!kHold) weights(jb, held[0]);
      const f32x4 uf = *(const f32x4*)(u + (rb * 16 + m) * kU + jb * 16 + g * 4);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) acc[nb] = mfma(held[kHold ? jb : 0][nb][s], uf[s], acc[nb]);
    }
    // lane: row m of the block, columns of the instruction's rows 4 g + i
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (FLAT)
        *(f32x4*)(my + m * kTile + 16 * g + 4 * q) = f32x4{acc[0][q], acc[1][q], acc[2][q], acc[3][q]};
      else
        *(f32x4*)(my + m * kTile + 16 * q + 4 * g) = acc[q];
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = rb * 16 + q * 4 + g, c = c0 + 4 * m, n = a.N - c;
      if (t >= run.count || n <= 0) continue;
      const int64_t row = order[t];
      f32x4 y = *(const f32x4*)(my + (q * 4 + g) * kTile + 4 * m);
      if (a.base) y += load4((const O*)a.base + row * a.base_ld + c, n);
      O* dst = (O*)a.out + row * a.out_ld + c;
      if (n >= 4) {
        O z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = narrow<O>(y[e]);
        __builtin_memcpy(dst, z, sizeof(z));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < n) dst[e] = narrow<O>(y[e]);
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
  }
}

struct OuterArgs {
  const void* src;  // [T, N]
  int64_t ld;
  const float* w;   // [T, rp] by place
  int32_t n, r, rp, N;
  float* out;       // [n, N, r], or [n, r, N] where FLAT
  float* part;      // [slots] of the same
  int32_t accumulate;
};

// The sum over a run of rows of src[row][c] w[place][j], for 256 columns.
template <class S, bool FLAT, int JB>
__global__ __launch_bounds__(kThreads) void outer(OuterArgs a, RunList l) {
  if ((int)blockIdx.x >= *l.n_runs) return;
  const Run run = l.runs[blockIdx.x];
  if (run.key >= a.n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c0 = (blockIdx.y * kWaves + wave) * 64, j0 = blockIdx.z * JB * 16;
  if (c0 >= a.N) return;
  const int c = c0 + 4 * m;
  f32x4 acc[JB][4] = {};
  for (int t0 = 0; t0 < run.count; t0 += 4) {
    const int t = t0 + g;
    const bool there = t < run.count;
    const int place = run.first + (there ? t : 0);
    const f32x4 sf = there && c < a.N ? load4((const S*)a.src + l.order[place] * a.ld + c, a.N - c) : f32x4{};
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) {
      const int j = j0 + jb * 16 + m;
      const float wf = there && j < a.r ? a.w[(int64_t)place * a.rp + j] : 0.f;
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
        acc[jb][nb] = FLAT ? mfma(sf[nb], wf, acc[jb][nb]) : mfma(wf, sf[nb], acc[jb][nb]);
    }
  }
  const bool only = run.slot < 0, add = only && a.accumulate;
  float* out = only ? a.out + (int64_t)run.key * a.r * a.N : a.part + (int64_t)run.slot * a.r * a.N;
#pragma unroll
  for (int jb = 0; jb < JB; ++jb)
#pragma unroll
    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = j0 + jb * 16 + (FLAT ? m : 4 * g + i), cc = FLAT ? c0 + 4 * (4 * g + i) + nb : c + nb;
        if (j < a.r && cc < a.N) {
          float* p = out + (FLAT ? (int64_t)j * a.N + cc : (int64_t)cc * a.r + j);
          *p = add ? *p + acc[jb][nb][i] : acc[jb][nb][i];
        }
      }
}

// Adapters of several runs of rows: the runs' sums in order.
__global__ __launch_bounds__(kThreads) void join_outer(const float* part, float* out, int64_t size, int n, int accumulate,
                                                       RunList l) {
  if ((int)blockIdx.x >= *l.n_joins) return;
  const Join j = l.joins[blockIdx.x];
  if (j.key >= n) return;
  for (int64_t i = (int64_t)blockIdx.y * kThreads + threadIdx.x; i < size; i += (int64_t)gridDim.y * kThreads) {
    float s = 0.f;
    for (int p = j.first; p < j.end; p += kGradRows)
      s += part[run_slot(p, kGradRows, p + kGradRows >= j.end) * size + i];
    float* q = out + j.key * size + i;
    *q = accumulate ? *q + s : s;
  }
}

__global__ __launch_bounds__(kThreads) void zero_adapters(float* p, int64_t size, int n, const uint8_t* seen) {
  for (int k = blockIdx.x; k < n; k += gridDim.x) {
    if (seen[k]) continue;
    for (int64_t i = (int64_t)blockIdx.y * kThreads + threadIdx.x; i < size; i += (int64_t)gridDim.y * kThreads)
      p[k * size + i] = 0.f;
  }
}

#define TIM_LAUNCH(...)                      \
  do {                                       \
    __VA_ARGS__;                             \
    const hipError_t e_ = hipGetLastError(); \
    if (e_ != hipSuccess) return e_;         \
  } while (0)

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
template <class T, class G>
hipError_t run_contract(const ContractArgs& a, const RunList& l, int chunks, hipStream_t s) {
  const unsigned runs = (unsigned)l.max_runs;
  if (a.rp <= 16)
    TIM_LAUNCH((contract<T, G, 1><<<dim3(runs, chunks), kThreads, 0, s>>>(a, l)));
  else if (a.rp <= 32)
    TIM_LAUNCH((contract<T, G, 2><<<dim3(runs, chunks), kThreads, 0, s>>>(a, l)));
  else
    TIM_LAUNCH((contract<T, G, 4><<<dim3(runs, chunks, (a.rp + 63) / 64), kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class T, class O, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  const dim3 grid((unsigned)l.max_runs, (unsigned)((a.N + kWaves * 64 - 1) / (kWaves * 64)));
  if (a.rp <= 16)
    TIM_LAUNCH((expand<T, O, FLAT, 1><<<grid, kThreads, 0, s>>>(a, l)));
  else if (a.rp <= 32)
    TIM_LAUNCH((expand<T, O, FLAT, 2><<<grid, kThreads, 0, s>>>(a, l)));
  else if (a.rp <= 64)
    TIM_LAUNCH((expand<T, O, FLAT, 4><<<grid, kThreads, 0, s>>>(a, l)));
  else
    TIM_LAUNCH((expand<T, O, FLAT, 16><<<grid, kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class T, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, int dtype, const RunList& l, hipStream_t s) {
  switch (dtype) {
    case TIM_F32: return run_expand<T, float, FLAT>(a, l, s);
    case TIM_BF16: return run_expand<T, __bf16, FLAT>(a, l, s);
    default: return run_expand<T, _Float16, FLAT>(a, l, s);
  }
}
template <class S, bool FLAT>
hipError_t run_outer(const OuterArgs& a, const RunList& l, hipStream_t s) {
  const unsigned runs = (unsigned)l.max_runs, tiles = (unsigned)((a.N + kWaves * 64 - 1) / (kWaves * 64));
  if (a.rp <= 16)
    TIM_LAUNCH((outer<S, FLAT, 1><<<dim3(runs, tiles), kThreads, 0, s>>>(a, l)));
  else if (a.rp <= 32)
    TIM_LAUNCH((outer<S, FLAT, 2><<<dim3(runs, tiles), kThreads, 0, s>>>(a, l)));
  else
    TIM_LAUNCH((outer<S, FLAT, 4><<<dim3(runs, tiles, (a.rp + 63) / 64), kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class S, bool FLAT>
hipError_t weight_gradient(const OuterArgs& a, const RunList& l, int64_t T, const uint8_t* seen, hipStream_t s) {
  const int64_t size = (int64_t)a.r * a.N;
  const unsigned across = (unsigned)(size < 256 * 1024 ? (size + 255) / 256 : 1024);
  hipError_t e = run_outer<S, FLAT>(a, l, s);
  if (e != hipSuccess) return e;
  if (T > kGradRows)
    TIM_LAUNCH((join_outer<<<dim3((unsigned)l.max_joins, across), kThreads, 0, s>>>(a.part, a.out, size, a.n,
                                                                                    a.accumulate, l)));
  if (!a.accumulate)
    TIM_LAUNCH((zero_adapters<<<dim3((unsigned)(a.n < 1024 ? a.n : 1024), across), kThreads, 0, s>>>(a.out, size, a.n,
                                                                                                     seen)));
  return hipSuccess;
}

template <class T>
hipError_t add_typed(const tim_adapters& ad, const void* x, int64_t x_ld, int64_t n_rows, const void* base,
                     int64_t base_ld, void* out, int out_dtype, int64_t out_ld, const AdapterPlan& p, char* ws,
                     hipStream_t s) {
  const RunList l = run_list(p.g, ws, 0);
  const ShrinkArgs sa = {x, x_ld, n_rows, ad.a, ad.n, ad.r, p.rp, ad.d, (float*)(ws + p.u_part)};
  const hipError_t e = run_shrink<T>(sa, l, p.x_chunks, s);
  if (e != hipSuccess) return e;
  const ExpandArgs ea = {sa.part, n_rows, p.x_chunks, ad.n,    ad.r, p.rp,  ad.N,
                         ad.scales, ad.b,  base,       base_ld, out,  out_ld};
  return run_expand<T, false>(ea, out_dtype, l, s);
}

template <class T, class G>
hipError_t backward_typed(const tim_adapters& ad, const AdapterGradArgs& a, int gx_dtype, const AdapterPlan& p, char* ws,
                          hipStream_t s) {
  const RunList l = run_list(p.g, ws, 0), rows = run_list(p.g, ws, 1);
  float *u = (float*)(ws + p.u), *v = (float*)(ws + p.v);
  const uint8_t* seen = (const uint8_t*)(ws + p.seen);
  hipError_t e;
  if (a.grad_b) {
    const ShrinkArgs sa = {a.x, a.x_ld, a.T, ad.a, ad.n, ad.r, p.rp, ad.d, (float*)(ws + p.u_part)};
    e = run_shrink<T>(sa, l, p.x_chunks, s);
    if (e != hipSuccess) return e;
    TIM_LAUNCH((sum_chunks<<<(unsigned)l.max_runs, kThreads, 0, s>>>(sa.part, a.T, p.rp, p.x_chunks, ad.n, ad.scales, u,
                                                                     l)));
  }
  if (a.grad_x || a.grad_a) {
    const ContractArgs ca = {a.grad, a.grad_ld, a.T, ad.b, ad.n, ad.r, p.rp, ad.N, (float*)(ws + p.v_part)};
    e = run_contract<T, G>(ca, l, p.g_chunks, s);
    if (e != hipSuccess) return e;
    TIM_LAUNCH((sum_chunks<<<(unsigned)l.max_runs, kThreads, 0, s>>>(ca.part, a.T, p.rp, p.g_chunks, ad.n, ad.scales, v,
                                                                     l)));
  }
  if (a.grad_x) {
    const ExpandArgs ea = {v, a.T, 1, ad.n, ad.r, p.rp, ad.d, nullptr, ad.a, a.accumulate_x ? a.grad_x : nullptr,
                           a.gx_ld, a.grad_x, a.gx_ld};
    e = run_expand<T, true>(ea, gx_dtype, l, s);
    if (e != hipSuccess) return e;
  }
  if (a.grad_a) {
    const OuterArgs oa = {a.x, a.x_ld, v, ad.n, ad.r, p.rp, ad.d, a.grad_a, (float*)(ws + p.a_part), a.accumulate_ab};
    e = weight_gradient<T, true>(oa, rows, a.T, seen, s);
    if (e != hipSuccess) return e;
  }
  if (a.grad_b) {
    const OuterArgs oa = {a.grad, a.grad_ld, u, ad.n, ad.r, p.rp, ad.N, a.grad_b, (float*)(ws + p.b_part),
                          a.accumulate_ab};
    e = weight_gradient<G, false>(oa, rows, a.T, seen, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class T>
hipError_t backward_grad(const tim_adapters& ad, const AdapterGradArgs& a, int grad_dtype, int gx_dtype,
                         const AdapterPlan& p, char* ws, hipStream_t s) {
  switch (grad_dtype) {
    case TIM_F32: return backward_typed<T, float>(ad, a, gx_dtype, p, ws, s);
    case TIM_BF16: return backward_typed<T, __bf16>(ad, a, gx_dtype, p, ws, s);
    default: return backward_typed<T, _Float16>(ad, a, gx_dtype, p, ws, s);
  }
}

}  // namespace

hipError_t launch_adapters_add(const tim_adapters& ad, const void* x, int64_t x_ld, const int32_t* rows, int64_t T,
                               const void* base, int64_t base_ld, void* out, int out_dtype, int64_t out_ld, void* ws,
                               hipStream_t s) {
  const AdapterPlan p = plan_adapters(T, ad.d, ad.N, ad.n, ad.r, false);
  const hipError_t e = launch_grouping(p.g, rows, true, nullptr, ws, s);
  if (e != hipSuccess) return e;
  if (ad.dtype == TIM_BF16)
    return add_typed<__bf16>(ad, x, x_ld, T, base, base_ld, out, out_dtype, out_ld, p, (char*)ws, s);
  return add_typed<_Float16>(ad, x, x_ld, T, base, base_ld, out, out_dtype, out_ld, p, (char*)ws, s);
}

hipError_t launch_adapters_backward(const tim_adapters& ad, const AdapterGradArgs& a, int grad_dtype, int gx_dtype,
                                    void* ws, hipStream_t s) {
  const AdapterPlan p = plan_adapters(a.T, ad.d, ad.N, ad.n, ad.r, true);
  const hipError_t e = launch_grouping(p.g, a.rows, true, (uint8_t*)ws + p.seen, ws, s);
  if (e != hipSuccess) return e;
  if (ad.dtype == TIM_BF16) return backward_grad<__bf16>(ad, a, grad_dtype, gx_dtype, p, (char*)ws, s);
  return backward_grad<_Float16>(ad, a, grad_dtype, gx_dtype, p, (char*)ws, s);
}

}  // namespace tim
