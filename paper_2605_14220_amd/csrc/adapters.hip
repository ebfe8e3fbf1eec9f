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
// The same where all N elements are known to lie in the array: without the
// branches, so that many loads are in flight at once. WHOLE picks one by a
// condition that is the same in every lane.
template <bool WHOLE, class V, int N, class T>
__device__ __forceinline__ V load_n(const T* p, int n) {
  if constexpr (WHOLE) {
    V r;
    __builtin_memcpy(&r, p, N * sizeof(T));
    return r;
  } else {
    return load_some<V, N>(p, n);
  }
}
template <class T>
using x4 = T __attribute__((ext_vector_type(4)));
// A wave's results of JB blocks of 16 ranks for RB blocks of 16 rows, summed
// over the workgroup's waves in wave order and stored as part[place][rank], zeros
// for the ranks from r on.
template <int JB>
__device__ __forceinline__ void store_sums(f32x4 (&acc)[JB][4], f32x4 (*lds)[JB][4][64], float* part, int r, int rp,
                                           int j0, int count, int lane, int wave) {
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
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e >= r) s[e] = 0.f;
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
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0 || run.key >= a.n) return;
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
  const T* wr[JB];
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int j = j0 + jb * 16 + m;
    wr[jb] = w + (int64_t)(j < a.r ? j : a.r - 1) * a.d;
  }
  f32x4 acc[JB][4] = {};
  constexpr int kEach = kShrinkChunk / kWaves;
  const int from = at.tile * kShrinkChunk + wave * kEach;
  auto step = [&](auto whole, int k0) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int k = k0 + g * 8, n = a.d - k;
    x8<T> wf[JB], xf[4];
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) wf[jb] = load_n<WHOLE, x8<T>, 8>(wr[jb] + k, n);
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks) xf[rb] = load_n<WHOLE, x8<T>, 8>(xr[rb] + k, n);
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[jb][rb] = mfma(wf[jb], xf[rb], acc[jb][rb]);
  };
  if (from + kEach <= a.d) {
#pragma unroll 4
    for (int k0 = 0; k0 < kEach; k0 += 32) step(std::true_type{}, from + k0);
  } else {
    for (int k0 = from; k0 < a.d && k0 < from + kEach; k0 += 32) step(std::false_type{}, k0);
  }
  store_sums<JB>(acc, lds, a.part + ((int64_t)at.tile * a.T + run.first) * a.rp, a.r, a.rp, j0, run.count, lane, wave);
}

// out[place][j] = scale of the place's adapter * the sum of its chunks: in order
// over `inner` chunks (1 or 2), then a sixteenth of these sums a group of 16 lanes, each
// in order, then the groups in order. 64 consecutive elements a workgroup.
__global__ __launch_bounds__(kThreads) void sum_chunks(const float* part, int64_t T, int rp, int chunks, int inner, int n,
                                                       const float* scales, float* out, RunList l) {
  __shared__ f32x4 lds[16][16];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0) return;
  const int i = ((int)at.tile * 16 + (int)threadIdx.x % 16) * 4, group = threadIdx.x / 16;
  if (run.key >= n || (int)at.tile * 64 >= run.count * rp) return;
  const int outer = (chunks + inner - 1) / inner, per = (outer + 15) / 16 * inner;
  const int from = group * per, to = from + per < chunks ? from + per : chunks;
  const float* p = part + (int64_t)run.first * rp + i;
  const int64_t step = T * rp;
  f32x4 s = {};
  if (i < run.count * rp) {
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
  if (group > 0 || i >= run.count * rp) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x];
  *(f32x4*)(out + (int64_t)run.first * rp + i) = s * (scales ? scales[run.key] : 1.f);
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

// out[row][c] = base[row][c] + sum_j u[place][j] w[c][j] for the rows of a run and
// NT tiles of 64 columns a wave. The waves work by themselves: u and the first
// tile's weights and rows of base are requested together, later ones a step
// (16 rows of a tile) ahead, before the step's stores. The matrix instructions'
// results pass through LDS, so that rows are read and written 64 columns at a time.
template <class T, class O, bool FLAT, int JB, int NT>
__global__ __launch_bounds__(kThreads) void expand(ExpandArgs a, RunList l) {
  constexpr int kTile = 64 + 4;    // a row of the 16 x 64 results
  constexpr bool kHold = JB <= 4;  // u and a tile's weights stay in registers for all rows
  __shared__ float tile[kWaves][16 * kTile];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c_first = (at.tile * kWaves + wave) * NT * 64;
  if (c_first >= a.N) return;
  const int my_row = l.order[run.first + (lane < run.count ? lane : run.count - 1)];  // of the run's row `lane`
  const O* base = (const O*)a.base;
  if (run.key >= a.n) {  // no adapter
    for (int t = 0; t < run.count; ++t) {
      const int64_t row = __shfl(my_row, t);
      for (int c = c_first + lane; c < a.N && c < c_first + NT * 64; c += 64)
        ((O*)a.out)[row * a.out_ld + c] = base ? base[row * a.base_ld + c] : (O)0.f;
    }
    return;
  }
  const int blocks = (run.count + 15) / 16, tiles = (a.N - c_first + 63) / 64 < NT ? (a.N - c_first + 63) / 64 : NT;
  const T* w = (const T*)a.w + (int64_t)run.key * a.r * a.N;
  // raw[nb][s]: the weight of rank jb * 16 + 4 g + s in column c0 + 16 nb + m; FLAT: raw[s][nb] in column c0 + 4 m + nb.
  // Without FLAT the four ranks may reach into the next columns' weights (up to 15 columns on): zeros take their place.
  auto weights = [&](int c0, int jb, x4<T>(&raw)[4]) {
    const int j = jb * 16 + g * 4;
    if (c0 + 64 + (FLAT ? 0 : 16) <= a.N) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        raw[q] = FLAT ? load_n<true, x4<T>, 4>(w + (int64_t)(j + q < a.r ? j + q : a.r - 1) * a.N + c0 + 4 * m, 4)
                      : load_n<true, x4<T>, 4>(w + (int64_t)(c0 + q * 16 + m) * a.r + j, 4);
      if (a.r != a.rp) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int s = 0; s < 4; ++s)
            if (j + (FLAT ? q : s) >= a.r) raw[q][s] = (T)0.f;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = FLAT ? c0 + 4 * m : c0 + q * 16 + m;
        raw[q] = x4<T>{};
        if (FLAT && j + q < a.r) raw[q] = load_some<x4<T>, 4>(w + (int64_t)(j + q) * a.N + c, a.N - c);
        if (!FLAT && c < a.N) raw[q] = load_some<x4<T>, 4>(w + (int64_t)c * a.r + j, a.r - j);
      }
    }
  };
  const float scale = a.scales ? a.scales[run.key] : 1.f;
  // row m of a block, ranks jb * 16 + 4 g on
  auto load_u = [&](int rb, int jb) {
    const int t = rb * 16 + m < run.count ? rb * 16 + m : run.count - 1;
    const float* p = a.u + ((int64_t)run.first + t) * a.rp + jb * 16 + g * 4;
    f32x4 s = *(const f32x4*)p;
#pragma unroll 4
    for (int c = 1; c < a.chunks; ++c) s += *(const f32x4*)(p + (int64_t)c * a.T * a.rp);
    return s * scale;
  };
  x4<T> raw[kHold ? JB : 1][4];
  x4<O> old[4];
  // what lane (m, g) reads and writes of a step: row 4 q + g, columns 4 m .. 4 m + 3
  auto load_base = [&](int c0, int rb) {
    const int c = c0 + 4 * m;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = rb * 16 + q * 4;
      if (t >= run.count) break;
      const O* p = base + __shfl(my_row, t + g) * a.base_ld + c;
      old[q] = c0 + 64 <= a.N ? load_n<true, x4<O>, 4>(p, 4) : load_some<x4<O>, 4>(p, a.N - c);
    }
  };
  if constexpr (kHold)
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) weights(c_first, jb, raw[jb]);
  if (base) load_base(c_first, 0);
  f32x4 u[kHold ? 4 : 1][kHold ? JB : 1];
  if constexpr (kHold)
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) u[rb][jb] = jb * 16 < a.rp ? load_u(rb, jb) : f32x4{};
  float* const my = tile[wave];
  for (int ct = 0; ct < tiles; ++ct) {
    const int c0 = c_first + ct * 64;
    f32x4 wf[kHold ? JB : 1][4];
    auto widen = [&](int k) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int s = 0; s < 4; ++s) wf[k][q][s] = (float)raw[k][q][s];
    };
    if constexpr (kHold) {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) widen(jb);
      if (ct + 1 < tiles)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) weights(c0 + 64, jb, raw[jb]);
    }
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      if (rb >= blocks) break;
      f32x4 acc[4] = {};
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) {
        if (jb * 16 >= a.rp) break;
        if constexpr (!kHold) {
          weights(c0, jb, raw[0]);
          widen(0);
          u[0][0] = load_u(rb, jb);
        }
        const f32x4 uf = u[kHold ? rb : 0][kHold ? jb : 0];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int nb = 0; nb < 4; ++nb) {
            const f32x4(&h)[4] = wf[kHold ? jb : 0];
            acc[nb] = mfma(FLAT ? h[s][nb] : h[nb][s], uf[s], acc[nb]);
          }
      }
      // lane: row m of the block, columns of the instruction's rows 4 g + i
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (FLAT)
          *(f32x4*)(my + m * kTile + 16 * g + 4 * q) = f32x4{acc[0][q], acc[1][q], acc[2][q], acc[3][q]};
        else
          *(f32x4*)(my + m * kTile + 16 * q + 4 * g) = acc[q];
      }
      lanes_in_order();
      f32x4 y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        y[q] = *(const f32x4*)(my + (q * 4 + g) * kTile + 4 * m);
        if (base) y[q] += f32x4{(float)old[q][0], (float)old[q][1], (float)old[q][2], (float)old[q][3]};
      }
      lanes_in_order();
      if (base) {
        if (rb + 1 < blocks)
          load_base(c0, rb + 1);
        else if (ct + 1 < tiles)
          load_base(c0 + 64, 0);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (rb * 16 + q * 4 >= run.count) break;
        const int t = rb * 16 + q * 4 + g, c = c0 + 4 * m, n = a.N - c;
        const int64_t row = __shfl(my_row, t);
        if (t >= run.count || n <= 0) continue;
        O* dst = (O*)a.out + row * a.out_ld + c;
        x4<O> z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = narrow<O>(y[q][e]);
        if (n >= 4) {
          __builtin_memcpy(dst, &z, sizeof(z));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n) dst[e] = z[e];
        }
      }
    }
  }
}

struct PassArgs {
  const void* src;  // [T, N]
  int64_t ld, T;
  const float* w;   // [T, rp] by place
  const void* b;    // [n, N, r], the contraction's
  float* part;      // [chunks, T, rp], the contraction's sums
  int32_t n, r, rp, N;
  float* out;       // [n, N, r], or [n, r, N] without the contraction
  float* out_part;  // [slots] of the same
  int32_t accumulate;
};

// One pass over the columns of src = grad: for a run of one adapter's rows and
// CT * 256 columns
//   out[c][j]      sum over the rows of src[row][c] w[place][j]
//   part[place][j] sum over the columns of src[row][c] b[c][j]    (CONTRACT)
// and without the contraction the first alone, [j][c], of src = x.
//
// 64 rows of 256 columns at a time lie in LDS, read from memory once, and are
// read from there along the rows for one product and along the columns for the
// other. A wave takes 64 columns of the first and 16 rows of the second.
//
// FAST, where all is bf16: both on the bf16 matrix instructions, w as the sum of
// three bf16 numbers, which holds all of its 24 bits. Otherwise on the fp32 ones.
constexpr int kPassRows = 64;
template <class S, class W, bool CONTRACT, int JB, int CT>
struct Pass {
  static constexpr bool FAST = std::is_same_v<S, __bf16> && std::is_same_v<W, __bf16>;
  typedef std::conditional_t<FAST, __bf16, float> E;  // of the tile and of w in LDS
  static constexpr int kTerms = FAST ? 3 : 1;
  static constexpr int kPad = 16 / (int)sizeof(E);
  static constexpr int kRow = kPassCols + kPad;  // elements from row to row of the tile
  static constexpr int kW = kPassRows + kPad;    // of w, [term][j][row]
  static constexpr int kB = CT * kPassCols + 8;  // of b, [j][c]
  static constexpr int kLoads = kPassRows * kPassCols * (int)sizeof(S) / 16 / kThreads;  // 16 bytes a thread
  static constexpr int kV = 16 / (int)sizeof(S);
};
template <class S, class W, bool CONTRACT, int JB, int CT>
__global__ __launch_bounds__(kThreads) void pass(PassArgs a, RunList l) {
  typedef Pass<S, W, CONTRACT, JB, CT> P;
  typedef typename P::E E;
  typedef S sv __attribute__((ext_vector_type(P::kV)));
  typedef E ev __attribute__((ext_vector_type(P::kV)));
  __shared__ __attribute__((aligned(16))) E tile[kPassRows * P::kRow];
  __shared__ __attribute__((aligned(16))) E wt[P::kTerms * JB * 16 * P::kW];
  __shared__ __attribute__((aligned(16))) W bt[CONTRACT ? JB * 16 * P::kB : 1];
  __shared__ int32_t rows[kMaxPassRows];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0 || run.key >= a.n) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane % 16, g = lane / 16;
  const int c_first = at.tile * CT * kPassCols, j0 = blockIdx.z * JB * 16;
  const int tiles = (a.N - c_first + kPassCols - 1) / kPassCols < CT ? (a.N - c_first + kPassCols - 1) / kPassCols : CT;
  const int32_t* order = l.order + run.first;
  const float* w = a.w + (int64_t)run.first * a.rp + j0;

  // rows past the run's end, up to a whole tile, are read as its last one
  for (int t = tid; t < (run.count + kPassRows - 1) / kPassRows * kPassRows; t += kThreads)
    rows[t] = order[t < run.count ? t : run.count - 1];
  if constexpr (CONTRACT) {
    // a thread takes 8 ranks of a column; the loads first, then their way into LDS
    constexpr int kEach = JB * 16 * CT * kPassCols / 8 / kThreads;
    const W* b = (const W*)a.b + ((int64_t)run.key * a.N + c_first) * a.r + j0;
    x8<W> x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = tid + k * kThreads, j = i % (JB * 2) * 8, c = i / (JB * 2);
      x[k] = c_first + c < a.N ? load_some<x8<W>, 8>(b + (int64_t)c * a.r + j, a.r - j0 - j) : x8<W>{};
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = tid + k * kThreads, j = i % (JB * 2) * 8, c = i / (JB * 2);
#pragma unroll
      for (int e = 0; e < 8; ++e) bt[(j + e) * P::kB + c] = x[k][e];
    }
  }
  __syncthreads();  // rows

  // the tile's loads: thread t takes column group t % kAcross of the rows t / kAcross + k * kDown
  constexpr int kAcross = kPassCols / P::kV, kDown = kThreads / kAcross;
  sv held[P::kLoads];
  f32x4 held_w[JB];
  const int lc = tid % kAcross * P::kV, lr = tid / kAcross;
  auto load_tile = [&](int t0, int ct) {
    const int c = c_first + ct * kPassCols + lc;
    const S* src = (const S*)a.src + c;
    if (c_first + (ct + 1) * kPassCols <= a.N) {
#pragma unroll
      for (int k = 0; k < P::kLoads; ++k) held[k] = load_n<true, sv, P::kV>(src + rows[t0 + lr + k * kDown] * a.ld, 0);
    } else {
#pragma unroll
      for (int k = 0; k < P::kLoads; ++k)
        held[k] = load_some<sv, P::kV>(src + rows[t0 + lr + k * kDown] * a.ld, a.N - c);
    }
    if (ct == 0) {
      const int t = t0 + lane;
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) {
        const int j = jb * 16 + wave * 4;
        held_w[jb] = a.w && t < run.count && j0 + j < a.rp ? *(const f32x4*)(w + (int64_t)t * a.rp + j) : f32x4{};
      }
    }
  };
  auto store_tile = [&](int t0, int ct) {
    if (t0 + kPassRows > run.count) {  // rows past the run's end
#pragma unroll
      for (int k = 0; k < P::kLoads; ++k)
        if (t0 + lr + k * kDown >= run.count) held[k] = sv{};
    }
#pragma unroll
    for (int k = 0; k < P::kLoads; ++k) {
      ev x;
#pragma unroll
      for (int e = 0; e < P::kV; ++e) x[e] = (E)held[k][e];
      *(ev*)(tile + (lr + k * kDown) * P::kRow + lc) = x;
    }
    if (ct == 0) {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int to = (jb * 16 + wave * 4 + e) * P::kW + lane;
          const float x = held_w[jb][e];
          if constexpr (P::FAST) {
            const __bf16 hi = (__bf16)x;
            const bool finite = __builtin_isfinite((float)hi);
            const float r1 = finite ? x - (float)hi : 0.f;
            const __bf16 mid = (__bf16)r1;
            wt[to] = hi;
            wt[JB * 16 * P::kW + to] = mid;
            wt[2 * JB * 16 * P::kW + to] = (__bf16)(r1 - (float)mid);
          } else {
            wt[to] = x;
          }
        }
    }
  };

  f32x4 acc[CT][JB][4] = {};  // out
  f32x4 total[JB];            // part, over the tiles so far
  auto add_up = [](f32x4(&total)[JB], const f32x4(&sum)[JB], int ct) {
#pragma unroll
    for (int jb = 0; jb < JB; ++jb) total[jb] = ct == 0 ? sum[jb] : total[jb] + sum[jb];
  };
  load_tile(0, 0);
  for (int t0 = 0; t0 < run.count; t0 += kPassRows) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      if (ct >= tiles) break;
      __syncthreads();
      store_tile(t0, ct);
      __syncthreads();
      if (ct + 1 < tiles)
        load_tile(t0, ct + 1);
      else if (t0 + kPassRows < run.count)
        load_tile(t0 + kPassRows, 0);
      if constexpr (P::FAST) {
#pragma unroll
        for (int ks = 0; ks < kPassRows / 32; ++ks) {
          x4<E> x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = *(const x4<E>*)(tile + (ks * 32 + g * 8 + e) * P::kRow + wave * 64 + 4 * m);
          bf16x8 f[4];
#pragma unroll
          for (int nb = 0; nb < 4; ++nb)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[nb][e] = x[e][nb];
#pragma unroll
          for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int q = 0; q < 3; ++q) {
              const bf16x8 wf = *(const bf16x8*)(wt + ((q * JB + jb) * 16 + m) * P::kW + ks * 32 + g * 8);
#pragma unroll
              for (int nb = 0; nb < 4; ++nb)
                acc[ct][jb][nb] = CONTRACT ? mfma(wf, f[nb], acc[ct][jb][nb]) : mfma(f[nb], wf, acc[ct][jb][nb]);
            }
        }
        if constexpr (CONTRACT) {
          f32x4 sum[JB] = {};
#pragma unroll
          for (int ks = 0; ks < kPassCols / 32; ++ks) {
            const bf16x8 x = *(const bf16x8*)(tile + (wave * 16 + m) * P::kRow + ks * 32 + g * 8);
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
              sum[jb] = mfma(*(const bf16x8*)(bt + (jb * 16 + m) * P::kB + ct * kPassCols + ks * 32 + g * 8), x, sum[jb]);
          }
          add_up(total, sum, ct);
        }
      } else {
#pragma unroll 4
        for (int q = 0; q < kPassRows / 4; ++q) {
          const f32x4 x = *(const f32x4*)(tile + (q * 4 + g) * P::kRow + wave * 64 + 4 * m);
#pragma unroll
          for (int jb = 0; jb < JB; ++jb) {
            const float wf = wt[(jb * 16 + m) * P::kW + q * 4 + g];
#pragma unroll
            for (int nb = 0; nb < 4; ++nb)
              acc[ct][jb][nb] = CONTRACT ? mfma(wf, x[nb], acc[ct][jb][nb]) : mfma(x[nb], wf, acc[ct][jb][nb]);
          }
        }
        if constexpr (CONTRACT) {
          f32x4 sum[JB] = {};
#pragma unroll 4
          for (int ks = 0; ks < kPassCols / 16; ++ks) {
            const f32x4 x = *(const f32x4*)(tile + (wave * 16 + m) * P::kRow + ks * 16 + g * 4);
#pragma unroll
            for (int jb = 0; jb < JB; ++jb) {
              const x4<W> bf = *(const x4<W>*)(bt + (jb * 16 + m) * P::kB + ct * kPassCols + ks * 16 + g * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) sum[jb] = mfma((float)bf[e], x[e], sum[jb]);
            }
          }
          add_up(total, sum, ct);
        }
      }
    }
    if constexpr (CONTRACT) {
      const int t = t0 + wave * 16 + m;
      float* p = a.part + ((int64_t)at.tile * a.T + run.first + t) * a.rp + j0 + g * 4;
#pragma unroll
      for (int jb = 0; jb < JB; ++jb)
        if (t < run.count && j0 + jb * 16 < a.rp) *(f32x4*)(p + jb * 16) = total[jb];
    }
  }

  if (!a.out) return;
  const bool only = run.slot < 0, add = only && a.accumulate;
  float* out = only ? a.out + (int64_t)run.key * a.r * a.N : a.out_part + (int64_t)run.slot * a.r * a.N;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int jb = 0; jb < JB; ++jb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // four elements next to each other in memory: of the rank, or of the columns
        const int c0 = c_first + ct * kPassCols + wave * 64;
        const int j = j0 + jb * 16 + (CONTRACT ? 4 * g : m), c = c0 + (CONTRACT ? 4 * m + q : 16 * g + 4 * q);
        if (j >= a.r || c >= a.N) continue;
        const f32x4 y = CONTRACT ? acc[ct][jb][q]
                                 : f32x4{acc[ct][jb][0][q], acc[ct][jb][1][q], acc[ct][jb][2][q], acc[ct][jb][3][q]};
        float* p = out + (CONTRACT ? (int64_t)c * a.r + j : (int64_t)j * a.N + c);
        const int left = CONTRACT ? a.r - j : a.N - c;
        if (left >= 4) {
          f32x4 z = y;
          if (add) z = load_n<true, f32x4, 4>(p, 4) + y;
          __builtin_memcpy(p, &z, sizeof(z));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = add ? p[e] + y[e] : y[e];
        }
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
template <class T, class O, bool FLAT, int JB, int NT>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, NT * kWaves * 64));
  TIM_LAUNCH((expand<T, O, FLAT, JB, NT><<<grid, kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class T, class O, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  // a wave takes four tiles where that leaves 16 waves for each of 256 CUs
  const bool many = l.max_runs * chunks_of(a.N, 4 * 64) >= 4096;
  if (a.rp <= 16) return many ? run_expand<T, O, FLAT, 1, 4>(a, l, s) : run_expand<T, O, FLAT, 1, 1>(a, l, s);
  if (a.rp <= 32) return many ? run_expand<T, O, FLAT, 2, 4>(a, l, s) : run_expand<T, O, FLAT, 2, 1>(a, l, s);
  if (a.rp <= 64) return run_expand<T, O, FLAT, 4, 1>(a, l, s);
  return run_expand<T, O, FLAT, 16, 1>(a, l, s);
}
template <class T, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, int dtype, const RunList& l, hipStream_t s) {
  switch (dtype) {
    case TIM_F32: return run_expand<T, float, FLAT>(a, l, s);
    case TIM_BF16: return run_expand<T, __bf16, FLAT>(a, l, s);
    default: return run_expand<T, _Float16, FLAT>(a, l, s);
  }
}
template <class S, class W, bool CONTRACT, int JB, int CT>
hipError_t run_pass(const PassArgs& a, const RunList& l, hipStream_t s) {
  const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, CT * kPassCols), (unsigned)((a.rp + 63) / 64));
  TIM_LAUNCH((pass<S, W, CONTRACT, JB, CT><<<grid, kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class S, class W, bool CONTRACT>
hipError_t run_pass(const PassArgs& a, int tiles, const RunList& l, hipStream_t s) {
  if (a.rp <= 16) {
    if constexpr (CONTRACT)
      if (tiles == 2) return run_pass<S, W, CONTRACT, 1, 2>(a, l, s);
    return run_pass<S, W, CONTRACT, 1, 1>(a, l, s);
  }
  if (a.rp <= 32) {
    if constexpr (CONTRACT)
      if (tiles == 2) return run_pass<S, W, CONTRACT, 2, 2>(a, l, s);
    return run_pass<S, W, CONTRACT, 2, 1>(a, l, s);
  }
  return run_pass<S, W, CONTRACT, 4, 1>(a, l, s);
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
  const RunList l = run_list(p.g, ws, 0), la = run_list(p.g, ws, 1), lb = run_list(p.g, ws, 2);
  float *u = (float*)(ws + p.u), *v = (float*)(ws + p.v);
  hipError_t e;
  if (a.grad_b) {
    const ShrinkArgs sa = {a.x, a.x_ld, a.T, ad.a, ad.n, ad.r, p.rp, ad.d, (float*)(ws + p.u_part)};
    e = run_shrink<T>(sa, l, p.x_chunks, s);
    if (e != hipSuccess) return e;
    TIM_LAUNCH((sum_chunks<<<dim3((unsigned)l.max_runs, p.rp), kThreads, 0, s>>>(sa.part, a.T, p.rp, p.x_chunks, 1, ad.n, ad.scales, u,
                                                                     l)));
  } else {
    u = nullptr;
  }
  const PassArgs pb = {a.grad, a.grad_ld, a.T,      u,    ad.b, (float*)(ws + p.v_part),   ad.n,
                       ad.r,   p.rp,      ad.N,     a.grad_b, (float*)(ws + p.b_part), a.accumulate_ab};
  e = run_pass<G, T, true>(pb, p.of_grad.tiles, lb, s);
  if (e != hipSuccess) return e;
  if (a.grad_x || a.grad_a)
    TIM_LAUNCH((sum_chunks<<<dim3((unsigned)l.max_runs, p.rp), kThreads, 0, s>>>(pb.part, a.T, p.rp, p.g_chunks,
                                                                                 kChunkPair / p.of_grad.tiles, ad.n,
                                                                                 ad.scales, v, l)));
  if (a.grad_x) {
    const ExpandArgs ea = {v, a.T, 1, ad.n, ad.r, p.rp, ad.d, nullptr, ad.a, a.accumulate_x ? a.grad_x : nullptr,
                           a.gx_ld, a.grad_x, a.gx_ld};
    e = run_expand<T, true>(ea, gx_dtype, l, s);
    if (e != hipSuccess) return e;
  }
  float* a_part = (float*)(ws + p.a_part);
  if (a.grad_a) {
    const PassArgs pa = {a.x,  a.x_ld, a.T,  v,        nullptr, nullptr,        ad.n,
                         ad.r, p.rp,   ad.d, a.grad_a, a_part,  a.accumulate_ab};
    e = run_pass<T, T, false>(pa, 1, la, s);
    if (e != hipSuccess) return e;
  }
  if (!a.grad_a && !a.grad_b) return hipSuccess;
  FinishArgs f = {{a_part, pb.out_part},
                  {a.grad_a, a.grad_b},
                  {(int64_t)ad.r * ad.d, (int64_t)ad.r * ad.N},
                  {p.of_x.log_rows, p.of_grad.log_rows},
                  {la, lb},
                  ad.n,
                  0,
                  a.accumulate_ab,
                  (const uint8_t*)(ws + p.seen)};
  f.joins = (int)(la.max_joins > lb.max_joins ? la.max_joins : lb.max_joins);
  const int zeros = a.accumulate_ab ? 0 : ad.n < 1024 ? ad.n : 1024;
  const int64_t most = f.size[0] > f.size[1] ? f.size[0] : f.size[1];
  const unsigned across = (unsigned)(most < 512 * kThreads ? (most + kThreads - 1) / kThreads : 512);
  if (f.joins + zeros > 0) TIM_LAUNCH((finish<<<dim3(f.joins + zeros, across, 2), kThreads, 0, s>>>(f)));
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
