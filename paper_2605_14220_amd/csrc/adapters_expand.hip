// Adapters: the product that ends in rows of N (or d) elements, out = base + u w^T.

#include <hip/hip_runtime.h>

#include "adapters.h"

namespace tim {
namespace {

// out[row][c] = base[row][c] + sum_j u[row][j] w[c][j] for the rows of a run and
// nt tiles of 64 columns a wave. The waves work by themselves: u and the first
// tile's weights and rows of base are requested together, later ones a step
// (16 rows of a tile) ahead, before the step's stores. The matrix instructions'
// results pass through LDS, so that rows are read and written 64 columns at a time.
template <class T, class O, bool FLAT, int JB>
__global__ __launch_bounds__(kThreads) void expand(ExpandArgs a, RunList l, int nt) {
  constexpr int kTile = 64 + 4;    // a row of the 16 x 64 results
  constexpr bool kHold = JB <= 4;  // u and a tile's weights stay in registers for all rows
  __shared__ float tile[kWaves][16 * kTile];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c_first = (at.tile * kWaves + wave) * nt * 64;
  if (c_first >= a.N) return;
  const int my_row = l.order[run.first + (lane < run.count ? lane : run.count - 1)];  // of the run's row `lane`
  const O* base = (const O*)a.base;
  if (run.key >= a.n) {  // no adapter
    for (int t = 0; t < run.count; ++t) {
      const int64_t row = __shfl(my_row, t);
      for (int c = c_first + lane; c < a.N && c < c_first + nt * 64; c += 64)
        ((O*)a.out)[row * a.out_ld + c] = base ? base[row * a.base_ld + c] : (O)0.f;
    }
    return;
  }
  const int blocks = (run.count + 15) / 16, tiles = (a.N - c_first + 63) / 64 < nt ? (a.N - c_first + 63) / 64 : nt;
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
    const float* p = a.u + (int64_t)__shfl(my_row, rb * 16 + m) * a.rp + jb * 16 + g * 4;
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

template <class T, class O, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  // a wave takes four tiles where that leaves 16 waves for each of 256 CUs (48 rows of 32 adapters at d = 5120 on a
  // head of 152064: 80 us against 95), of a high rank always one (its weights and rows of u fill the registers)
  const int nt = a.rp <= 32 && l.max_runs * chunks_of(a.N, 4 * 64) >= 4096 ? 4 : 1;
  const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, nt * kWaves * 64));
  if (a.rp <= 16)
    TIM_LAUNCH((expand<T, O, FLAT, 1><<<grid, kThreads, 0, s>>>(a, l, nt)));
  else if (a.rp <= 32)
    TIM_LAUNCH((expand<T, O, FLAT, 2><<<grid, kThreads, 0, s>>>(a, l, nt)));
  else if (a.rp <= 64)
    TIM_LAUNCH((expand<T, O, FLAT, 4><<<grid, kThreads, 0, s>>>(a, l, nt)));
  else
    TIM_LAUNCH((expand<T, O, FLAT, 16><<<grid, kThreads, 0, s>>>(a, l, nt)));
  return hipSuccess;
}
template <class T, class O>
hipError_t run_expand(const ExpandArgs& a, bool flat, const RunList& l, hipStream_t s) {
  return flat ? run_expand<T, O, true>(a, l, s) : run_expand<T, O, false>(a, l, s);
}
template <class T>
hipError_t run_expand(const ExpandArgs& a, int out_dtype, bool flat, const RunList& l, hipStream_t s) {
  switch (out_dtype) {
    case TIM_F32: return run_expand<T, float>(a, flat, l, s);
    case TIM_BF16: return run_expand<T, __bf16>(a, flat, l, s);
    default: return run_expand<T, _Float16>(a, flat, l, s);
  }
}

}  // namespace

hipError_t launch_expand(const ExpandArgs& a, int dtype, int out_dtype, bool flat, const RunList& l, hipStream_t s) {
  return dtype == TIM_BF16 ? run_expand<__bf16>(a, out_dtype, flat, l, s)
                           : run_expand<_Float16>(a, out_dtype, flat, l, s);
}

}  // namespace tim
