// Adapters: the product that ends in rows of N (or d) elements, out = base + u w^T.

#include <hip/hip_runtime.h>

#include "adapters.h"

namespace tim {
namespace {

// out[row][c] = base[row][c] + sum_j u[row][j] w[c][j] for the rows of a run and
// 64 columns a wave. Weights and the first rows of base are requested beside u,
// later rows of base a step (16 rows of a tile) ahead, before the step's stores.
// The matrix instructions' results pass through LDS, so that rows are read and
// written 64 columns at a time. Memory bounds it: 4096 rows on a head of 151936
// (rank 16, fp32) take 895 us, 5.6 TB/s.
//
// The four waves share u in LDS, where its partial sums are added up once (200
// rows of 8 adapters of rank 64, d = N = 4096: 25 us a call, 30 with each wave's
// own). AHEAD: a wave takes 4 / JB tiles, all their weights requested first.
// Registers for four workgroups a CU where nothing spills (333 rows, d 1536, N
// 50257, rank 9, fp16: 29 us against 31).
template <class T, class O, bool FLAT, int JB, bool AHEAD>
__global__ __launch_bounds__(kThreads, !AHEAD && JB <= 2 ? 4 : 1) void expand(ExpandArgs a, RunList l) {
  constexpr int kTile = 64 + 4;    // a row of the 16 x 64 results
  constexpr bool kHold = JB <= 4;  // a tile's weights stay in registers for all rows
  constexpr int NT = AHEAD ? 4 / JB : 1;
  // Four ranks of a row of u: on the bf16 instructions three terms, which hold all 24 bits, a third of the time of the
  // fp32 instructions (fp16's range does not hold such terms).
  constexpr bool FAST = std::is_same_v<T, __bf16>;
  typedef std::conditional_t<FAST, bf16x4, f32x4> U;
  constexpr int kTerms = FAST ? 3 : 1;
  constexpr int kU = JB * 4 * kTerms + 1;  // of them, a row in LDS, apart in the banks
  __shared__ float tile[kWaves][16 * kTile];
  __shared__ U shared_u[64 * kU];
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c_first = (at.tile * kWaves + wave) * NT * 64;
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
  // four ranks from j on of the run's row t
  auto load_u = [&](int t, int j) {
    const float* p = a.u + (int64_t)__shfl(my_row, t) * a.rp + j;
    f32x4 s = *(const f32x4*)p;
#pragma unroll 8
    for (int c = 1; c < a.chunks; ++c) s += *(const f32x4*)(p + (int64_t)c * a.T * a.rp);
    return s * scale;
  };
  x4<T> raw[NT][kHold ? JB : 1][4];
  x4<O> old[4];
  // what lane (m, g) reads and writes of a step: row 4 q + g, columns 4 m .. 4 m + 3; with one block the same rows in every
  // tile
  int32_t only[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) only[q] = __shfl(my_row, 4 * q + g);
  auto row_of = [&](int rb, int q) { return blocks == 1 ? only[q] : __shfl(my_row, rb * 16 + q * 4 + g); };
  auto load_base = [&](int c0, int rb) {
    const int c = c0 + 4 * m;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = rb * 16 + q * 4;
      if (t >= run.count) break;
      const O* p = base + row_of(rb, q) * a.base_ld + c;
      old[q] = c0 + 64 <= a.N ? load_n<true, x4<O>, 4>(p, 4) : load_some<x4<O>, 4>(p, a.N - c);
    }
  };
  if constexpr (kHold)
#pragma unroll
    for (int ct = 0; ct < NT; ++ct)
      if (ct == 0 || ct < tiles)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) weights(c_first + ct * 64, jb, raw[ct][jb]);
  if (base) load_base(c_first, 0);
  auto in_terms = [](f32x4 x, U(&t)[kTerms]) {
    if constexpr (FAST) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __bf16 q[3];
        split3(x[e], q);
#pragma unroll
        for (int k = 0; k < 3; ++k) t[k][e] = q[k];
      }
    } else {
      t[0] = x;
    }
  };
  const int across = a.rp / 4;
  for (int i = threadIdx.x; i < blocks * 16 * across; i += kThreads)
    in_terms(load_u(i / across, i % across * 4), *(U(*)[kTerms])(shared_u + i / across * kU + i % across * kTerms));
  __syncthreads();
  if (c_first >= a.N) return;
  auto from_lds = [&](int rb, int jb) -> const U(&)[kTerms] {
    return *(const U(*)[kTerms])(shared_u + (rb * 16 + m) * kU + (jb * 4 + g) * kTerms);
  };
  float* const my = tile[wave];
#pragma unroll
  for (int ct = 0; ct < NT; ++ct) {
    if (AHEAD && ct >= tiles) break;
    const int c0 = c_first + ct * 64;
    // operands: the weights as they are, or turned (FLAT), or in fp32
    typedef std::conditional_t<FAST, bf16x4, f32x4> W;
    W wf[kHold ? JB : 1][4];
    auto operands = [&](int jb) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const T x = FLAT ? raw[ct][jb][s][q] : raw[ct][jb][q][s];
          if constexpr (FAST)
            wf[jb][q][s] = x;
          else
            wf[jb][q][s] = (float)x;
        }
    };
    if constexpr (kHold) {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) operands(jb);
    }
#pragma unroll 1
    for (int rb = 0; rb < blocks; ++rb) {
      f32x4 acc[4] = {};
      auto multiply = [&](const W(&h)[4], const U(&x)[kTerms]) {
        if constexpr (FAST) {
#pragma unroll
          for (int k = 0; k < kTerms; ++k)
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) acc[nb] = mfma(h[nb], x[k], acc[nb]);
        } else {
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) acc[nb] = mfma(h[nb][s], x[0][s], acc[nb]);
        }
      };
      if constexpr (kHold) {
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
          if (jb * 16 < a.rp) multiply(wf[jb], from_lds(rb, jb));
      } else {
#pragma unroll 1
        for (int jb = 0; jb * 16 < a.rp; ++jb) {
          weights(c0, jb, raw[0][0]);
          operands(0);
          multiply(wf[0], from_lds(rb, jb));
        }
      }
      // lane: row m of the block, columns of the instruction's rows 4 g + i
      auto turn = [&]() {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (FLAT)
            *(f32x4*)(my + m * kTile + 16 * g + 4 * q) = f32x4{acc[0][q], acc[1][q], acc[2][q], acc[3][q]};
          else
            *(f32x4*)(my + m * kTile + 16 * q + 4 * g) = acc[q];
        }
        lanes_in_order();
      };
      turn();
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
        else if (AHEAD && ct + 1 < tiles)
          load_base(c0 + 64, 0);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (rb * 16 + q * 4 >= run.count) break;
        const int t = rb * 16 + q * 4 + g, c = c0 + 4 * m, n = a.N - c;
        const int64_t row = row_of(rb, q);
        if constexpr (FAST) {
          if (__builtin_expect(__ballot(has_nan(y[q])) != 0, 0)) {  // see sign_of
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) acc[nb] = f32x4{};
            auto signs = [&](const W(&h)[4], const U(&x)[kTerms]) {
              const U u = signs_of<U, 4>(x[0]);
#pragma unroll
              for (int nb = 0; nb < 4; ++nb) acc[nb] = mfma(h[nb], u, acc[nb]);
            };
            if constexpr (kHold) {
#pragma unroll
              for (int jb = 0; jb < JB; ++jb)
                if (jb * 16 < a.rp) signs(wf[jb], from_lds(rb, jb));
            } else {
#pragma unroll 1
              for (int jb = 0; jb * 16 < a.rp; ++jb) {
                weights(c0, jb, raw[0][0]);
                operands(0);
                signs(wf[0], from_lds(rb, jb));
              }
            }
            turn();
            const f32x4 s = *(const f32x4*)(my + (q * 4 + g) * kTile + 4 * m);
            lanes_in_order();
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (y[q][e] != y[q][e] && __builtin_isinf(s[e]) && t < run.count && e < n)
                y[q][e] = s[e] + (base ? (float)base[row * a.base_ld + c + e] : 0.f);
          }
        }
        if (t >= run.count || n <= 0) continue;
        O* dst = (O*)a.out + row * a.out_ld + c;
        x4<O> z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = narrow<O>(y[q][e]);
        if (n >= 4) {
          if (a.past) {
            asm volatile("" ::: "memory");  // or the compiler makes one store of the two
            typedef x4<O> by_element __attribute__((aligned(sizeof(O))));
            __builtin_nontemporal_store(z, (by_element*)dst);
            asm volatile("" ::: "memory");
          } else {
            __builtin_memcpy(dst, &z, sizeof(z));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n) dst[e] = z[e];
        }
      }
    }
  }
}

// out[row][c] = base[row][c] + sum_j u[row][j] w[j][c] on the bf16 matrix
// instructions, for u as three bf16 numbers each, which hold all of its 24 bits
// (ExpandArgs::terms). The rows of grad_x: 64 columns a wave, for all rows of a run.
//
// A lane takes 8 ranks of 4 columns and turns them in registers. Its results are
// 16 columns of a row, stored as they are. KS: steps of 32 ranks; 0 for up to 16,
// where one step holds the first and the second number and one the third.
template <class O, int KS, int NT>
__global__ __launch_bounds__(kThreads, KS < 2 ? 4 : 1) void expand_flat(ExpandArgs a, RunList l) {
  constexpr int kSteps = KS == 0 ? 1 : KS, kTerms = KS == 0 ? 2 : 3;
  const Place at = place_of();
  const Run run = run_of(l, at.item);
  if (run.count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane % 16, g = lane / 16;
  const int c_first = ((int)at.tile * kWaves + wave) * NT * 64;
  if (c_first >= a.N) return;
  const int my_row = l.order[run.first + (lane < run.count ? lane : run.count - 1)];  // of the run's row `lane`
  const int blocks = (run.count + 15) / 16;
  const bool there = run.key < a.n;
  auto load_weights = [&](int ct, bf16x8(&wf)[kSteps][4]) {
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
      const int c0 = c_first + ct * 64, j0 = ks * 32 + (KS == 0 ? g % 2 : g) * 8;
      const __bf16* w = (const __bf16*)a.w + (int64_t)run.key * a.r * a.N + c0 + 4 * m;
      x4<__bf16> x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __bf16* p = w + (int64_t)(j0 + e < a.r ? j0 + e : a.r - 1) * a.N;
        x[e] = c0 + 64 <= a.N ? load_n<true, x4<__bf16>, 4>(p, 4) : load_some<x4<__bf16>, 4>(p, a.N - c0 - 4 * m);
        if (a.r != a.rp && j0 + e >= a.r) x[e] = x4<__bf16>{};
      }
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int e = 0; e < 8; ++e) wf[ks][nb][e] = x[e][nb];
      if (KS == 2 && j0 >= a.rp)  // a rank of up to 48
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) wf[ks][nb] = bf16x8{};
    }
  };
  auto load_u = [&](int rb, bf16x8(&u)[kSteps][kTerms]) {
    const __bf16* p = (const __bf16*)a.terms + (int64_t)__shfl(my_row, rb * 16 + m) * 3 * a.rp;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int q = 0; q < kTerms; ++q) {
        const int term = KS == 0 ? 2 * q + g / 2 : q, j = KS == 0 ? g % 2 * 8 : ks * 32 + g * 8;
        u[ks][q] = term < 3 && j < a.rp ? *(const bf16x8*)(p + term * a.rp + j) : bf16x8{};
      }
  };
  auto multiply = [&](const bf16x8(&wf)[kSteps][4], const bf16x8(&u)[kSteps][kTerms], f32x4(&acc)[4]) {
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int q = 0; q < kTerms; ++q)
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) acc[nb] = mfma(wf[ks][nb], u[ks][q], acc[nb]);
  };
  bf16x8 wf[NT][kSteps][4], u[4][kSteps][kTerms];
  if (there) {
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) load_weights(ct, wf[ct]);
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      if (rb < blocks) load_u(rb, u[rb]);
  }
  uint64_t nan = 0;  // sums that are NaN: added to base they count as 0 at first
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) {
    if (rb >= blocks) break;
    const int64_t row = __shfl(my_row, rb * 16 + m);
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      f32x4 acc[4] = {};
      if (there) {
        multiply(wf[ct], u[rb], acc);
        nan |= __ballot(has_nan(acc[0]) || has_nan(acc[1]) || has_nan(acc[2]) || has_nan(acc[3]));
      }
      const int c = c_first + ct * 64 + 16 * g, n = a.N - c;
      if (rb * 16 + m >= run.count || n <= 0) continue;
      O* dst = (O*)a.out + row * a.out_ld + c;
      const O* base = a.base ? (const O*)a.base + row * a.base_ld + c : nullptr;
      constexpr int E = 16 / (int)sizeof(O);  // columns a store
      typedef O ov __attribute__((ext_vector_type(E)));
      if (n >= 16) {
#pragma unroll
        for (int s = 0; s < 16 / E; ++s) {
          ov z, old = {};
          if (base) old = load_n<true, ov, E>(base + s * E, E);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int k = s * E + e;  // acc[k % 4][k / 4]
            const float y = acc[k % 4][k / 4];
            z[e] = base ? (there && y == y ? narrow<O>((float)old[e] + y) : old[e]) : narrow<O>(y);
          }
          __builtin_memcpy(dst + s * E, &z, sizeof(z));
        }
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < n) {
            const float y = acc[k % 4][k / 4];
            dst[k] = base ? (there && y == y ? narrow<O>((float)base[k] + y) : base[k]) : narrow<O>(y);
          }
      }
    }
  }
  if (__builtin_expect(nan == 0, 1)) return;
  // the same sums once more, and what those that are NaN are (sign_of)
#pragma unroll 1
  for (int ct = 0; ct < NT; ++ct) {
    load_weights(ct, wf[0]);
#pragma unroll 1
    for (int rb = 0; rb < blocks; ++rb) {
      load_u(rb, u[0]);
      f32x4 acc[4] = {}, signs[4] = {};
      multiply(wf[0], u[0], acc);
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        i32x4 first = __builtin_bit_cast(i32x4, signs_of<bf16x8, 8>(u[0][ks][0]));
        if (KS == 0)  // the lanes of the second terms take the first ones too
#pragma unroll
          for (int e = 0; e < 4; ++e) first[e] = __shfl(first[e], lane % 32);
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) signs[nb] = mfma(wf[0][ks][nb], __builtin_bit_cast(bf16x8, first), signs[nb]);
      }
      const int64_t row = __shfl(my_row, rb * 16 + m);
      const int c = c_first + ct * 64 + 16 * g;
      O* dst = (O*)a.out + row * a.out_ld + c;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float y = acc[k % 4][k / 4], s = signs[k % 4][k / 4];
        if (y == y || rb * 16 + m >= run.count || c + k >= a.N) continue;
        dst[k] = narrow<O>((a.base ? (float)dst[k] : 0.f) + (__builtin_isinf(s) ? s : y));
      }
    }
  }
}

template <class T, class O, bool FLAT, bool AHEAD>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  const int tiles = !AHEAD ? 1 : a.rp <= 16 ? 4 : 2;
  const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, tiles * kWaves * 64));
  if constexpr (!FLAT || !std::is_same_v<T, __bf16>) {  // those have terms up to rank 64
    if (a.rp <= 16) {
      TIM_LAUNCH((expand<T, O, FLAT, 1, AHEAD><<<grid, kThreads, 0, s>>>(a, l)));
      return hipSuccess;
    }
    if (a.rp <= 32) {
      TIM_LAUNCH((expand<T, O, FLAT, 2, AHEAD><<<grid, kThreads, 0, s>>>(a, l)));
      return hipSuccess;
    }
    if (a.rp <= 64) {
      TIM_LAUNCH((expand<T, O, FLAT, 4, false><<<grid, kThreads, 0, s>>>(a, l)));
      return hipSuccess;
    }
  }
  TIM_LAUNCH((expand<T, O, FLAT, 16, false><<<grid, kThreads, 0, s>>>(a, l)));
  return hipSuccess;
}
template <class T, class O, bool FLAT>
hipError_t run_expand(const ExpandArgs& a, const RunList& l, hipStream_t s) {
  if constexpr (FLAT && std::is_same_v<T, __bf16>) {
    if (a.terms) {
      // a wave takes two tiles where that leaves a workgroup of four waves four times for each of 256 CUs (8192
      // rows of rank 32, d = 4096: 138 us a call against 142; 146 with registers for three workgroups a CU)
      const int tiles = a.rp <= 32 && l.max_runs * chunks_of(a.N, 2 * kWaves * 64) >= 1024 ? 2 : 1;
      const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, tiles * kWaves * 64));
      if (a.rp <= 16 && tiles == 2)
        TIM_LAUNCH((expand_flat<O, 0, 2><<<grid, kThreads, 0, s>>>(a, l)));
      else if (a.rp <= 16)
        TIM_LAUNCH((expand_flat<O, 0, 1><<<grid, kThreads, 0, s>>>(a, l)));
      else if (a.rp <= 32 && tiles == 2)
        TIM_LAUNCH((expand_flat<O, 1, 2><<<grid, kThreads, 0, s>>>(a, l)));
      else if (a.rp <= 32)
        TIM_LAUNCH((expand_flat<O, 1, 1><<<grid, kThreads, 0, s>>>(a, l)));
      else
        TIM_LAUNCH((expand_flat<O, 2, 1><<<grid, kThreads, 0, s>>>(a, l)));
      return hipSuccess;
    }
  }
  // A wave takes several tiles where that leaves 16 waves for each of 256 CUs and the runs hold less than a block of 16
  // rows: what it waits for are then the weights, otherwise the rows. (48 rows of 32 adapters at d = 5120 on a head of
  // 152064 61 us against 74, 4096 rows of 4 adapters at d = 4096 on one of 151936 984 against 900; of a high rank the
  // weights of several tiles do not fit the registers.) max_runs counts each adapter of the set once, for the host does not
  // know which have rows: long runs of few adapters out of a large set take several tiles too (4096 rows of 4 adapters out
  // of 200 989 us, 1024 rows of 2 out of 100 on 50257 columns 141 against 107).
  if (!FLAT && a.rp <= 32 && l.max_runs * chunks_of(a.N, 4 * 64) >= 4096 && a.T < 16 * l.max_runs)
    return run_expand<T, O, FLAT, !FLAT>(a, l, s);
  return run_expand<T, O, FLAT, false>(a, l, s);
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

hipError_t launch_expand(const ExpandArgs& args, int dtype, int out_dtype, bool flat, const RunList& l, hipStream_t s) {
  ExpandArgs a = args;
  // 4096 rows of 151936 fp32 logits, with several tiles a wave, 983 us against 996; 48 rows 68 against 65
  a.past = a.T * a.N * dtype_bytes(out_dtype) > kCaches;
  return dtype == TIM_BF16 ? run_expand<__bf16>(a, out_dtype, flat, l, s)
                           : run_expand<_Float16>(a, out_dtype, flat, l, s);
}

}  // namespace tim
