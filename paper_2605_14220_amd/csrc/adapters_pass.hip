// Adapters: the pass over the rows that the backward makes once for both products that need it.

#include <hip/hip_runtime.h>

#include "adapters.h"

namespace tim {
namespace {

// One pass over the columns of src = grad: for a run of one adapter's rows and
// CT tiles of columns
//   out[c][j]      sum over the rows of src[row][c] w[row][j]
//   part[row][j] sum over the columns of src[row][c] b[c][j]    (CONTRACT)
// and without the contraction the first alone, [j][c], of src = x.
//
// 64 rows of 256 (otherwise 128) columns at a time lie in LDS, read from memory once, and are
// read from there along the rows for one product and along the columns for the
// other. A wave takes a quarter of the columns of the first and 16 rows of the
// second.
//
// FAST, where all is bf16: both on the bf16 matrix instructions, w as the sum of
// three bf16 numbers, which holds all of its 24 bits. Otherwise on the fp32 ones,
// whose tile of 128 columns has the same bytes: three workgroups fit a CU, with 256
// columns one. 2047 rows on a head of 151936 (rank 16, bf16) take 150 us, 4.2 TB/s;
// 150 rows on one of 50257 (rank 9, fp32) 20 us, the latency of one workgroup's
// four tiles: two blocks of rows, two tiles of columns.
constexpr int kPassRows = 64;
template <class S, class W, bool CONTRACT, int JB, int CT>
struct Pass {
  static constexpr bool FAST = std::is_same_v<S, __bf16> && std::is_same_v<W, __bf16>;
  typedef std::conditional_t<FAST, __bf16, float> E;  // of the tile and of w in LDS
  static constexpr int kCols = FAST ? kPassCols : kPassColsF32;  // of a tile
  static constexpr int NB = kCols / 64;  // blocks of 16 columns a wave
  static constexpr int kTerms = FAST ? 3 : 1;
  static constexpr int kPad = 16 / (int)sizeof(E);
  static constexpr int kRow = kCols + kPad;  // elements from row to row of the tile
  static constexpr int kW = kPassRows + kPad;    // of w, [term][j][row]
  static constexpr int kB = CT * kCols + 8;  // of b, [j][c]
  static constexpr int kLoads = kPassRows * kCols * (int)sizeof(S) / 16 / kThreads;  // 16 bytes a thread
  static constexpr int kV = 16 / (int)sizeof(S);
  static constexpr int kLds = (kPassRows * kRow + kTerms * JB * 16 * kW) * (int)sizeof(E) +
                              (CONTRACT ? JB * 16 * kB : 1) * (int)sizeof(W) + kMaxPassRows * 4;
};
static_assert(kPassesAtOnce == 256 * (160 * 1024 / Pass<__bf16, __bf16, true, 1, 1>::kLds) &&
                  kPassesAtOnce == 256 * (160 * 1024 / Pass<float, __bf16, true, 1, 1>::kLds),
              "workgroups of one tile that 256 CUs hold");
template <class S, class W, bool CONTRACT, int JB, int CT>
__global__ __launch_bounds__(kThreads) void pass(PassArgs a, RunList l) {
  typedef Pass<S, W, CONTRACT, JB, CT> P;
  typedef typename P::E E;
  constexpr int kCols = P::kCols, NB = P::NB;
  typedef E en __attribute__((ext_vector_type(NB)));
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
  const int c_first = at.tile * CT * kCols, j0 = blockIdx.z * JB * 16;
  const int tiles = (a.N - c_first + kCols - 1) / kCols < CT ? (a.N - c_first + kCols - 1) / kCols : CT;
  const int32_t* order = l.order + run.first;
  const float* w = a.w + j0;

  // rows past the run's end, up to a whole tile, are read as its last one
  for (int t = tid; t < (run.count + kPassRows - 1) / kPassRows * kPassRows; t += kThreads)
    rows[t] = order[t < run.count ? t : run.count - 1];
  if constexpr (CONTRACT) {
    // a thread takes 8 ranks of a column; the loads first, then their way into LDS
    constexpr int kEach = JB * 16 * CT * kCols / 8 / kThreads;
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
  constexpr int kAcross = kCols / P::kV, kDown = kThreads / kAcross;
  sv held[P::kLoads];
  f32x4 held_w[JB];
  const int lc = tid % kAcross * P::kV, lr = tid / kAcross;
  auto load_tile = [&](int t0, int ct) {
    const int c = c_first + ct * kCols + lc;
    const S* src = (const S*)a.src + c;
    const bool whole = c_first + (ct + 1) * kCols <= a.N;
    if (whole && a.past) {
      asm volatile("" ::: "memory");  // or the compiler makes one of the two branches' loads
#pragma unroll
      for (int k = 0; k < P::kLoads; ++k) held[k] = load_past<sv, P::kV>(src + rows[t0 + lr + k * kDown] * a.ld);
      asm volatile("" ::: "memory");
    } else if (whole) {
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
        held_w[jb] = a.w && t < run.count && j0 + j < a.rp ? *(const f32x4*)(w + (int64_t)rows[t] * a.rp + j) : f32x4{};
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
            __bf16 t[3];
            split3(x, t);
#pragma unroll
            for (int k = 0; k < 3; ++k) wt[k * JB * 16 * P::kW + to] = t[k];
          } else {
            wt[to] = x;
          }
        }
    }
  };

  f32x4 acc[CT][JB][NB] = {};  // out
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
            x[e] = *(const x4<E>*)(tile + (ks * 32 + g * 8 + e) * P::kRow + wave * (16 * NB) + 4 * m);
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
          for (int ks = 0; ks < kCols / 32; ++ks) {
            const bf16x8 x = *(const bf16x8*)(tile + (wave * 16 + m) * P::kRow + ks * 32 + g * 8);
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
              sum[jb] = mfma(*(const bf16x8*)(bt + (jb * 16 + m) * P::kB + ct * kCols + ks * 32 + g * 8), x, sum[jb]);
          }
          add_up(total, sum, ct);
        }
      } else {
#pragma unroll 4
        for (int q = 0; q < kPassRows / 4; ++q) {
          const en x = *(const en*)(tile + (q * 4 + g) * P::kRow + wave * (16 * NB) + NB * m);
#pragma unroll
          for (int jb = 0; jb < JB; ++jb) {
            const float wf = wt[(jb * 16 + m) * P::kW + q * 4 + g];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              acc[ct][jb][nb] = CONTRACT ? mfma(wf, x[nb], acc[ct][jb][nb]) : mfma(x[nb], wf, acc[ct][jb][nb]);
          }
        }
        if constexpr (CONTRACT) {
          f32x4 sum[JB] = {};
#pragma unroll 4
          for (int ks = 0; ks < kCols / 16; ++ks) {
            const f32x4 x = *(const f32x4*)(tile + (wave * 16 + m) * P::kRow + ks * 16 + g * 4);
#pragma unroll
            for (int jb = 0; jb < JB; ++jb) {
              const x4<W> bf = *(const x4<W>*)(bt + (jb * 16 + m) * P::kB + ct * kCols + ks * 16 + g * 4);
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
      if (t < run.count) {
        float* p = a.part + ((int64_t)at.tile * a.T + rows[t]) * a.rp + j0 + g * 4;
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
          if (j0 + jb * 16 < a.rp) *(f32x4*)(p + jb * 16) = total[jb];
      }
    }
  }

  if (!a.out) return;
  const bool only = run.slot < 0, add = only && a.accumulate;
  float* out = only ? a.out + (int64_t)run.key * a.r * a.N : a.out_part + (int64_t)run.slot * a.r * a.N;
  // runs of E elements next to each other in memory: four of the rank, or NB of the columns
  constexpr int E4 = CONTRACT ? 4 : NB;
  typedef float fe __attribute__((ext_vector_type(E4)));
  constexpr int kQ = CONTRACT ? NB : 4;
  auto column = [&](int ct, int q) {
    return c_first + ct * kCols + wave * (16 * NB) + (CONTRACT ? NB * m + q : NB * (4 * g + q));
  };
  auto rank = [&](int jb) { return j0 + jb * 16 + (CONTRACT ? 4 * g : m); };
  uint64_t again = 0;  // a bit an element that came out as NaN (sign_of); added, it counts as 0 at first
  if constexpr (P::FAST) {
    static_assert(NB == 4 && kQ == 4 && E4 == 4 && CT * JB <= 4, "a bit an element");
    bool any = false;
#pragma unroll
    for (int i = 0; i < CT * JB * 4; ++i) any |= has_nan(acc[i / 4 / JB][i / 4 % JB][i % 4]);
    if (__builtin_expect(any, 0)) {
#pragma unroll
      for (int i = 0; i < CT * JB * 16; ++i) {
        const int ct = i / 16 / JB, jb = i / 16 % JB, q = i / 4 % 4, e = i % 4;
        const float y = CONTRACT ? acc[ct][jb][q][e] : acc[ct][jb][e][q];
        if (y != y) again |= 1ull << i;
      }
    }
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int jb = 0; jb < JB; ++jb)
#pragma unroll
      for (int q = 0; q < kQ; ++q) {
        const int j = rank(jb), c = column(ct, q);
        if (j >= a.r || c >= a.N) continue;
        fe y;
#pragma unroll
        for (int e = 0; e < E4; ++e) y[e] = CONTRACT ? acc[ct][jb][q][e] : acc[ct][jb][e][q];
        float* p = out + (CONTRACT ? (int64_t)c * a.r + j : (int64_t)j * a.N + c);
        const int left = CONTRACT ? a.r - j : a.N - c;
        if (P::FAST && add) {
#pragma unroll
          for (int e = 0; e < E4; ++e) y[e] = y[e] == y[e] ? y[e] : 0.f;
        }
        if (left >= E4) {
          if (add) y += load_n<true, fe, E4>(p, E4);
          __builtin_memcpy(p, &y, sizeof(y));
        } else {
#pragma unroll
          for (int e = 0; e < E4; ++e)
            if (e < left) p[e] = add ? p[e] + y[e] : y[e];
        }
      }
  if (__builtin_expect(again == 0, 1)) return;
  // the blocks of 16 elements that hold NaN once more, from w itself
#pragma unroll 1
  for (int i = 0; i < CT * JB; ++i, again >>= 16) {
    const int j = rank(i % JB), c = column(i / JB, 0);
    if (!(again & 0xffff) || j >= a.r || c >= a.N) continue;
    float sum[16] = {};
#pragma unroll 4
    for (int t = 0; t < run.count; ++t) {
      const S* src = (const S*)a.src + rows[t] * a.ld + c;
      const float* wr = a.w + (int64_t)rows[t] * a.rp + j;
      if constexpr (CONTRACT) {
        const x4<S> x = load_some<x4<S>, 4>(src, a.N - c);
        const f32x4 y = *(const f32x4*)wr;
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[k] = fmaf((float)x[k / 4], y[k % 4], sum[k]);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const x4<S> x = load_some<x4<S>, 4>(src + 4 * q, a.N - c - 4 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[q * 4 + e] = fmaf((float)x[e], *wr, sum[q * 4 + e]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int jk = j + (CONTRACT ? k % 4 : 0), ck = c + (CONTRACT ? k / 4 : k);
      if (!(again >> k & 1) || jk >= a.r || ck >= a.N) continue;
      float* p = out + (CONTRACT ? (int64_t)ck * a.r + jk : (int64_t)jk * a.N + ck);
      *p = add ? *p + sum[k] : sum[k];
    }
  }
}

template <class S, class W, bool CONTRACT, int JB, int CT>
hipError_t run_pass(const PassArgs& a, const RunList& l, hipStream_t s) {
  const dim3 grid((unsigned)l.max_runs, (unsigned)chunks_of(a.N, CT * Pass<S, W, CONTRACT, JB, CT>::kCols), (unsigned)((a.rp + 63) / 64));
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
  if (a.rp <= 32) return run_pass<S, W, CONTRACT, 2, 1>(a, l, s);
  return run_pass<S, W, CONTRACT, 4, 1>(a, l, s);
}

template <class W>
hipError_t run_pass(const PassArgs& a, int src_dtype, bool contract, int tiles, const RunList& l, hipStream_t s) {
  if (!contract) return run_pass<W, W, false>(a, 1, l, s);
  switch (src_dtype) {
    case TIM_F32: return run_pass<float, W, true>(a, tiles, l, s);
    case TIM_BF16: return run_pass<__bf16, W, true>(a, tiles, l, s);
    default: return run_pass<_Float16, W, true>(a, tiles, l, s);
  }
}

}  // namespace

hipError_t launch_pass(const PassArgs& args, int src_dtype, int dtype, bool contract, int tiles, const RunList& l,
                       hipStream_t s) {
  PassArgs a = args;
  // the gradients of 2047 rows on a head of 151936 208 us against 220; 150 rows on 50257 61 against 58
  a.past = a.T * a.N * dtype_bytes(src_dtype) > kCaches;
  return dtype == TIM_BF16 ? run_pass<__bf16>(a, src_dtype, contract, tiles, l, s)
                           : run_pass<_Float16>(a, src_dtype, contract, tiles, l, s);
}

}  // namespace tim
