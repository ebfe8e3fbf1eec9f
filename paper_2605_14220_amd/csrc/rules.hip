// Changed logits on gfx950: penalties, biases and grammar masks applied to the
// logits of T rows, the softmax statistics of the result and their gradient.
//
// Mathematics, per entry (include/tim_policy.h has the order and the roundings):
//   x = rule(z): penalties of the tokens in the row's history, bias, 1/tau, mask
//   logprobs: per chunk m = max x, s = sum e^(x-m), u = sum e^(x-m) (x-m); a
//             merge over the chunks gives lse = M + log S, H = log S - U / S
//   backward: dz = slope (g [v = tok] - p (g + e (log p + H))), p = e^(x-lse)
//
// All three are one pass over the logits (read once; adjust and backward write
// as many) and bound by HBM. A workgroup takes one chunk of TIM_RULE_CHUNK
// vocabulary entries of consecutive rows, its part of a row in registers. The
// sparse changes live in LDS, one word per entry of the chunk: bit 31 = token
// of the prompt, the rest = count in the output (integer atomics, so the order
// of the tokens does not matter), and in a second word the last bias entry of
// that id (an integer maximum). A chunk's workgroup reads the row's whole
// history and keeps what falls into it; rows whose history extends the last
// row's (the rows of one response in a packed stream) add only the new tokens.

#include <hip/hip_runtime.h>

#include "kernels.h"
#include "policy.h"

namespace tim {
namespace {

constexpr int kChunk = TIM_RULE_CHUNK;
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kPer = kChunk / kThreads;  // entries per thread
constexpr int kMaxGroup = 16;            // rows of one workgroup
constexpr int kMaxChunks = (TIM_MAX_VOCAB + kChunk - 1) / kChunk;
static_assert(kMaxChunks <= 64, "the merge holds a row's chunks in one wave");
constexpr uint32_t kPromptBit = 0x80000000u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_inff();
// Below this distance from the maximum e^x is 0 in fp32; it takes the place
// of -inf in the products p * log p.
constexpr float kFloor = -200.f;

enum class Op { kAdjust, kStats, kGrad };

__device__ __forceinline__ float exp_hw(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

template <class T>
__device__ __forceinline__ float widen(T x) { return (float)x; }

// N consecutive elements at p, which is aligned to its element only.
template <class T, int N>
struct Vec {
  T v[N];
};
template <class T, int N>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p) {
  Vec<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, N>& r) { __builtin_memcpy(p, &r, sizeof(r)); }

struct Stat {
  float m, s, u;
};

// (m, s, u) of two disjoint sets of entries. A side with no finite maximum has
// s = u = 0 (or NaN), so any finite shift keeps it.
__device__ __forceinline__ Stat shift(const Stat& a, float m) {
  const float dm = fmaxf(a.m - m, -1e30f);
  const float k = exp_hw(dm);
  return {m, a.s * k, k * (a.u + a.s * dm)};
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}

// Tokens history[from .. to) that fall into the chunk [v0, v0 + n): before
// split marked, from there on counted.
__device__ __forceinline__ void count_tokens(uint32_t* cnt, const int32_t* __restrict__ history, int64_t from,
                                             int64_t split, int64_t to, int v0, int n) {
  for (int64_t i = from + threadIdx.x; i < to; i += kThreads) {
    const uint32_t t = (uint32_t)history[i] - (uint32_t)v0;
    if (t < (uint32_t)n) {
      if (i < split)
        atomicOr(&cnt[t], kPromptBit);
      else
        atomicAdd(&cnt[t], 1u);
    }
  }
}

// What a workgroup needs of one of its rows, read once for all of them.
struct Row {
  int64_t begin, split, end;  // of the history
  int64_t bias0, bias1;
  int64_t mask;               // row of the mask, -1: none
  float rho, inv_rho, freq, pres;
  int tok;                    // relative to the chunk; negative or past it: elsewhere
  float lse, ent, g, e;
  int zero;                   // the gradient is 0 everywhere
};

template <Op OP>
__device__ __forceinline__ Row read_row(const RuleArgs& a, int64_t row, int v0, bool hist, bool bias) {
  Row w = {};
  w.mask = -1;
  if (a.r.mask) {
    const int64_t m = a.r.mask_rows ? (int64_t)a.r.mask_rows[row] : row;
    if (m >= 0 && m < a.r.n_masks) w.mask = m;
  }
  // a penalty that is left out takes the value that changes nothing
  w.rho = 1.f;
  if (hist) {
    const int64_t N = a.r.history_len;
    w.begin = clamp64(a.r.hist_begin[row], 0, N);
    w.split = a.r.hist_split ? clamp64(a.r.hist_split[row], w.begin, N) : w.begin;
    w.end = clamp64(a.r.hist_end[row], w.split, N);
    if (a.r.repetition) w.rho = a.r.repetition[row];
    if (a.r.frequency) w.freq = a.r.frequency[row];
    if (a.r.presence) w.pres = a.r.presence[row];
  }
  w.inv_rho = 1.f / w.rho;
  if (bias) {
    w.bias0 = clamp64(a.r.bias_begin[row], 0, a.r.bias_len);
    w.bias1 = clamp64(a.r.bias_end[row], w.bias0, a.r.bias_len);
  }
  w.tok = -1;
  if constexpr (OP != Op::kAdjust) {
    const bool valid = (unsigned)a.tokens[row] < (unsigned)a.V;
    if (valid) w.tok = a.tokens[row] - v0;
    if constexpr (OP == Op::kGrad) {
      w.lse = a.lse[row];
      w.g = valid ? a.grad_logp[row] : 0.f;
      if (a.grad_entropy) {
        w.e = a.grad_entropy[row];
        w.ent = a.entropy[row];
      }
      w.zero = (w.g == 0.f && w.e == 0.f) || w.lse == kNegInf;
    }
  }
  return w;
}

template <Op OP, class TI, class TO, bool SPARSE>
__global__ __launch_bounds__(kThreads) void rules_kernel(const RuleArgs a, int n_chunks, int rows_per_group) {
  constexpr int E = 16 / (int)sizeof(TI);  // entries per load
  constexpr int NV = kPer / E;             // loads per thread
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ Row rows[kMaxGroup];
  __shared__ Stat wstat[kWaves];
  __shared__ float tok_x;

  const int chunk = (int)(blockIdx.x % (unsigned)n_chunks);
  const int64_t r0 = (int64_t)(blockIdx.x / (unsigned)n_chunks) * rows_per_group;
  const int n_rows = (int)(a.T - r0 < rows_per_group ? a.T - r0 : rows_per_group);
  const int v0 = chunk * kChunk;
  const int n = a.V - v0 < kChunk ? a.V - v0 : kChunk;
  const bool hist = SPARSE && a.r.history != nullptr;
  const bool bias = SPARSE && a.r.bias_ids != nullptr;
  uint32_t* cnt = lds;
  uint32_t* last = lds + (hist ? kChunk : 0);
  if ((int)threadIdx.x < n_rows) rows[threadIdx.x] = read_row<OP>(a, r0 + threadIdx.x, v0, hist, bias);
  __syncthreads();

  int64_t pb = -1, ps = 0, pe = 0;  // the history counted in cnt; pb < 0: none, cnt not cleared
  int64_t qb = -1, qe = -1;         // the bias list in last

  for (int i = 0; i < n_rows; ++i) {
    const int64_t row = r0 + i;
    const Row& w = rows[i];
    const TI* z = (const TI*)a.logits + row * a.ld + v0;
    TO* out = OP == Op::kStats ? nullptr : (TO*)a.out + row * a.out_ld + v0;
    if (OP == Op::kGrad && w.zero) {
      for (int c = threadIdx.x; c < n; c += kThreads) out[c] = (TO)0.f;
      continue;
    }

    Vec<TI, E> in[NV];
    uint32_t open[NV];  // bit k: entry k of the load is allowed and lies in the vocabulary
    const bool some_off = w.mask >= 0 || n < kChunk;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * kThreads + (int)threadIdx.x) * E;
      if (c + E <= n) {
        in[j] = load_vec<TI, E>(z + c);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) in[j].v[k] = c + k < n ? z[c + k] : (TI)0.f;
      }
      open[j] = c + E <= n ? ~0u : c < n ? (1u << (n - c)) - 1u : 0u;
      if (w.mask >= 0 && c < n) open[j] &= a.r.mask[w.mask * a.r.mask_ld + ((v0 + c) >> 5)] >> ((v0 + c) & 31);
    }

    if (hist) {
      const int64_t b = w.begin, s = w.split, t = w.end;
      int64_t from = pe;
      if (b != pb || s != ps || t < pe) {
        for (int c = threadIdx.x * 4; c < kChunk; c += kThreads * 4) *(uint4*)(cnt + c) = uint4{0, 0, 0, 0};
        from = b;
        __syncthreads();
      }
      count_tokens(cnt, a.r.history, from, s, t, v0, n);
      pb = b;
      ps = s;
      pe = t;
    }
    if (bias) {
      const int64_t b = w.bias0, t = w.bias1;
      if (b != qb || t != qe) {
        for (int c = threadIdx.x * 4; c < kChunk; c += kThreads * 4) *(uint4*)(last + c) = uint4{0, 0, 0, 0};
        __syncthreads();
        for (int64_t k = b + threadIdx.x; k < t; k += kThreads) {
          const uint32_t id = (uint32_t)a.r.bias_ids[k] - (uint32_t)v0;
          if (id < (uint32_t)n) atomicMax(&last[id], (uint32_t)k + 1u);
        }
        qb = b;
        qe = t;
      }
    }
    if constexpr (SPARSE) __syncthreads();

    float x[kPer];
    float m = kNegInf;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * kThreads + (int)threadIdx.x) * E;
      float* y = x + j * E;
      float slope[E];
#pragma unroll
      for (int k = 0; k < E; ++k) {
        y[k] = widen(in[j].v[k]);
        slope[k] = a.inv_tau;
      }
      if (hist) {
        uint32_t u[E], any = 0;
#pragma unroll
        for (int k = 0; k < E; k += 4) __builtin_memcpy(u + k, __builtin_assume_aligned(cnt + c + k, 16), 16);
#pragma unroll
        for (int k = 0; k < E; ++k) any |= u[k];
        if (any) {
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const float up = y[k] / w.rho, down = y[k] * w.rho;
            const bool pos = y[k] > 0.f;
            float v = u[k] ? (pos ? up : down) : y[k];
            if constexpr (OP == Op::kGrad) slope[k] = u[k] ? (pos ? w.inv_rho : w.rho) * a.inv_tau : a.inv_tau;
            const uint32_t count = u[k] & ~kPromptBit;
            const float less = v - w.freq * (float)count - w.pres;
            y[k] = count ? less : v;
          }
        }
      }
      if (bias) {
        uint32_t u[E], any = 0;
#pragma unroll
        for (int k = 0; k < E; k += 4) __builtin_memcpy(u + k, __builtin_assume_aligned(last + c + k, 16), 16);
#pragma unroll
        for (int k = 0; k < E; ++k) any |= u[k];
        if (any) {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (u[k]) y[k] = y[k] + a.r.bias_values[u[k] - 1];
        }
      }
#pragma unroll
      for (int k = 0; k < E; ++k) y[k] = y[k] * a.inv_tau;
      if (some_off) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const bool off = !((open[j] >> k) & 1u);
          y[k] = off ? kNegInf : y[k];
          slope[k] = off ? 0.f : slope[k];
        }
      }
      if constexpr (OP == Op::kStats) {
#pragma unroll
        for (int k = 0; k < E; ++k) m = fmaxf(m, y[k]);
      } else {
        Vec<TO, E> o;
        if constexpr (OP == Op::kAdjust) {
#pragma unroll
          for (int k = 0; k < E; ++k) o.v[k] = narrow<TO>(y[k]);
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const float q = y[k] - w.lse;
            const float p = exp_hw(q);
            float up = c + k == w.tok ? w.g : 0.f;
            up = up - p * (w.g + w.e * (fmaxf(q, kFloor) + w.ent));
            o.v[k] = narrow<TO>(slope[k] == 0.f ? 0.f : up * slope[k]);
          }
        }
        if (c + E <= n) {
          store_vec<TO, E>(out + c, o);
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (c + k < n) out[c + k] = o.v[k];
        }
      }
    }

    if constexpr (OP == Op::kStats) {
      m = wave_max(m);
      const float at = m == kNegInf ? 0.f : m;
      float s = 0.f, u = 0.f;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const float q = x[k] - at;
        const float p = exp_hw(q);
        s += p;
        u = fmaf(p, fmaxf(q, kFloor), u);
      }
      s = wave_sum(s);
      u = wave_sum(u);
      if ((threadIdx.x & 63) == 0) wstat[threadIdx.x >> 6] = {m, s, u};
      const int tok = w.tok;
      if (tok >= 0 && tok < n && tok / E % kThreads == (int)threadIdx.x) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if (tok / E / kThreads * E + tok % E == k) tok_x = x[k];
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        float top = wstat[0].m;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) top = fmaxf(top, wstat[v].m);
        Partial p = {top, 0.f, 0.f, tok >= 0 && tok < n ? tok_x : 0.f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          const Stat t = shift(wstat[v], top);
          p.s += t.s;
          p.u += t.u;
        }
        ((Partial*)a.part)[row * n_chunks + chunk] = p;
      }
    }
    // the next row changes what this one read from LDS
    if (SPARSE || OP == Op::kStats) __syncthreads();
  }
}

// One wave per row: lane c holds chunk c's partial.
__global__ __launch_bounds__(256) void rules_merge(const Partial* __restrict__ part, const int32_t* __restrict__ tokens,
                                                   int64_t T, int V, int n_chunks, float* __restrict__ logp,
                                                   float* __restrict__ entropy, float* __restrict__ lse) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= T) return;
  Partial p = {kNegInf, 0.f, 0.f, 0.f};
  if (lane < n_chunks) p = part[row * n_chunks + lane];
  const float top = wave_max(p.m);
  const Stat t = shift({p.m, p.s, p.u}, top);
  const float S = wave_sum(t.s);
  const float U = wave_sum(t.u);
  const int tok = tokens[row];
  const bool valid = (unsigned)tok < (unsigned)V;
  const float x = __shfl(p.ztok, valid ? tok / kChunk : 0);
  if (lane == 0) {
    const bool none = top == kNegInf && S == 0.f;  // nothing allowed
    const float log_s = logf(S);
    logp[row] = !valid ? __builtin_nanf("") : none ? kNegInf : (x - top) - log_s;
    if (entropy) entropy[row] = none ? 0.f : log_s - U / S;
    if (lse) lse[row] = none ? kNegInf : top + log_s;
  }
}

int rule_lds_bytes(const RuleArgs& a) {
  return ((a.r.history ? 1 : 0) + (a.r.bias_ids ? 1 : 0)) * kChunk * 4;
}

// `a` from row t0 on.
RuleArgs rows_from(const RuleArgs& a, int64_t t0, int64_t rows, int in_bytes, int out_bytes) {
  RuleArgs b = a;
  b.T = rows;
  b.logits = (const char*)a.logits + t0 * a.ld * in_bytes;
  auto at = [t0](auto*& p) {
    if (p) p += t0;
  };
  at(b.r.hist_begin);
  at(b.r.hist_split);
  at(b.r.hist_end);
  at(b.r.repetition);
  at(b.r.frequency);
  at(b.r.presence);
  at(b.r.bias_begin);
  at(b.r.bias_end);
  if (b.r.mask && !b.r.mask_rows) {  // row i takes mask i
    const int64_t skip = t0 < b.r.n_masks ? t0 : b.r.n_masks;
    b.r.mask += skip * b.r.mask_ld;
    b.r.n_masks -= skip;
    if (b.r.n_masks == 0) b.r.mask = nullptr;
  }
  at(b.r.mask_rows);
  at(b.tokens);
  if (b.part) b.part = (Partial*)b.part + t0 * rule_chunks_of(a.V);
  if (b.out) b.out = (char*)a.out + t0 * a.out_ld * out_bytes;
  at(b.lse);
  at(b.entropy);
  at(b.grad_logp);
  at(b.grad_entropy);
  return b;
}

template <Op OP, class TI, class TO>
hipError_t launch_rules(const RuleArgs& a, hipStream_t s) {
  const int n_chunks = rule_chunks_of(a.V);
  // a grid holds fewer than 2^32 threads
  const int64_t step = ((int64_t)1 << 22) / n_chunks;
  for (int64_t t0 = 0; t0 < a.T; t0 += step) {
    const int64_t rows = a.T - t0 < step ? a.T - t0 : step;
    const RuleArgs b = rows_from(a, t0, rows, (int)sizeof(TI), (int)sizeof(TO));
    int group = 1;
    if (b.r.history) {
      const int64_t fill = rows * n_chunks / 4096;
      group = fill < 1 ? 1 : fill > kMaxGroup ? kMaxGroup : (int)fill;
    }
    const unsigned grid = (unsigned)((rows + group - 1) / group * n_chunks);
    const int lds = rule_lds_bytes(b);
    if (lds)
      rules_kernel<OP, TI, TO, true><<<grid, kThreads, lds, s>>>(b, n_chunks, group);
    else
      rules_kernel<OP, TI, TO, false><<<grid, kThreads, 0, s>>>(b, n_chunks, group);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_logits_adjust(const RuleArgs& a, int dtype, hipStream_t s) {
  if (dtype == TIM_F32) return launch_rules<Op::kAdjust, float, float>(a, s);
  if (dtype == TIM_BF16) return launch_rules<Op::kAdjust, __bf16, __bf16>(a, s);
  return launch_rules<Op::kAdjust, _Float16, _Float16>(a, s);
}

hipError_t launch_logits_logprobs(const RuleArgs& a, int dtype, float* logp, float* entropy, float* lse,
                                  hipStream_t s) {
  const hipError_t e = dtype == TIM_F32    ? launch_rules<Op::kStats, float, float>(a, s)
                       : dtype == TIM_BF16 ? launch_rules<Op::kStats, __bf16, float>(a, s)
                                           : launch_rules<Op::kStats, _Float16, float>(a, s);
  if (e != hipSuccess) return e;
  const int n_chunks = rule_chunks_of(a.V);
  const int64_t step = (int64_t)1 << 25;  // rows per launch: a grid holds fewer than 2^32 threads
  for (int64_t t0 = 0; t0 < a.T; t0 += step) {
    const int64_t rows = a.T - t0 < step ? a.T - t0 : step;
    rules_merge<<<(unsigned)((rows + 3) / 4), 256, 0, s>>>((const Partial*)a.part + t0 * n_chunks, a.tokens + t0, rows,
                                                           a.V, n_chunks, logp + t0, entropy ? entropy + t0 : nullptr,
                                                           lse ? lse + t0 : nullptr);
    const hipError_t m = hipGetLastError();
    if (m != hipSuccess) return m;
  }
  return hipSuccess;
}

template <class TI>
static hipError_t launch_backward_from(const RuleArgs& a, int grad_dtype, hipStream_t s) {
  if (grad_dtype == TIM_F32) return launch_rules<Op::kGrad, TI, float>(a, s);
  if (grad_dtype == TIM_BF16) return launch_rules<Op::kGrad, TI, __bf16>(a, s);
  return launch_rules<Op::kGrad, TI, _Float16>(a, s);
}

hipError_t launch_logits_logprobs_backward(const RuleArgs& a, int dtype, int grad_dtype, hipStream_t s) {
  if (dtype == TIM_F32) return launch_backward_from<float>(a, grad_dtype, s);
  if (dtype == TIM_BF16) return launch_backward_from<__bf16>(a, grad_dtype, s);
  return launch_backward_from<_Float16>(a, grad_dtype, s);
}

}  // namespace tim
