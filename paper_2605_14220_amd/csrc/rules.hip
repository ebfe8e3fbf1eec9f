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

template <Op OP, class TI, class TO, bool SPARSE>
__global__ __launch_bounds__(kThreads) void rules_kernel(const RuleArgs a, int n_chunks, int rows_per_group) {
  constexpr int E = 16 / (int)sizeof(TI);  // entries per load
  constexpr int NV = kPer / E;             // loads per thread
  extern __shared__ uint32_t lds[];
  __shared__ Stat wstat[kWaves];
  __shared__ float tok_x;

  const int chunk = (int)(blockIdx.x % (unsigned)n_chunks);
  const int64_t r0 = (int64_t)(blockIdx.x / (unsigned)n_chunks) * rows_per_group;
  const int64_t r1 = r0 + rows_per_group < a.T ? r0 + rows_per_group : a.T;
  const int v0 = chunk * kChunk;
  const int n = a.V - v0 < kChunk ? a.V - v0 : kChunk;
  const bool hist = SPARSE && a.r.history != nullptr;
  const bool bias = SPARSE && a.r.bias_ids != nullptr;
  uint32_t* cnt = lds;
  uint32_t* last = lds + (hist ? kChunk : 0);

  int64_t pb = -1, ps = 0, pe = 0;  // the history counted in cnt; pb < 0: none, cnt not cleared
  int64_t qb = -1, qe = -1;         // the bias list in last

  for (int64_t row = r0; row < r1; ++row) {
    const TI* z = (const TI*)a.logits + row * a.ld + v0;
    TO* out = OP == Op::kStats ? nullptr : (TO*)a.out + row * a.out_ld + v0;
    float lse = 0.f, ent = 0.f, g = 0.f, e = 0.f;
    int tok = -1;  // of the row, relative to the chunk
    if constexpr (OP != Op::kAdjust) tok = (unsigned)a.tokens[row] < (unsigned)a.V ? a.tokens[row] - v0 : -1;
    if constexpr (OP == Op::kGrad) {
      lse = a.lse[row];
      g = (unsigned)a.tokens[row] < (unsigned)a.V ? a.grad_logp[row] : 0.f;
      if (a.grad_entropy) {
        e = a.grad_entropy[row];
        ent = a.entropy[row];
      }
      if ((g == 0.f && e == 0.f) || lse == kNegInf) {
        for (int i = threadIdx.x; i < n; i += kThreads) out[i] = (TO)0.f;
        continue;
      }
    }
    const int64_t mrow = a.r.mask ? (a.r.mask_rows ? (int64_t)a.r.mask_rows[row] : row) : -1;
    const bool masked = a.r.mask && mrow >= 0 && mrow < a.r.n_masks;

    Vec<TI, E> in[NV];
    uint32_t word[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = (j * kThreads + (int)threadIdx.x) * E;
      word[j] = ~0u;
      if (i + E <= n) {
        in[j] = load_vec<TI, E>(z + i);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) in[j].v[k] = i + k < n ? z[i + k] : (TI)0.f;
      }
      if (masked && i < n) word[j] = a.r.mask[mrow * a.r.mask_ld + ((v0 + i) >> 5)] >> ((v0 + i) & 31);
    }

    if (hist) {
      const int64_t N = a.r.history_len;
      const int64_t b = clamp64(a.r.hist_begin[row], 0, N);
      const int64_t s = a.r.hist_split ? clamp64(a.r.hist_split[row], b, N) : b;
      const int64_t t = clamp64(a.r.hist_end[row], s, N);
      int64_t from = pe;
      if (b != pb || s != ps || t < pe) {
        for (int i = threadIdx.x; i < kChunk; i += kThreads) cnt[i] = 0;
        from = b;
        __syncthreads();
      }
      count_tokens(cnt, a.r.history, from, s, t, v0, n);
      pb = b;
      ps = s;
      pe = t;
    }
    if (bias) {
      const int64_t b = clamp64(a.r.bias_begin[row], 0, a.r.bias_len);
      const int64_t t = clamp64(a.r.bias_end[row], b, a.r.bias_len);
      if (b != qb || t != qe) {
        for (int i = threadIdx.x; i < kChunk; i += kThreads) last[i] = 0;
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
    const float rho = hist && a.r.repetition ? a.r.repetition[row] : 1.f;
    const float inv_rho = 1.f / rho;
    const float freq = hist && a.r.frequency ? a.r.frequency[row] : 0.f;
    const float pres = hist && a.r.presence ? a.r.presence[row] : 0.f;

    float x[kPer], slope[OP == Op::kGrad ? kPer : 1];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = (j * kThreads + (int)threadIdx.x) * E;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        float y = widen(in[j].v[k]);
        float sl = 1.f;
        if (hist) {
          const uint32_t w = cnt[i + k];
          if (w) {
            if (a.r.repetition) {
              sl = y > 0.f ? inv_rho : rho;
              y = y > 0.f ? y / rho : y * rho;
            }
            const uint32_t c = w & ~kPromptBit;
            if (c) {
              if (a.r.frequency) y = y - freq * (float)c;
              if (a.r.presence) y = y - pres;
            }
          }
        }
        if (bias) {
          const uint32_t w = last[i + k];
          if (w) y = y + a.r.bias_values[w - 1];
        }
        y = y * a.inv_tau;
        const bool off = !((word[j] >> k) & 1u) || i + k >= n;
        x[j * E + k] = off ? kNegInf : y;
        if constexpr (OP == Op::kGrad) slope[j * E + k] = off ? 0.f : sl * a.inv_tau;
      }
    }

    if constexpr (OP == Op::kAdjust) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = (j * kThreads + (int)threadIdx.x) * E;
        Vec<TO, E> o;
#pragma unroll
        for (int k = 0; k < E; ++k) o.v[k] = narrow<TO>(x[j * E + k]);
        if (i + E <= n) {
          store_vec<TO, E>(out + i, o);
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (i + k < n) out[i + k] = o.v[k];
        }
      }
    } else if constexpr (OP == Op::kGrad) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = (j * kThreads + (int)threadIdx.x) * E;
        Vec<TO, E> o;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const float q = x[j * E + k] - lse;
          const float p = exp_hw(q);
          float up = i + k == tok ? g : 0.f;
          up = up - p * (g + e * (fmaxf(q, kFloor) + ent));
          const float sl = slope[j * E + k];
          o.v[k] = narrow<TO>(sl == 0.f ? 0.f : up * sl);
        }
        if (i + E <= n) {
          store_vec<TO, E>(out + i, o);
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (i + k < n) out[i + k] = o.v[k];
        }
      }
    } else {
      float m = kNegInf;
#pragma unroll
      for (int k = 0; k < kPer; ++k) m = fmaxf(m, x[k]);
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
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = (j * kThreads + (int)threadIdx.x) * E;
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (i + k == tok) tok_x = x[j * E + k];
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        float top = wstat[0].m;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, wstat[w].m);
        Partial p = {top, 0.f, 0.f, tok >= 0 && tok < n ? tok_x : 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const Stat t = shift(wstat[w], top);
          p.s += t.s;
          p.u += t.u;
        }
        ((Partial*)a.part)[row * n_chunks + chunk] = p;
      }
    }
    // the next row changes what this one read from LDS
    if (row + 1 < r1) __syncthreads();
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
      group = fill < 1 ? 1 : fill > 16 ? 16 : (int)fill;
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
