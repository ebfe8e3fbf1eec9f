// Changed logits on gfx950: penalties, biases and grammar masks applied to the
// logits of T rows, the softmax statistics of the result and their gradient.
//
// Mathematics, per entry (include/tim_policy.h has the order and the roundings):
//   y = rule(z): penalties of the tokens in the row's history, bias, mask;
//       x = y / tau
//   logprobs: per chunk m = max y, and with t = (y - m) log2(e) / tau the sums
//             s = sum 2^t, u = sum 2^t t; a merge over the chunks gives
//             lse = M / tau + log S, H = log S - ln 2 U / S
//   backward: dz = slope (g [v = tok] - p (g + e (log p + H))), p = e^(x-lse),
//             and where lse is too coarse for it the row's M and log S anew
//
// All three are one pass over the logits (read once; adjust and backward write
// as many) and bound by HBM. A workgroup takes one chunk of TIM_RULE_CHUNK
// vocabulary entries of consecutive rows. The sparse changes live in LDS, one
// word per entry of the chunk: bit 31 = token of the prompt, the rest = count in
// the output (integer atomics, so the order of the tokens does not matter), and
// in a second word the last bias entry of that id (an integer maximum). A
// chunk's workgroup reads the row's whole history and keeps what falls into it;
// rows whose history extends the last row's (the rows of one response in a
// packed stream) add only the new tokens.
//
// Few entries of a row are touched. A bitmap tells a thread which of its
// entries are, and it walks those by themselves, picking each out of its
// registers; with the penalties' code inside the pass over the row, once per
// entry of a load, 4096 rows of 151936 logits with up to 1280 tokens of history
// took 574 us against 533 (before other steps made both faster).
//
// Reads reach 7 TB/s (4096 rows of 151936 fp32 logits without rules 349 us). With histories, and for 16-bit logits, the
// vector instructions of the row loop bound the statistics (442 us fp32, 386 us bf16, 251 us bf16 without rules),
// so whole chunks, all but the last of a row, take a path without bounds per load (with them 458, 447 and 296 us).

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.h"
#include "policy.h"
#include "tilepass.h"

namespace tim {
namespace {

constexpr int kChunk = TIM_RULE_CHUNK;
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
static_assert(kWaves == 8, "the workgroup's merge rotates over eight lanes");
constexpr int kPer = kChunk / kThreads;  // entries per thread
constexpr int kMaxGroup = 16;            // rows of one workgroup
constexpr int kMaxChunks = (TIM_MAX_VOCAB + kChunk - 1) / kChunk;
static_assert(kMaxChunks <= 64, "the merge holds a row's chunks in one wave");
constexpr float kLn2 = 0.6931471805599453f;
constexpr uint32_t kPromptBit = 0x80000000u;
// 2^kFloor is 0 in fp32; it takes the place of -inf in the products p * log p.
constexpr float kFloor = -300.f;

enum class Op { kAdjust, kStats, kGrad };

template <class T>
__device__ __forceinline__ float widen(T x) { return (float)x; }

// N consecutive elements of a chunk at entry c of it: p the chunk's first, the
// same in every lane (one 32-bit offset per lane then makes the address), and
// aligned to its element only.
template <class T, int N>
struct Vec {
  T v[N];
};
template <class T>
__device__ __forceinline__ T* entry(T* p, int c) {
  return (T*)((std::conditional_t<std::is_const_v<T>, const char, char>*)p + (uint32_t)(c * (int)sizeof(T)));
}
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x2 i32x2_by2 __attribute__((aligned(2)));
typedef i32x4 i32x4_by2 __attribute__((aligned(2)));
// Streaming loads: the pass does not read its logits again (log-probs of 4096
// rows of 151936 fp32 logits 442 us against 459, 64 rows 16.1 against 18.4).
template <class T, int N>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p, int c) {
  static_assert(sizeof(Vec<T, N>) == 16, "one load");
  Vec<T, N> r;
  const i32x4 q = __builtin_nontemporal_load((const i32x4_by2*)entry(p, c));
  __builtin_memcpy(&r, &q, 16);
  return r;
}
// past: past the caches, for outputs too large to be found there again.
template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, int c, const Vec<T, N>& r, bool past) {
  if (!past) {
    __builtin_memcpy(entry(p, c), &r, sizeof(r));
    return;
  }
  constexpr int kWide = sizeof(r) < 16 ? (int)sizeof(r) : 16;
  typedef std::conditional_t<kWide == 8, i32x2, i32x4> V;
  typedef std::conditional_t<kWide == 8, i32x2_by2, i32x4_by2> U;
#pragma unroll
  for (int b = 0; b < (int)sizeof(r); b += kWide) {
    V q;
    __builtin_memcpy(&q, (const char*)&r + b, kWide);
    __builtin_nontemporal_store(q, (U*)((char*)entry(p, c) + b));
  }
}

// Softmax statistics of a set of entries, the logits short of the temperature:
// m = max y, and with t = (y - m) log2(e) / tau: s = sum 2^t, u = sum 2^t t.
// Differences first, then the factor, so that rows of the type's lowest value
// do not overflow.
struct Stat {
  float m, s, u;
};

// The statistics over a higher maximum, c = log2(e) / tau. A set without a
// finite maximum has s = u = 0 (or NaN), so any finite shift keeps it.
__device__ __forceinline__ Stat shift(const Stat& a, float m, float c) {
  const float t = fmaxf((a.m - m) * c, -1e30f);
  const float k = exp2_hw(t);
  return {m, a.s * k, k * (a.u + a.s * t)};
}

// Over the wave, the same in every lane: rotations within 16 lanes, then the
// four groups of them.
template <int N>
__device__ __forceinline__ float ror(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xF, 0xF, false));
#else
  return x;
#endif
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, ror<8>(x));
  x = fmaxf(x, ror<4>(x));
  x = fmaxf(x, ror<2>(x));
  x = fmaxf(x, ror<1>(x));
  return group_max(x);
}
__device__ __forceinline__ float wave_sum(float x) {
  x += ror<8>(x);
  x += ror<4>(x);
  x += ror<2>(x);
  x += ror<1>(x);
  return group_sum(x);
}

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}

// A token less the chunk's first entry, if it falls into the chunk's n: marked
// as the prompt's, or counted.
__device__ __forceinline__ void count_token(uint32_t* cnt, uint32_t* touched, uint32_t t, bool given, int n) {
  if (t < (uint32_t)n) {
    atomicOr(&touched[t >> 5], 1u << (t & 31));
    if (given)
      atomicOr(&cnt[t], kPromptBit);
    else
      atomicAdd(&cnt[t], 1u);
  }
}

// Tokens history[from .. to), the prompt's before split. Two loads a thread are
// in flight at a time: more take registers from the rows' (with two 64 rows of
// 151936 logits take 16.1 us, with four 17.2, with eight 17.8; 4096 rows 442,
// 448 and 477).
__device__ __forceinline__ void count_tokens(uint32_t* cnt, uint32_t* touched, const int32_t* __restrict__ history,
                                             int64_t from, int64_t split, int64_t to, int v0, int n) {
  constexpr int kStep = 2 * kThreads;
  for (int64_t i = from; i < to; i += kStep) {
    const int left = to - i < kStep ? (int)(to - i) : kStep;
    const int given = split <= i ? 0 : split - i < kStep ? (int)(split - i) : kStep;  // of them, the prompt's
    const int32_t* h = history + i;
    uint32_t t[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int c = k * kThreads + (int)threadIdx.x;
      t[k] = c < left ? (uint32_t)*entry(h, c) - (uint32_t)v0 : ~0u;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) count_token(cnt, touched, t[k], k * kThreads + (int)threadIdx.x < given, n);
  }
}

// p[i] for an index that is the same in every lane, through the scalar cache:
// no kernel writes these arrays while it reads them, and what an earlier launch
// wrote (the merge lse and entropy) is seen from the start of the next.
template <class T>
__device__ __forceinline__ T scalar(const T* p, int64_t i) {
  typedef const __attribute__((address_space(4))) T* constant;
  return ((constant)(uint64_t)p)[i];
}

// The kernel's arguments where the launch left them, read again where they are
// used (through the scalar cache): they are more than the scalar registers hold,
// and a spilled one costs a vector instruction each way. Opaque, so that the
// reads are not gathered in one place.
typedef const __attribute__((address_space(4))) RuleArgs* ArgsPtr;
__device__ __forceinline__ ArgsPtr kernel_args() {
#if defined(__HIP_DEVICE_COMPILE__)
  ArgsPtr p = (ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
#else
  ArgsPtr p = nullptr;
#endif
  asm volatile("" : "+s"(p));
  return p;
}

// What a row's changes are.
struct Row {
  int64_t begin, split, end;  // of the history
  int64_t bias0, bias1;
  int64_t mask;               // row of the mask, -1: none
  float rho, freq, pres;
};

__device__ __forceinline__ Row read_row(int64_t row, bool hist, bool bias) {
  const ArgsPtr a = kernel_args();
  Row w = {};
  w.mask = -1;
  if (a->r.mask) {
    const int64_t m = a->r.mask_rows ? (int64_t)scalar(a->r.mask_rows, row) : row;
    if (m >= 0 && m < a->r.n_masks) w.mask = m;
  }
  // a penalty that is left out takes the value that changes nothing
  w.rho = 1.f;
  if (hist) {
    const int64_t N = a->r.history_len;
    w.begin = clamp64(scalar(a->r.hist_begin, row), 0, N);
    w.split = a->r.hist_split ? clamp64(scalar(a->r.hist_split, row), w.begin, N) : w.begin;
    w.end = clamp64(scalar(a->r.hist_end, row), w.split, N);
    if (a->r.repetition) w.rho = scalar(a->r.repetition, row);
    if (a->r.frequency) w.freq = scalar(a->r.frequency, row);
    if (a->r.presence) w.pres = scalar(a->r.presence, row);
  }
  if (bias) {
    w.bias0 = clamp64(scalar(a->r.bias_begin, row), 0, a->r.bias_len);
    w.bias1 = clamp64(scalar(a->r.bias_end, row), w.bias0, a->r.bias_len);
  }
  return w;
}

// y with the penalties of an entry whose word in the row's counts is u; the
// factor the repetition penalty puts on the entry's slope in `factor`.
__device__ __forceinline__ float penalise(float y, uint32_t u, const Row& w, float inv_rho, float& factor) {
  const bool pos = y > 0.f;
  factor = pos ? inv_rho : w.rho;
  const float v = pos ? y / w.rho : y * w.rho;
  const uint32_t count = u & ~kPromptBit;
  return count ? v - w.freq * (float)count - w.pres : v;
}

// x where the bit is set, else z.
__device__ __forceinline__ float choose(uint32_t bits, int k, float x, float z) {
  const int m = __builtin_amdgcn_sbfe((int)bits, k, 1);
  return __int_as_float((m & __float_as_int(x)) | (~m & __float_as_int(z)));
}

// LDS words of a history or a bias list: one per entry, and their bitmap.
constexpr int kWords = kChunk + kChunk / 32;
__device__ __forceinline__ void clear_words(uint32_t* words, int tid) {
  for (int c = tid * 4; c < kWords; c += kThreads * 4) *(uint4*)(words + c) = uint4{0, 0, 0, 0};
}

// The entries of a bias list that fall into a chunk's n from v0 on: the last one of each id.
__device__ __forceinline__ void mark_biases(uint32_t* last, const int32_t* ids, int64_t from, int64_t to, int v0, int n,
                                            int tid) {
  for (int64_t k = from + tid; k < to; k += kThreads) {
    const uint32_t id = (uint32_t)ids[k] - (uint32_t)v0;
    if (id < (uint32_t)n) {
      atomicOr(&last[kChunk + (id >> 5)], 1u << (id & 31));
      atomicMax(&last[id], (uint32_t)k + 1u);
    }
  }
}

// |lse| from which a row's gradient does not go by it. p = e^(x - lse) is
// relatively as far off as fp32's lse is absolutely, by two roundings: 2^-14
// short of this, but at fp32's lowest value lse holds no log n any more, and
// over a temperature below 1 it is infinite.
constexpr float kFarLse = 1024.f;

// The whole gradient of such a row in one workgroup, which first forms the
// row's maximum y and log S as the statistics do: p = e^((y - top) / tau - log
// S). One workgroup, so that the gradient may lie where the logits do. A model's
// rows hardly come here: 150 rows of 50257 fp16 logits with histories, all of
// them far, take 123 us against 17, 2047 of 151936 fp32 logits 1640 against 350.
template <class TI, class TO, bool SPARSE>
__device__ __forceinline__ void far_row(int64_t row, uint32_t* lds, Stat* wstat) {
  const ArgsPtr a = kernel_args();
  const int tid = threadIdx.x;
  const bool hist = SPARSE && a->r.history != nullptr;
  const bool bias = SPARSE && a->r.bias_ids != nullptr;
  uint32_t* cnt = lds;
  uint32_t* last = lds + (hist ? kWords : 0);
  const Row w = read_row(row, hist, bias);
  const int token = scalar(a->tokens, row);
  const float g = (unsigned)token < (unsigned)a->V ? scalar(a->grad_logp, row) : 0.f;
  const float e = a->grad_entropy ? scalar(a->grad_entropy, row) : 0.f;
  const float ent = a->grad_entropy ? scalar(a->entropy, row) : 0.f;
  const float inv_tau = a->inv_tau, log2e_tau = kLog2e * inv_tau;
  const float inv_rho = 1.f / w.rho;
  const TI* z = (const TI*)a->logits + row * a->ld;
  TO* out = (TO*)a->out + row * a->out_ld;
  const uint32_t* mask = a->r.mask + w.mask * a->r.mask_ld;
  // each(v, open, y, factor of the slope) for the thread's entries of every chunk
  auto walk = [&](auto&& each) {
    for (int v0 = 0; v0 < a->V; v0 += kChunk) {
      const int n = a->V - v0 < kChunk ? a->V - v0 : kChunk;
      if constexpr (SPARSE) {
        __syncthreads();  // the last chunk's words have been read
        if (hist) clear_words(cnt, tid);
        if (bias) clear_words(last, tid);
        __syncthreads();
        if (hist) count_tokens(cnt, cnt + kChunk, a->r.history, w.begin, w.split, w.end, v0, n);
        if (bias) mark_biases(last, a->r.bias_ids, w.bias0, w.bias1, v0, n, tid);
        __syncthreads();
      }
      for (int c = tid; c < n; c += kThreads) {
        const int v = v0 + c;
        float y = widen(z[v]), factor = 1.f;
        if constexpr (SPARSE) {
          const uint32_t u = hist ? cnt[c] : 0u;
          if (u) y = penalise(y, u, w, inv_rho, factor);
          const uint32_t b = bias ? last[c] : 0u;
          if (b) y = y + a->r.bias_values[b - 1];
        }
        each(v, w.mask < 0 || (mask[v >> 5] >> (v & 31) & 1u), y, factor);
      }
    }
  };
  float m = kNegInf, s = 0.f;  // of the thread's entries; a NaN or +inf makes s NaN
  walk([&](int, bool open, float y, float) {
    if (!open || y == kNegInf) return;
    const float top = fmaxf(m, y);
    s = s * exp2_hw((m - top) * log2e_tau) + exp2_hw((y - top) * log2e_tau);
    m = top;
  });
  const float wave_top = wave_max(m);
  s = wave_sum(shift({m, s, 0.f}, wave_top, log2e_tau).s);
  if ((tid & 63) == 0) wstat[tid >> 6] = {wave_top, s, 0.f};
  __syncthreads();
  float top = kNegInf, S = 0.f;
#pragma unroll
  for (int j = 0; j < kWaves; ++j) top = fmaxf(top, wstat[j].m);
#pragma unroll
  for (int j = 0; j < kWaves; ++j) S += shift(wstat[j], top, log2e_tau).s;
  const bool none = top == kNegInf && S == 0.f;  // nothing allowed
  const float log_s = logf(S);
  walk([&](int v, bool open, float y, float factor) {
    float r = 0.f;
    if (open && !none) {
      const float q = (y - top) * inv_tau - log_s;
      const float p = exp2_hw(q * kLog2e);
      r = e == 0.f ? -p * g : -p * (g + e * (fmaxf(q, kFloor) + ent));
      r = (v == token ? g + r : r) * (factor * inv_tau);
    }
    out[v] = narrow<TO>(r);
  });
  __syncthreads();  // wstat and the words have been read
}

// Three workgroups a CU (80 registers): with two 4096 rows of 151936 logits take 546 us against 442, 64 rows 18.6
// against 16.1, the gradient of 2047 rows 361 against 337; four spill.
template <Op OP, class TI, class TO, bool SPARSE>
__global__ __launch_bounds__(kThreads, 6) void rules_kernel(const RuleArgs args, int n_chunks, int rows_per_group) {
  const ArgsPtr a = kernel_args();  // args
  (void)args;
  constexpr int E = 16 / (int)sizeof(TI);  // entries per load
  constexpr int NV = kPer / E;             // loads per thread
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ Stat wstat[2][kWaves];  // by row in turn, so that a row need not wait for the last one's merge
  __shared__ float tok_x[2];
  // of the group's rows, stored at the end: a wait for the next row's loads would be one for the store too
  __shared__ Partial parts[OP == Op::kStats && SPARSE ? kMaxGroup : 1];

  const int chunk = (int)(blockIdx.x % (unsigned)n_chunks);
  const int64_t r0 = (int64_t)(blockIdx.x / (unsigned)n_chunks) * rows_per_group;
  const int n_rows = (int)(a->T - r0 < rows_per_group ? a->T - r0 : rows_per_group);
  const int v0 = chunk * kChunk;
  int n = a->V - v0 < kChunk ? a->V - v0 : kChunk;
  int tid = threadIdx.x;
  const bool hist = SPARSE && a->r.history != nullptr;
  const bool bias = SPARSE && a->r.bias_ids != nullptr;
  uint32_t* cnt = lds;
  uint32_t* last = lds + (hist ? kWords : 0);
  const float log2e_tau = kLog2e * a->inv_tau;

  Vec<TI, E> in[NV];  // the row's logits, requested ahead
  auto request = [&](int64_t row) {
    const ArgsPtr a = kernel_args();
    const TI* z = (const TI*)a->logits + row * a->ld + v0;
    if (n == kChunk) {
#pragma unroll
      for (int j = 0; j < NV; ++j) in[j] = load_vec<TI, E>(z, (j * kThreads + tid) * E);
      return;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * kThreads + tid) * E;
      if (c + E <= n) {
        in[j] = load_vec<TI, E>(z, c);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) in[j].v[k] = c + k < n ? entry(z, c)[k] : (TI)0.f;
      }
    }
  };
  request(r0);
  auto clear = [&](uint32_t* words) { clear_words(words, tid); };
  if (hist) clear(cnt);
  if (bias) clear(last);
  if constexpr (SPARSE) __syncthreads();

  int64_t pb = -1, ps = 0, pe = 0;  // the history counted in cnt; pb < 0: none yet
  int64_t qb = -1, qe = -1;         // the bias list in last; qb < 0: none yet
  Row w = read_row(r0, hist, bias);
  // With `ahead`, the tokens by which this row's history extends the last one's, at most one per thread, were
  // requested with the row.
  bool ahead = false;
  uint32_t token_ahead = ~0u;
  uint32_t far = 0;  // backward: bit i: row i of the group is left to the end, where no register holds its state

  for (int i = 0; i < n_rows; ++i) {
    // Opaque copies: the entries' bounds and offsets are worked out where they are used, not once for all rows and
    // kept in (spilled) registers.
    asm volatile("" : "+s"(n), "+v"(tid));
    const int64_t row = r0 + i;
    const ArgsPtr a = kernel_args();
    const float inv_tau = a->inv_tau;
    const bool past = OP != Op::kStats && a->past_caches;
    TO* out = OP == Op::kStats ? nullptr : (TO*)a->out + row * a->out_ld + v0;
    int tok = -1;  // relative to the chunk; negative or past it: elsewhere
    float lse = 0.f, ent = 0.f, g = 0.f, e = 0.f;
    if constexpr (OP != Op::kAdjust) {
      const int token = scalar(a->tokens, row);
      const bool valid = (unsigned)token < (unsigned)a->V;
      if (valid) tok = token - v0;
      if constexpr (OP == Op::kGrad) {
        lse = scalar(a->lse, row);
        g = valid ? scalar(a->grad_logp, row) : 0.f;
        if (a->grad_entropy) {
          e = scalar(a->grad_entropy, row);
          ent = scalar(a->entropy, row);
        }
        const bool zero = g == 0.f && e == 0.f;
        if (zero || fabsf(lse) >= kFarLse) {
          if (zero)
            for (int c = tid; c < n; c += kThreads) *entry(out, c) = (TO)0.f;
          else
            far |= 1u << i;
          if (i + 1 < n_rows) {
            request(row + 1);
            w = read_row(row + 1, hist, bias);
            ahead = false;
          }
          continue;
        }
      }
    }

    // bit k: entry k of the load is allowed and lies in the vocabulary
    uint32_t open[NV];
    const uint32_t* mask = a->r.mask + w.mask * a->r.mask_ld + v0 / 32;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * kThreads + tid) * E;
      open[j] = ~0u;
      if (n < kChunk) open[j] = c + E <= n ? ~0u : c < n ? (1u << (n - c)) - 1u : 0u;
      if (w.mask >= 0 && c < n) open[j] &= *entry(mask, c >> 5) >> (c & 31);
    }

    if (hist) {
      const int64_t b = w.begin, s = w.split, t = w.end;
      int64_t from = pe;
      if (b != pb || s != ps || t < pe) {
        from = b;
        if (pb >= 0) {
          clear(cnt);
          __syncthreads();
        }
      }
      if (ahead)
        count_token(cnt, cnt + kChunk, token_ahead, from + tid < s, n);
      else
        count_tokens(cnt, cnt + kChunk, a->r.history, from, s, t, v0, n);
      pb = b;
      ps = s;
      pe = t;
    }
    if (bias) {
      const int64_t b = w.bias0, t = w.bias1;
      if (b != qb || t != qe) {
        if (qb >= 0) {
          clear(last);
          __syncthreads();
        }
        mark_biases(last, a->r.bias_ids, b, t, v0, n, tid);
        qb = b;
        qe = t;
      }
    }
    if constexpr (SPARSE) __syncthreads();

    float x[kPer];  // entry k of the thread: number k % E of its load k / E
    uint32_t opened = 0, touched = 0;
    constexpr uint32_t kAll = (1u << E) - 1u, kAllOpen = (uint32_t)((1ull << kPer) - 1u);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      opened |= (open[j] & kAll) << (j * E);
      if constexpr (SPARSE) {
        const int c = (j * kThreads + tid) * E;
        const uint32_t t = (hist ? cnt[kChunk + (c >> 5)] : 0u) | (bias ? last[kChunk + (c >> 5)] : 0u);
        touched |= (t >> (c & 31) & kAll) << (j * E);
      }
#pragma unroll
      for (int k = 0; k < E; ++k) x[j * E + k] = widen(in[j].v[k]);
    }
    const bool some_off = __any(opened != kAllOpen);
    const float inv_rho = SPARSE ? 1.f / w.rho : 1.f;

    // The gradient of an entry: y short of the temperature.
    auto grad = [&](float y) {
      const float q = fmaf(y, inv_tau, -lse);
      const float p = exp2_hw(q * kLog2e);
      return e == 0.f ? -p * g : -p * (g + e * (fmaxf(q, kFloor) + ent));
    };
    float r[OP == Op::kGrad ? kPer : 1];
    if constexpr (OP == Op::kGrad) {
      if (e == 0.f) {
        const float gs = -g * inv_tau;
#pragma unroll
        for (int k = 0; k < kPer; ++k) r[k] = exp2_hw(fmaf(x[k], inv_tau, -lse) * kLog2e) * gs;
      } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) r[k] = grad(x[k]) * inv_tau;
      }
      if (tok >= 0 && tok < n && tok / E % kThreads == tid) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if ((k / E * kThreads + tid) * E + k % E == tok) r[k] = (g + grad(x[k])) * inv_tau;
      }
    }
    if constexpr (SPARSE) {
      // the touched ones by themselves, picked out of the registers and put back
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        for (uint32_t left = touched >> (j * E) & kAll; left; left &= left - 1) {
          const int at = __builtin_ctz(left);
          const int c = (j * kThreads + tid) * E + at;
          float y = x[j * E];
#pragma unroll
          for (int k = 1; k < E; ++k) y = k == at ? x[j * E + k] : y;
          float factor = 1.f;
          const uint32_t u = hist ? cnt[c] : 0u;
          if (u) y = penalise(y, u, w, inv_rho, factor);
          const uint32_t b = bias ? last[c] : 0u;
          if (b) y = y + a->r.bias_values[b - 1];
          if constexpr (OP == Op::kGrad) {
            y = (c == tok ? g + grad(y) : grad(y)) * (factor * inv_tau);
#pragma unroll
            for (int k = 0; k < E; ++k) r[j * E + k] = k == at ? y : r[j * E + k];
          } else {
#pragma unroll
            for (int k = 0; k < E; ++k) x[j * E + k] = k == at ? y : x[j * E + k];
          }
        }
      }
    }
    if constexpr (OP == Op::kAdjust) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = x[k] * inv_tau;
    }
    if (some_off) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if constexpr (OP == Op::kGrad)
          r[k] = choose(opened, k, r[k], 0.f);
        else
          x[k] = choose(opened, k, x[k], kNegInf);
      }
    }
    // The next row is requested before this one is stored: memory operations end in order, and loads behind the stores
    // would wait for them (the gradient of 2047 rows of 151936 fp32 logits 343 us against 337; of bf16 logits the same).
    if (i + 1 < n_rows) {
      request(row + 1);
      w = read_row(row + 1, hist, bias);
      ahead = hist && w.begin == pb && w.split == ps && w.end >= pe && w.end - pe <= kThreads;
      if (ahead) token_ahead = tid < (int)(w.end - pe) ? (uint32_t)*entry(a->r.history + pe, tid) - (uint32_t)v0 : ~0u;
    }
    if constexpr (OP != Op::kStats) {
      auto rounded = [&](int j) {
        Vec<TO, E> o;
#pragma unroll
        for (int k = 0; k < E; ++k) o.v[k] = narrow<TO>(OP == Op::kGrad ? r[j * E + k] : x[j * E + k]);
        return o;
      };
      // The loads have to be there, the stores behind them need not be done. Where both are in a straight line the
      // compiler's wait is that one.
      auto arrived = [&] {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          i32x4 q;
          __builtin_memcpy(&q, &in[j], 16);
          asm volatile("" : "+v"(q));
          __builtin_memcpy(&in[j], &q, 16);
        }
        if constexpr (SPARSE) asm volatile("" : "+v"(token_ahead));
      };
      if (n == kChunk) {
#pragma unroll
        for (int j = 0; j < NV; ++j) store_vec<TO, E>(out, (j * kThreads + tid) * E, rounded(j), past);
        arrived();
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (j * kThreads + tid) * E;
          const Vec<TO, E> o = rounded(j);
          if (c + E <= n) {
            store_vec<TO, E>(out, c, o, past);
          } else {
#pragma unroll
            for (int k = 0; k < E; ++k)
              if (c + k < n) entry(out, c)[k] = o.v[k];
          }
        }
        arrived();
      }
    }

    if constexpr (OP == Op::kStats) {
      float m = x[0], low = x[0];
#pragma unroll
      for (int k = 1; k < kPer; ++k) {
        m = fmaxf(m, x[k]);
        low = fminf(low, x[k]);
      }
      m = wave_max(m);
      const float at = m == kNegInf ? 0.f : m;
      float s = 0.f, u = 0.f;
      if (__any(!((low - at) * log2e_tau > kFloor))) {  // entries whose 2^t is 0, t perhaps -inf (or a NaN)
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          const float t = (x[k] - at) * log2e_tau;
          const float p = exp2_hw(t);
          s += p;
          u = fmaf(p, fmaxf(t, kFloor), u);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          const float t = (x[k] - at) * log2e_tau;
          const float p = exp2_hw(t);
          s += p;
          u = fmaf(p, t, u);
        }
      }
      s = wave_sum(s);
      u = wave_sum(u);
      const int par = i & 1;
      if ((tid & 63) == 0) wstat[par][tid >> 6] = {m, s, u};
      if (tok >= 0 && tok < n && tok / E % kThreads == tid) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if ((k / E * kThreads + tid) * E + k % E == tok) tok_x[par] = x[k];
      }
      __syncthreads();
      if (tid < 64) {  // lane l merges wave l % kWaves' with the others'
        const Stat mine = wstat[par][tid % kWaves];
        float top = fmaxf(mine.m, ror<4>(mine.m));
        top = fmaxf(top, ror<2>(top));
        top = fmaxf(top, ror<1>(top));
        Stat t = shift(mine, top, log2e_tau);
        t.s += ror<4>(t.s);
        t.s += ror<2>(t.s);
        t.s += ror<1>(t.s);
        t.u += ror<4>(t.u);
        t.u += ror<2>(t.u);
        t.u += ror<1>(t.u);
        if (tid == 0)
          (SPARSE ? parts[i] : ((Partial*)a->part)[row * n_chunks + chunk]) =
              Partial{top, t.s, t.u, tok >= 0 && tok < n ? tok_x[par] : 0.f};
      }
    } else if (SPARSE) {
      __syncthreads();  // the next row changes what this one read from LDS
    }
  }
  if constexpr (OP == Op::kGrad) {
    for (; far; far &= far - 1) {  // a row's chunks share its work out by the rows; a launch's rows fit 32 bits
      const int64_t row = r0 + __builtin_ctz(far);
      const unsigned chunks = (unsigned)(kernel_args()->V + kChunk - 1) / kChunk;
      if ((unsigned)row % chunks == (unsigned)v0 / kChunk) far_row<TI, TO, SPARSE>(row, lds, wstat[0]);
    }
  }
  if constexpr (OP == Op::kStats && SPARSE) {
    __syncthreads();
    if (tid < n_rows) ((Partial*)a->part)[(r0 + tid) * n_chunks + chunk] = parts[tid];
  }
}

// One wave per row: lane c holds chunk c's partial.
__global__ __launch_bounds__(256) void rules_merge(const Partial* __restrict__ part, const int32_t* __restrict__ tokens,
                                                   int64_t T, int V, int n_chunks, float inv_tau,
                                                   float* __restrict__ logp, float* __restrict__ entropy,
                                                   float* __restrict__ lse) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= T) return;
  Partial p = {kNegInf, 0.f, 0.f, 0.f};
  if (lane < n_chunks) p = part[row * n_chunks + lane];
  const float top = wave_max(p.m);
  const Stat t = shift({p.m, p.s, p.u}, top, kLog2e * inv_tau);
  const float S = wave_sum(t.s);
  const float U = wave_sum(t.u);
  const int tok = tokens[row];
  const bool valid = (unsigned)tok < (unsigned)V;
  const float y = __shfl(p.ztok, valid ? tok / kChunk : 0);
  if (lane == 0) {
    const bool none = top == kNegInf && S == 0.f;  // nothing allowed
    const float log_s = logf(S);
    logp[row] = !valid ? __builtin_nanf("") : none ? kNegInf : (y - top) * inv_tau - log_s;
    if (entropy) entropy[row] = none ? 0.f : log_s - kLn2 * (U / S);
    if (lse) lse[row] = none ? kNegInf : top * inv_tau + log_s;
  }
}

int rule_lds_bytes(const RuleArgs& a) {
  return ((a.r.history ? 1 : 0) + (a.r.bias_ids ? 1 : 0)) * kWords * 4;
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
    RuleArgs b = rows_from(a, t0, rows, (int)sizeof(TI), (int)sizeof(TO));
    b.past_caches = a.T * a.V * (int64_t)sizeof(TO) > kCacheBytes;
    // Rows of one workgroup: histories that extend one another are counted once for the group, and the next row's
    // logits are on their way while a row is worked on, but only where the workgroups fill the CUs many times over.
    // At 4096 workgroups: log-probs of 4096 rows of 151936 logits 442 us (at 1024 workgroups 450, at 8192 437, one row
    // each 557), the gradient of 2047 rows 337 us (at 1024 410, at 8192 357, one row each 327).
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
                                                           a.V, n_chunks, a.inv_tau, logp + t0,
                                                           entropy ? entropy + t0 : nullptr,
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
