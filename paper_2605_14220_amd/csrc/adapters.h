// Low-rank adapters of many requests beside a shared projection, and their
// gradients, on gfx950. Rows are grouped by adapter (grouping.h); a workgroup
// takes a run of rows of one adapter:
//
//   shrink  u = x a^T            up to 64 rows, 512 elements of d
//   expand  out = base + u b^T   up to 64 rows, 256 columns (512 or 1024 where runs are short);
//           grad_x (+)= v a      for bf16 up to rank 64 by expand_flat, 256 or 512 columns
//   pass    v = grad b           up to 512 rows of one or two tiles of 256 columns (of 128 on the fp32
//           grad_b = grad^T u    instructions): grad is read once for both
//           grad_a = v^T x       the same pass over x, without the first product
//
// x, a and b are 16 bits wide; their products with each other run on the 16-bit
// matrix instructions, and so does bf16 grad times bf16 b. u and v stay in fp32.
// Where all else is bf16 the products that they enter run on the bf16 instructions,
// each as the sum of three bf16 numbers (split3); with fp16, and with grad of
// another type than the adapters', on the fp32 ones (16x16x4), for fp16's exponents
// do not hold such terms as they are. What a call moves, not what it computes,
// bounds it.

#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "vocab.h"

namespace tim {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
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
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 mfma(bf16x4 a, bf16x4 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s4 __attribute__((ext_vector_type(4)));
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4, a), __builtin_bit_cast(s4, b), c, 0, 0, 0);
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
// Past the caches, for rows that are too many to be found there again.
template <class V, int N, class T>
__device__ __forceinline__ V load_past(const T* p) {
  typedef V by_element __attribute__((aligned(sizeof(T))));
  return __builtin_nontemporal_load((const by_element*)p);
}
constexpr int64_t kCaches = (int64_t)256 << 20;
template <class T>
using x4 = T __attribute__((ext_vector_type(4)));
// x as the sum of three bf16 numbers, exactly where none overflows or is subnormal
// (24 bits are three times 8); an infinity or NaN alone in the first. In a product
// with an infinity terms of 0 or of the other sign give NaN, see sign_of.
__device__ __forceinline__ void split3(float x, __bf16 (&t)[3]) {
  t[0] = (__bf16)x;
  const float r = __builtin_isfinite((float)t[0]) ? x - (float)t[0] : 0.f;
  t[1] = (__bf16)r;
  t[2] = (__bf16)(r - (float)t[1]);
}

// A sum of products with such terms is NaN only where an operand is not finite. Then
// the sum with sign_of(x) in place of x, which no finite numbers make overflow, tells
// what it is: an infinity of that sign, or NaN (pass, whose rows are many, takes x
// itself). It is taken where a tile's sums hold NaN, for those elements alone: the
// others keep their bits. The look for NaN costs 0 to 1.7% of a call (48 rows on a
// head of 152064 60.5 us with it and without, 8192 rows' gradients 140.1 and 137.8);
// a NaN for each of 2047 rows takes their gradients from 212 to 900 us.
__device__ __forceinline__ __bf16 sign_of(float x) {
  return (__bf16)(x == 0.f || !__builtin_isfinite(x) ? x : __builtin_copysignf(0x1p-20f, x));
}
template <class V, int N>
__device__ __forceinline__ V signs_of(V x) {
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = sign_of((float)x[e]);
  return x;
}
__device__ __forceinline__ bool has_nan(f32x4 y) {
  return __builtin_isunordered(y[0], y[1]) || __builtin_isunordered(y[2], y[3]);
}

struct ExpandArgs {
  const float* u;     // [chunks, T, rp], summed and scaled here
  const void* terms;  // or null: u as bf16 [T, 3, rp], whose sums of three it is
  int64_t T;
  int32_t chunks, n, r, rp, N;
  const float* scales;
  const void* w;   // [n, N, r], or [n, r, N] where FLAT
  const void* base;
  int64_t base_ld;
  void* out;
  int64_t out_ld;
  int32_t past;  // out is larger than the caches
};

struct PassArgs {
  const void* src;  // [T, N]
  int64_t ld, T;
  const float* w;   // [T, rp]
  const void* b;    // [n, N, r], the contraction's
  float* part;      // [chunks, T, rp], the contraction's sums
  int32_t n, r, rp, N;
  float* out;       // [n, N, r], or [n, r, N] without the contraction
  float* out_part;  // [slots] of the same
  int32_t accumulate;
  int32_t past;  // src is larger than the caches
};

// The products over the runs of a list, see adapters_expand.hip and adapters_pass.hip.
hipError_t launch_expand(const ExpandArgs& a, int dtype, int out_dtype, bool flat, const RunList& l, hipStream_t s);
hipError_t launch_pass(const PassArgs& a, int src_dtype, int dtype, bool contract, int tiles, const RunList& l,
                       hipStream_t s);

#define TIM_LAUNCH(...)                      \
  do {                                       \
    __VA_ARGS__;                             \
    const hipError_t e_ = hipGetLastError(); \
    if (e_ != hipSuccess) return e_;         \
  } while (0)

}  // namespace tim
