// 4-bit microscaled floating point on gfx950: quantisation, the values of the
// codes, and the logits of a quantised head.
//
// Quantisation: 2^E = 2^(floor(log2 top) - 2) places a block's largest
// magnitude in [4, 8), the upper binade of E2M1; x 2^-E is exact in fp32, and
// the conversion to E2M1 is the hardware's (nearest even, saturating at 6).
// HBM-bound: 2 bytes read and 17/32 written per bf16 element. Four lanes share
// a block, so a wave reads and writes consecutive memory.
//
// Product: v_mfma_scale_f32_16x16x128_f8f6f4 on 4-bit operands, W as its first
// operand: lane l holds 32 elements, one scale block, of row l % 16, and its
// four results are consecutive vocabulary entries of one hidden row.

#include <hip/hip_runtime.h>

#include "kernels.h"
#include "policy.h"

namespace tim {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kGroup = 8;       // elements of one lane: a quarter of a block
constexpr int kGroupsEach = 4;  // groups per thread
constexpr int64_t kLaunchBlocks = (int64_t)1 << 23;  // a grid holds fewer than 2^32 threads

template <class T>
struct Group {
  T v[kGroup];
};

// Codes of the lane's eight elements and the scale byte of its block, from the
// block's largest magnitude: the four lanes' maximum of the bits, which order
// as the values do (a NaN or infinity tops them all).
__device__ __forceinline__ uint32_t quantise_group(const float (&x)[kGroup], uint32_t& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kGroup; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    top = b > top ? b : top;
  }
  uint32_t o = __shfl_xor(top, 1);
  top = o > top ? o : top;
  o = __shfl_xor(top, 2);
  top = o > top ? o : top;
  const uint32_t ex = top >> 23;  // biased exponent; 0 below 2^-126, where E is clamped anyway
  if (ex == 255) {
    scale = 255;
    return 0;
  }
  scale = ex > 2 ? ex - 2 : 0;
  const int e = 127 - (int)scale;
  uint32_t c = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, ldexpf(x[0], e), ldexpf(x[1], e), 1.f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, ldexpf(x[2], e), ldexpf(x[3], e), 1.f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, ldexpf(x[4], e), ldexpf(x[5], e), 1.f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, ldexpf(x[6], e), ldexpf(x[7], e), 1.f, 3);
#endif
  return c;
}

// Groups of eight elements, `per_row` of them in a row of stride ld; rows
// without gaps are one long row (per_row the total).
template <class T>
__global__ __launch_bounds__(kThreads) void quantise(const T* __restrict__ x, int64_t groups, int64_t first,
                                                     int64_t per_row, int64_t ld, uint8_t* __restrict__ codes,
                                                     uint8_t* __restrict__ scales) {
  const int64_t g0 = first + (int64_t)blockIdx.x * (kThreads * kGroupsEach) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int64_t g = g0 + j * kThreads;
    // a block's four lanes are on the same side of the end, which is a multiple of 4
    if (g >= groups) continue;
    const int64_t row = per_row == groups ? 0 : g / per_row;
    Group<T> in;
    __builtin_memcpy(&in, x + row * ld + (g - row * per_row) * kGroup, sizeof(in));
    float f[kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) f[i] = (float)in.v[i];
    uint32_t scale;
    const uint32_t c = quantise_group(f, scale);
    __builtin_memcpy(codes + g * 4, &c, 4);
    if ((g & 3) == 0) scales[g >> 2] = (uint8_t)scale;
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void dequantise(const uint8_t* __restrict__ codes,
                                                       const uint8_t* __restrict__ scales, int64_t groups,
                                                       int64_t first, T* __restrict__ out) {
  const int64_t g0 = first + (int64_t)blockIdx.x * (kThreads * kGroupsEach) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int64_t g = g0 + j * kThreads;
    if (g >= groups) continue;
    uint32_t c;
    __builtin_memcpy(&c, codes + g * 4, 4);
    const int s = scales[g >> 2];
    Group<T> o;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      // magnitudes 0 .. 7 in halves: 0 1 2 3 4 6 8 12
      const uint32_t m = (c >> (4 * i)) & 7u;
      const float a = ldexpf((float)((0xC8643210u >> (4 * m)) & 15u), s - 128);
      const float v = s == 255 ? __builtin_nanf("") : a;
      o.v[i] = (T)((c >> (4 * i)) & 8u ? -v : v);
    }
    __builtin_memcpy(out + g * kGroup, &o, sizeof(o));
  }
}

__device__ __forceinline__ f32x4 mfma_fp4(i32x4 a, int sa, i32x4 b, int sb, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
  const i32x8 b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, sa, 0, sb);
#else
  return c;
#endif
}

// One wave per 16 vocabulary entries and 16 hidden rows.
template <class T>
__global__ __launch_bounds__(256) void mxfp4_product(const Mxfp4LogitsArgs a) {
  const int lane = threadIdx.x & 63;
  const int v0 = ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)) * 16;
  const int64_t t0 = (int64_t)blockIdx.y * 16;
  if (v0 >= a.V) return;
  const int r = lane & 15, q = lane >> 4;
  // rows past the end repeat the last one; their results are not written
  const int64_t w = v0 + r < a.V ? v0 + r : a.V - 1;
  const int64_t h = t0 + r < a.T ? t0 + r : a.T - 1;
  const uint8_t* wc = a.w_codes + w * (a.d / 2) + q * 16;
  const uint8_t* hc = a.h_codes + h * (a.d / 2) + q * 16;
  const uint8_t* ws = a.w_scales + w * (a.d / 32) + q;
  const uint8_t* hs = a.h_scales + h * (a.d / 32) + q;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.d / 128; ++k)
    acc = mfma_fp4(*(const i32x4*)(wc + k * 64), ws[k * 4], *(const i32x4*)(hc + k * 64), hs[k * 4], acc);
  if (t0 + r >= a.T) return;
  T* out = (T*)a.logits + (t0 + r) * a.ld;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int v = v0 + 4 * q + i;
    if (v < a.V) out[v] = narrow<T>(acc[i] * a.inv_tau);
  }
}

template <class T>
hipError_t quantise_as(const void* x, int64_t rows, int d, int64_t ld, uint8_t* codes, uint8_t* scales,
                       hipStream_t s) {
  const int64_t groups = rows * d / kGroup;
  const int64_t per_row = ld == d ? groups : d / kGroup;
  const int64_t blocks = (groups + kThreads * kGroupsEach - 1) / (kThreads * kGroupsEach);
  for (int64_t b = 0; b < blocks; b += kLaunchBlocks) {
    const unsigned grid = (unsigned)(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
    quantise<T><<<grid, kThreads, 0, s>>>((const T*)x, groups, b * kThreads * kGroupsEach, per_row, ld, codes, scales);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t dequantise_as(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* out, hipStream_t s) {
  const int64_t groups = rows * d / kGroup;
  const int64_t blocks = (groups + kThreads * kGroupsEach - 1) / (kThreads * kGroupsEach);
  for (int64_t b = 0; b < blocks; b += kLaunchBlocks) {
    const unsigned grid = (unsigned)(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
    dequantise<T><<<grid, kThreads, 0, s>>>(codes, scales, groups, b * kThreads * kGroupsEach, (T*)out);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t product_as(const Mxfp4LogitsArgs& a, hipStream_t s) {
  const int64_t across = (a.V + 63) / 64;  // at most 8192
  const int64_t rows = kLaunchBlocks / across < 65535 ? kLaunchBlocks / across * 16 : 65535 * 16;
  for (int64_t t0 = 0; t0 < a.T; t0 += rows) {
    Mxfp4LogitsArgs b = a;
    b.T = a.T - t0 < rows ? a.T - t0 : rows;
    b.h_codes = a.h_codes + t0 * (a.d / 2);
    b.h_scales = a.h_scales + t0 * (a.d / 32);
    b.logits = (T*)a.logits + t0 * a.ld;
    mxfp4_product<T><<<dim3((unsigned)across, (unsigned)((b.T + 15) / 16)), 256, 0, s>>>(b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_mxfp4_quantize(const void* x, int dtype, int64_t rows, int d, int64_t ld, uint8_t* codes,
                                 uint8_t* scales, hipStream_t s) {
  if (dtype == TIM_F32) return quantise_as<float>(x, rows, d, ld, codes, scales, s);
  if (dtype == TIM_BF16) return quantise_as<__bf16>(x, rows, d, ld, codes, scales, s);
  return quantise_as<_Float16>(x, rows, d, ld, codes, scales, s);
}

hipError_t launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* out,
                                   int dtype, hipStream_t s) {
  if (dtype == TIM_F32) return dequantise_as<float>(codes, scales, rows, d, out, s);
  return dequantise_as<__bf16>(codes, scales, rows, d, out, s);
}

hipError_t launch_mxfp4_logits(const Mxfp4LogitsArgs& a, int dtype, hipStream_t s) {
  if (dtype == TIM_F32) return product_as<float>(a, s);
  if (dtype == TIM_BF16) return product_as<__bf16>(a, s);
  return product_as<_Float16>(a, s);
}

}  // namespace tim
