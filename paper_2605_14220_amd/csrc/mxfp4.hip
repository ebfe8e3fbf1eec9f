// 4-bit microscaled floating point on gfx950: quantisation and the values of
// the codes.
//
// Quantisation: 2^E = 2^(floor(log2 top) - 2) places a block's largest
// magnitude in [4, 8), the upper binade of E2M1; x 2^-E is exact in fp32 where
// it is no subnormal (and then its code is 0 either way), and the conversion to E2M1 is the hardware's (nearest even, saturating at 6).
// HBM-bound: 2 bytes read and 17/32 written per bf16 element (6.2 TB/s; rows
// with gaps, whose places are a division away, 5.9). Four lanes share a block,
// so a wave reads and writes consecutive memory.

#include <hip/hip_runtime.h>

#include "kernels.h"
#include "policy.h"

namespace tim {
namespace {

constexpr int kThreads = 256;
constexpr int kGroup = 8;       // elements of one lane: a quarter of a block
// Groups per thread: 151936 rows of 4096 bf16 elements, each call again and again, quantised in 253 us with two (280
// with four, 287 with eight), dequantised in 272 with four (286 with two, 293 with eight); fp32 rows 518 and 719 us.
constexpr int kGroupsIn = 2, kGroupsOut = 4;
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
  [[maybe_unused]] const int e = 127 - (int)scale;
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
  const int64_t g0 = first + (int64_t)blockIdx.x * (kThreads * kGroupsIn) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < kGroupsIn; ++j) {
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
  const int64_t g0 = first + (int64_t)blockIdx.x * (kThreads * kGroupsOut) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < kGroupsOut; ++j) {
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

template <class T>
hipError_t quantise_as(const void* x, int64_t rows, int d, int64_t ld, uint8_t* codes, uint8_t* scales,
                       hipStream_t s) {
  const int64_t groups = rows * d / kGroup;
  const int64_t per_row = ld == d ? groups : d / kGroup;
  const int64_t blocks = (groups + kThreads * kGroupsIn - 1) / (kThreads * kGroupsIn);
  for (int64_t b = 0; b < blocks; b += kLaunchBlocks) {
    const unsigned grid = (unsigned)(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
    quantise<T><<<grid, kThreads, 0, s>>>((const T*)x, groups, b * kThreads * kGroupsIn, per_row, ld, codes, scales);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t dequantise_as(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* out, hipStream_t s) {
  const int64_t groups = rows * d / kGroup;
  const int64_t blocks = (groups + kThreads * kGroupsOut - 1) / (kThreads * kGroupsOut);
  for (int64_t b = 0; b < blocks; b += kLaunchBlocks) {
    const unsigned grid = (unsigned)(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
    dequantise<T><<<grid, kThreads, 0, s>>>(codes, scales, groups, b * kThreads * kGroupsOut, (T*)out);
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

}  // namespace tim
