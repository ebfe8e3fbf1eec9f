// Logits of a 4-bit head on gfx950: z[t][v] = (sum_k h[t][k] w[v][k]) / tau
// over MXFP4 rows, on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// The MFMA takes 128 elements of 16 rows of each side, 32 elements (one scale
// block, 16 bytes of codes) per lane with the block's scale byte, and adds to
// fp32. W is its first operand: a lane's four results are consecutive
// vocabulary entries of one hidden row. Every logit is one accumulation chain
// over ascending 128-element steps in every shape below, so its bits do not
// depend on the shape.
//
// A stage is 256 elements of the tile's rows: 128 bytes of codes per row, DMA
// loaded into LDS and XOR-swizzled as in tilepass.h, and 8 scale bytes per
// row beside them. Few rows are bound by the stream of W; many by the MFMAs
// and, with them, by the fp32 logits going out.

#include <hip/hip_runtime.h>

#include "kernels.h"
#include "policy.h"
#include "tilepass.h"

namespace tim {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStageCodes = 128;  // bytes of a row's codes in a stage (two k-steps)
constexpr int kStageScales = 8;   // and of its scales

// A workgroup of WV x WT waves, each NA x NB blocks of 16 x 16, and PER_CU
// workgroups on a CU.
template <int WV_, int WT_, int NA_, int NB_, int PER_CU_>
struct Fp4Tile {
  static constexpr int WV = WV_, WT = WT_, NA = NA_, NB = NB_, PER_CU = PER_CU_;
  static constexpr int NW = WV * WT;
  static constexpr int TA = WV * NA * 16;  // vocabulary entries
  static constexpr int TB = WT * NB * 16;  // hidden rows
  // DMA loads of a stage: 1 KB of codes (8 rows) or 256 bytes of scales (32 rows) each
  static constexpr int CA = TA / 8, CB = TB / 8, SA = (TA + 31) / 32, SC = (TB + 31) / 32;
  // Stage layout: W codes, hidden codes, W scales, hidden scales
  static constexpr int kCodesB = CA * 1024, kScalesA = kCodesB + CB * 1024, kScalesB = kScalesA + SA * 256;
  static constexpr int SB = kScalesB + SC * 256;
  static constexpr int FIT = 160 * 1024 / PER_CU / SB;
  static constexpr int NBUF = FIT < 8 ? FIT : 8;
  // Loads per wave, each kind dealt round the waves; a kind that does not fill its last round has blocks loaded
  // twice (with the same bytes)
  static constexpr int LA = (CA + NW - 1) / NW, LB = (CB + NW - 1) / NW, XA = (SA + NW - 1) / NW,
                       XB = (SC + NW - 1) / NW;
  static constexpr int L = LA + LB + XA + XB;
  static_assert(NW % 2 == 0, "a wave's blocks of 8 rows are all even or all odd ones, so one swizzle serves them");
  static_assert(NBUF >= 2, "double buffering at least");
};

// a += the product of one k-step, the scales in byte S of sa and sb.
template <int S>
__device__ __forceinline__ f32x4 mfma_fp4(i32x4 a, int sa, i32x4 b, int sb, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
  const i32x8 b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, S, sa, S, sb);
#else
  return c;
#endif
}

// Where a tile's stages come from: the operands' resources, each over the
// tile's own rows, so that loads of rows past its end return zeros (the range
// is checked on the per-lane offsets; the stage is in the scalar offset), and
// the lane's offsets within the first round of loads. The last stage of an odd
// number of k-steps holds one: its second half would lie in the next row, or
// past the last one, and repeats the first half instead.
struct Fp4Source {
  rsrc_t ac, bc, as, bs;  // codes and scales of W and of the hidden rows
  int code, code_tail, scale, scale_tail;
  int rowc, rows;         // bytes of a row's codes and scales
};

template <class TL>
__device__ __forceinline__ Fp4Source fp4_source(const Mxfp4LogitsArgs& a, int v0, int64_t t0, int wave, int lane) {
  Fp4Source o;
  o.rowc = a.d / 2;
  o.rows = a.d / 32;
  const int va = a.V - v0 < TL::TA ? a.V - v0 : TL::TA;
  const int tb = a.T - t0 < TL::TB ? (int)(a.T - t0) : TL::TB;
  o.ac = make_rsrc(a.w_codes + (int64_t)v0 * o.rowc, (uint64_t)va * o.rowc);
  o.as = make_rsrc(a.w_scales + (int64_t)v0 * o.rows, (uint64_t)va * o.rows);
  o.bc = make_rsrc(a.h_codes + t0 * o.rowc, (uint64_t)tb * o.rowc);
  o.bs = make_rsrc(a.h_scales + t0 * o.rows, (uint64_t)tb * o.rows);
  const int r = wave * 8 + (lane >> 3), c = (lane & 7) ^ swz(r);
  o.code = (lane >> 3) * o.rowc + c * 16;
  o.code_tail = (lane >> 3) * o.rowc + (c & 3) * 16;
  o.scale_tail = (lane >> 1) * o.rows;
  o.scale = o.scale_tail + (lane & 1) * 4;
  return o;
}

// Load q of a wave's request of a stage into `buf`.
template <class TL>
__device__ __forceinline__ void fp4_load(unsigned char* buf, const Fp4Source& o, int stage, bool tail, int wave, int q) {
#if defined(__HIP_DEVICE_COMPILE__)
  // block b of kind of n: past the last one, a block of an earlier round (for NW even, of the same parity)
  auto block = [wave](int j, int n) {
    const int b = j * TL::NW + wave;
    return n % TL::NW == 0 || b < n ? b : n >= TL::NW ? b - TL::NW : n >= 2 ? (wave & 1) : 0;
  };
  const int code = tail ? o.code_tail : o.code, scale = tail ? o.scale_tail : o.scale;
  if (q < TL::LA) {
    const int b = block(q, TL::CA);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.ac, (lds_void*)(buf + b * 1024), 16, (uint32_t)(code + b * 8 * o.rowc),
                                             stage * kStageCodes, 0, 0);
  } else if (q < TL::LA + TL::LB) {
    const int b = block(q - TL::LA, TL::CB);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.bc, (lds_void*)(buf + TL::kCodesB + b * 1024), 16,
                                             (uint32_t)(code + b * 8 * o.rowc), stage * kStageCodes, 0, 0);
  } else if (q < TL::LA + TL::LB + TL::XA) {
    const int b = block(q - TL::LA - TL::LB, TL::SA);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.as, (lds_void*)(buf + TL::kScalesA + b * 256), 4,
                                             (uint32_t)(scale + b * 32 * o.rows), stage * kStageScales, 0, 0);
  } else {
    const int b = block(q - TL::LA - TL::LB - TL::XA, TL::SC);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.bs, (lds_void*)(buf + TL::kScalesB + b * 256), 4,
                                             (uint32_t)(scale + b * 32 * o.rows), stage * kStageScales, 0, 0);
  }
#endif
}

// A wave's operands of one k-step, and the scales of the stage's two: byte 0
// for the first k-step, byte 1 for the second. The hidden rows' codes alternate
// between two sets by k-step; W's are refilled in place.
template <class TL>
struct Fp4Operands {
  i32x4 fa[TL::NA], fb[2][TL::NB];
  int sa[TL::NA], sb[TL::NB];
};

// Addresses of a lane's operands in a stage buffer.
struct Fp4Lane {
  int code[2];  // k-step 0 and 1, within a block of 16 rows
  int scale;
  uint32_t pick;  // bytes g of two dwords
};
__device__ __forceinline__ Fp4Lane fp4_lane(int lane) {
  const int r = lane & 15, g = lane >> 4;
  return {{r * kStageCodes + (g ^ swz(r)) * 16, r * kStageCodes + ((4 + g) ^ swz(r)) * 16}, r * kStageScales,
          0x0C0C0400u + 0x0101u * (uint32_t)g};
}
__device__ __forceinline__ int fp4_scales(i32x2 raw, uint32_t pick) {
  return (int)__builtin_amdgcn_perm((uint32_t)raw[1], (uint32_t)raw[0], pick);
}

// One k-step (P: the stage's first or second), unit by unit; with LOAD the
// wave's share of a stage request into lb, with READ the next step's operands
// from rb (with P = 1 the next stage's, scales too).
template <class TL, int P, bool LOAD, bool READ>
__device__ __forceinline__ void fp4_step(Fp4Operands<TL>& f, f32x4 (&acc)[TL::NA][TL::NB], unsigned char* lb,
                                         const Fp4Source& o, int stage, bool tail, const unsigned char* rb,
                                         const Fp4Lane& at, int wave, int wv, int wt) {
  constexpr int NA = TL::NA, NB = TL::NB, NM = NA * NB, L = TL::L;
  static_assert(NA <= NM && NB <= NM, "a unit for every read");
  const unsigned char* ca = rb + wv * NA * 2048 + at.code[P ^ 1];
  const unsigned char* cb = rb + TL::kCodesB + wt * NB * 2048 + at.code[P ^ 1];
  const unsigned char* xa = rb + TL::kScalesA + wv * NA * 128 + at.scale;
  const unsigned char* xb = rb + TL::kScalesB + wt * NB * 128 + at.scale;
  i32x2 ra[NA], rs[NB];
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    const int bi = i / NB, bq = i % NB, bj = (bi & 1) ? NB - 1 - bq : bq;
    acc[bi][bj] = mfma_fp4<P>(f.fa[bi], f.sa[bi], f.fb[P][bj], f.sb[bj], acc[bi][bj]);
    if (LOAD) {
#pragma unroll
      for (int q = 0; q < L; ++q)
        if (q * NM / L == i) fp4_load<TL>(lb, o, stage, tail, wave, q);
    }
    if (READ) {
      if (i < NB) f.fb[P ^ 1][i] = *(const i32x4*)(cb + i * 2048);
      if (bq == NB - 1) f.fa[bi] = *(const i32x4*)(ca + bi * 2048);
      if (P == 1) {
        if (i >= NM - NB) rs[i - (NM - NB)] = *(const i32x2*)(xb + (i - (NM - NB)) * 128);
        if (i >= NM - NA) ra[i - (NM - NA)] = *(const i32x2*)(xa + (i - (NM - NA)) * 128);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (READ && P == 1) {
#pragma unroll
    for (int j = 0; j < NB; ++j) f.sb[j] = fp4_scales(rs[j], at.pick);
#pragma unroll
    for (int j = 0; j < NA; ++j) f.sa[j] = fp4_scales(ra[j], at.pick);
  }
}

template <class TL, class T>
__global__ __launch_bounds__(TL::NW * 64, TL::PER_CU * TL::NW / 4) void fp4_logits(const Mxfp4LogitsArgs a, int n_vt,
                                                                                    int n_tt) {
  constexpr int NA = TL::NA, NB = TL::NB, NBUF = TL::NBUF, L = TL::L, SB = TL::SB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[NBUF * SB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wv = wave % TL::WV, wt = wave / TL::WV;
  const int lane = threadIdx.x & 63;

  // logical tile id: contiguous ranges per XCD, walked in groups of vocabulary tiles
  const int n_tiles = n_vt * n_tt;
  const int x = blockIdx.x & 7, tq = n_tiles >> 3, trm = n_tiles & 7;
  int vt, tt;
  tile_of_lid<kGroupV>(x * tq + (x < trm ? x : trm) + (int)(blockIdx.x >> 3), n_vt, n_tt, vt, tt);
  const int v0 = vt * TL::TA;
  const int64_t t0 = (int64_t)tt * TL::TB;
  const int nk = (a.d + 255) / 256;
  // whole stages; with an odd number of k-steps the last stage has one
  const int whole = a.d / 256;
  const Fp4Source o = fp4_source<TL>(a, v0, t0, wave, lane);

#pragma unroll
  for (int s = 0; s < NBUF; ++s) {
    const int st = s < nk ? s : nk - 1;
#pragma unroll
    for (int q = 0; q < L; ++q) fp4_load<TL>(lds + s * SB, o, st, st >= whole, wave, q);
  }
  wait_vmem<(NBUF - 1) * L>();  // stage 0 landed
  __syncthreads();

  f32x4 acc[NA][NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{};
  const Fp4Lane at = fp4_lane(lane);
  Fp4Operands<TL> f;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    f.fb[0][j] = *(const i32x4*)(lds + TL::kCodesB + (wt * NB + j) * 2048 + at.code[0]);
    f.sb[j] = fp4_scales(*(const i32x2*)(lds + TL::kScalesB + (wt * NB + j) * 128 + at.scale), at.pick);
  }
#pragma unroll
  for (int j = 0; j < NA; ++j) {
    f.fa[j] = *(const i32x4*)(lds + (wv * NA + j) * 2048 + at.code[0]);
    f.sa[j] = fp4_scales(*(const i32x2*)(lds + TL::kScalesA + (wv * NA + j) * 128 + at.scale), at.pick);
  }
  int bk = 0;  // buffer of the current stage
  for (int k = 0; k < whole; ++k) {
    unsigned char* cb = lds + bk * SB;
    fp4_step<TL, 0, false, true>(f, acc, cb, o, 0, false, cb, at, wave, wv, wt);
    // this wave's reads of stage k and its DMA of stage k + 1 are done; the barrier makes that stage visible and
    // frees this one's buffer, which takes stage k + NBUF (past the end: the last stage again, never read)
    wait_lgkm0_vmem<(NBUF - 2) * L>();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (++bk == NBUF) bk = 0;
    const int st = k + NBUF < nk ? k + NBUF : nk - 1;
    fp4_step<TL, 1, true, true>(f, acc, cb, o, st, st >= whole, lds + bk * SB, at, wave, wv, wt);
  }
  if (whole < nk) fp4_step<TL, 0, false, false>(f, acc, lds, o, 0, false, lds, at, wave, wv, wt);
  wait_vmem<0>();  // no global->LDS request may outlive the workgroup

  // lane l holds hidden row l % 16 of a block and its vocabulary entries 4 (l / 16) .. + 3
  const int vl = v0 + wv * NA * 16 + 4 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t t = t0 + (wt * NB + j) * 16 + (lane & 15);
    if (t >= a.T) continue;
    T* out = (T*)a.logits + t * a.ld;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int v = vl + i * 16;
      T z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = narrow<T>(acc[i][j][e] * a.inv_tau);
      if (v + 4 <= a.V) {
        __builtin_memcpy(out + v, z, sizeof(z));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < a.V) out[v + e] = z[e];
      }
    }
  }
}

template <class TL, class T>
hipError_t launch_tiles(const Mxfp4LogitsArgs& a, hipStream_t s) {
  const int n_vt = (a.V + TL::TA - 1) / TL::TA;
  // a grid holds fewer than 2^32 threads
  const int64_t rows = (((int64_t)1 << 32) / (64 * TL::NW) - 1) / n_vt * TL::TB;
  for (int64_t t0 = 0; t0 < a.T; t0 += rows) {
    Mxfp4LogitsArgs b = a;
    b.T = a.T - t0 < rows ? a.T - t0 : rows;
    b.h_codes = a.h_codes + t0 * (a.d / 2);
    b.h_scales = a.h_scales + t0 * (a.d / 32);
    b.logits = (T*)a.logits + t0 * a.ld;
    const int n_tt = (int)((b.T + TL::TB - 1) / TL::TB);
    fp4_logits<TL, T><<<(unsigned)(n_vt * n_tt), TL::NW * 64, 0, s>>>(b, n_vt, n_tt);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

#ifndef FP4_SHAPE
#define FP4_SHAPE 0
#endif
template <class T>
hipError_t product_as(const Mxfp4LogitsArgs& a, hipStream_t s) {
  if (a.T <= 16) return launch_tiles<Fp4Tile<4, 1, 2, 1, 3>, T>(a, s);
  if (a.T <= 32) return launch_tiles<Fp4Tile<4, 1, 2, 2, 3>, T>(a, s);
  if (a.T <= 64) return launch_tiles<Fp4Tile<4, 1, 2, 4, 2>, T>(a, s);
  if (a.T <= 128) return launch_tiles<Fp4Tile<4, 1, 4, 8, 1>, T>(a, s);
  return launch_tiles<Fp4Tile<2, 2, 8, 8, 1>, T>(a, s);
}

}  // namespace

hipError_t launch_mxfp4_logits(const Mxfp4LogitsArgs& a, int dtype, hipStream_t s) {
  if (dtype == TIM_F32) return product_as<float>(a, s);
  if (dtype == TIM_BF16) return product_as<__bf16>(a, s);
  return product_as<_Float16>(a, s);
}

}  // namespace tim
