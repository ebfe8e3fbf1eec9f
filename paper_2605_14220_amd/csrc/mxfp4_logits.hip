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
// loaded into LDS and XOR-swizzled as in tilepass.h. Scales are few bytes but
// many requests: 8 bytes a row and stage in 4-byte loads cost 2000 rows at
// d = 4096 a fifth of their time, and reading a row's four bytes to use one of
// them a tenth. So they come in groups of 512 elements, 16 bytes a row, and
// the wave that loaded a row's group turns it (a 4 x 4 transpose of bytes), so
// that a lane reads the four bytes of its block column with one ds_read_b32
// and the MFMA picks the k-step's by its byte select.
//
// Few rows are bound by the stream of W. Many are bound by the k-loop of the
// 256 x 256 tile: at V = 151936 2000 rows take 439, 753 and 1325 us for d =
// 2048, 4096 and 8192, in 18.6 rounds of tiles 2.0 us a stage, of which the
// MFMAs need 1.3 (two buffers fit, so every boundary waits for all loads), and
// 7.8 us a tile besides, its first loads and its logits.

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.h"
#include "policy.h"
#include "tilepass.h"

namespace tim {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStageCodes = 128;  // bytes of a row's codes in a stage (two k-steps)
constexpr int kGroupScales = 16;  // bytes of a row's scales in a group (two stages)
// Vocabulary tiles per group in the workgroup -> tile order. What a round of workgroups writes is runs of this many
// tiles in the rows of a few: 2000 rows at d = 4096, V = 151936 753 us against 789 for 8 and 830 for 4, 1000 rows 405,
// 431 and 431 (8000 rows 2857, 2848 and 2921; one or two row tiles the same).
constexpr int kGroupFp4 = 16;

// A workgroup of WV x WT waves, each NA x NB blocks of 16 x 16, and PER_CU
// workgroups on a CU. ONCE: one tile takes all hidden rows, so W is read once
// and its loads pass the caches by (1 row of d = 2048 and V = 151936 31.1 us
// against 34.6, 64 of d = 4096 79 against 83, 128 and 200 the same; a W of less
// than the caches, called for again at once, would be found there: 28.5 against
// 26.7); where tiles share W they find it in L2 (2000 rows 753 us against 899).
template <int WV_, int WT_, int NA_, int NB_, int PER_CU_, bool ONCE_>
struct Fp4Tile {
  static constexpr int WV = WV_, WT = WT_, NA = NA_, NB = NB_, PER_CU = PER_CU_;
  static constexpr int kAuxW = ONCE_ ? 2 : 0;  // the cache policy of W's loads: 2, non-temporal
  static constexpr int NW = WV * WT;
  static constexpr int TA = WV * NA * 16;  // vocabulary entries
  static constexpr int TB = WT * NB * 16;  // hidden rows
  // DMA loads of 1 KB: of a stage's codes (8 rows each), and of a group's scales (64 rows each)
  static constexpr int CA = TA / 8, CB = TB / 8, SA = (TA + 63) / 64, SC = (TB + 63) / 64;
  // per wave, each kind dealt round the waves; a kind of codes that does not fill its last round has blocks loaded
  // twice (with the same bytes), scales that do not have loads into a spare KB
  static constexpr int LA = (CA + NW - 1) / NW, LB = (CB + NW - 1) / NW, LX = (SA + SC + NW - 1) / NW;
  static constexpr int L = LA + LB;
  static constexpr int kCodesB = CA * 1024;
  static constexpr int SB = kCodesB + CB * 1024;  // a stage buffer: W codes, hidden codes
  static constexpr int XB = (SA + SC) * 1024;     // a group's scales: W, hidden
  static constexpr int kSpare = (SA + SC) % NW ? 1024 : 0;
  // NBUF stages and SBUF groups: group j + 1 is requested with stage 2 j + 1, NBUF stages ahead, into the buffer
  // of group j + 1 - SBUF, whose last reads are in stage 2 (j + 1 - SBUF) - 1
  static constexpr int lds_bytes(int n) { return n * SB + (n / 2 + 1) * XB + kSpare; }
  static constexpr int kRoom = 160 * 1024 / PER_CU;
  static constexpr int NBUF = lds_bytes(6) <= kRoom ? 6 : lds_bytes(5) <= kRoom ? 5 : lds_bytes(4) <= kRoom ? 4
                              : lds_bytes(3) <= kRoom                                                       ? 3
                                                                                                            : 2;
  static constexpr int SBUF = NBUF / 2 + 1;
  static constexpr int kScales = NBUF * SB, kSpareAt = kScales + SBUF * XB;
  static constexpr int LDS = kSpareAt + kSpare;
  static_assert(NW % 2 == 0, "a wave's blocks of 8 rows are all even or all odd ones, so one swizzle serves them");
  static_assert(LDS <= kRoom, "double buffering at least");
};

// c + the product of one k-step, the scales in byte S of sa and sb.
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

// Four consecutive logits from v on, as far as they lie in the vocabulary.
template <class T>
__device__ __forceinline__ void store_logits(T* row, int v, int V, const f32x4& acc, float inv_tau) {
  T z[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) z[e] = narrow<T>(acc[e] * inv_tau);
  if (v + 4 <= V) {
    __builtin_memcpy(row + v, z, sizeof(z));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < V) row[v + e] = z[e];
  }
}

// Between a wave's lanes that hand data on through LDS. The hardware takes a
// wave's LDS accesses in order, so this is no instruction: it keeps the
// compiler, which sees each lane by itself, from moving one across it.
__device__ __forceinline__ void lanes_ordered() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// A wave's logits leave through LDS, 16 hidden rows at a time, so that a store
// writes runs of NA * 16 logits of a row: straight from the accumulators it
// would write 64 bytes in each of 16 rows. NT: past the caches, for logits too
// large to be found there again (2000 rows at d = 4096, V = 151936, 1.2 GB: 753
// us against 780; with the scattered stores, before other steps, 960 against 890).
typedef i32x4 i32x4_by2 __attribute__((aligned(2)));  // logits are aligned to their element
typedef i32x4 i32x4_by4 __attribute__((aligned(4)));
template <class TL, class T>
struct Fp4Out {
  static constexpr int E = 16 / (int)sizeof(T);                  // logits per lane and store
  static constexpr int kRow = TL::NA * 16 * (int)sizeof(T) + 16;  // 16 bytes apart in the banks
  static constexpr int kBytes = 16 * kRow;
  static constexpr int kLanes = TL::NA * 16 / E;  // lanes a row
  static_assert(TL::NW * kBytes <= TL::LDS && 64 % kLanes == 0, "the waves' rows fit, whole rows a store");
};
template <class TL, class T, bool NT>
__device__ __forceinline__ void store_tile(unsigned char* lds, const f32x4 (&acc)[TL::NA][TL::NB], T* logits, int64_t ld,
                                           int V, int64_t rows, int v0, int64_t t0, float inv_tau, int lane) {
  using O = Fp4Out<TL, T>;
  constexpr int kRows = 64 / O::kLanes;  // rows a store
  const int v = v0 + lane % O::kLanes * O::E;
#pragma unroll
  for (int j = 0; j < TL::NB; ++j) {
    // lane l holds hidden row l % 16 of a block and its vocabulary entries 4 (l / 16) .. + 3
#pragma unroll
    for (int i = 0; i < TL::NA; ++i) {
      T z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = narrow<T>(acc[i][j][e] * inv_tau);
      __builtin_memcpy(__builtin_assume_aligned(lds + (lane & 15) * O::kRow + (i * 16 + 4 * (lane >> 4)) * sizeof(T),
                                                4 * sizeof(T)),
                       z, sizeof(z));
    }
    lanes_ordered();
#pragma unroll
    for (int r = lane / O::kLanes; r < 16; r += kRows) {
      const int64_t t = t0 + j * 16 + r;
      const i32x4 q = *(const i32x4*)(lds + r * O::kRow + lane % O::kLanes * 16);
      if (t >= rows) continue;
      T* out = logits + t * ld + v;
      if (v + O::E <= V) {
        if constexpr (NT)
          __builtin_nontemporal_store(q, (std::conditional_t<sizeof(T) == 4, i32x4_by4, i32x4_by2>*)out);
        else
          __builtin_memcpy(out, &q, 16);
      } else {
        T z[O::E];
        __builtin_memcpy(z, &q, 16);
#pragma unroll
        for (int e = 0; e < O::E; ++e)
          if (v + e < V) out[e] = z[e];
      }
    }
    lanes_ordered();  // the next rows take the same place
  }
}

// Where a tile's stages come from: the operands' resources, each over the
// tile's own rows, so that loads of rows past its end return zeros (the range
// is checked on the per-lane offsets; the place along the row is in the scalar
// offset), and the lane's offsets within the first round of loads. The last
// stage of an odd number of k-steps holds one: its second half would lie in the
// next row, or past the last one, and repeats the first half instead; the last
// group of a row that is no whole number of them starts where it ends with the
// row, and is moved down as it is turned.
struct Fp4Source {
  rsrc_t ac, bc, as, bs;  // codes and scales of W and of the hidden rows
  int code, code_tail, scale;
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
  o.scale = lane * o.rows;
  return o;
}

// Load q of a wave's request of a stage's codes into `buf`.
template <class TL>
__device__ __forceinline__ void fp4_load(unsigned char* buf, const Fp4Source& o, int stage, bool tail, int wave, int q) {
#if defined(__HIP_DEVICE_COMPILE__)
  // block b of n of a kind: past the last one, a block of an earlier round (for NW even, of the same parity)
  auto block = [wave](int j, int n) {
    const int b = j * TL::NW + wave;
    return n % TL::NW == 0 || b < n ? b : n >= TL::NW ? b - TL::NW : (wave & 1);
  };
  const int code = tail ? o.code_tail : o.code;
  const bool first = q < TL::LA;
  const int b = first ? block(q, TL::CA) : block(q - TL::LA, TL::CB);
  const uint32_t at = (uint32_t)(code + b * 8 * o.rowc);
  if (first)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.ac, (lds_void*)(buf + b * 1024), 16, at, stage * kStageCodes, 0, TL::kAuxW);
  else
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.bc, (lds_void*)(buf + TL::kCodesB + b * 1024), 16, at,
                                             stage * kStageCodes, 0, 0);
#endif
}

// The wave's request of a group's scales into the group's buffer, and, once it
// has landed, the turning of those rows: dword s of a row holds the four bytes
// of k-step s, and will hold those of block column s.
template <class TL>
__device__ __forceinline__ void fp4_load_scales(unsigned char* lds, int slot, const Fp4Source& o, int group, int wave) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int at = 16 * group < o.rows - 16 ? 16 * group : o.rows - 16;
#pragma unroll
  for (int q = 0; q < TL::LX; ++q) {
    const int b = q * TL::NW + wave;
    unsigned char* dst = lds + (b < TL::SA + TL::SC ? TL::kScales + slot * TL::XB + b * 1024 : TL::kSpareAt);
    const bool first = b < TL::SA;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(first ? o.as : o.bs, (lds_void*)dst, 16,
                                             (uint32_t)(o.scale + (first ? b : b - TL::SA) * 64 * o.rows), at, 0, 0);
  }
#endif
}
template <class TL>
__device__ __forceinline__ i32x4* fp4_turned(unsigned char* lds, int slot, int q, int wave, int lane) {
  const int b = q * TL::NW + wave;
  return (i32x4*)(lds + (b < TL::SA + TL::SC ? TL::kScales + slot * TL::XB + b * 1024 : TL::kSpareAt) + lane * 16);
}
__device__ __forceinline__ i32x4 fp4_turn(i32x4 w, int down) {
  if (down == 1) w = {w[1], w[2], w[3], w[3]};
  if (down == 2) w = {w[2], w[3], w[3], w[3]};
  if (down >= 3) w = {w[3], w[3], w[3], w[3]};
  const uint32_t lo01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t lo23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  return {(int)__builtin_amdgcn_perm(lo23, lo01, 0x05040100u), (int)__builtin_amdgcn_perm(lo23, lo01, 0x07060302u),
          (int)__builtin_amdgcn_perm(hi23, hi01, 0x05040100u), (int)__builtin_amdgcn_perm(hi23, hi01, 0x07060302u)};
}
// Dwords by which a group starts before its place.
__device__ __forceinline__ int fp4_down(const Fp4Source& o, int group) {
  return 16 * group < o.rows - 16 ? 0 : (16 * group - (o.rows - 16)) / 4;
}

// A wave's operands: one k-step's codes, the hidden rows' alternating between
// two sets by k-step and W's refilled in place, and a group's scales.
template <class TL>
struct Fp4Operands {
  i32x4 fa[TL::NA], fb[2][TL::NB];
  int sa[TL::NA], sb[TL::NB];
};

// Offsets of a lane's operands within a block of 16 rows.
struct Fp4Lane {
  int code[2];  // of k-step 0 and 1 of a stage
  int scale;
};
__device__ __forceinline__ Fp4Lane fp4_lane(int lane) {
  const int r = lane & 15, g = lane >> 4;
  return {{r * kStageCodes + (g ^ swz(r)) * 16, r * kStageCodes + ((4 + g) ^ swz(r)) * 16}, r * kGroupScales + g * 4};
}

// K-step P of a group, unit by unit, and beside it the next k-step's operands:
// from this stage's buffer rb, or (P odd) the next one's, and after the group's
// last k-step the next group's scales from xb. P odd also issues the wave's
// share of a stage request into lb; P = 2 turns the next group's scales in
// slot `turn`.
template <class TL, int P>
__device__ __forceinline__ void fp4_step(Fp4Operands<TL>& f, f32x4 (&acc)[TL::NA][TL::NB], unsigned char* lds,
                                         unsigned char* lb, const Fp4Source& o, int stage, bool tail,
                                         const unsigned char* rb, const unsigned char* xb, int turn, int down,
                                         const Fp4Lane& at, int wave, int wv, int wt, int lane) {
  constexpr int NA = TL::NA, NB = TL::NB, NM = NA * NB, L = TL::L, Q = P & 1;
  static_assert(NA <= NM && NB <= NM, "a unit for every read");
  const unsigned char* ca = rb + wv * NA * 2048 + at.code[Q ^ 1];
  const unsigned char* cb = rb + TL::kCodesB + wt * NB * 2048 + at.code[Q ^ 1];
  const unsigned char* xa = xb + wv * NA * 256 + at.scale;
  const unsigned char* xt = xb + TL::SA * 1024 + wt * NB * 256 + at.scale;
  int na[NA], nb[NB];
  i32x4 raw[TL::LX];
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    const int bi = i / NB, bq = i % NB, bj = (bi & 1) ? NB - 1 - bq : bq;
    acc[bi][bj] = mfma_fp4<P>(f.fa[bi], f.sa[bi], f.fb[Q][bj], f.sb[bj], acc[bi][bj]);
    if (Q == 1) {
#pragma unroll
      for (int q = 0; q < L; ++q)
        if (q * NM / L == i) fp4_load<TL>(lb, o, stage, tail, wave, q);
    }
    if (P == 2 && i == 0) {
#pragma unroll
      for (int q = 0; q < TL::LX; ++q) raw[q] = *fp4_turned<TL>(lds, turn, q, wave, lane);
    }
    if (P == 2 && i == NM - 1) {
#pragma unroll
      for (int q = 0; q < TL::LX; ++q) *fp4_turned<TL>(lds, turn, q, wave, lane) = fp4_turn(raw[q], down);
    }
    if (i < NB) f.fb[Q ^ 1][i] = *(const i32x4*)(cb + i * 2048);
    if (bq == NB - 1) f.fa[bi] = *(const i32x4*)(ca + bi * 2048);
    if (P == 3) {
      if (i >= NM - NB) nb[i - (NM - NB)] = *(const int*)(xt + (i - (NM - NB)) * 256);
      if (i >= NM - NA) na[i - (NM - NA)] = *(const int*)(xa + (i - (NM - NA)) * 256);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (P == 3) {
#pragma unroll
    for (int j = 0; j < NB; ++j) f.sb[j] = nb[j];
#pragma unroll
    for (int j = 0; j < NA; ++j) f.sa[j] = na[j];
  }
}

// This wave's LDS accesses and its DMA up to the next stage's are done; the
// barrier makes that stage (and turned scales) visible and frees this one's
// buffer. The count ignores scale requests, which only makes the wait stricter.
template <class TL>
__device__ __forceinline__ void fp4_boundary() {
  wait_lgkm0_vmem<(TL::NBUF - 2) * TL::L>();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <class TL, class T, bool NT>
__global__ __launch_bounds__(TL::NW * 64, TL::PER_CU * TL::NW / 4) void fp4_logits(const Mxfp4LogitsArgs a, int n_vt,
                                                                                    int n_tt) {
  constexpr int NA = TL::NA, NB = TL::NB, NBUF = TL::NBUF, SBUF = TL::SBUF, L = TL::L, SB = TL::SB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[TL::LDS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wv = wave % TL::WV, wt = wave / TL::WV;
  const int lane = threadIdx.x & 63;

  // logical tile id: contiguous ranges per XCD, walked in groups of vocabulary tiles
  const int n_tiles = n_vt * n_tt;
  const int x = blockIdx.x & 7, tq = n_tiles >> 3, trm = n_tiles & 7;
  int vt, tt;
  tile_of_lid<kGroupFp4>(x * tq + (x < trm ? x : trm) + (int)(blockIdx.x >> 3), n_vt, n_tt, vt, tt);
  const int v0 = vt * TL::TA;
  const int64_t t0 = (int64_t)tt * TL::TB;
  const int nk = (a.d + 255) / 256;
  // whole stages; with an odd number of k-steps the last stage has one
  const int whole = a.d / 256;
  const Fp4Source o = fp4_source<TL>(a, v0, t0, wave, lane);

  // stage s is requested after group (s + 1) / 2 for s odd
  fp4_load_scales<TL>(lds, 0, o, 0, wave);
#pragma unroll
  for (int s = 0; s < NBUF; ++s) {
    if (s & 1) fp4_load_scales<TL>(lds, (s + 1) / 2 % SBUF, o, (s + 1) / 2, wave);
    const int st = s < nk ? s : nk - 1;
#pragma unroll
    for (int q = 0; q < L; ++q) fp4_load<TL>(lds + s * SB, o, st, st >= whole, wave, q);
  }
  wait_vmem<(NBUF - 1) * L>();  // group 0 and stage 0 landed
  asm volatile("" ::: "memory");  // and no read of them is moved up
#pragma unroll
  for (int q = 0; q < TL::LX; ++q) {
    i32x4* p = fp4_turned<TL>(lds, 0, q, wave, lane);
    *p = fp4_turn(*p, 0);
  }
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
    f.sb[j] = *(const int*)(lds + TL::kScales + TL::SA * 1024 + (wt * NB + j) * 256 + at.scale);
  }
#pragma unroll
  for (int j = 0; j < NA; ++j) {
    f.fa[j] = *(const i32x4*)(lds + (wv * NA + j) * 2048 + at.code[0]);
    f.sa[j] = *(const int*)(lds + TL::kScales + (wv * NA + j) * 256 + at.scale);
  }
  // buffers of the current stage and of the current group; past the row's end, stage requests repeat the last stage
  // and operand reads take what a buffer holds, none of it used
  int bk = 0, sk = 0;
  auto next = [](int i, int n) { return i + 1 == n ? 0 : i + 1; };
  for (int k = 0;; k += 2) {
    {
      unsigned char* cb = lds + bk * SB;
      fp4_step<TL, 0>(f, acc, lds, cb, o, 0, false, cb, lds, 0, 0, at, wave, wv, wt, lane);
      if (k == whole) break;
      fp4_boundary<TL>();
      if constexpr (NBUF & 1) fp4_load_scales<TL>(lds, (sk + (NBUF + 1) / 2) % SBUF, o, (k + NBUF + 1) / 2, wave);
      bk = next(bk, NBUF);
      const int st = k + NBUF < nk ? k + NBUF : nk - 1;
      fp4_step<TL, 1>(f, acc, lds, cb, o, st, st >= whole, lds + bk * SB, lds, 0, 0, at, wave, wv, wt, lane);
      if (k + 1 == nk) break;
    }
    {
      unsigned char* cb = lds + bk * SB;
      sk = next(sk, SBUF);
      // the next group's scales were requested before this stage
      fp4_step<TL, 2>(f, acc, lds, cb, o, 0, false, cb, lds, sk, fp4_down(o, k / 2 + 1), at, wave, wv, wt, lane);
      if (k + 1 == whole) break;
      fp4_boundary<TL>();
      if constexpr (!(NBUF & 1)) fp4_load_scales<TL>(lds, (sk + NBUF / 2) % SBUF, o, (k + NBUF + 2) / 2, wave);
      bk = next(bk, NBUF);
      const int st = k + 1 + NBUF < nk ? k + 1 + NBUF : nk - 1;
      fp4_step<TL, 3>(f, acc, lds, cb, o, st, st >= whole, lds + bk * SB, lds + TL::kScales + sk * TL::XB, 0, 0, at,
                      wave, wv, wt, lane);
      if (k + 2 == nk) break;
    }
  }
  wait_vmem<0>();  // no global->LDS request may outlive the workgroup

  __syncthreads();  // nor reach the LDS after this
  store_tile<TL, T, NT>(lds + wave * Fp4Out<TL, T>::kBytes, acc, (T*)a.logits, a.ld, a.V, a.T, v0 + wv * NA * 16,
                    t0 + wt * NB * 16, a.inv_tau, lane);
}

// Rows shorter than a group of scales: one wave per block of 16 x 16, operands
// from memory. For few rows that is near W's stream (1 row of d = 384 and V =
// 151936 8.7 us, 6.4 at the copy's rate); W is read again for every 16 rows and
// logits leave in 64-byte runs, so many rows are far from it (2000 rows of d =
// 256 672 us and of d = 384 740, where rows of 512 take 258 in tiles).
template <class T>
__global__ __launch_bounds__(256) void fp4_logits_short(const Mxfp4LogitsArgs a) {
  const int lane = threadIdx.x & 63;
  const int v0 = ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)) * 16;
  const int64_t t0 = (int64_t)blockIdx.y * 16;
  if (v0 >= a.V) return;
  const int r = lane & 15, g = lane >> 4;
  // rows past the end repeat the last one; their results are not written
  const int64_t w = v0 + r < a.V ? v0 + r : a.V - 1;
  const int64_t h = t0 + r < a.T ? t0 + r : a.T - 1;
  const uint8_t* wc = a.w_codes + w * (a.d / 2) + g * 16;
  const uint8_t* hc = a.h_codes + h * (a.d / 2) + g * 16;
  const uint8_t* ws = a.w_scales + w * (a.d / 32) + g;
  const uint8_t* hs = a.h_scales + h * (a.d / 32) + g;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.d / 128; ++k)
    acc = mfma_fp4<0>(*(const i32x4*)(wc + k * 64), ws[k * 4], *(const i32x4*)(hc + k * 64), hs[k * 4], acc);
  if (t0 + r < a.T) store_logits<T>((T*)a.logits + (t0 + r) * a.ld, v0 + 4 * g, a.V, acc, a.inv_tau);
}

template <class TL, class T, bool NT = false>
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
    fp4_logits<TL, T, NT><<<(unsigned)(n_vt * n_tt), TL::NW * 64, 0, s>>>(b, n_vt, n_tt);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t launch_short(const Mxfp4LogitsArgs& a, hipStream_t s) {
  const int64_t across = (a.V + 63) / 64;  // at most 8192
  const int64_t down = ((int64_t)1 << 23) / across;  // a grid holds fewer than 2^32 threads
  const int64_t rows = (down < 65535 ? down : 65535) * 16;
  for (int64_t t0 = 0; t0 < a.T; t0 += rows) {
    Mxfp4LogitsArgs b = a;
    b.T = a.T - t0 < rows ? a.T - t0 : rows;
    b.h_codes = a.h_codes + t0 * (a.d / 2);
    b.h_scales = a.h_scales + t0 * (a.d / 32);
    b.logits = (T*)a.logits + t0 * a.ld;
    fp4_logits_short<T><<<dim3((unsigned)across, (unsigned)((b.T + 15) / 16)), 256, 0, s>>>(b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t product_as(const Mxfp4LogitsArgs& a, hipStream_t s) {
  switch (fp4_kernel(a.T, a.d, a.V, sizeof(T), device_cu_count())) {
    case Fp4Kernel::kShort: return launch_short<T>(a, s);
    case Fp4Kernel::kRows16: return launch_tiles<Fp4Tile<4, 1, 2, 1, 3, true>, T>(a, s);
    case Fp4Kernel::kRows32: return launch_tiles<Fp4Tile<4, 1, 2, 2, 3, true>, T>(a, s);
    case Fp4Kernel::kRows64: return launch_tiles<Fp4Tile<4, 1, 2, 4, 2, true>, T>(a, s);
    case Fp4Kernel::kRows128: return launch_tiles<Fp4Tile<4, 1, 2, 8, 2, true>, T>(a, s);
    case Fp4Kernel::kSmall: return launch_tiles<Fp4Tile<4, 1, 2, 8, 2, false>, T>(a, s);
    case Fp4Kernel::kLargePast: return launch_tiles<Fp4Tile<2, 4, 8, 4, 1, false>, T, true>(a, s);
    case Fp4Kernel::kLargeOnce: return launch_tiles<Fp4Tile<2, 4, 8, 4, 1, true>, T>(a, s);
    case Fp4Kernel::kLarge: return launch_tiles<Fp4Tile<2, 4, 8, 4, 1, false>, T>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mxfp4_logits(const Mxfp4LogitsArgs& a, int dtype, hipStream_t s) {
  if (dtype == TIM_F32) return product_as<float>(a, s);
  if (dtype == TIM_BF16) return product_as<__bf16>(a, s);
  return product_as<_Float16>(a, s);
}

}  // namespace tim
