// Sizes, shapes and workspaces of the adapters' calls, from their sizes alone.
#pragma once

#include <cstddef>
#include <cstdint>

#include "grouping.h"
#include "tim_policy.h"

namespace tim {

constexpr int kLogAdapterRun = 6;   // 64 rows of one adapter that a workgroup takes together
constexpr int kShrinkChunk = 512;  // elements of d whose products one workgroup sums

inline int rank_padded(int r) { return (r + 15) / 16 * 16; }
inline int chunks_of(int64_t n, int chunk) { return (int)((n + chunk - 1) / chunk); }

// The pass over grad sums grad b over tiles of 256 columns (128 where it runs on
// the fp32 instructions), and two tiles in order, whatever a workgroup takes: 1 or
// 2 tiles of up to 2^log_rows rows of one adapter. More tiles leave fewer partial
// sums of grad b, more rows fewer of the weights' gradients; both have to leave
// work for 256 CUs.
//
// Up to rank 16 three workgroups of one tile fit a CU (51 KB of LDS, 45 on the fp32
// instructions). Where one tile each would be more than the 768 that run at once, a
// second round would follow for the rest, and workgroups take two. A call of 150 rows
// of 2 adapters, rank 16, d 1536, one tile a workgroup and two, us:
//   740 of one tile   fp32 51.4, 51.7   bf16 53.8, 53.5
//   770               fp32 57.9, 50.9   bf16 58.6, 51.6
//   1540              fp32 72.0, 66.2   bf16 72.6, 67.3
// (700 rows, whose runs end in part of a block: 1100 fp32 84.5, 91.4 and bf16 97.8,
// 111.5; 1540 fp32 104, 92 and bf16 114, 114. 2047 rows on a head of 151936: 161 us
// with two tiles, with one 159 and 13 more to add up the sums, with four 183.) Each
// adapter of the set is taken for one with rows, for the host does not know which
// have some: 150 rows of 2 adapters out of a set of 24 on 16000 columns, fp32, take
// 55.0 us with the two tiles that follow, 51.4 with one.
constexpr int kPassCols = 256, kPassColsF32 = 128, kTilePair = 2;
constexpr int kPassesAtOnce = 3 * 256;
constexpr int kLogMaxPassRows = 9, kMaxPassRows = 1 << kLogMaxPassRows;
struct PassShape {
  int tiles, log_rows;
};
inline PassShape pass_shape(int64_t T, int64_t N, int n, int cols, int rp, bool contract) {
  PassShape s = {1, kLogMaxPassRows};
  auto workgroups = [&](int tiles, int log_rows) { return ((T >> log_rows) + 1) * chunks_of(N, tiles * cols); };
  const int64_t runs = (T >> s.log_rows) + (n < T ? n : T);
  if (contract && rp <= 16 && runs * chunks_of(N, cols) > kPassesAtOnce) s.tiles = 2;
  while (s.log_rows > 7 && workgroups(s.tiles, s.log_rows) < 512) --s.log_rows;
  return s;
}
// The columns of its tiles: whether grad and the adapters are bf16.
inline int pass_cols(int dtype, int adapter_dtype) {
  return dtype == TIM_BF16 && adapter_dtype == TIM_BF16 ? kPassCols : kPassColsF32;
}

// Workspaces: the grouping, then fp32 [chunks, T, rank_padded] of partial sums
// of x a^T, and for the backward those of grad b, both sums, and the partial
// weight gradients of adapters with several runs of rows.
struct AdapterPlan {
  Grouping g;  // runs of kAdapterRun rows; the backward's for grad_a and for grad_b
  int rp, x_chunks, g_chunks;
  bool rows_alone;  // u by rows, beside the grouping
  PassShape of_x, of_grad;
  size_t u_part, v_part, u, v, v_terms, a_part, b_part, seen, bytes;
};
// cols: of the pass over grad (pass_cols); 0 for the forward.
inline AdapterPlan plan_adapters(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r, int cols) {
  const bool backward = cols != 0;
  AdapterPlan p = {};
  p.rp = rank_padded(r);
  p.x_chunks = chunks_of(d, kShrinkChunk);
  // the pass over x runs on the bf16 instructions or not as x is, whatever grad is; its runs may be the same
  p.of_x = pass_shape(T, d, n, kPassCols, p.rp, false);
  if (backward) {
    p.of_grad = pass_shape(T, N, n, cols, p.rp, true);
    p.g_chunks = chunks_of(N, p.of_grad.tiles * cols);
  }
  const int log_C[3] = {kLogAdapterRun, p.of_x.log_rows, p.of_grad.log_rows};
  p.g = plan_grouping(T, n, backward ? 3 : 1, log_C);
  // few rows, whose adapters' weights for each come to at most 32 MB from the caches
  p.rows_alone = T <= 1024 && T * p.rp * d * 2 <= (int64_t)32 << 20;
  size_t at = p.g.bytes;
  const size_t rows = group_align((size_t)T * p.rp * 4);
  p.u_part = at, at += rows * p.x_chunks;
  if (backward) {
    p.v_part = at, at += rows * p.g_chunks;
    p.u = at, at += rows;
    p.v = at, at += rows;
    p.v_terms = at, at += group_align((size_t)T * p.rp * 6);
    p.a_part = at, at += p.g.max_joins[1] > 0 ? group_align((size_t)run_slots(T, log_C[1]) * r * d * 4) : 0;
    p.b_part = at, at += p.g.max_joins[2] > 0 ? group_align((size_t)run_slots(T, log_C[2]) * r * N * 4) : 0;
    p.seen = at, at += group_align((size_t)n);
  }
  p.bytes = at;
  return p;
}

// Bytes of the backward's workspace, for either kind of pass over grad.
inline size_t adapters_backward_workspace(int64_t T, int32_t d, int32_t N, int32_t n, int32_t r) {
  const size_t a = plan_adapters(T, d, N, n, r, kPassCols).bytes, b = plan_adapters(T, d, N, n, r, kPassColsF32).bytes;
  return a > b ? a : b;
}

}  // namespace tim
