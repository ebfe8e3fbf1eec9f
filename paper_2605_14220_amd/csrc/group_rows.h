// The grouping of few rows (group_small_rows) by one workgroup of kSmallThreads,
// for the kernel that does that alone and for those that do it beside other work.
#pragma once

#include <hip/hip_runtime.h>

#include "grouping.h"

namespace tim {

constexpr int kSmallThreads = 1024;
constexpr int kSmallWaves = kSmallThreads / 64;

// The lanes whose digit (of `bits` bits) is this lane's, among those of `active`.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, uint64_t active) {
  uint64_t peers = active;
  for (int b = 0; b < bits; ++b) {
    const bool set = (digit >> b) & 1;
    const uint64_t m = __ballot(set);
    peers &= set ? m : ~m;
  }
  return peers;
}
__device__ __forceinline__ int lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

__device__ __forceinline__ uint32_t key_of(const int32_t* keys, int64_t i, int32_t n) {
  const uint32_t k = (uint32_t)keys[i];
  return k < (uint32_t)n ? k : (uint32_t)n;
}

// Counts a wave's items of consecutive steps per digit: `count` is the wave's own.
__device__ __forceinline__ void count_step(uint32_t digit, int bits, bool there, volatile uint32_t* count) {
  const uint64_t peers = same_digit(digit, bits, __ballot(there));
  if (there && lanes_below(peers) == 0) count[digit] += __popcll(peers);
  lanes_in_order();
}
// The item's place: `place` holds the wave's next place of each digit.
__device__ __forceinline__ uint32_t place_step(uint32_t digit, int bits, bool there, volatile uint32_t* place) {
  const uint64_t peers = same_digit(digit, bits, __ballot(there));
  const int below = lanes_below(peers);
  const uint32_t at = there ? place[digit] : 0;
  lanes_in_order();
  if (there && below == 0) place[digit] = at + __popcll(peers);
  lanes_in_order();
  return at + below;
}

// The lists to make of the sorted keys.
struct Lists {
  int32_t n, lists;
  int32_t log_C[kMaxRunLists];
  Run* runs[kMaxRunLists];
  Join* joins[kMaxRunLists];
};
// What the grouping of few rows takes.
struct GroupArgs {
  const int32_t* keys;
  int32_t T, passes, digit, limit;  // keys from `limit` on are not listed
  Lists lists;
  int32_t* order;
  uint8_t* seen;
  int32_t* counters;
};
GroupArgs group_args(const Grouping& g, const int32_t* keys, bool keep_rest, uint8_t* seen, void* ws);

// One workgroup. Items are the key above the row index, 32 bits: keys below 2^20
// with 4096 rows, below 2^18 with 16384.
template <int LOG_ROWS>
__device__ __forceinline__ void group_rows(const GroupArgs& a) {
  const int T = a.T, digit_bits = a.digit;
  const Lists& L = a.lists;
  uint8_t* seen = a.seen;
  constexpr int kRows = 1 << LOG_ROWS;
  __shared__ uint32_t item[2][kRows + 64];
  __shared__ uint32_t place[kSmallWaves][256];
  __shared__ uint32_t wave_total[kSmallWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bins = 1 << digit_bits;
  // each wave takes consecutive items, a multiple of 64
  const int per_wave = ((T + kSmallWaves - 1) / kSmallWaves + 63) / 64 * 64;
  const int from = wave * per_wave, to = from + per_wave < T ? from + per_wave : T;
#pragma unroll 4
  for (int i = tid; i < T; i += kSmallThreads) item[0][i] = key_of(a.keys, i, L.n) << LOG_ROWS | i;
  if (seen)
    for (int i = tid; i * 4 < L.n; i += kSmallThreads) ((uint32_t*)seen)[i] = 0;
  int cur = 0;
  for (int pass = 0; pass < a.passes; ++pass, cur ^= 1) {
    const int shift = LOG_ROWS + pass * digit_bits;
    for (int b = lane; b < bins; b += 64) place[wave][b] = 0;
    __syncthreads();
    for (int i = from; i < to; i += 64) {
      const bool there = i + lane < to;
      const uint32_t x = there ? item[cur][i + lane] : 0;
      count_step((x >> shift) & (bins - 1), digit_bits, there, place[wave]);
    }
    __syncthreads();
    // places: digits in order, the waves' items of one digit in wave order
    uint32_t sum = 0, incl = 0, c[kSmallWaves] = {};
    if (tid < 256) {
      if (tid < bins) {
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) c[w] = place[w][tid];
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) {
          const uint32_t x = c[w];
          c[w] = sum;
          sum += x;
        }
      }
      incl = sum;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const uint32_t y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 63) wave_total[wave] = incl;
    }
    __syncthreads();
    if (tid < bins) {
      uint32_t before = incl - sum;
      for (int w = 0; w < wave; ++w) before += wave_total[w];
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) place[w][tid] = before + c[w];
    }
    __syncthreads();
    for (int i = from; i < to; i += 64) {
      const bool there = i + lane < to;
      const uint32_t x = there ? item[cur][i + lane] : 0;
      const uint32_t at = place_step((x >> shift) & (bins - 1), digit_bits, there, place[wave]);
      if (there) item[cur ^ 1][at] = x;
    }
    __syncthreads();
  }
  const uint32_t* sorted = item[cur];
  int32_t* head = (int32_t*)item[cur ^ 1];  // the first place of each key that occurs
  // the sum of x over the threads before this one and the earlier `total`, which grows by the sum over all threads
  auto scan = [&](uint32_t x, uint32_t& total) {
    uint32_t incl = x;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const uint32_t y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
    __syncthreads();  // the last scan's sums are read
    if (lane == 63) wave_total[wave] = incl;
    __syncthreads();
    uint32_t before = total + incl - x;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
      const uint32_t y = wave_total[w];
      before += w < wave ? y : 0;
      total += y;
    }
    return before;
  };
  // a wave's items again: how many keys begin in them, then where
  auto begins = [&](int i, uint32_t& x) {
    x = i < to ? sorted[i] : 0;
    return i < to && (i == 0 || sorted[i - 1] >> LOG_ROWS != x >> LOG_ROWS);
  };
  uint32_t here = 0, heads = 0, x;
  for (int i = from; i < to; i += 64) here += (uint32_t)__popcll(__ballot(begins(i + lane, x)));
  uint32_t next = scan(lane == 0 ? here : 0, heads);
  next = __shfl(next, 0);
  for (int i = from; i < to; i += 64) {
    const bool is = begins(i + lane, x);
    const uint64_t mask = __ballot(is);
    if (i + lane < to) a.order[i + lane] = x & (kRows - 1);
    if (is) {
      head[next + lanes_below(mask)] = i + lane;
      if (seen && (int32_t)(x >> LOG_ROWS) < L.n) seen[x >> LOG_ROWS] = 1;
    }
    next += (uint32_t)__popcll(mask);
  }
  if (tid == 0) head[heads] = T;
  __syncthreads();
  // the keys from `limit` on are the last ones: key n alone
  if ((int32_t)(sorted[T - 1] >> LOG_ROWS) >= a.limit) --heads;
  for (int l = 0; l < L.lists; ++l) {
    const int log_C = L.log_C[l], C = 1 << log_C;
    uint32_t total = 0;  // runs, and joins from bit 16 on
    for (uint32_t base = 0; base < heads; base += kSmallThreads) {
      const uint32_t h = base + tid;
      int first = 0, end = 0, key = 0;
      if (h < heads) {
        first = head[h];
        end = head[h + 1];
        key = sorted[first] >> LOG_ROWS;
      }
      const int runs = (end - first + C - 1) >> log_C;
      const uint32_t at = scan(runs + (runs > 1 ? 1 << 16 : 0), total);
      auto put = [&](int q, int first, int end, int key, int runs, int at) {
        const int f = first + q * C;
        L.runs[l][at + q] = {f, end - f < C ? end - f : C, key, runs > 1 ? run_slot(f, log_C, q == runs - 1) : -1};
      };
      constexpr int kOwn = 4;  // runs that the key's thread lists; more are the whole wave's work
      for (int q = 0; q < kOwn; ++q)
        if (q < runs) put(q, first, end, key, runs, at & 0xffff);
      if (runs > 1) L.joins[l][at >> 16] = {first, end, key, 0};
      for (uint64_t more = __ballot(runs > kOwn); more != 0; more &= more - 1) {
        const int src = __builtin_ctzll(more);
        const int f = __shfl(first, src), e = __shfl(end, src), k = __shfl(key, src), n = __shfl(runs, src);
        const int a = __shfl((int)(at & 0xffff), src);
        for (int q = kOwn + lane; q < n; q += 64) put(q, f, e, k, n, a);
      }
    }
    if (tid == 0) {
      a.counters[2 * l] = total & 0xffff;
      a.counters[2 * l + 1] = total >> 16;
    }
  }
}

}  // namespace tim
