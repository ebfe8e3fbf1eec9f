// Stable sort of row indices by key, least significant digit first, and the
// lists of runs. Up to group_small_rows rows are one workgroup's work in LDS; more
// are sorted in one or two passes of two launches each (counts per block, then
// places), blocks in row order, then listed.
//
// Within a wave 64 consecutive items find the ones of their own digit by one
// ballot per bit, so equal digits keep their order without atomics.

#include <hip/hip_runtime.h>

#include "group_rows.h"

namespace tim {
namespace {

constexpr int kSortThreads = 256;
constexpr int kSortWaves = kSortThreads / 64;

template <int LOG_ROWS>
__global__ __launch_bounds__(kSmallThreads) void group_small(GroupArgs a) {
  group_rows<LOG_ROWS>(a);
}

// ------------------------------------------------------------ many rows

// One pass's input: the keys themselves (first pass), or key and row pairs.
struct Source {
  const int32_t* keys;
  const uint2* pairs;
  int64_t T;
  int32_t n, per_block, shift, bits;
};
__device__ __forceinline__ uint2 item_of(const Source& s, int64_t i) {
  return s.pairs ? s.pairs[i] : uint2{key_of(s.keys, i, s.n), (uint32_t)i};
}

// hist[block][digit]: items of each digit; the first launch of a grouping also
// clears the counters and `seen`.
__global__ __launch_bounds__(kSortThreads) void sort_count(Source s, uint32_t* hist, int32_t* counters,
                                                           uint8_t* seen) {
  __shared__ uint32_t count[kSortWaves][1024];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bins = 1 << s.bits;
  if (counters && blockIdx.x == 0 && threadIdx.x < 2 * kMaxRunLists) counters[threadIdx.x] = 0;
  if (seen)
    for (int i = blockIdx.x * kSortThreads + threadIdx.x; i * 4 < s.n; i += gridDim.x * kSortThreads)
      ((uint32_t*)seen)[i] = 0;
  for (int b = lane; b < bins; b += 64) count[wave][b] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * s.per_block;
  const int64_t to = base + s.per_block < s.T ? base + s.per_block : s.T;
  for (int64_t i = base + wave * 64; i < to; i += kSortThreads) {
    const bool there = i + lane < to;
    const uint32_t x = there ? item_of(s, i + lane).x : 0;
    count_step((x >> s.shift) & (bins - 1), s.bits, there, count[wave]);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads)
    hist[((size_t)blockIdx.x << s.bits) + b] = count[0][b] + count[1][b] + count[2][b] + count[3][b];
}

// The items in the pass's order: pairs, or (last pass) rows and keys apart.
__global__ __launch_bounds__(kSortThreads) void sort_place(Source s, const uint32_t* hist, uint2* pairs, int32_t* order,
                                                           uint32_t* keys) {
  __shared__ uint32_t place[kSortWaves][1024];
  __shared__ uint32_t wave_total[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bins = 1 << s.bits;
  for (int b = lane; b < bins; b += 64) place[wave][b] = 0;
  __syncthreads();
  // a wave takes consecutive quarters here, so that its items precede the next wave's
  const int64_t base = (int64_t)blockIdx.x * s.per_block + (int64_t)wave * (s.per_block / kSortWaves);
  const int64_t end = base + s.per_block / kSortWaves;
  const int64_t to = end < s.T ? end : s.T;
  for (int64_t i = base; i < to; i += 64) {
    const bool there = i + lane < to;
    const uint32_t x = there ? item_of(s, i + lane).x : 0;
    count_step((x >> s.shift) & (bins - 1), s.bits, there, place[wave]);
  }
  __syncthreads();
  // four consecutive digits a thread: items of smaller digits, and of the same one in earlier blocks
  const int per = bins > kSortThreads ? bins / kSortThreads : 1;
  uint32_t all[4] = {}, mine[4] = {}, sum = 0;
  if (threadIdx.x * per < (unsigned)bins) {
    for (unsigned k = 0; k < gridDim.x; ++k) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < per) {
          const uint32_t c = hist[((size_t)k << s.bits) + threadIdx.x * per + e];
          all[e] += c;
          if (k < blockIdx.x) mine[e] += c;
        }
    }
    sum = all[0] + all[1] + all[2] + all[3];
  }
  uint32_t incl = sum;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t y = __shfl_up(incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 63) wave_total[wave] = incl;
  __syncthreads();
  uint32_t before = incl - sum;
  for (int w = 0; w < wave; ++w) before += wave_total[w];
  if (threadIdx.x * per < (unsigned)bins) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < per) {
        uint32_t at = before + mine[e];
        before += all[e];
        for (int w = 0; w < kSortWaves; ++w) {
          const uint32_t c = place[w][threadIdx.x * per + e];
          place[w][threadIdx.x * per + e] = at;
          at += c;
        }
      }
  }
  __syncthreads();
  for (int64_t i = base; i < to; i += 64) {
    const bool there = i + lane < to;
    const uint2 x = there ? item_of(s, i + lane) : uint2{0, 0};
    const uint32_t at = place_step((x.x >> s.shift) & (bins - 1), s.bits, there, place[wave]);
    if (there) {
      if (pairs) {
        pairs[at] = x;
      } else {
        order[at] = (int32_t)x.y;
        keys[at] = x.x;
      }
    }
  }
}

// Lists the run that place p starts, if any, and the join of the runs that it ends. first: the first place of p's key.
template <class Keys, class Append>
__device__ __forceinline__ void list_place(const Lists& L, Keys key_at, int32_t T, int32_t p, bool there, uint32_t key,
                                           int32_t first, Append append) {
  for (int l = 0; l < L.lists; ++l) {
    const int log_C = L.log_C[l], C = 1 << log_C;
    const bool starts = there && ((p - first) & (C - 1)) == 0;
    Run r = {p, 0, (int32_t)key, -1};
    bool ends = false;  // the last run of several
    if (starts) {
      // the first place in (p, p + C] that is not of the key
      int lo = p + 1, hi = p + C < T ? p + C : T;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (key_at(mid) == key) lo = mid + 1; else hi = mid;
      }
      r.count = lo - p;
      const bool last = !(lo < T && key_at(lo) == key);
      if (p != first || !last) r.slot = run_slot(p, log_C, last);
      ends = last && p != first;
    }
    const int at = append(2 * l, starts);
    if (starts) L.runs[l][at] = r;
    const int j = append(2 * l + 1, ends);
    if (ends) L.joins[l][j] = {first, p + r.count, (int32_t)key, 0};
  }
}

// The inclusive maximum over the wave's lanes up to this one.
__device__ __forceinline__ int32_t wave_scan_max(int32_t x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int32_t y = __shfl_up(x, o);
    if (lane >= o && y > x) x = y;
  }
  return x;
}

constexpr int kListThreads = 256;
__global__ __launch_bounds__(kListThreads) void list_runs(const uint32_t* keys, int32_t T, int32_t limit, Lists L,
                                                          uint8_t* seen, int32_t* counters) {
  __shared__ int32_t wave_first[kListThreads / 64];
  __shared__ int32_t carry;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t base = blockIdx.x * kListThreads, p = base + tid;
  auto key_at = [&](int q) { return keys[q]; };
  if (wave == 0) {
    // the first place of the key at the block's start: 64 probes at a time
    const uint32_t key = keys[base];
    int lo = 0, hi = base;  // the answer is in [lo, hi]
    while (lo < hi) {
      const int step = (hi - lo + 63) / 64;
      const int q = lo + lane * step;
      const uint64_t at_or_after = __ballot(q >= hi || keys[q] >= key);
      // the first probe at or after the answer, and the one before it
      const int f = at_or_after ? __builtin_ctzll(at_or_after) : 64;
      const int new_hi = f == 64 ? hi : (lo + f * step < hi ? lo + f * step : hi);
      if (f > 0) lo = lo + (f - 1) * step + 1;
      hi = new_hi;
    }
    if (lane == 0) carry = lo;
  }
  const uint32_t key = p < T ? keys[p] : 0xffffffffu;
  const bool head = p < T && (p == 0 || keys[p - 1] != key);
  int first = wave_scan_max(head ? p : 0, lane);
  if (lane == 63) wave_first[wave] = first;
  __syncthreads();
  int before = carry;
  for (int w = 0; w < wave; ++w) before = wave_first[w] > before ? wave_first[w] : before;
  first = first > before ? first : before;
  const bool there = p < T && (int32_t)key < limit;
  if (head && there && seen && (int32_t)key < L.n) seen[key] = 1;
  auto append = [&](int c, bool add) {
    const uint64_t m = __ballot(add);
    int at = 0;
    if (m != 0 && lane == 0) at = atomicAdd(&counters[c], (int)__popcll(m));
    return __shfl(at, 0) + lanes_below(m);
  };
  list_place(L, key_at, T, p, there, key, first, append);
}

}  // namespace

#define TIM_TRY(call)                  \
  do {                                 \
    call;                              \
    const hipError_t e_ = hipGetLastError(); \
    if (e_ != hipSuccess) return e_;   \
  } while (0)

GroupArgs group_args(const Grouping& g, const int32_t* keys, bool keep_rest, uint8_t* seen, void* ws) {
  char* w = (char*)ws;
  GroupArgs a = {};
  a.keys = keys;
  a.T = (int32_t)g.T;
  a.passes = g.passes;
  a.digit = g.digit;
  a.limit = keep_rest ? g.n + 1 : g.n;
  a.lists.n = g.n;
  a.lists.lists = g.lists;
  for (int l = 0; l < g.lists; ++l) {
    a.lists.log_C[l] = g.log_C[l];
    a.lists.runs[l] = (Run*)(w + g.runs[l]);
    a.lists.joins[l] = (Join*)(w + g.joins[l]);
  }
  a.order = (int32_t*)(w + g.order);
  a.seen = seen;
  a.counters = (int32_t*)(w + g.counters);
  return a;
}

hipError_t launch_grouping(const Grouping& g, const int32_t* keys, bool keep_rest, uint8_t* seen, void* ws,
                           hipStream_t s) {
  const GroupArgs a = group_args(g, keys, keep_rest, seen, ws);
  if (g.small) {
    if (g.T <= 4096)
      TIM_TRY((group_small<12><<<1, kSmallThreads, 0, s>>>(a)));
    else
      TIM_TRY((group_small<14><<<1, kSmallThreads, 0, s>>>(a)));
    return hipSuccess;
  }
  char* w = (char*)ws;
  uint32_t* sorted = (uint32_t*)(w + g.keys);
  uint2* pairs = (uint2*)(w + g.pairs);
  uint32_t* hist = (uint32_t*)(w + g.hist);
  for (int pass = 0; pass < g.passes; ++pass) {
    const bool last = pass + 1 == g.passes;
    const Source src = {keys, pass == 0 ? nullptr : pairs, g.T, g.n, g.per_block, pass * g.digit, g.digit};
    TIM_TRY((sort_count<<<g.blocks, kSortThreads, 0, s>>>(src, hist, pass == 0 ? a.counters : nullptr,
                                                          pass == 0 ? seen : nullptr)));
    TIM_TRY((sort_place<<<g.blocks, kSortThreads, 0, s>>>(src, hist, last ? nullptr : pairs, a.order, sorted)));
  }
  TIM_TRY((list_runs<<<(unsigned)((g.T + kListThreads - 1) / kListThreads), kListThreads, 0, s>>>(
      sorted, (int32_t)g.T, a.limit, a.lists, seen, a.counters)));
  return hipSuccess;
}

}  // namespace tim
