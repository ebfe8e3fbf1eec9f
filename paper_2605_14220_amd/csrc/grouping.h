// Rows grouped by a key (a row's token, or its adapter): a stable sort of the
// row indices by key and the list of runs that the operators work on.
//
// A run is at most C (a power of two) consecutive places of the sorted order with one key, and
// runs start every C places from the key's first: what a run holds depends on
// the key's own rows only. The lists' order in memory is not fixed (it is made
// with an atomic counter), so nothing may depend on it but which workgroup
// takes which run.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace tim {

// A run: places first .. first + count - 1 of the order, all of `key`. slot < 0:
// the key's only run. Otherwise one of several, whose partial result goes to
// `slot` (run_slot) and is joined with the others' by the key's entry of the
// list of joins.
struct alignas(16) Run {
  int32_t first, count, key, slot;
};
// The key whose rows are the places first .. end - 1, more than one run.
struct alignas(16) Join {
  int32_t first, end, key, pad;
};

// Slots of runs of C places. Of the keys with several runs, at most one full
// run starts in each C places, and at most one last (shorter or full) run of a key.
// C is a power of two, given by its logarithm.
__host__ __device__ inline int32_t run_slot(int32_t first, int log_C, bool last) {
  return (first >> log_C) * 2 + (last ? 1 : 0);
}
inline int64_t run_slots(int64_t T, int log_C) { return ((T >> log_C) + 1) * 2; }

// Rows that one workgroup sorts in LDS, by the sorting passes it takes. With one
// pass (up to 255 keys) 8192 rows take 18 us, in launches of their own 24; with
// more, 32 bits hold a key and the row's index only up to 4096 rows.
inline int64_t group_small_rows(int passes) { return passes == 1 ? 16384 : 4096; }
constexpr int kMaxRunLists = 3;

// Sizes and workspace of a grouping of T rows by keys in [0, n); keys outside
// are those of key n, whose runs are listed only with keep_rest.
struct Grouping {
  int64_t T;
  int32_t n;
  int32_t lists;                // lists of runs
  int32_t log_C[kMaxRunLists];  // logarithms of their lengths
  int64_t max_runs[kMaxRunLists], max_joins[kMaxRunLists];
  bool small;                   // one workgroup's work
  int32_t bits, passes, digit;  // of a key, sorting passes, bits a pass
  int32_t blocks, per_block;    // of the sort of many rows
  // offsets into the workspace
  size_t counters, order, keys, pairs, hist, runs[kMaxRunLists], joins[kMaxRunLists], bytes;
};

inline size_t group_align(size_t x) { return (x + 255) & ~(size_t)255; }

inline Grouping plan_grouping(int64_t T, int32_t n, int lists, const int* log_C) {
  Grouping g = {};
  g.T = T;
  g.n = n;
  g.lists = lists;
  while (((int64_t)1 << g.bits) < (int64_t)n + 1) ++g.bits;  // key n too
  size_t at = 0;
  g.counters = at, at += 256;
  g.order = at, at += group_align((size_t)T * 4);
  // digits of at most 8 bits: a bin for each of 256 threads to add up
  g.passes = (g.bits + 7) / 8;
  g.small = T <= group_small_rows(g.passes);
  if (g.small) {
    g.digit = (g.bits + g.passes - 1) / g.passes;
    g.blocks = 1;
    g.per_block = (int32_t)T;
  } else {
    g.passes = (g.bits + 9) / 10;
    g.digit = (g.bits + g.passes - 1) / g.passes;
    // at most 256 blocks, whose counts each block adds up by itself
    const int64_t per = (T + 255) / 256;
    g.per_block = (int32_t)((per + 1023) / 1024 * 1024);
    g.blocks = (int32_t)((T + g.per_block - 1) / g.per_block);
    g.keys = at, at += group_align((size_t)T * 4);
    g.pairs = at, at += g.passes > 1 ? group_align((size_t)T * 8) : 0;
    g.hist = at, at += group_align(((size_t)g.blocks << g.digit) * 4);
  }
  const int64_t distinct = T < (int64_t)n + 1 ? T : (int64_t)n + 1;
  for (int l = 0; l < lists; ++l) {
    const int64_t C = (int64_t)1 << log_C[l];
    g.log_C[l] = log_C[l];
    g.max_runs[l] = T / C + distinct;
    g.max_joins[l] = T / (C + 1) < distinct ? T / (C + 1) : distinct;
    g.runs[l] = at, at += group_align((size_t)g.max_runs[l] * sizeof(Run));
    g.joins[l] = at, at += group_align((size_t)g.max_joins[l] * sizeof(Join));
  }
  g.bytes = at;
  return g;
}

// The lists on the device.
struct RunList {
  const int32_t* order;
  const Run* runs;
  const Join* joins;
  const int32_t* n_runs;
  const int32_t* n_joins;
  int64_t max_runs, max_joins;
};
#if defined(__HIPCC__)
// The run (or other item) and the tile of it that a workgroup of a grid of
// (items, tiles) takes: consecutive workgroups take consecutive tiles. They go to
// the eight XCDs in turn; with the items first, of which a list leaves some
// empty, 8 items with 4 runs among them would leave four XCDs without work (the
// pass over grad of 2047 rows on a head of 151936 took 242 us so).
struct Place {
  uint32_t item, tile;
};
__device__ __forceinline__ Place place_of() {
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
  return {id / gridDim.y, id % gridDim.y};
}
// Keeps the compiler from moving LDS accesses of a wave across it; the hardware
// takes a wave's LDS accesses in order.
__device__ __forceinline__ void lanes_in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// A run of the list (count 0: past its end), asked for beside the list's length rather than after it.
__device__ __forceinline__ Run run_of(const RunList& l, uint32_t item) {
  Run r = l.runs[item];
  const int32_t n = *l.n_runs;
  asm volatile("" ::"s"(n), "s"(r.first));  // both loads before the branch
  if ((int)item >= n) r.count = 0;
  return r;
}
#endif
inline RunList run_list(const Grouping& g, const void* ws, int l) {
  const char* w = (const char*)ws;
  const int32_t* c = (const int32_t*)(w + g.counters);
  return {(const int32_t*)(w + g.order), (const Run*)(w + g.runs[l]), (const Join*)(w + g.joins[l]), c + 2 * l,
          c + 2 * l + 1, g.max_runs[l], g.max_joins[l]};
}

// seen (may be null): a byte per key in [0, n), set to 1 for the keys that
// occur and 0 for the others; room for whole words, 4-byte aligned.
hipError_t launch_grouping(const Grouping& g, const int32_t* keys, bool keep_rest, uint8_t* seen, void* ws,
                           hipStream_t s);

}  // namespace tim
