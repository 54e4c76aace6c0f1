// Where the rows of packed sequences lie, for kernels whose blocks take row
// tiles of sequences that the host has not seen the lengths of.
#pragma once
#include "common.cuh"

namespace tadm {

// Rows first .. first + n - 1 of sequence b, inside 0 .. total and at most max_rows of them.
struct SeqRows {
  int first, n;
};
__device__ __forceinline__ SeqRows seq_rows(const int32_t* cu, int b, int total, int max_rows) {
  const int c0 = min(max(cu[b], 0), total), c1 = min(max(cu[b + 1], c0), total);
  return {c0, min(c1 - c0, max_rows)};
}

// The sequence of row `row`: cu[b] <= row < cu[b + 1]; -1: it is in none.  Warp-collective, for a row that the warp's lanes
// share; 32 boundaries per step, so that 1024 sequences take two reads one after the other.
__device__ __forceinline__ int seq_of_row(const int32_t* cu, int batch, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = batch + 1;                                  // the boundaries <= row end in lo .. lo + n
  while (n > 0) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool le = at < lo + n && cu[at] <= row;
    const int hits = __popc(__ballot_sync(0xffffffffu, le));
    if (hits == 0) return lo - 1;
    const int last = lo + (hits - 1) * step;                  // a boundary <= row; the next one asked about is not
    n = min(lo + n, last + step) - (last + 1);
    lo = last + 1;
  }
  return lo - 1 < batch ? lo - 1 : -1;
}

// Row tile `tile` of all sequences' tiles, sequence by sequence; tiles_of(b)
// says how many sequence b has.  Returns the sequence (-1: there are fewer
// tiles) and the tile's index in it.  Warp-collective, 32 sequences per step.
template <class F>
__device__ __forceinline__ int find_tile(int batch, int64_t tile, F&& tiles_of, int* within) {
  const int lane = threadIdx.x & 31;
  int64_t before = 0;
  for (int base = 0; base < batch; base += 32) {
    const int b = base + lane;
    int64_t x = b < batch ? tiles_of(b) : 0;
    const int64_t mine = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + x > tile);
    if (past) {
      const int src = __ffs(past) - 1;
      *within = static_cast<int>(__shfl_sync(0xffffffffu, tile - (before + x - mine), src));
      return base + src;
    }
    before += __shfl_sync(0xffffffffu, x, 31);
  }
  *within = 0;
  return -1;
}

// The same for tiles whose work grows with their index: 32 sequences at a time, their tiles in falling order of index (of
// those with the same index, by sequence).  Warp-collective.
template <class F>
__device__ __forceinline__ int find_largest(int batch, int tile, F&& tiles_of, int* within) {
  const int lane = threadIdx.x & 31;
  for (int base = 0; base < batch; base += 32) {
    const int n = base + lane < batch ? tiles_of(base + lane) : 0;
    const int all = __reduce_add_sync(0xffffffffu, n);
    if (tile >= all) {
      tile -= all;
      continue;
    }
    int lo = 0, hi = __reduce_max_sync(0xffffffffu, n), above = 0;   // tiles with an index >= lo: more than `tile`; >= hi: `above`
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2, more = __reduce_add_sync(0xffffffffu, max(n - mid, 0));
      if (more > tile) {
        lo = mid;
      } else {
        hi = mid;
        above = more;
      }
    }
    const unsigned have = __ballot_sync(0xffffffffu, n > lo);
    const bool mine = n > lo && __popc(have & ((1u << lane) - 1)) == tile - above;
    *within = lo;
    return base + __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
  }
  *within = 0;
  return -1;
}

}  // namespace tadm
