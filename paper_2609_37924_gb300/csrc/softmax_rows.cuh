// What the tcgen05 attention kernels share whose softmax has a query row per thread.
#pragma once
#include "common.cuh"

namespace tadm {

// One arrival per warp: the lanes' reads (TMEM) and writes (shared memory,
// each fenced for the async proxy by its own lane) precede the elected
// lane's arrive.  128 arrivals per tile and barrier serialise on the barrier
// word; one per warp does not.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// barrier `id` of T threads, and its vote
template <int T>
__device__ __forceinline__ void bar_group(int id) {
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "n"(T) : "memory");
}
template <int T>
__device__ __forceinline__ bool vote_group(int id, bool p) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred a, b;\n\t"
      "setp.ne.u32 a, %1, 0;\n\t"
      "barrier.cta.red.or.pred b, %3, %2, a;\n\t"
      "selp.u32 %0, 1, 0, b;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(p)), "n"(T), "r"(id)
      : "memory");
  return r != 0;
}

// Max of 64 scores of one row (two chunks of 32); MASKED: only the columns lo <= c < lim count.
template <bool MASKED>
__device__ __forceinline__ void max64(const uint32_t (&ra)[32], const uint32_t (&rb)[32], int lo, int lim,
                                      float (&mx)[4]) {
#pragma unroll
  for (int k = 0; k < 32; ++k) {
    float a = __uint_as_float(ra[k]), b = __uint_as_float(rb[k]);
    if (MASKED) {
      a = k < lim && k >= lo ? a : -INFINITY;
      b = 32 + k < lim && 32 + k >= lo ? b : -INFINITY;
    }
    mx[k & 3] = fmax3(mx[k & 3], a, b);
  }
}

}  // namespace tadm
