// Groups of MMAs of the attention kernels over packed rows and over pages.
#pragma once
#include "common.cuh"

namespace tadm {

// A value that is the same in every lane, in a uniform register: what the MMA
// warp computes from it (loop counts, ring places, descriptors) then needs no
// move into one ahead of every MMA.
__device__ __forceinline__ int uniform(int x) { return static_cast<int>(__reduce_or_sync(0xffffffffu, static_cast<uint32_t>(x))); }
__device__ __forceinline__ int2 uniform(int2 x) { return make_int2(uniform(x.x), uniform(x.y)); }

// The MMAs of a tile in one block: the lane is elected once, and operands differ by constants in the low words of their
// descriptors (the high word: 1024 bytes from one 8-row group to the next, descriptor version, 128-byte swizzle).  With
// a 64-bit descriptor built per MMA their issue took longer than the MMAs.
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
// low word of a K-major tile at saddr (16 further elements: 32 bytes on; 64: 16384 on)
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return (saddr & 0x3FFFFu) >> 4 | 1u << 16; }
// low word of a tile of V as it lies in memory, an MN-major operand: lines of 64 dims per key (16 further keys: 2048
// bytes on), 64 further dims 16384 bytes on
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr) { return (saddr & 0x3FFFFu) >> 4 | (16384u >> 4) << 16; }

// D = A B^T over 64 dims (four MMAs), A and B in shared memory; acc: add to D
__device__ __forceinline__ void umma4_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, e, t;\n\t.reg .b64 da, db;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %5, %5;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, t;\n\t"
      "add.u32 x, %1, 4;\n\tadd.u32 y, %2, 4;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, t;\n\t"
      "add.u32 x, %1, 6;\n\tadd.u32 y, %2, 6;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, t;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHi)
      : "memory");
}
// D += A B over 64 keys (four MMAs), A = P in TMEM (8 columns per 16 keys), B = V, MN-major
__device__ __forceinline__ void umma4_ts_mn(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, e, t;\n\t.reg .b64 db;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %5, %5;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t"
      "add.u32 x, %1, 8;\n\tadd.u32 y, %2, 128;\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, t;\n\t"
      "add.u32 x, %1, 16;\n\tadd.u32 y, %2, 256;\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, t;\n\t"
      "add.u32 x, %1, 24;\n\tadd.u32 y, %2, 384;\n\tmov.b64 db, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, t;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHi)
      : "memory");
}

// The same over 32 keys with P in two terms: 16 columns of the first, then 16 of the second
__device__ __forceinline__ void umma4_ts_two(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, e, t;\n\t.reg .b64 db, dc;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %5, %5;\n\t"
      "add.u32 y, %2, 128;\n\tmov.b64 db, {%2, %5};\n\tmov.b64 dc, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t"
      "add.u32 x, %1, 8;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], dc, %3, t;\n\t"
      "add.u32 x, %1, 16;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, t;\n\t"
      "add.u32 x, %1, 24;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], dc, %3, t;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHi)
      : "memory");
}

// D = A B^T over STEPS x 32 dims of 8-bit floats (idesc says which), A and B in shared memory, both K-major with rows of HD bytes; hi: the high
// word of their descriptors (32 further dims: 32 bytes on)
template <int STEPS>
__device__ __forceinline__ void umma_f8_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, uint32_t acc) {
  if constexpr (STEPS == 4) {
    asm volatile(
        "{\n\t.reg .pred p, e, t;\n\t.reg .b64 da, db;\n\t.reg .b32 x, y;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %5, %5;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n\t"
        "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, t;\n\t"
        "add.u32 x, %1, 4;\n\tadd.u32 y, %2, 4;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, t;\n\t"
        "add.u32 x, %1, 6;\n\tadd.u32 y, %2, 6;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, t;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(hi)
        : "memory");
  } else {
    static_assert(STEPS == 2, "rows of 64 or 128 bytes");
    asm volatile(
        "{\n\t.reg .pred p, e, t;\n\t.reg .b64 da, db;\n\t.reg .b32 x, y;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, %5, %5;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n\t"
        "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %5};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, t;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(hi)
        : "memory");
  }
}

}  // namespace tadm
