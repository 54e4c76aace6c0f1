// One token per row of logits, drawn with the row's own temperature, top-k,
// top-p and min-p from a given random number.
//
//   order   ids by falling logit, equal ones by rising id
//   w_v     exp((l_v - max) / T)
//   kept    the longest first part of the order with rank < k, w >= min_p and
//           exclusive mass < p S (S: the mass that k and min_p leave)
//   token   the first kept id, in the order of ids, whose cumulative weight
//           exceeds u * mass(kept)
//
// Every set is a first part of the order, so it is one cut: a key (the logit's
// bits as an ordered integer) and, among the ids of that key, a last id.
//
// A cut or a draw next to a border must not depend on rounding: with weights
// of fp32 a row of 10^5 like tokens draws another one every few thousand
// rows.  Weights are right to 2^-28 (2^-30.6 in the mean over logits, without a
// bias), and their sums are 64-bit integers in units of 2^-44, or pairs of fp32
// sums good to 2^-37 a lane (bulk).  So a border has to lie within some 2^-34 of
// the mass where a hundred distinct logits or more carry it; where a few do,
// equal ones among them, whose errors are one, within 2^-29 (two values with
// half of the mass each: a quarter of the difference of their errors).
//
// Rows of up to 4096 ids: one block a row, sample_finish_kernel.  Longer ones:
//   sample_scan_kernel     per 8192 ids: maximum, mass per 512 ids, histogram of
//                          the mass by value in 512 bins;
//   sample_plan_kernel     per row: from those the mass to be kept, and between
//                          which values the cut lies (three bins); where few ids are
//                          kept at all, a value below the cut;
//   sample_collect_kernel  per 8192 ids: the mass above those values per 512
//                          ids, and a list of the ids in between;
//   sample_finish_kernel   per row: the cut within the list, by histograms over the
//                          key until 128 elements or one key are left; the 512
//                          ids in which the draw falls; the token.
// Where a list overflows or the guess was wrong, the last one takes the whole
// row by the same histograms (logits beyond some 2^17 T, where a chunk's weights
// or bins are not counted; cuts of thousands of ids by top-k under a second
// setting).  Of few rows the last three are one kernel, sample_rest_kernel.
//
// Bound: of few rows the chain of small steps, each a barrier or two (a row of 32768
// ids 16 to 20 us, of which the scan 4); of many the instructions of the two passes
// over the logits (512 rows of 128000, fp32, a nucleus each: 230 us, of which scan
// 111 with 46 instructions an id at 73 % of the issue slots, collect 87 with 36 at
// 73 %; one reading of the logits is 39).  Rows of up to 4096 ids: the same steps over all of
// a row's ids (one row of 1024 9.0 us with top-p, 5.4 without; 512 of 4096 47 and 30; 4096
// of 4096 294 and 200).  Weights above the cut summed where they
// lie, without moving them together, 292 us with two blocks an SM.  The row in the
// shared memory of a cluster of 8 blocks instead, read from HBM once, took 691
// us: 38 rows at a time, each some 45 us of passes that end in a cluster
// barrier.  A pair of values per instruction (f32x2) executes as many
// instructions as one.
#include <cstdint>

#include "common.cuh"
#include "requests.h"

namespace tadm {
namespace {

constexpr int NT = 512, NW = NT / 32, NB = 512, LIST = 128;
constexpr int PER = 16;                    // ids of a lane
constexpr int CHUNK = NT * PER, SEG = 32 * PER;   // ids of a block, of a warp
constexpr int CAP = 4096;                  // ids on a row's list
constexpr int SEGS = (kSampleMaxVocab + SEG - 1) / SEG;
constexpr uint64_t ONE = 1ull << 44;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int rows, vocab, mask_id, chunks;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* tok;
  float* prob;
  // scratch
  struct ChunkInfo* info;                  // [rows][chunks]
  uint64_t *seg, *kept;                    // [rows][chunks * NW] mass of a warp's ids: as scanned; kAll: in the row's units, kWindow: above the list
  uint32_t* hist;                          // [rows][chunks][NB]
  struct RowPlan* plan;                    // [rows]
  uint2* list;                             // [rows][CAP] key, id
};
// Maximum of a chunk; its weights count from 2^(mj / 16), its bins from gj down; far: one of them does not fit, the row is taken
// whole if anything in the chunk counts.
struct ChunkInfo {
  float max;
  int mj, gj, far;
};
enum Mode : int { kEmpty, kAll, kListed, kWindow, kWhole };
// kAll: every id is kept, the masses are the scan's.  kListed: what may be kept is on the list.  kWindow: what lies above
// the list is kept, too; of the mass, `target` is, or, under min-p, top-p of `mass`, or the cut is by `count`.  kWhole: the last kernel takes the row by itself.
struct RowPlan {
  float max, lo, hi;                       // the list: lo <= logit <= hi
  float c_hi, c_lo, none;                  // the scale; see none_of()
  int mode, mj, listed;
  int more;                                // ids below lo may be kept, too
  int left;                                // kWindow: 1 where `mass` is wanted
  uint32_t low;                            // the least key that min-p keeps
  uint64_t target;
  unsigned long long mass, count;          // kWindow, where the cut is by them: mass that min-p leaves, ids above hi
  int done;                                // chunks that are through (the kernels of few rows)
};

// ------------------------------------------------------------------ keys
// Logits as integers of the same order.  bf16: 16 bits, so that a key is one value.
template <class T>
struct Key;
template <>
struct Key<float> {
  static __device__ __forceinline__ uint32_t of(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
  }
  static __device__ __forceinline__ float value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
  }
};
template <>
struct Key<bf16> {
  static __device__ __forceinline__ uint32_t of(float v) { return Key<float>::of(v) >> 16; }
  static __device__ __forceinline__ float value(uint32_t k) {
    return Key<float>::value(k & 0x8000u ? k << 16 : (k << 16) | 0xffffu);
  }
};

// 16 bytes of logits
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
  }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

// The logits of a row: NaN and the masked id count as -inf, -0 as 0.
template <class T>
struct Logits {
  using V = Vec<T>;
  const T* p;
  int vocab, mask_id;
  bool vec;                                // rows on 16 bytes
  __device__ __forceinline__ Logits(const SampleArgs& a, int row)
      : p(static_cast<const T*>(a.logits) + row * a.ld), vocab(a.vocab), mask_id(a.mask_id),
        vec((reinterpret_cast<uintptr_t>(p) & 15) == 0) {}
  __device__ __forceinline__ float one(int id) const {
    const float ninf = __int_as_float(0xff800000);
    return id < vocab && id != mask_id ? fmaxf(to_f32(p[id]) + 0.0f, ninf) : ninf;
  }
  // V::N ids from id on, a multiple of V::N
  __device__ __forceinline__ uint4 load(int id) const {
    if (vec && id + V::N <= vocab) return __ldg(reinterpret_cast<const uint4*>(p + id));
    alignas(16) T v[V::N];
#pragma unroll
    for (int e = 0; e < V::N; ++e) v[e] = id + e < vocab ? p[id + e] : from_f32<T>(__int_as_float(0xff800000));
    return *reinterpret_cast<const uint4*>(v);
  }
  template <bool ZERO = true>              // false: -0 stays
  __device__ __forceinline__ void get(const uint4& q, int id, float* v) const {
    const float ninf = __int_as_float(0xff800000);
    float x[V::N];
    V::get(q, x);
#pragma unroll
    for (int e = 0; e < V::N; ++e) v[e] = fmaxf(ZERO ? x[e] + 0.0f : x[e], ninf);
    if (static_cast<uint32_t>(mask_id - id) < V::N) {
#pragma unroll
      for (int e = 0; e < V::N; ++e)
        if (id + e == mask_id) v[e] = ninf;
    }
  }
};

// ------------------------------------------------------------------ weights
// 2^(j/16) in units of 2^-43, rounded; and over 1 + j/16 in fp32, with what the product of the two leaves over itself
__constant__ const uint64_t kPow[16] = {
    0x80000000000ull, 0x85aac367cc5ull, 0x8b95c1e3ea9ull, 0x91c3d373ab1ull,
    0x9837f0518dcull, 0x9ef5326091aull, 0xa5fed6a9b15ull, 0xad583eea42aull,
    0xb504f333f9eull, 0xbd08a39f581ull, 0xc5672a11550ull, 0xce248c151f8ull,
    0xd744fccad6aull, 0xe0ccdeec2a9ull, 0xeac0c6e7dd2ull, 0xf5257d15248ull};
__constant__ const float2 kPowF[16] = {
    {1.0f, 0.0f}, {0.982845902f, 4.62854715e-08f}, {0.969340205f, -1.19921575e-08f}, {0.958979905f, 4.72978243e-08f},
    {0.951365709f, 3.19341815e-08f}, {0.946177363f, 3.62105723e-08f}, {0.943156064f, -3.09907193e-08f}, {0.942090809f, -7.47521334e-09f},
    {0.942809045f, 1.71142709e-08f}, {0.945168734f, -3.04768335e-08f}, {0.949052811f, 5.23333421e-09f}, {0.954364657f, 6.10759177e-09f},
    {0.961024463f, -1.47196051e-08f}, {0.968966722f, -5.25879518e-09f}, {0.978137672f, -6.12825968e-09f}, {0.988493681f, 5.14060927e-09f}};
// 2^f - 1 = f (A1 + f (A2 + f (A3 + f A4))) for |f| <= 1/32: ln2^n / n!, eased so that the neglected terms spread (Chebyshev);
// with the coefficients in fp32 right to 2^-33.7, which is little beside what its evaluation rounds (2^-30.6, 2^-28.3 at most)
constexpr float A1 = 0.693147182f, A2 = 0.240226507f, A3 = 0.0555057377f, A4 = 0.00961835496f;
constexpr float kMagic = 12582912.0f;      // 1.5 * 2^23: added to a number, leaves the nearest whole one in the low bits
constexpr int kMagicBits = 0x4b400000;
constexpr int kFar = 1 << 22;              // |mj|, |gj| below this

// Settings of a row.
struct Row {
  float hi, lo;                            // log2(e) / T in two terms
  int k;
  float p, mp, t;
};
// log2(e) / t in two terms
__device__ __forceinline__ void log2e_over(float t, float& hi, float& lo) {
  constexpr double kLog2e = 1.4426950408889634074;
  constexpr float L = static_cast<float>(kLog2e), LL = static_cast<float>(kLog2e - static_cast<double>(L));
  hi = L / t;
  lo = hi > 0.0f && hi < 3e38f ? (fmaf(-hi, t, L) + LL) / t : 0.0f;   // the division's remainder
}
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row) {
  Row r;
  r.t = a.temperature ? a.temperature[row] : 1.0f;
  r.p = a.top_p ? a.top_p[row] : 1.0f;
  r.mp = a.min_p ? a.min_p[row] : 0.0f;
  const int k = a.top_k ? a.top_k[row] : 0;                   // (asked for with the others)
  r.k = !(r.t > 0x1p-100f) || r.p <= 0.0f ? 1 : k;
  if (r.k < 0 || r.k >= a.vocab) r.k = 0;
  log2e_over(r.t, r.hi, r.lo);
  return r;
}
// p / q, right to an ulp of fp32 (a quotient of doubles takes four times as long).
__device__ __forceinline__ float ratio(uint64_t p, uint64_t q) {
  const float ph = __ull2float_rn(p), qh = __ull2float_rn(q);
  const float pl = static_cast<float>(static_cast<int64_t>(p - static_cast<uint64_t>(ph))), ql = static_cast<float>(static_cast<int64_t>(q - static_cast<uint64_t>(qh)));
  const float x = ph / qh;
  return x + (fmaf(-x, qh, ph) + fmaf(-x, ql, pl)) / qh;
}
// f m rounded down (UP: up), for 0 <= f < 1: f's 24 bits times m's 64, shifted.
template <bool UP>
__device__ __forceinline__ uint64_t times(float f, uint64_t m) {
  const uint32_t b = __float_as_uint(f), e = b >> 23;
  const uint64_t mant = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int down = 150 - static_cast<int>(e ? e : 1);         // f = mant 2^-down, down >= 24
  const uint64_t lo = mant * m, hi = __umul64hi(mant, m);
  if (down >= 128) return UP && mant != 0 && m != 0;
  const uint64_t q = down >= 64 ? hi >> (down - 64) : (hi << (64 - down)) | (lo >> down);
  const bool rest = down >= 64 ? lo != 0 || (down > 64 && hi << (128 - down) != 0) : lo << (64 - down) != 0;
  return q + (UP && rest);
}
// Which part of `mass` is kept: at least a unit, at most all of it.
__device__ __forceinline__ uint64_t target_of(float p, uint64_t mass) { return min(max(times<true>(p, mass), static_cast<uint64_t>(1)), mass); }
// Ids of less than 2^-depth of the maximum are of no account: too light for a nucleus (those that weigh less than
// (1 - p) / vocab together weigh less than 1 - p of the mass), or for any draw.
__device__ __forceinline__ float depth_of(const SampleArgs& a, const Row& r) {
  return r.k == 0 && r.mp <= 0.0f && r.p < 1.0f ? fminf(44.0f, __log2f(static_cast<float>(a.vocab) / (1.0f - r.p)) + 0.5f) : 44.0f;
}

// What weights count from: 2^(mj / 16), next to the weight of a maximum.  t = c x - mj / 16 without the rounding of a
// difference: j = 16 t to the nearest whole number, f = c x - (mj + j) / 16 by one fma (whose product is exact), plus c's
// second term.  shift: the maximum where it is far from zero (then mj = 0, and logits that weigh anything are near it).  by:
// what logits are multiplied with, and temperatures, too.
struct Scale {
  float hi, lo, hi16, k_c, mh, shift, by;
  __device__ __forceinline__ Scale(float c_hi, float c_lo, int mj, float from, float factor = 1.0f)
      : hi(c_hi), lo(c_lo), hi16(16.0f * c_hi), k_c(kMagic - static_cast<float>(mj)), mh(static_cast<float>(mj) * 0.0625f), shift(from), by(factor) {}
};
__device__ __forceinline__ int mj_of(float c_hi, float c_lo, float max) {
  const float m = 16.0f * max * c_hi;
  return fabsf(m) < static_cast<float>(kFar) - 2.0f ? __float2int_rn(m) : kFar;
}
// Of a row taken by itself.  Where its temperature is above 10^30 logits that count may lie further apart than the largest number,
// and log2(e) / T has no second term: both are taken 2^-64 times.  (What a logit loses by that weighs nothing.)
__device__ __forceinline__ Scale far_scale(const Row& r, float max) {
  if (r.hi > 1e-30f) return Scale(r.hi, r.lo, 0, max);
  constexpr float by = 0x1p-64f;
  float hi, lo;
  log2e_over(r.t * by, hi, lo);
  const int mj = mj_of(hi, lo, max * by);
  return mj == kFar ? Scale(hi, lo, 0, max * by, by) : Scale(hi, lo, mj, 0.0f, by);
}

// The weight of a logit in units of 2^-44, rounded: 2^f - 1 (2^-28.3 of rounding at most) in 36 fraction bits, times 2^(j/16) from
// the table, shifted.
__device__ __forceinline__ uint64_t weight(const Scale& s, const uint64_t* pow, float l) {
  const float x = fmaf(l, s.by, -s.shift);
  if (!(fmaf(x, s.hi, -s.mh) > -46.0f)) return 0;
  const float q = fmaf(x, s.hi16, s.k_c), jf = q - kMagic;
  const int j = __float_as_int(q) - kMagicBits;
  const float g = fmaf(x, s.lo, fmaf(x, s.hi, fmaf(jf, -0.0625f, -s.mh)));
  const float r = g * fmaf(g, fmaf(g, fmaf(g, A4, A3), A2), A1);
  const uint64_t t = pow[j & 15];
  const uint64_t w = t + static_cast<uint64_t>((static_cast<int64_t>(t >> 12) * __float2int_rn(r * 68719476736.0f)) >> 24);
  const int down = -(j >> 4) - 1;          // w counts 2^-44 of 2^(n + 1)
  return down <= 0 ? w << -down : (w + (1ull << (down - 1))) >> down;
}

// Adds to a word of shared memory.
__device__ __forceinline__ void add_shared(uint32_t at, uint32_t x) { asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(at), "r"(x) : "memory"); }

// Sums the weights of a lane's values, in units of 2^-44.  weight()'s arithmetic, with the table's rest added to 2^f - 1: a
// weight is a + a r, a in fp32, r as good as there; h the sum's rounding, l what that lost.  The sum of h begins at 96, so that
// what its roundings (2^-17) lose is had by two subtractions; the lost parts' sum carries errors of about 2^-38 a lane.
struct Sums {
  float big = 96.0f, small = 0.0f;
  __device__ __forceinline__ void add(float x, const Scale& s, const float2* pow) {
    const float q = fmaf(x, s.hi16, s.k_c);
    const uint32_t b = __float_as_uint(q);
    const float g = fmaf(x, s.lo, fmaf(x, s.hi, fmaf(q, -0.0625f, kMagic * 0.0625f - s.mh)));
    const float2 t = pow[b & 15];
    const float r = fmaf(g, fmaf(g, fmaf(g, fmaf(g, A4, A3), A2), A1), t.y);
    // 2^n (1 + i/16), j = 16 n + i: j with its last four bits at the top of the fraction (the magic number's drop out)
    const float a = __uint_as_float(b * (1u << 19) + ((127u << 23) - (static_cast<uint32_t>(kMagicBits) << 19))) * t.x;
    const float h = fmaf(a, r, a), l = fmaf(a, r, a - h);
    const float next = big + h;
    small += (h - (next - big)) + l;
    big = next;
  }
  // over the warp, in every lane: 16 weights of up to 1.03 a lane in units of 2^-17: 2^26 over the warp; the rest 2^30 a lane
  __device__ __forceinline__ uint64_t all() const {
    const uint32_t whole = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(__float2int_rn((big - 96.0f) * 131072.0f)));
    const int rest = __float2int_rn(small * 17592186044416.0f);
    const int high = __reduce_add_sync(0xffffffffu, rest >> 16);
    const uint32_t low = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(rest) & 0xffffu);
    const int64_t sum = (static_cast<int64_t>(whole) << 27) + (static_cast<int64_t>(high) << 16) + low;
    return sum > 0 ? static_cast<uint64_t>(sum) : 0;
  }
};
// stands for a value that is not summed: 2^-60 of max, in no bin (deep: 60 / hi)
__device__ __forceinline__ float none_of(float max, float deep) { return fmaxf(max - deep, -3.0e38f); }
// A value's weight over that of its bin's middle, in 2^-14: as a float's bits where that float counts 2^-149.
constexpr float kUnit = 0x1p-135f;         // 2^14 of them


// Sum of the weights of the values that a warp's lanes hold.
// BINS: also a histogram by value, bins counted down from gj / per; a value adds its weight over that of its bin's
// middle, linear in its place within the bin, in 2^-14.  NB words, and 32 for what lies past them.
template <bool BINS>
__device__ __forceinline__ uint64_t bulk(const float (&v)[PER], const Scale& s, const float2* pow, float none, float per, float slope, int gj, uint32_t hist) {
  const float b_c = kMagic + static_cast<float>(gj), past = kMagic + static_cast<float>(NB + (threadIdx.x & 31));   // (a word per lane: no branch, no conflicts)
  hist -= 4u * static_cast<uint32_t>(kMagicBits);
  Sums sums;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const float x = fmaxf(v[e], none);
    if constexpr (BINS) {
      const float q = fmaf(x, -per, b_c), d = fmaf(x, -per, b_c - q);       // d: from the bin's middle, in bins
      add_shared(hist + 4u * __float_as_uint(q < kMagic + NB ? q : past), __float_as_uint(fmaf(d, slope, kUnit)));
    }
    sums.add(x, s, pow);
  }
  return sums.all();
}
// Of those above `cut` alone: they are moved together first (room: SEG words of the warp's), since in a nucleus' or a top-k's
// row they are few.
__device__ __forceinline__ uint64_t bulk_above(const float (&v)[PER], const Scale& s, const float2* pow, float none, float cut, float* room) {
  const int lane = threadIdx.x & 31;
  cut = fmaxf(cut, none);
  int n = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) n += v[e] > cut;
  int incl = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  const int all = __shfl_sync(0xffffffffu, incl, 31);
  if (all == 0) return 0;
  float* to = room + incl - n;
  __syncwarp();
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (v[e] > cut) *to++ = v[e];
  __syncwarp();
  Sums sums;
#pragma unroll 4
  for (int i = 0; i < all; i += 32) sums.add(i + lane < all ? room[i + lane] : none, s, pow);
  return sums.all();
}
// the largest logit below `v`
__device__ __forceinline__ float below(float v) { return v == 0.0f ? -1.4e-45f : Key<float>::value(Key<float>::of(v) - 1); }

__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// inclusive over the lanes
__device__ __forceinline__ uint64_t warp_scan_u64(uint64_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
// The smallest key in lo .. hi for which pred holds; it holds for hi and is monotone.  Warp-collective.
template <class F>
__device__ __forceinline__ uint32_t first_key(uint32_t lo, uint32_t hi, F&& pred) {
  const uint32_t lane = threadIdx.x & 31;
  while (lo < hi) {
    const uint32_t step = (hi - lo) / 32 + 1;
    const uint64_t at64 = static_cast<uint64_t>(lo) + static_cast<uint64_t>(lane + 1) * step - 1;
    const uint32_t at = at64 < hi ? static_cast<uint32_t>(at64) : hi;
    const int first = __ffs(__ballot_sync(0xffffffffu, pred(at))) - 1;
    const uint32_t top = __shfl_sync(0xffffffffu, at, first);
    lo += first * step;
    hi = top;
  }
  return lo;
}

// Sum over the block's threads up to this one, and over all.  Block-collective; `room` may be used again after a __syncthreads.
__device__ __forceinline__ uint64_t scan_block(uint64_t own, uint64_t* room, uint64_t* all = nullptr) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint64_t incl = warp_scan_u64(own);
  if (lane == 31) room[warp] = incl;
  __syncthreads();
  const uint64_t x = warp_scan_u64(lane < NW ? room[lane] : 0);
  if (all) *all = __shfl_sync(0xffffffffu, x, 31);
  const uint64_t before = __shfl_sync(0xffffffffu, x, warp > 0 ? warp - 1 : 0);
  return warp > 0 ? incl + before : incl;
}

// ------------------------------------------------------------------ the passes over the logits
// This lane's ids: PER of its warp's 512, V::N next to each other, 32 V::N from piece to piece.  NaN may come as it is: maxima
// leave it out, and no comparison holds for it.
template <class T>
__device__ __forceinline__ void load_chunk(const Logits<T>& l, int base, float (&v)[PER]) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31;
  uint4 q[PER / N];
  if (l.vec && base + SEG <= l.vocab && static_cast<uint32_t>(l.mask_id - base) >= SEG) {   // a whole segment, nothing masked in it
    const uint4* p = reinterpret_cast<const uint4*>(l.p + base) + lane;
#pragma unroll
    for (int i = 0; i < PER / N; ++i) q[i] = __ldg(p + i * 32);
#pragma unroll
    for (int i = 0; i < PER / N; ++i) {
      float x[N];
      Vec<T>::get(q[i], x);
#pragma unroll
      for (int e = 0; e < N; ++e) v[i * N + e] = x[e];
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < PER / N; ++i) {
      float x[N];
      l.template get<false>(l.load(base + (i * 32 + lane) * N), base + (i * 32 + lane) * N, x);
#pragma unroll
      for (int k = 0; k < PER / N; ++k)
        if (k == i)
#pragma unroll
          for (int e = 0; e < N; ++e) v[k * N + e] = x[e];
    }
  }
}
__device__ __forceinline__ bool wants_mass(const Row& r) { return r.k == 0; }          // draws or cuts by the mass of everything
__device__ __forceinline__ bool wants_bins(const Row& r) { return r.k > 1 || (r.k == 0 && (r.p < 1.0f || r.mp > 0.0f)); }

// What a block of the first pass needs of its row's settings; made by its first warp.
struct ScanRow {
  float hi, lo, per, slope, deep;          // per: bins per logit; slope: see bulk()
  int sums;                                // 0: none, 1: the mass, 2: with bins
};
template <class T>
__global__ void __launch_bounds__(NT, 3) sample_scan_kernel(const SampleArgs a) {
  __shared__ uint32_t s_hist[NB + 32];
  __shared__ float2 s_pow[16];
  __shared__ float s_max[NW];
  __shared__ ScanRow s_row;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks;
  if (threadIdx.x < 16) s_pow[threadIdx.x] = kPowF[threadIdx.x];
  s_hist[threadIdx.x] = 0;
  pdl_enter();
  const Logits<T> l(a, row);
  float v[PER];
  load_chunk(l, chunk * CHUNK + warp * SEG, v);
  if (warp == 0) {
    const Row r = row_of(a, row);
    const float depth = depth_of(a, r);
    if (lane == 0) s_row = ScanRow{r.hi, r.lo, r.hi * ((NB - 2) / depth), kUnit * (-0.693147181f / (NB - 2)) * depth, 60.0f / r.hi, r.k == 1 ? 0 : wants_bins(r) ? 2 : 1};
  }
  const float ninf = __int_as_float(0xff800000);
  float top = ninf;
#pragma unroll
  for (int e = 0; e < PER; ++e) top = fmaxf(top, v[e]);
  top = warp_max(top);
  if (lane == 0) s_max[warp] = top;
  __syncthreads();
  top = warp_max(s_max[lane & (NW - 1)]);
  const ScanRow r = s_row;
  ChunkInfo info{top, 0, 0, 0};
  uint64_t sum = 0;
  if (top > ninf) {
    const float g = top * r.per;
    info.mj = mj_of(r.hi, r.lo, top);
    info.gj = fabsf(g) < static_cast<float>(kFar) ? __float2int_ru(g) : kFar;   // (up: no value rounds to a bin before the first)
    info.far = info.mj == kFar || info.gj == kFar || !(r.hi > 1e-30f);
    if (!info.far && r.sums > 0) {
      const Scale s(r.hi, r.lo, info.mj, 0.0f);
      const float none = none_of(top, r.deep);
      sum = r.sums == 2 ? bulk<true>(v, s, s_pow, none, r.per, r.slope, info.gj, smem_u32(s_hist)) : bulk<false>(v, s, s_pow, none, 1.0f, 0.0f, 0, 0);
    }
  }
  if (lane == 0) a.seg[(static_cast<int64_t>(row) * a.chunks + chunk) * NW + warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.info[static_cast<int64_t>(row) * a.chunks + chunk] = info;
    if (chunk == 0) a.plan[row].listed = 0, a.plan[row].mass = 0, a.plan[row].count = 0, a.plan[row].done = 0;
  }
  if (r.sums == 2) a.hist[(static_cast<int64_t>(row) * a.chunks + chunk) * NB + threadIdx.x] = s_hist[threadIdx.x];
}

// a number of units of 2^(from / 16) in units of 2^(to / 16), from <= to
__device__ __forceinline__ uint64_t rescale(uint64_t sum, int from, int to) {
  const int d = from - to, n = d >> 4;                        // 2^n 2^(j/16), n <= 0
  const uint64_t t = kPow[d & 15];                            // 2^-43
  // sum * t: 128 bits, down by 43 - n
  const uint64_t hi = __umul64hi(sum, t), lo = sum * t;
  const int down = 43 - n;
  if (down >= 128) return 0;
  if (down >= 64) return hi >> (down - 64);
  return (hi << (64 - down)) | (lo >> down);
}

// The least key whose weight is at least min-p of the maximum's.  Warp-collective.
template <class T>
__device__ __forceinline__ uint32_t low_key(const Row& r, const Scale& s, const uint64_t* pow, float max) {
  const uint32_t top = Key<T>::of(max), bottom = Key<T>::of(__int_as_float(0xff800000)) + 1;
  if (!(r.mp > 0.0f)) return bottom;
  if (!(max < __int_as_float(0x7f800000))) return top;
  if (r.mp >= 1.0f) return r.hi > 0.0f ? top : bottom;        // (T infinite: every id weighs as much as the first)
  const uint64_t least = ::max(times<true>(r.mp, weight(s, pow, max)), static_cast<uint64_t>(1));
  auto enough = [&](uint32_t key) { return weight(s, pow, Key<T>::value(key)) >= least; };
  // (near max + T ln(min-p), if it is there)
  const uint32_t near = Key<T>::of(max + __log2f(r.mp) / r.hi), from = ::max(bottom, near - ::min(near, 400u)), to = ::min(top, near + 400u);
  if (from < to && enough(to) && (from == bottom || !enough(from - 1))) return first_key(from, to, enough);
  return first_key(bottom, top, enough);
}

struct Planner {
  uint64_t room[NW], front, pow[16];
  float max[NW], part;
  int bin, deep, three;
  ChunkInfo info[(kSampleMaxVocab + CHUNK - 1) / CHUNK];
};
// A row's plan, in every thread; `writes`: this block leaves the masses of kAll.  Block-collective.
template <class T>
__device__ __forceinline__ RowPlan plan_row(const SampleArgs& a, int row, const Row& r, Planner& sh, bool writes) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) sh.bin = NB, sh.deep = 0, sh.three = 0;
  if (threadIdx.x < 16) sh.pow[threadIdx.x] = kPow[threadIdx.x];
  const ChunkInfo* info = a.info + static_cast<int64_t>(row) * a.chunks;
  const uint64_t* seg = a.seg + static_cast<int64_t>(row) * a.chunks * NW;
  const float ninf = __int_as_float(0xff800000);
  const ChunkInfo mine = threadIdx.x < a.chunks ? info[threadIdx.x] : ChunkInfo{ninf, 0, 0, 0};   // (a row has fewer chunks than threads)
  const uint64_t seg0 = static_cast<int>(threadIdx.x) < a.chunks * NW ? seg[threadIdx.x] : 0;   // (asked for with the others)
  if (threadIdx.x < a.chunks) sh.info[threadIdx.x] = mine;
  float top = warp_max(mine.max);
  if (lane == 0) sh.max[warp] = top;
  __syncthreads();
  top = warp_max(sh.max[lane & (NW - 1)]) + 0.0f;             // (-0 as 0, which its ids' keys are of)
  RowPlan plan{top, top, top, r.hi, r.lo, none_of(top, 60.0f / r.hi), kEmpty, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  // (a chunk without masses counts if it lies within 2^-64 of the maximum, or that is not to be told: infinities)
  const bool far = __syncthreads_or(mine.far && !((top - mine.max) * r.hi >= 64.0f)) != 0;
  if (top > ninf && (r.k == 1 || top == -ninf)) {
    plan.mode = kListed;                                      // the ids of the maximum
    plan.mj = far ? kFar : mj_of(r.hi, r.lo, top);
  } else if (top > ninf && far) {
    plan.mode = kWhole;
    plan.mj = kFar;
  } else if (top > ninf) {
    const int mj = mj_of(r.hi, r.lo, top);
    const float per = r.hi * ((NB - 2) / depth_of(a, r));
    const int gj = __float2int_ru(top * per);
    plan.mj = mj;
    // every mass in the units of the row's maximum
    auto mass_of = [&](int i) {
      const ChunkInfo c = sh.info[i / NW];
      return c.max > ninf && !c.far ? rescale(i < NT ? seg0 : seg[i], c.mj, mj) : 0;
    };
    uint64_t mass = 0;
    if (wants_mass(r)) {
      uint64_t own = 0;
      for (int i = threadIdx.x; i < a.chunks * NW; i += NT) {
        own += mass_of(i);
      }
      scan_block(own, sh.room, &mass);
      __syncthreads();
    }
    plan.low = low_key<T>(r, Scale(r.hi, r.lo, mj, 0.0f), sh.pow, top);
    plan.mode = kAll;
    plan.lo = ninf, plan.hi = -ninf;
    if (wants_bins(r)) {
      // a bin per thread: its number of ids, about, and its mass in 2^-32
      uint64_t n = 0;
#pragma unroll 4
      for (int c = 0; c < a.chunks; ++c) {
        const ChunkInfo x = sh.info[c];
        const int bin = static_cast<int>(threadIdx.x) - (gj - x.gj);
        if (x.max > ninf && !x.far && bin >= 0 && bin < NB) n += a.hist[(static_cast<int64_t>(row) * a.chunks + c) * NB + bin];
      }
      auto edge = [&](float bin) { return (static_cast<float>(gj) - bin) / per; };
      const uint64_t count = (n + 8192) >> 14, in_front = scan_block(count, sh.room);
      __syncthreads();
      int b = NB;
      // the place in its bin, too: the guess of a mass is good to some 10^-4
      auto cross = [&](uint64_t own, uint64_t incl, uint64_t target) {
        if (incl >= target && incl - own < target) {
          sh.bin = threadIdx.x;
          sh.part = static_cast<float>(target - (incl - own)) / static_cast<float>(own);
        }
      };
      if (r.k > 1) {
        cross(count, in_front, r.k);
      } else if (r.p < 1.0f) {
        const float mid = ex2_approx(fmaf(edge(static_cast<float>(threadIdx.x)), r.hi, -0.0625f * static_cast<float>(mj))) * 262144.0f;
        uint64_t guess = static_cast<uint64_t>(static_cast<float>(n) * mid);
        if (r.mp <= 0.0f) {
          plan.target = target_of(r.p, mass);
        } else {                           // of what min-p leaves: its part of its last bin
          const float last = static_cast<float>(gj) - Key<T>::value(plan.low) * per + 0.5f - static_cast<float>(threadIdx.x);
          guess = last >= 1.0f ? guess : last > 0.0f ? static_cast<uint64_t>(static_cast<float>(guess) * last) : 0;
        }
        uint64_t all;
        const uint64_t incl = scan_block(guess, sh.room, &all);
        const uint64_t target = r.mp <= 0.0f ? plan.target >> 12 : target_of(r.p, all);
        cross(guess, incl, target);
        // What is left over of a bin may be no more than the guess is off by: the cut is then in the next bin that has anything.
        // (5 of 6144 peaked rows of 128000, p 0.8 to 0.95, were taken whole without this, 0.3 ms each: calls of 512 rows took
        // 228 us or, with such a row, 315 to 405.)
        const uint64_t late = min(target + (target >> 10) + 1, all);
        if (incl >= late && incl - guess < late) sh.deep = threadIdx.x;
      }
      float lo = ninf;
      if (r.mp > 0.0f) lo = Key<T>::value(plan.low);
      __syncthreads();
      b = sh.bin;
      plan.mode = kListed;
      // ids from a value on, about
      auto ids_from = [&](float value) {
        const int low = min(NB - 1, max(0, static_cast<int>(static_cast<float>(gj) - value * per) + 1));
        __syncthreads();
        if (threadIdx.x == low) sh.front = in_front;
        __syncthreads();
        return sh.front;
      };
      const bool few_mp = r.mp > 0.0f && ids_from(lo) < CAP * 3 / 4;
      if (few_mp || (r.k == 0 && r.p >= 1.0f)) {
        // min-p alone cuts, or leaves a list
        if (!few_mp) {                     // everything from lo on lies above an empty list
          plan.mode = kWindow;
          plan.hi = below(lo);
          lo = -ninf;
        } else {
          plan.hi = -ninf;
        }
      } else if (b >= NB - 2) {
        if (r.k == 0) plan.mode = kWhole;
        lo = fmaxf(lo, edge(NB - 0.5f));   // (k: nothing below counts)
        plan.hi = -ninf;
        if (ids_from(lo) >= CAP * 3 / 4) plan.mode = kWhole;
      } else {
        // three bins; all from there on where those are few (or a second cut follows); else, of crowded bins, as many as the
        // list takes around the place of the cut
        const float edge_lo = fmaxf(lo, edge((sh.deep < NB - 2 ? max(b, sh.deep) : b) + 1.5f));
        plan.more = edge_lo > lo;
        const bool again = r.k > 0 && (r.p < 1.0f || r.mp > 0.0f);
        if (ids_from(edge_lo) < (again ? CAP * 3 / 4 : LIST * 4)) {
          if (r.k == 0 && r.mp > 0.0f) plan.mode = kWindow;   // (the mass is not the list's)
          lo = edge_lo;
          plan.hi = -ninf;
        } else if (again) {
          plan.mode = kWhole;
        } else {
          if (threadIdx.x == max(0, b - 1) || threadIdx.x == b || threadIdx.x == b + 1) atomicAdd(&sh.three, static_cast<int>(min(count, static_cast<uint64_t>(1 << 24))));
          __syncthreads();
          const float most = CAP * 0.6f, three = static_cast<float>(sh.three);
          const float half = three <= most ? 1.5f : fmaxf(0.05f, 1.5f * most / three), mid = three <= most ? b : b - 0.5f + sh.part;
          plan.mode = kWindow;
          lo = fmaxf(lo, edge(mid + half));
          plan.hi = edge(mid - half);
        }
      }
      plan.lo = lo;
      plan.left = plan.mode == kWindow && r.k == 0 && r.mp > 0.0f && r.p < 1.0f;
    }
    if (plan.mode == kAll && writes) {
      uint64_t* kept = a.kept + static_cast<int64_t>(row) * a.chunks * NW;
      for (int i = threadIdx.x; i < a.chunks * NW; i += NT) kept[i] = mass_of(i);
    }
  }
  return plan;
}
template <class T>
__global__ void __launch_bounds__(NT) sample_plan_kernel(const SampleArgs a) {
  __shared__ Planner sh;
  pdl_enter();
  const RowPlan plan = plan_row<T>(a, blockIdx.x, row_of(a, blockIdx.x), sh, true);
  if (threadIdx.x == 0) a.plan[blockIdx.x] = plan;
}

struct Collector {
  float2 pow[16];
  int n, at;
};
// A chunk's part, by plan `to`; c_max: the chunk's maximum; room: CHUNK words.  Block-collective.
template <class T>
__device__ __forceinline__ void collect_chunk(const SampleArgs& a, int row, int chunk, const RowPlan& to, float c_max, int k, Collector& sh, float* room) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float p_lo = to.lo, p_hi = to.hi;
  uint64_t* seg = a.kept + (static_cast<int64_t>(row) * a.chunks + chunk) * NW + warp;
  const bool above = to.mode == kWindow;
  // (a chunk with nothing to list or to add; what min-p leaves may lie lower)
  const float low = Key<T>::value(to.low), least = to.left ? low : above ? fminf(p_lo, p_hi) : p_lo;
  if (c_max < least) {
    if (above && lane == 0) *seg = 0;
    return;
  }
  const Logits<T> l(a, row);
  const int base = chunk * CHUNK + warp * SEG;
  float v[PER];
  load_chunk(l, base, v);
  uint32_t in = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) in |= v[e] >= p_lo && v[e] <= p_hi ? 1u << e : 0u;
  __syncthreads();
  const int mine = __popc(in);
  int at = 0;
  if (__any_sync(0xffffffffu, mine > 0)) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    int first = 0;
    if (lane == 31) first = atomicAdd(&sh.n, incl);
    at = __shfl_sync(0xffffffffu, first, 31) + incl - mine;
  }
  __syncthreads();
  if (threadIdx.x == 0 && sh.n > 0) sh.at = atomicAdd(&a.plan[row].listed, sh.n);   // (on its way while the sums are made)
  if (above) {
    const Scale s(to.c_hi, to.c_lo, to.mj, 0.0f);
    // (a loop, so that the sums' code is there once)
#pragma unroll 1
    for (int turn = 0; turn < 1 + to.left; ++turn) {
      const uint64_t sum = bulk_above(v, s, sh.pow, to.none, turn ? below(low) : p_hi, room + warp * SEG);
      if (lane == 0 && turn == 0) *seg = sum;
      if (lane == 0 && turn == 1 && sum) atomicAdd(&a.plan[row].mass, static_cast<unsigned long long>(sum));
    }
    if (k > 0) {
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < PER; ++e) n += v[e] > p_hi;
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0 && n) atomicAdd(&a.plan[row].count, static_cast<unsigned long long>(n));
    }
  }
  __syncthreads();
  if (mine > 0) {
    uint2* list = a.list + static_cast<int64_t>(row) * CAP;
    at += sh.at;
    constexpr int N = Vec<T>::N;
    for (; in; in &= in - 1) {             // (few: read once more)
      const int e = __ffs(in) - 1, id = base + ((e / N) * 32 + lane) * N + e % N;
      if (at < CAP) list[at] = make_uint2(Key<T>::of(l.one(id)), id);
      ++at;
    }
  }
}
template <class T>
__global__ void __launch_bounds__(NT, 3) sample_collect_kernel(const SampleArgs a) {
  __shared__ Collector sh;
  __shared__ float s_room[CHUNK];
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks;
  if (threadIdx.x < 16) sh.pow[threadIdx.x] = kPowF[threadIdx.x];
  if (threadIdx.x == 0) sh.n = 0;
  pdl_enter();
  // (what is read of the plan, the chunk and the settings is asked for at once)
  const RowPlan& from = a.plan[row];
  RowPlan to;
  to.mode = from.mode, to.lo = from.lo, to.hi = from.hi, to.none = from.none, to.c_hi = from.c_hi, to.c_lo = from.c_lo;
  to.mj = from.mj, to.left = from.left, to.low = from.low;
  const float c_max = a.info[static_cast<int64_t>(row) * a.chunks + chunk].max;
  const int k = a.top_k ? a.top_k[row] : 0;
  if (to.mode == kListed || to.mode == kWindow) collect_chunk<T>(a, row, chunk, to, c_max, k, sh, s_room);
}

// ------------------------------------------------------------------ the cut and the draw
struct Cut {
  uint32_t key;
  int id;                                  // ids of that key up to this one are kept
};
constexpr int ALL = 0x7fffffff;

struct Finish {
  uint64_t pow[16];
  // mass by bin: whole rows 64 bits; lists, whose counts allow it, three words of 16 bits' sums (64-bit additions to shared
  // memory are loops)
  union {
    uint64_t mass[NB];
    uint32_t mass3[3][NB];
  };
  uint64_t seg[(SEGS + NT - 1) / NT * NT], room[NW];
  uint32_t seg2[2][(SEGS + NT - 1) / NT * NT];                // of lists: 22 bits, and the others
  uint64_t all_w[LIST];
  uint32_t count[NB];
  uint32_t key[CAP], id[CAP];
  uint32_t few_key[LIST], few_id[LIST];
  float max[NW];
  int n, few;
  // what one thread decides
  uint64_t d_above, d_left, d_w, d_best;
  uint32_t d_bin, d_count, d_key, d_id;
};

template <class T>
struct Finisher {
  Finish& sh;
  Logits<T> l;
  Scale s;
  float max;
  bool whole;                              // the row itself, not its list

  __device__ __forceinline__ uint64_t w(float v) const {
    return max == __int_as_float(0x7f800000) ? (v == max ? ONE : 0) : weight(s, sh.pow, v);
  }
  __device__ __forceinline__ static bool kept(const Cut& c, uint32_t key, int id) { return key > c.key || (key == c.key && id <= c.id); }
  // f(key, id) of this thread's candidates
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if (!whole) {
      for (int i = threadIdx.x; i < sh.n; i += NT) f(sh.key[i], static_cast<int>(sh.id[i]));
      return;
    }
    constexpr int N = Vec<T>::N;
    for (int id = threadIdx.x * N; id < l.vocab; id += NT * N) {
      float v[N];
      l.get(l.load(id), id, v);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (v[e] > __int_as_float(0xff800000)) f(Key<T>::of(v[e]), id + e);
    }
  }
  __device__ __forceinline__ uint64_t sum(uint64_t own) const {
    uint64_t all;
    scan_block(own, sh.room, &all);
    __syncthreads();
    return all;
  }

  // The cut that keeps, of the candidates that `from` keeps, the first ones of the order: `target` of them (BY_MASS: as many
  // as have less than `target` of mass in front of them; `above`: mass of what is kept beside the candidates).  Keys outside
  // lo .. hi are not looked at.  False: the cut is not there.
  template <bool BY_MASS>
  __device__ bool narrow(const Cut& from, uint32_t lo, uint32_t hi, uint64_t above, uint64_t target, Cut* cut) {
    uint32_t inside = whole ? 0xffffffffu : sh.n;   // candidates in the window, at most
    if (above >= target) return false;
    bool by_value = hi == Key<T>::of(max); // first by value, in steps of equal ratios of weights; then by key
    float per = 0.0f;
    int only = -1;                         // the bin by value that the few candidates are in
    auto value_bin = [&](uint32_t key) { return min(NB - 1, static_cast<int>((max - Key<T>::value(key)) * per)); };
    while (lo < hi && inside > LIST) {
      sh.count[threadIdx.x] = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) sh.mass3[i][threadIdx.x] = 0;
      if (threadIdx.x == 0) sh.d_count = 0;
      __syncthreads();
      const float range = max - Key<T>::value(lo);
      by_value = by_value && range < 3e38f;
      per = by_value ? (NB - 1) / range : 0.0f;
      int shift = 0;
      while (((hi - lo) >> shift) >= NB) ++shift;
      each([&](uint32_t key, int id) {
        if (key < lo || key > hi || !kept(from, key, id)) return;
        const int bin = by_value ? value_bin(key) : static_cast<int>((hi - key) >> shift);
        atomicAdd(&sh.count[bin], 1u);
        if (BY_MASS) {
          const uint64_t x = w(Key<T>::value(key));
          if (whole) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[bin]), static_cast<unsigned long long>(x));
          } else {
            atomicAdd(&sh.mass3[0][bin], static_cast<uint32_t>(x) & 0xffffu);
            atomicAdd(&sh.mass3[1][bin], static_cast<uint32_t>(x >> 16) & 0xffffu);
            atomicAdd(&sh.mass3[2][bin], static_cast<uint32_t>(x >> 32));
          }
        }
      });
      __syncthreads();
      uint64_t own = sh.count[threadIdx.x];
      if (BY_MASS)
        own = whole ? sh.mass[threadIdx.x]
                    : sh.mass3[0][threadIdx.x] + (static_cast<uint64_t>(sh.mass3[1][threadIdx.x]) << 16) + (static_cast<uint64_t>(sh.mass3[2][threadIdx.x]) << 32);
      const uint64_t incl = scan_block(own, sh.room);
      if (above + incl >= target && above + incl - own < target) {
        sh.d_bin = threadIdx.x;
        sh.d_count = sh.count[threadIdx.x];
        sh.d_above = above + incl - own;
      }
      __syncthreads();
      const uint32_t bin = sh.d_bin;
      inside = sh.d_count;
      if (inside == 0) return false;
      above = sh.d_above;
      if (by_value) {
        const int b = static_cast<int>(bin);
        if (inside <= LIST) {
          only = b;
          break;
        }
        const uint32_t lo2 = first_key(lo, hi, [&](uint32_t k) { return value_bin(k) <= b; });
        if (b > 0) hi = first_key(lo2, hi, [&](uint32_t k) { return value_bin(k) <= b - 1; }) - 1;
        lo = lo2;
        by_value = false;
      } else {
        const uint32_t top = hi - (bin << shift);
        lo = ::max(lo, top - min(top, (1u << shift) - 1));
        hi = top;
      }
      __syncthreads();                     // (d_bin and the histogram are written again)
    }
    if (lo >= hi) {
      // one key: of its ids the first ones, in the order of ids
      uint64_t need = target - above;
      if (BY_MASS) {
        const uint64_t one = w(Key<T>::value(lo));
        if (one == 0) return false;
        need = (need + one - 1) / one;
      }
      // by id as above by key
      uint32_t first = 0, last = static_cast<uint32_t>(l.vocab - 1), front = 0;
      while (first < last) {
        sh.count[threadIdx.x] = 0;
        if (threadIdx.x == 0) sh.d_count = 0;
        __syncthreads();
        int shift = 0;
        while (((last - first) >> shift) >= NB) ++shift;
        each([&](uint32_t key, int id) {
          if (key == lo && kept(from, key, id) && static_cast<uint32_t>(id) >= first && static_cast<uint32_t>(id) <= last)
            atomicAdd(&sh.count[(id - first) >> shift], 1u);
        });
        __syncthreads();
        const uint64_t own = sh.count[threadIdx.x], incl = scan_block(own, sh.room);
        if (front + incl >= need && front + incl - own < need) {
          sh.d_bin = threadIdx.x;
          sh.d_count = static_cast<uint32_t>(own);
          sh.d_above = front + incl - own;
        }
        __syncthreads();
        if (sh.d_count == 0) return false; // fewer than that
        front = static_cast<uint32_t>(sh.d_above);
        first += sh.d_bin << shift;
        last = min(last, first + (1u << shift) - 1);
        __syncthreads();
      }
      *cut = {lo, static_cast<int>(first)};
      return true;
    }
    // a few candidates: each of them finds what is in front of it
    if (threadIdx.x == 0) sh.few = 0, sh.d_id = 0xffffffffu;
    __syncthreads();
    each([&](uint32_t key, int id) {
      if (key < lo || key > hi || !kept(from, key, id) || (only >= 0 && value_bin(key) != only)) return;
      const int i = atomicAdd(&sh.few, 1);
      sh.few_key[i] = key;
      sh.few_id[i] = id;
      sh.all_w[i] = BY_MASS ? w(Key<T>::value(key)) : 1;
    });
    __syncthreads();
    // four threads a candidate
    const int i = threadIdx.x >> 2, n = sh.few;
    uint64_t front = 0;
    if (i < n) {
      const uint32_t key = sh.few_key[i], id = sh.few_id[i];
      for (int j = threadIdx.x & 3; j < n; j += 4)
        if (sh.few_key[j] > key || (sh.few_key[j] == key && sh.few_id[j] < id)) front += sh.all_w[j];
    }
    front += __shfl_xor_sync(0xffffffffu, front, 1);
    front += __shfl_xor_sync(0xffffffffu, front, 2);
    if (i < n && (threadIdx.x & 3) == 0 && above + front < target && above + front + sh.all_w[i] >= target) {
      sh.d_key = sh.few_key[i];
      sh.d_id = sh.few_id[i];
    }
    __syncthreads();
    *cut = {sh.d_key, static_cast<int>(sh.d_id)};
    const bool found = sh.d_id != 0xffffffffu;
    __syncthreads();
    return found;
  }
};

// The cut and the token.  DIRECT: rows of up to CAP ids, nothing ran ahead (and `plan` is made here); sh.n is 0 and sh.pow there.
// What other blocks left is read from L2.  Block-collective.
template <class T, bool DIRECT>
__device__ __forceinline__ void finish_row(const SampleArgs& a, int row, const Row& r, RowPlan plan, Finish& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float ninf = __int_as_float(0xff800000);
  const Logits<T> l(a, row);
  const float u = a.u[row];
  if constexpr (DIRECT) {
    float top = ninf;
    for (int id = threadIdx.x; id < a.vocab; id += NT) top = fmaxf(top, l.one(id));
    top = warp_max(top);
    if (lane == 0) sh.max[warp] = top;
    __syncthreads();
    top = warp_max(sh.max[lane & (NW - 1)]);
    for (int id = threadIdx.x; id < a.vocab; id += NT) {
      const float v = l.one(id);
      if (v > ninf && (r.k != 1 || v == top)) {
        const int i = atomicAdd(&sh.n, 1);
        sh.key[i] = Key<T>::of(v);
        sh.id[i] = id;
      }
    }
    plan = RowPlan{top, ninf, -ninf, r.hi, r.lo, ninf, top > ninf ? kListed : kEmpty, r.hi > 1e-30f ? mj_of(r.hi, r.lo, top) : kFar, 0, 0, 0, 0, 0, 0, 0, 0};
  } else {
    const uint2* list = a.list + static_cast<int64_t>(row) * CAP;
    if (plan.mode == kListed || plan.mode == kWindow) {
      uint2 x = __ldcg(list + threadIdx.x);                     // (asked for before its length is known)
      if (plan.listed > CAP) plan.mode = kWhole;
      else
        for (int i = threadIdx.x; i < plan.listed; i += NT) {
          if (i >= NT) x = __ldcg(list + i);
          sh.key[i] = x.x;
          sh.id[i] = x.y;
        }
    }
    if (threadIdx.x == 0) sh.n = plan.listed;
  }
  __syncthreads();
  if (plan.mode == kEmpty) {
    if (threadIdx.x == 0) {
      a.tok[row] = -1;
      if (a.prob) a.prob[row] = 0.0f;
    }
    return;
  }
  const bool far = plan.mj == kFar;
  Finisher<T> f{sh, l, far ? far_scale(r, plan.max) : Scale(r.hi, r.lo, plan.mj, 0.0f), plan.max, plan.mode == kWhole};
  const uint32_t khi = Key<T>::of(plan.max), kinf = Key<T>::of(ninf) + 1;
  if (r.k == 1) {                          // the lowest id of the maximum
    if (threadIdx.x == 0) sh.d_id = 0xffffffffu;
    __syncthreads();
    f.each([&](uint32_t key, int id) {
      if (key == khi) atomicMin(&sh.d_id, static_cast<uint32_t>(id));
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      a.tok[row] = static_cast<int>(sh.d_id);
      if (a.prob) a.prob[row] = 1.0f;
    }
    return;
  }
  // ---- the cut: min-p, top-k, top-p
  const uint64_t* seg = DIRECT ? nullptr : a.kept + static_cast<int64_t>(row) * a.chunks * NW;
  const int segs = (a.vocab + SEG - 1) / SEG;
  uint64_t above = 0;
  if (!DIRECT && plan.mode == kWindow) {
    uint64_t own = 0;
    for (int i = threadIdx.x; i < segs; i += NT) own += __ldcg(seg + i);
    above = f.sum(own);
  }
  const Cut low{DIRECT || far || plan.mode == kWhole ? low_key<T>(r, f.s, sh.pow, plan.max) : ::max(plan.low, kinf), ALL};
  Cut cut = low;
  bool window = plan.mode == kWindow;
  if (plan.mode != kAll) {
    for (;;) {                             // the list; where that fails, the row
      bool ok = true;
      cut = low;
      Cut to{};
      uint32_t lo = window ? ::max(cut.key, Key<T>::of(plan.lo)) : cut.key;
      const uint32_t hi = window ? Key<T>::of(plan.hi) : khi;
      if (r.k > 0) {
        ok = f.template narrow<false>(cut, lo, hi, window ? plan.count : 0, r.k, &to);
        if (ok) cut = to;
        else ok = !window && (f.whole || !plan.more);           // (fewer than k candidates: all of them)
      }
      if (ok && r.p < 1.0f && !(window && r.k > 0)) {           // (a window is there for one cut)
        uint64_t target = plan.target;
        if (window) {
          if (r.mp > 0.0f) target = target_of(r.p, plan.mass);
        } else {
          if (DIRECT || f.whole || far || r.k > 0 || r.mp > 0.0f) {
            uint64_t own = 0;
            f.each([&](uint32_t key, int id) { own += f.kept(cut, key, id) ? f.w(Key<T>::value(key)) : 0; });
            const uint64_t mass = f.sum(own);
            target = target_of(r.p, mass);
          }
          lo = cut.key;
          if (r.hi > 1e-30f) lo = ::max(lo, Key<T>::of(plan.max - 46.0f / r.hi));
          lo = min(lo, khi);
        }
        ok = f.template narrow<true>(cut, lo, hi, window ? above : 0, target, &to);
        if (ok) cut = to;
        else ok = f.whole;
      }
      if (ok) break;
      f.whole = true;
      window = false;
    }
  }
  // ---- the draw: the masses of 512 ids each
  for (int i = threadIdx.x; i < static_cast<int>(sizeof(sh.seg) / 8); i += NT)
    sh.seg[i] = !DIRECT && (window || plan.mode == kAll) && i < segs ? __ldcg(seg + i) : 0, sh.seg2[0][i] = sh.seg2[1][i] = 0;
  __syncthreads();
  if (f.whole) {
    constexpr int N = Vec<T>::N;
    for (int i = warp; i < segs; i += NW) {
      uint64_t own = 0;
      for (int id = i * SEG + lane * N; id < (i + 1) * SEG; id += 32 * N) {
        float v[N];
        l.get(l.load(id), id, v);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (v[e] > ninf && f.kept(cut, Key<T>::of(v[e]), id + e)) own += f.w(v[e]);
      }
      own = warp_sum_u64(own);
      if (lane == 0) sh.seg[i] = own;
    }
  } else if (plan.mode != kAll) {
    f.each([&](uint32_t key, int id) {
      if (!f.kept(cut, key, id)) return;
      const uint64_t x = f.w(Key<T>::value(key));
      atomicAdd(&sh.seg2[0][id / SEG], static_cast<uint32_t>(x) & 0x3fffffu);
      atomicAdd(&sh.seg2[1][id / SEG], static_cast<uint32_t>(x >> 22));
    });
  }
  __syncthreads();
  constexpr int EACH = (SEGS + NT - 1) / NT;                  // a thread's segments
  uint64_t own = 0, mass;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int at = threadIdx.x * EACH + i;
    sh.seg[at] += sh.seg2[0][at] + (static_cast<uint64_t>(sh.seg2[1][at]) << 22);
    own += sh.seg[at];
  }
  const uint64_t incl = scan_block(own, sh.room, &mass);
  const uint64_t target = u >= 1.0f ? mass - 1 : min(mass - 1, times<false>(u > 0.0f ? u : 0.0f, mass));
  if (incl > target && incl - own <= target) {
    uint64_t left = target - (incl - own);
    int i = 0;
    while (i + 1 < EACH && left >= sh.seg[threadIdx.x * EACH + i]) left -= sh.seg[threadIdx.x * EACH + i++];
    sh.d_bin = threadIdx.x * EACH + i;
    sh.d_left = left;
  }
  if (threadIdx.x == 0) sh.d_best = 0, sh.d_w = 0;
  __syncthreads();
  // its ids, one a thread.  (Their weights may add up to a little less than the segment's mass.)
  static_assert(SEG == NT, "one id a thread");
  const int id = static_cast<int>(sh.d_bin) * SEG + threadIdx.x;
  const float v = l.one(id);
  const uint32_t key = Key<T>::of(v);
  const bool in = v > ninf && f.kept(cut, key, id);
  const uint64_t x = in ? f.w(v) : 0;
  uint64_t all;
  const uint64_t upto = scan_block(x, sh.room, &all);
  if (all == 0) {                          // ids that weigh next to nothing: the heaviest of them
    if (in) atomicMax(reinterpret_cast<unsigned long long*>(&sh.d_best), static_cast<unsigned long long>(key) << 32 | (0xffffffffu - id));
  } else {
    const uint64_t left = min(sh.d_left, all - 1);
    if (upto > left && upto - x <= left) {
      sh.d_best = 0xffffffffu - id;
      sh.d_w = x;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.tok[row] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(sh.d_best));
    if (a.prob) a.prob[row] = ratio(sh.d_w, mass);
  }
}
template <class T, bool DIRECT>
__global__ void __launch_bounds__(NT) sample_finish_kernel(const SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  Finish& sh = *reinterpret_cast<Finish*>(smem);
  if (threadIdx.x < 16) sh.pow[threadIdx.x] = kPow[threadIdx.x];
  if (threadIdx.x == 0) sh.n = 0;
  pdl_enter();
  finish_row<T, DIRECT>(a, blockIdx.x, row_of(a, blockIdx.x), DIRECT ? RowPlan{} : a.plan[blockIdx.x], sh);
}

// Few rows: plan, collect and finish in one launch.  Every block plans its row for itself; the one that is through last with its
// chunk finishes the row.  (No block waits for another.)
template <class T>
__global__ void __launch_bounds__(NT, 2) sample_rest_kernel(const SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  Finish& sh = *reinterpret_cast<Finish*>(smem);
  static_assert(sizeof(Planner) <= sizeof(Finish) && CHUNK * 4 <= sizeof(Finish), "the parts take turns");
  __shared__ Collector s_c;
  __shared__ int s_last;
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks;
  if (threadIdx.x < 16) s_c.pow[threadIdx.x] = kPowF[threadIdx.x];
  if (threadIdx.x == 0) s_c.n = 0;
  pdl_enter();
  const Row r = row_of(a, row);
  RowPlan plan = plan_row<T>(a, row, r, *reinterpret_cast<Planner*>(smem), chunk == 0);
  __syncthreads();
  if (plan.mode == kListed || plan.mode == kWindow) {
    const float c_max = a.info[static_cast<int64_t>(row) * a.chunks + chunk].max;
    collect_chunk<T>(a, row, chunk, plan, c_max, r.k, s_c, reinterpret_cast<float*>(smem));
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicAdd(&a.plan[row].done, 1) == a.chunks - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    plan.listed = __ldcg(&a.plan[row].listed);
    plan.mass = __ldcg(&a.plan[row].mass);
    plan.count = __ldcg(&a.plan[row].count);
  } else if (chunk != 0) {
    return;
  }
  if (threadIdx.x < 16) sh.pow[threadIdx.x] = kPow[threadIdx.x];
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  finish_row<T, false>(a, row, r, plan, sh);
}

template <class... KArgs, class... Args>
cudaError_t start(void (*kernel)(KArgs...), int64_t grid, size_t smem, cudaStream_t s, Args&&... args) {
  return launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(NT), smem, s, args...);
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }
int chunks_of(int vocab) { return vocab <= CAP ? 0 : (vocab + CHUNK - 1) / CHUNK; }
// The scratch memory's parts; returns its size.
size_t place(SampleArgs* a, int rows, int vocab, uint8_t* base) {
  const size_t chunks = chunks_of(vocab), n = static_cast<size_t>(rows);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up(bytes);
    return base + here;
  };
  a->info = reinterpret_cast<ChunkInfo*>(take(n * chunks * sizeof(ChunkInfo)));
  a->seg = reinterpret_cast<uint64_t*>(take(n * chunks * NW * sizeof(uint64_t)));
  a->kept = reinterpret_cast<uint64_t*>(take(n * chunks * NW * sizeof(uint64_t)));
  a->hist = reinterpret_cast<uint32_t*>(take(n * chunks * NB * sizeof(uint32_t)));
  a->plan = reinterpret_cast<RowPlan*>(take(n * sizeof(RowPlan)));
  a->list = reinterpret_cast<uint2*>(take(n * CAP * sizeof(uint2)));
  return at;
}

template <class T>
cudaError_t run(const SampleArgs& a, cudaStream_t s) {
  static PerDevice ready;
  int dev = 0;
  const int sms = current_sms(&dev);
  cudaError_t e = cudaSuccess;
  const int smem = static_cast<int>(sizeof(Finish));
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(sample_finish_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_rest_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_finish_kernel<T, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return e;
  if (a.chunks == 0) return start(sample_finish_kernel<T, true>, a.rows, smem, s, a);
  const int64_t blocks = static_cast<int64_t>(a.rows) * a.chunks;
  if ((e = start(sample_scan_kernel<T>, blocks, 0, s, a)) != cudaSuccess) return e;
  // a block an SM: two launches for four (3 us less of the host's time per call), and every block's own plan costs no more than
  // one per row.  4 rows of 32768 ids and 9 of 128000 18.3 -> 17.3 and 27 -> 26 us; at three blocks an SM 32.6 -> 33 and 34 -> 39.
  if (blocks <= sms) return start(sample_rest_kernel<T>, blocks, smem, s, a);
  if ((e = start(sample_plan_kernel<T>, a.rows, 0, s, a)) != cudaSuccess) return e;
  if ((e = start(sample_collect_kernel<T>, blocks, 0, s, a)) != cudaSuccess) return e;
  return start(sample_finish_kernel<T, false>, a.rows, smem, s, a);
}

}  // namespace

size_t sample_scratch(int rows, int vocab) {
  SampleArgs a;
  return chunks_of(vocab) ? place(&a, rows, vocab, nullptr) : 0;
}

const char* sample_rows(const SampleCall& c, cudaStream_t s) {
  SampleArgs a{};
  a.logits = c.logits, a.ld = c.ld, a.rows = c.rows, a.vocab = c.vocab, a.mask_id = c.mask_id, a.chunks = chunks_of(c.vocab);
  a.temperature = c.temperature, a.top_k = c.top_k, a.top_p = c.top_p, a.min_p = c.min_p, a.u = c.u, a.tok = c.tok, a.prob = c.prob;
  if (a.chunks) place(&a, c.rows, c.vocab, static_cast<uint8_t*>(c.scratch));
  const cudaError_t e = c.bf16 ? run<bf16>(a, s) : run<float>(a, s);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
