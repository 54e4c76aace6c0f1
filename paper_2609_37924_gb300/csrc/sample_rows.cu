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
// Weights are whole numbers of 2^-44, accurate to about 2^-35 (weight() says
// how), and all sums are 64-bit integers.  So a sum does not depend on its
// order, cuts and draws repeat, and they differ from those of exact
// arithmetic only where a border lies within some 2^-40 of the mass: with
// fp32 weights a row of 10^5 like tokens draws another one every few thousand
// rows.
//
// A cluster of 1 to 8 blocks holds the row in shared memory: the logits leave
// HBM once, whatever the settings ask for.  Block c has the c-th part of the
// ids, warp w of it the w-th segment of that part.  What the blocks know
// together goes through distributed shared memory; every block reads all
// parts and comes to the same decisions.
//
// Whole rows are summed by bulk(): the same weights in pairs of fp32 sums, a
// third of weight()'s instructions.  The nucleus takes two passes: one sums
// the row and counts it by value in 512 bins, which places the cut within
// three of them; one sums what lies above those and lists what lies in them.
// top-k begins with the lanes' maxima, the k-th largest of which is a lower
// bound.  Listed elements are narrowed down by histograms over the key until
// 128 elements or one key are left.  Where a list overflows or a guess was
// wrong, the same histograms go over the whole row.
#include <cstdint>

#include "common.cuh"
#include "requests.h"

namespace tadm {
namespace {

constexpr int NT = 512, NW = NT / 32, NB = NT, LIST = 128, MAXC = 8;
constexpr uint64_t ONE = 1ull << 44;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int vocab, mask_id, seg;                 // seg: ids of a warp
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* tok;
  float* prob;
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

// 16 bytes of logits: NaN and the masked id count as -inf, -0 as 0
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
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
  static __device__ __forceinline__ uint4 put(const float (&v)[8]) {   // (the values are bf16)
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[2 * i]) >> 16 | __float_as_uint(v[2 * i + 1]);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// ------------------------------------------------------------------ weights
struct Scale {
  float max, hi, lo;                       // the row's maximum; log2(e) / T in two terms
};
// 2^(j/32) in units of 2^-43, rounded
__constant__ const uint64_t kPow[32] = {
    0x80000000000ull, 0x82cd8698ac3ull, 0x85aac367cc5ull, 0x88980e8092eull,
    0x8b95c1e3ea9ull, 0x8ea4398b45dull, 0x91c3d373ab1ull, 0x94f4efa8fefull,
    0x9837f0518dcull, 0x9b8d39b9d55ull, 0x9ef5326091aull, 0xa27043030c5ull,
    0xa5fed6a9b15ull, 0xa9a15ab4ea8ull, 0xad583eea42aull, 0xb123f581d2bull,
    0xb504f333f9eull, 0xb8fbaf47630ull, 0xbd08a39f581ull, 0xc12c4cca667ull,
    0xc5672a11550ull, 0xc9b9bd866e3ull, 0xce248c151f8ull, 0xd2a81d91f13ull,
    0xd744fccad6aull, 0xdbfbb797dafull, 0xe0ccdeec2a9ull, 0xe5b906e77c8ull,
    0xeac0c6e7dd2ull, 0xefe4b99bdceull, 0xf5257d15248ull, 0xfa83b2db723ull};

// exp((l - max) / T) * ONE, rounded.  t = (l - max) log2(e) / T in two fp32 terms p + e (the difference and the product are
// taken with their errors); p = n + j/32 + f with |f| <= 1/64; 2^f - 1 = f ln 2 + ... with the first term in two pieces,
// which go into 36 fraction bits; times 2^e = 1 + e ln 2, and 2^(j/32) from a table; shifted by n.  Errors: 2^-36 of the
// fraction's two roundings, 2^-38 of the neglected e^2, half a unit of the last shift.
__device__ __forceinline__ uint64_t weight(const Scale& s, const uint64_t* pow, float l) {
  if (l == s.max) return ONE;
  const float d = l - s.max, bb = d - l;
  const float dl = (l - (d - bb)) - (s.max + bb);
  const float p = d * s.hi;
  if (!(p > -46.0f)) return 0;
  float e = fmaf(d, s.hi, -p);
  e = fmaf(d, s.lo, e);
  e = fmaf(dl, s.hi, e);
  const float q = fmaf(p, 32.0f, 12582912.0f);                // 1.5 * 2^23: the nearest integer in the low bits
  const int j = __float_as_int(q) - 0x4b400000;
  const float f = fmaf(q - 12582912.0f, -0.03125f, p);
  constexpr float L = 0.693147180559945f, LL = static_cast<float>(0.6931471805599453094 - static_cast<double>(0.693147180559945f));
  const float r = f * L;
  float rest = fmaf(f, L, -r);
  rest = fmaf(f, LL, rest);
  rest = fmaf(e * L, 1.0f + r, rest);
  const float c = fmaf(f, fmaf(f, 0.00961812911f, 0.0555041087f), 0.240226507f);   // ln2^4/24, ln2^3/6, ln2^2/2
  rest = fmaf(f * f, c, rest);
  const int64_t frac = static_cast<int64_t>(__float2int_rn(r * 68719476736.0f)) + __float2int_rn(rest * 68719476736.0f);
  const uint64_t t = pow[j & 31];
  // t (1 + frac 2^-36) with the low 12 bits of t left out of the second product
  const uint64_t w = t + static_cast<uint64_t>((static_cast<int64_t>(t >> 12) * frac) >> 24);
  const int down = -(j >> 5) - 1;                             // w counts 2^-44 of 2^(n + 1)
  return down <= 0 ? w << -down : (w + (1ull << (down - 1))) >> down;
}

// 2^f - 1 = f (A1 + f (A2 + f (A3 + f A4))) for |f| <= 1/32: ln2^n / n!, the last two eased to spread the error of the next
// term (Chebyshev)
constexpr float A1 = 0.693147182f, A2 = 0.240226507f, A3 = 0.0555057377f, A4 = 0.00961835496f;

// ------------------------------------------------------------------ the cluster's shared memory
__device__ __forceinline__ uint32_t remote_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t remote_u64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
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

constexpr int CAP = 2048;                  // elements that a block lists
struct Shared {
  uint64_t pow[32];
  uint64_t mass[2][NB];                    // histograms, two in turn
  uint32_t count[2][NB];
  uint64_t sums[2][NW];                    // per warp
  uint64_t above[NW];                      // per warp: of what lies above the list
  uint64_t scan[NW];
  float scan_f[NW];
  float2 top;                              // largest and smallest of the lanes' maxima in the block
  float2 wtop[NW];
  uint32_t list_n, few_n;
  uint16_t list[CAP];                      // places in the block's part
  uint32_t few_key[LIST], few_id[LIST];
  uint64_t all_w[LIST];
  uint32_t all_key[LIST], all_id[LIST];
  uint32_t found_id[2];                    // what pick() found
  uint64_t found_w[2];
  uint64_t part[NW];
  float2 pow16[16];                        // bulk(): 2^(j/16) 2^-(M - Mh) in two fp32 terms
  float c_hi, c_lo, low;                   // log2(e) / T; the row's least logit that min-p keeps, less the maximum
  double low64;
  float mh;
  // what one thread decides for its block
  uint32_t d_bin, d_count, d_key, d_id;
  uint64_t d_above;
};
static_assert((sizeof(Shared) + 15) / 16 * 16 + (kSampleMaxVocab + MAXC * NW * 128 - 1) / (MAXC * NW * 128) * 128 * NW * 4 <= 232448, "shared memory");

struct Cut {
  uint32_t key;
  int id;                                  // ids of that key up to this one are kept
};
constexpr int ALL = 0x7fffffff;
constexpr float kFlat = 1e-30f;            // log2(e) / T above which a finite logit can stand for one that weighs nothing (bulk)

__device__ __forceinline__ uint64_t pair(float x) { return f2_pack(x, x); }
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <class T, int CS>
struct Row {
  using V = Vec<T>;
  Shared& sh;
  const uint4* data;                       // this block's part
  int first, seg, rank;                    // id of the part's first element
  Scale s;
  int turn;                                // of the arrays that pick() uses in turn: a sync lies between two uses of one
  bool listed;                             // each() goes over the list

  __device__ __forceinline__ uint64_t w(float l) const { return weight(s, sh.pow, l); }
  __device__ __forceinline__ static bool kept(const Cut& c, uint32_t key, int id) { return key > c.key || (key == c.key && id <= c.id); }
  __device__ __forceinline__ void sync() const {
    if constexpr (CS > 1) cluster_sync();
    else __syncthreads();
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(reinterpret_cast<const T*>(data)[i]); }
  // f(logit, id) of this warp's elements (listed: of this thread's listed ones) whose logit is at least `least`
  template <class F>
  __device__ __forceinline__ void each(float least, F&& f) const {
    if (listed) {
      const int n = sh.list_n;
      for (int i = threadIdx.x; i < n; i += NT) {
        const int p = sh.list[i];
        const float v = at(p);
        if (v >= least) f(v, first + p);
      }
      return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint4* p = data + warp * (seg / V::N);
    for (int i = lane; i < seg / V::N; i += 32) {
      float v[V::N];
      V::get(p[i], v);
#pragma unroll
      for (int e = 0; e < V::N; ++e)
        if (v[e] >= least) f(v[e], first + warp * seg + i * V::N + e);
    }
  }

  // Sum of the weights of this warp's elements above `cut` (a logit, exclusive), in units of ONE^-1, in lane 0.  With
  // BINS also a histogram by value, in bins of width 1 / per below the maximum (none past the last bin): an element adds its
  // weight over that of its bin's middle, linear in its place within the bin, in 2^-14.
  //
  // t = c x - M (c = log2(e) / T, M = c max; x a logit, less the maximum where c max is large) without the rounding of a
  // difference: j = 16 t to the nearest whole number, f = c x - Mh - j / 16 by one fma, Mh the multiple of 1/16 next to M,
  // plus c's second term; 2^f - 1 by a polynomial of degree 4 (error 2^-36 for |f| <= 1/32, coefficients below); times the
  // table's 2^(j/16) 2^(Mh - M) in two terms.  The sum is split at 2^-17: multiples of that add without rounding (at most
  // 104 of them a lane), the rest carries errors of about 2^-37 a lane.
  template <bool BINS>
  __device__ uint64_t bulk(float cut, float per, uint32_t* hist) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool far = fabsf(s.max * s.hi) >= 92.0f;            // then logits that weigh anything are near the maximum
    const float shift = far ? s.max : 0.0f, mh = sh.mh;
    const float none = fmaxf(s.max - shift - 60.0f / s.hi, -3.0e38f);   // stands for elements that are not summed: 2^-60
    const uint64_t k_shift = pair(-shift), k_hi16 = pair(16.0f * s.hi), k_c = pair(12582912.0f - 16.0f * mh), k_back = pair(-12582912.0f);
    const uint64_t k_n16 = pair(-0.0625f), k_nmh = pair(-mh), k_hi = pair(s.hi), k_lo = pair(s.lo), k_minus = pair(-1.0f);
    const uint64_t k_up = pair(96.0f), k_down = pair(-96.0f);
    const uint64_t a1 = pair(A1), a2 = pair(A2), a3 = pair(A3), a4 = pair(A4);
    const uint64_t b_per = pair(-per), b_c = pair(fmaf(s.max, per, 12582912.0f)), b_slope = pair(-16384.0f * 0.693147181f * s.hi / per);
    const uint64_t b_one = pair(12582912.0f + 16384.0f);
    uint64_t big = 0, small = 0;
    cut = fmaxf(cut, fminf(s.max - 60.0f / s.hi, below(s.max)));
    auto two = [&](float v0, float v1) {
      const bool in0 = v0 > cut, in1 = v1 > cut;
      if constexpr (BINS) {
        const uint64_t v = f2_pack(v0, v1), q = f2_fma(v, b_per, b_c);
        const uint64_t d = f2_fma(v, b_per, f2_fma(q, k_minus, b_c));     // from the bin's middle, in bins
        float q0, q1, m0, m1;
        f2_unpack(q, q0, q1);
        f2_unpack(f2_fma(d, b_slope, b_one), m0, m1);
        const uint32_t i0 = __float_as_uint(q0) - 0x4b400000u, i1 = __float_as_uint(q1) - 0x4b400000u;
        if (in0 && i0 < NB - 1) atomicAdd(&hist[i0], __float_as_uint(m0) - 0x4b400000u);
        if (in1 && i1 < NB - 1) atomicAdd(&hist[i1], __float_as_uint(m1) - 0x4b400000u);
      }
      float x0, x1;
      f2_unpack(f2_add(f2_pack(v0, v1), k_shift), x0, x1);
      const uint64_t x = f2_pack(in0 ? x0 : none, in1 ? x1 : none);
      const uint64_t q = f2_fma(x, k_hi16, k_c), j = f2_add(q, k_back);
      const uint64_t g = f2_fma(x, k_lo, f2_fma(x, k_hi, f2_fma(j, k_n16, k_nmh)));
      const uint64_t r = f2_mul(g, f2_fma(g, f2_fma(g, f2_fma(g, a4, a3), a2), a1));
      float q0, q1;
      f2_unpack(q, q0, q1);
      const uint32_t b0 = __float_as_uint(q0), b1 = __float_as_uint(q1);
      const float2 t0 = sh.pow16[b0 & 15], t1 = sh.pow16[b1 & 15];
      // 2^n, n = floor(j / 16): the magic number's bits drop out of the shifted word
      constexpr uint32_t BIAS = (127u << 23) - (0x4b400000u >> 4 << 23);
      const uint64_t p2 = f2_pack(__uint_as_float((b0 >> 4 << 23) + BIAS), __uint_as_float((b1 >> 4 << 23) + BIAS));
      const uint64_t a = f2_mul(f2_pack(t0.x, t1.x), p2), al = f2_mul(f2_pack(t0.y, t1.y), p2);
      const uint64_t t = f2_fma(a, r, al), h = f2_add(a, t), l = f2_add(f2_fma(h, k_minus, a), t);
      const uint64_t up = f2_add(f2_add(h, k_up), k_down);
      big = f2_add(big, up);
      small = f2_add(small, f2_add(f2_fma(up, k_minus, h), l));
    };
    const uint4* p = data + warp * (seg / V::N);
#pragma unroll 2
    for (int i = lane; i < seg / V::N; i += 32) {
      float v[V::N];
      V::get(p[i], v);
#pragma unroll
      for (int e = 0; e < V::N; e += 2) two(v[e], v[e + 1]);
    }
    float h0, h1, l0, l1;
    f2_unpack(big, h0, h1);
    f2_unpack(small, l0, l1);
    const int64_t whole = static_cast<int64_t>(__float2int_rn(h0 * 131072.0f)) + __float2int_rn(h1 * 131072.0f);
    return warp_sum_u64(static_cast<uint64_t>((whole << 27) + __float2ll_rn((l0 + l1) * 17592186044416.0f)));
  }
  // the largest logit below `v`
  __device__ __forceinline__ static float below(float v) {
    return v == 0.0f ? -1.4e-45f : Key<float>::value(Key<float>::of(v) - 1);
  }
  // Per warp into sums[turn]: the weights of what `cut` keeps.
  __device__ void sums_kept(const Cut& cut) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (listed) {                                             // all of it is on the list
      if (threadIdx.x < NW) sh.sums[turn][threadIdx.x] = sh.above[threadIdx.x];
      __syncthreads();
      each(Key<T>::value(cut.key), [&](float l, int id) {
        if (kept(cut, Key<T>::of(l), id))
          atomicAdd(reinterpret_cast<unsigned long long*>(&sh.sums[turn][(id - first) / seg]), static_cast<unsigned long long>(w(l)));
      });
      return;
    }
    const float v = Key<T>::value(cut.key);
    uint64_t mine = s.hi > kFlat ? bulk<false>(cut.id == ALL ? below(v) : v, 0.0f, nullptr) : 0;
    if (cut.id != ALL) {
      uint64_t ties = 0;
      each(v, [&](float l, int id) { ties += l == v && id <= cut.id ? 1 : 0; });
      mine += warp_sum_u64(ties) * w(v);
    }
    if (__shfl_sync(0xffffffffu, mine, 0) < 2ull * seg) {     // nearly nothing: exactly what weight() gives, so that it can be drawn from
      mine = 0;
      each(v, [&](float l, int id) { mine += kept(cut, Key<T>::of(l), id) ? w(l) : 0; });
      mine = warp_sum_u64(mine);
    }
    if (lane == 0) sh.sums[turn][warp] = mine;
  }

  // From the warps' sums[turn]: their sum over the cluster; with `id`, also the first element in the order of ids with which
  // the sum of f exceeds target(whole sum), and its f.  (The warps' sums may differ from f's in the last bits.)
  template <class F, class G>
  __device__ uint64_t pick(float least, F&& f, G&& target, int* id, uint64_t* value) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    sync();
    // every warp: lane l has the sums of CS * NW / 32 consecutive warps
    constexpr int PER = CS * NW >= 32 ? CS * NW / 32 : 1, LANES = CS * NW / PER;
    uint64_t part[PER], own = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = lane * PER + i;
      part[i] = lane < LANES ? remote_u64(cluster_addr(&sh.sums[turn][at % NW], at / NW)) : 0;
      own += part[i];
    }
    const uint64_t incl = warp_scan_u64(own), total = __shfl_sync(0xffffffffu, incl, 31);
    if (!id) {
      turn ^= 1;
      return total;
    }
    const uint64_t t = target(total);
    const unsigned past = __ballot_sync(0xffffffffu, incl > t);
    const int src = past ? __ffs(past) - 1 : 31;
    uint64_t left = t - (incl - own);
    int at = lane * PER;
#pragma unroll
    for (int i = 0; i + 1 < PER; ++i)
      if (left >= part[i] && at == lane * PER + i) {
        left -= part[i];
        ++at;
      }
    left = __shfl_sync(0xffffffffu, left, src);
    at = __shfl_sync(0xffffffffu, at, src);
    // the block that has it: its warps take the chunks of that segment
    if (at / NW == rank) {
      const int chunks = seg / (32 * V::N), per = (chunks + NW - 1) / NW, c0 = warp * per, c1 = min(chunks, c0 + per);
      const uint4* p = data + (at % NW) * (seg / V::N);
      const int base = first + (at % NW) * seg;
      auto lane_sum = [&](int c) {
        float v[V::N];
        V::get(p[c * 32 + lane], v);
        uint64_t a = 0;
#pragma unroll
        for (int e = 0; e < V::N; ++e)
          if (v[e] >= least) a += f(v[e], base + (c * 32 + lane) * V::N + e);
        return a;
      };
      uint64_t a = 0;
      for (int c = c0; c < c1; ++c) a += lane_sum(c);
      a = warp_sum_u64(a);
      if (lane == 0) sh.part[warp] = a;
      __syncthreads();
      const uint64_t x = lane < NW ? sh.part[lane] : 0, inc = warp_scan_u64(x), all = __shfl_sync(0xffffffffu, inc, 31);
      left = min(left, all - 1);
      const unsigned over = __ballot_sync(0xffffffffu, inc > left);
      if (!over && threadIdx.x == 0) sh.found_id[turn] = 0xffffffffu, sh.found_w[turn] = 0;
      const int who = __ffs(over) - 1;
      if (who == warp) {
        left -= __shfl_sync(0xffffffffu, inc - x, who);
        for (int c = c0; c < c1; ++c) {
          const uint64_t mine = lane_sum(c), in = warp_scan_u64(mine);
          const unsigned hit = __ballot_sync(0xffffffffu, in > left);
          if (hit) {
            if (lane == __ffs(hit) - 1) {
              uint64_t rem = left - (in - mine);
              float v[V::N];
              V::get(p[c * 32 + lane], v);
              bool open = true;
#pragma unroll
              for (int e = 0; e < V::N; ++e) {
                const int i = base + (c * 32 + lane) * V::N + e;
                const uint64_t x2 = open && v[e] >= least ? f(v[e], i) : 0;
                if (open && x2 > rem) {
                  sh.found_id[turn] = static_cast<uint32_t>(i);
                  sh.found_w[turn] = x2;
                  open = false;
                }
                rem -= x2;
              }
            }
            break;
          }
          left -= __shfl_sync(0xffffffffu, in, 31);
        }
      }
    }
    sync();
    *id = static_cast<int>(remote_u32(cluster_addr(&sh.found_id[turn], at / NW)));
    if (value) *value = remote_u64(cluster_addr(&sh.found_w[turn], at / NW));
    turn ^= 1;
    return total;
  }
  // Sums of f, which is 0 or 1, into the warps' sums.
  template <class F>
  __device__ void sums_of(float least, F&& f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool l = listed;
    listed = false;
    uint64_t mine = 0;
    each(least, [&](float v, int i) { mine += f(v, i); });
    listed = l;
    mine = warp_sum_u64(mine);
    if (lane == 0) sh.sums[turn][warp] = mine;
  }

  // Lists the elements from `least` to `most` that `from` keeps.  False (in every block): one of the lists is too short for them.
  __device__ bool make_list(const Cut& from, float least, float most) {
    listed = false;
    if (threadIdx.x == 0) sh.list_n = 0;
    if (threadIdx.x < NW) sh.above[threadIdx.x] = 0;
    __syncthreads();
    each(least, [&](float l, int id) {
      if (l > most || !kept(from, Key<T>::of(l), id)) return;
      const uint32_t i = atomicAdd(&sh.list_n, 1u);
      if (i < CAP) sh.list[i] = static_cast<uint16_t>(id - first);
    });
    sync();
    uint32_t n = 0;
#pragma unroll
    for (int r = 0; r < CS; ++r) n = max(n, remote_u32(cluster_addr(&sh.list_n, r)));
    listed = n <= CAP;
    return listed;
  }

  // Sum over the threads up to this one and over all (block-collective); the arrays may be used again after a __syncthreads.
  __device__ __forceinline__ uint64_t scan_block(uint64_t own) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t incl = warp_scan_u64(own);
    if (lane == 31) sh.scan[warp] = incl;
    __syncthreads();
    const uint64_t x = warp_scan_u64(lane < NW ? sh.scan[lane] : 0);
    return warp > 0 ? incl + __shfl_sync(0xffffffffu, x, warp - 1) : incl;
  }

  // The cut that keeps, of the elements that `from` keeps, the first ones of the order: `target` of them (BY_MASS: as many
  // as have less than `target` of mass in front of them).  At least one element is kept by `from`, target >= 1 and at most
  // all of them (their mass).  Keys outside lo .. hi need not be looked at; `above`: what lies above hi counts.  False: the cut is not
  // between lo and hi.
  template <bool BY_MASS>
  __device__ bool narrow(const Cut& from, uint32_t lo, uint32_t hi, uint64_t above, uint64_t target, Cut* cut) {
    const uint64_t start = above;
    uint32_t inside = 0xffffffffu;         // elements in the window
    bool by_value = hi == Key<T>::of(s.max);   // first by value, in steps of equal ratios of weights; then by key
    for (int level = 0; lo < hi && inside > LIST; ++level) {
      const int buf = level & 1;
      sh.count[buf][threadIdx.x] = 0;
      sh.mass[buf][threadIdx.x] = 0;
      if (threadIdx.x == 0) sh.d_count = 0;
      __syncthreads();
      const float range = s.max - Key<T>::value(lo);
      by_value = by_value && range < 3e38f;
      const float per = by_value ? (NB - 1) / range : 0.0f;
      int shift = 0;
      while (((hi - lo) >> shift) >= NB) ++shift;
      auto value_bin = [&](float l) { return min(NB - 1, static_cast<int>((s.max - l) * per)); };
      const float least = Key<T>::value(lo), most = Key<T>::value(hi);
      each(least, [&](float l, int id) {
        const uint32_t key = Key<T>::of(l);
        if (l > most || !kept(from, key, id)) return;
        const int bin = by_value ? value_bin(l) : static_cast<int>((hi - key) >> shift);
        atomicAdd(&sh.count[buf][bin], 1u);
        if (BY_MASS) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[buf][bin]), static_cast<unsigned long long>(w(l)));
      });
      sync();
      // a bin per thread, all blocks' together
      uint32_t n = 0;
      uint64_t m = 0;
#pragma unroll
      for (int r = 0; r < CS; ++r) {
        n += remote_u32(cluster_addr(&sh.count[buf][threadIdx.x], r));
        if (BY_MASS) m += remote_u64(cluster_addr(&sh.mass[buf][threadIdx.x], r));
      }
      const uint64_t own = BY_MASS ? m : n, incl = scan_block(own);
      if (above + incl >= target && above + incl - own < target) {
        sh.d_bin = threadIdx.x;
        sh.d_count = n;
        sh.d_above = above + incl - own;
      }
      __syncthreads();
      const uint32_t bin = sh.d_bin;
      inside = sh.d_count;
      if (inside == 0) return false;
      above = sh.d_above;
      if (by_value) {
        const int b = static_cast<int>(bin);
        const uint32_t lo2 = first_key(lo, hi, [&](uint32_t k) { return value_bin(Key<T>::value(k)) <= b; });
        if (b > 0) hi = first_key(lo2, hi, [&](uint32_t k) { return value_bin(Key<T>::value(k)) <= b - 1; }) - 1;
        lo = lo2;
        by_value = false;
      } else {
        const uint32_t top = hi - (bin << shift);
        lo = max(lo, top - min(top, (1u << shift) - 1));
        hi = top;
      }
      __syncthreads();                                        // (d_bin is written again)
    }
    const float least = Key<T>::value(lo), most = Key<T>::value(hi);
    if (lo >= hi) {
      if (above >= target) return false;
      // one key: of its ids the first ones, in the order of ids
      uint64_t need = target - above;
      if (BY_MASS) {
        const uint64_t each_w = w(least);
        if (each_w == 0) return false;
        need = (need + each_w - 1) / each_w;
      }
      auto one = [&](float l, int i) { return l == least && kept(from, Key<T>::of(l), i) ? 1ull : 0ull; };
      int id;
      sums_of(least, one);
      if (pick(least, one, [&](uint64_t all) { return min(all, need) - 1; }, &id, nullptr) < need && above == start) return false;
      *cut = {lo, id};
      return true;
    }
    // a few elements: each of them finds what is in front of it
    if (threadIdx.x == 0) sh.few_n = 0, sh.d_id = 0xffffffffu;
    __syncthreads();
    each(least, [&](float l, int id) {
      const uint32_t key = Key<T>::of(l);
      if (l > most || !kept(from, key, id)) return;
      const uint32_t i = atomicAdd(&sh.few_n, 1u);
      sh.few_key[i] = key;
      sh.few_id[i] = id;
    });
    sync();
    uint32_t n_all = 0, off = 0;
    int src = -1;
#pragma unroll
    for (int r = 0; r < CS; ++r) {
      const uint32_t n = remote_u32(cluster_addr(&sh.few_n, r));
      if (threadIdx.x >= n_all && threadIdx.x < n_all + n) {
        src = r;
        off = threadIdx.x - n_all;
      }
      n_all += n;
    }
    if (src >= 0) {
      const uint32_t key = remote_u32(cluster_addr(&sh.few_key[off], src));
      sh.all_key[threadIdx.x] = key;
      sh.all_id[threadIdx.x] = remote_u32(cluster_addr(&sh.few_id[off], src));
      sh.all_w[threadIdx.x] = BY_MASS ? w(Key<T>::value(key)) : 1;
    }
    __syncthreads();
    // four threads an element
    {
      const uint32_t i = threadIdx.x >> 2, part = threadIdx.x & 3;
      uint64_t front = 0;
      if (i < n_all) {
        const uint32_t key = sh.all_key[i], id = sh.all_id[i];
        for (uint32_t j = part; j < n_all; j += 4)
          if (sh.all_key[j] > key || (sh.all_key[j] == key && sh.all_id[j] < id)) front += sh.all_w[j];
      }
      front += __shfl_xor_sync(0xffffffffu, front, 1);
      front += __shfl_xor_sync(0xffffffffu, front, 2);
      if (i < n_all && part == 0 && above + front < target && above + front + sh.all_w[i] >= target) {
        sh.d_key = sh.all_key[i];
        sh.d_id = sh.all_id[i];
      }
    }
    sync();                                                   // (the few have been read by all)
    *cut = {sh.d_key, static_cast<int>(sh.d_id)};
    return cut->id >= 0;
  }

  // A key below which no element is among the first k: the lanes' maxima, `mine` of each, are counted by value.
  __device__ uint32_t bound_k(uint32_t lo, uint32_t hi, float mine, float least_mine, uint64_t k) {
    const float range = s.max - least_mine;
    if (!(range > 0.0f && range < 3e38f)) return lo;
    const float per = (NB - 1) / range;
    auto value_bin = [&](float l) { return min(NB - 1, static_cast<int>((s.max - l) * per)); };
    sh.count[0][threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.d_bin = NB;
    __syncthreads();
    if (mine >= least_mine) atomicAdd(&sh.count[0][value_bin(mine)], 1u);
    sync();
    uint32_t n = 0;
#pragma unroll
    for (int r = 0; r < CS; ++r) n += remote_u32(cluster_addr(&sh.count[0][threadIdx.x], r));
    const uint64_t incl = scan_block(n);
    if (incl >= k && incl - n < k) sh.d_bin = threadIdx.x;
    __syncthreads();
    const int b = static_cast<int>(sh.d_bin);
    sync();                                                   // (the counts may be written again)
    if (b >= NB - 1) return lo;
    return max(lo, first_key(lo, hi, [&](uint32_t key) { return value_bin(Key<T>::value(key)) <= b; }));
  }

  // The nucleus of a row that is not listed: p of the mass of what `from` keeps.
  __device__ Cut nucleus(const Cut& from, float p, int vocab) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t khi = Key<T>::of(s.max);
    auto nothing = [](float, int) { return 0ull; };
    auto any = [](uint64_t) { return 0ull; };
    auto target_of = [&](uint64_t mass) {
      const uint64_t t = static_cast<uint64_t>(ceil(static_cast<double>(p) * static_cast<double>(mass)));
      return min(max(t, static_cast<uint64_t>(1)), mass);
    };
    Cut cut{};
    // Ids that weigh less than (1 - p) / vocab of the maximum together weigh less than 1 - p of the mass: none is kept.
    const float depth = (__log2f(static_cast<float>(vocab) / (1.0f - p)) + 0.5f) / s.hi;
    const uint32_t low = max(from.key, Key<T>::of(s.max - depth));
    if (from.id == ALL && from.key < khi && s.hi > kFlat) {
      const float cutv = below(Key<T>::value(from.key)), per = (NB - 2) / depth;
      sh.count[0][threadIdx.x] = 0;
      if (threadIdx.x == 0) sh.d_bin = NB;
      __syncthreads();
      const uint64_t mine = bulk<true>(cutv, per, sh.count[0]);
      if (lane == 0) sh.sums[turn][warp] = mine;
      const uint64_t mass = pick(0.0f, nothing, any, nullptr, nullptr);
      const uint64_t target = target_of(mass);
      uint32_t n = 0;
#pragma unroll
      for (int r = 0; r < CS; ++r) n += remote_u32(cluster_addr(&sh.count[0][threadIdx.x], r));
      // a bin's mass, about, in 2^-32 of the maximum's
      const float b_c = fmaf(s.max, per, 12582912.0f), off = fmaf(-s.max, per, b_c - 12582912.0f);   // (of the maximum from its bin's middle)
      const float mid = ex2_approx((off - static_cast<float>(threadIdx.x)) / per * s.hi) * 262144.0f;
      const uint64_t guess = static_cast<uint64_t>(static_cast<float>(n) * mid), incl = scan_block(guess);
      if (incl >= target >> 12 && incl - guess < target >> 12) sh.d_bin = threadIdx.x;
      __syncthreads();
      const int b = static_cast<int>(sh.d_bin);
      if (b < NB - 2) {
        // the keys of the bins b - 1 .. b + 1
        auto bin = [&](uint32_t k) { return static_cast<int>(__float_as_uint(fmaf(Key<T>::value(k), -per, b_c)) - 0x4b400000u); };
        const uint32_t lo = first_key(low, khi, [&](uint32_t k) { return bin(k) <= b + 1; });
        const uint32_t hi = b > 1 ? first_key(lo, khi, [&](uint32_t k) { return bin(k) <= b - 2; }) - 1 : khi;
        if (make_list(from, Key<T>::value(lo), Key<T>::value(hi))) {
          const uint64_t over = hi < khi ? bulk<false>(Key<T>::value(hi), 0.0f, nullptr) : 0;
          if (lane == 0) sh.above[warp] = sh.sums[turn][warp] = over;
          const uint64_t above = pick(0.0f, nothing, any, nullptr, nullptr);
          if (above < target && narrow<true>(from, lo, hi, above, target, &cut)) return cut;
          listed = false;
        }
      }
    }
    sums_kept(from);
    const uint64_t mass = pick(0.0f, nothing, any, nullptr, nullptr);
    if (!narrow<true>(from, low, khi, 0, target_of(mass), &cut)) cut = from;
    return cut;
  }
};

template <class T, int CS>
__global__ void __launch_bounds__(NT) sample_kernel(const SampleArgs a) {
  using V = Vec<T>;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  uint4* data = reinterpret_cast<uint4*>(smem + (sizeof(Shared) + 15) / 16 * 16);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CS > 1 ? static_cast<int>(cluster_ctarank()) : 0, row = blockIdx.x / CS;
  if (threadIdx.x < 32) sh.pow[threadIdx.x] = kPow[threadIdx.x];
  pdl_enter();
  // ---- the row into shared memory, its maximum
  const int first = rank * NW * a.seg;
  const T* src = static_cast<const T*>(a.logits) + row * a.ld;
  const float ninf = __int_as_float(0xff800000);
  const float t = a.temperature ? a.temperature[row] : 1.0f, p = a.top_p ? a.top_p[row] : 1.0f, mp = a.min_p ? a.min_p[row] : 0.0f;
  const int k = !(t > 0x1p-100f) || p <= 0.0f ? 1 : a.top_k ? a.top_k[row] : 0;
  const float u0 = a.u[row];
  float top = ninf;
  {
    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    const int base = first + warp * a.seg, n = a.seg / V::N;
    uint4* dst = data + warp * n;
    auto take = [&](int i, const uint4& q) {
      float v[V::N];
      V::get(q, v);
      const int id = base + i * V::N;
#pragma unroll
      for (int e = 0; e < V::N; ++e) v[e] = fmaxf(v[e] + 0.0f, ninf);   // NaN: -inf
      if (static_cast<uint32_t>(a.mask_id - id) < V::N) {
#pragma unroll
        for (int e = 0; e < V::N; ++e)
          if (id + e == a.mask_id) v[e] = ninf;
      }
#pragma unroll
      for (int e = 0; e < V::N; ++e) top = fmaxf(top, v[e]);
      dst[i] = V::put(v);
    };
    auto one = [&](int i) {                                   // element by element: the row's end, and rows off 16 bytes
      float v[V::N];
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const int id = base + i * V::N + e;
        v[e] = id < a.vocab ? to_f32(src[id]) : ninf;
      }
      return V::put(v);
    };
    constexpr int U = 4;
    for (int i0 = lane; i0 < n; i0 += 32 * U) {
      uint4 q[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = i0 + 32 * k, id = base + i * V::N;
        if (i < n) q[k] = vec && id + V::N <= a.vocab ? __ldcs(reinterpret_cast<const uint4*>(src + id)) : one(i);
      }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i0 + 32 * k < n) take(i0 + 32 * k, q[k]);
    }
  }
  const float lane_top = top;
  {
    const float hi = warp_max(top), lo = -warp_max(top > ninf ? -top : ninf);
    if (lane == 0) sh.wtop[warp] = make_float2(hi, lo);
  }
  if (threadIdx.x == 0) {                                     // (double precision is slow here: one thread, for all)
    const double c = 1.4426950408889634074 / static_cast<double>(t);
    sh.c_hi = static_cast<float>(c);
    sh.c_lo = static_cast<float>(c - static_cast<double>(sh.c_hi));
    if (mp > 0.0f) sh.low64 = mp >= 1.0f ? 0.0 : static_cast<double>(t) * log(static_cast<double>(mp));
  }
  __syncthreads();
  if (warp == 0) {
    const float2 x = lane < NW ? sh.wtop[lane] : make_float2(ninf, -ninf);
    const float hi = warp_max(x.x), lo = -warp_max(-x.y);
    if (lane == 0) sh.top = make_float2(hi, lo);
  }
  Row<T, CS> r{sh, data, first, a.seg, rank, {}, 0, false};
  r.sync();
  float least_top = -ninf;
#pragma unroll
  for (int i = 0; i < CS; ++i) {
    top = fmaxf(top, __uint_as_float(remote_u32(cluster_addr(&sh.top.x, i))));
    least_top = fminf(least_top, __uint_as_float(remote_u32(cluster_addr(&sh.top.y, i))));
  }
  const bool writer = rank == 0 && threadIdx.x == 0;
  if (top == ninf) {                                          // nothing to draw from
    if (writer) {
      a.tok[row] = -1;
      if (a.prob) a.prob[row] = 0.0f;
    }
    r.sync();
    return;
  }
  const uint32_t khi = Key<T>::of(top);
  int id = -1;
  if (k == 1 || top == -ninf) {
    // the first of the order, the lowest id of the maximum; or, of an infinite maximum, ids of equal weight
    auto of_max = [&](float l, int) { return l == top ? 1ull : 0ull; };
    r.sums_of(top, of_max);
    uint64_t n = 1;
    r.pick(top, of_max, [&](uint64_t all) {
      if (k == 1) return static_cast<uint64_t>(0);
      n = k > 0 ? min(all, static_cast<uint64_t>(k)) : all;
      if (p < 1.0f) n = min(n, max(static_cast<uint64_t>(1), static_cast<uint64_t>(ceil(static_cast<double>(p) * static_cast<double>(n)))));
      const double x = (u0 > 0.0f ? static_cast<double>(u0) : 0.0) * static_cast<double>(n);
      return x >= static_cast<double>(n) ? n - 1 : static_cast<uint64_t>(x);
    }, &id, nullptr);
    if (writer) {
      a.tok[row] = id;
      if (a.prob) a.prob[row] = 1.0f / static_cast<float>(n);
    }
    r.sync();
    return;
  }
  r.s = {top, sh.c_hi, sh.c_lo};
  // ---- what bulk() needs of the row: M = c max (max less itself where it is large) to 1/16, and the table with the rest of it
  if (threadIdx.x < 16) {
    const float xm = fabsf(top * r.s.hi) >= 92.0f ? 0.0f : top;
    const float m = xm * r.s.hi, e = fmaf(xm, r.s.lo, fmaf(xm, r.s.hi, -m));
    const float mh = rintf(16.0f * m) * 0.0625f, rest = (m - mh) + e;      // |rest| <= 1/32
    const double f = -static_cast<double>(rest) * 0.693147180559945309417;
    const double x = 1.0 + f * (1.0 + f * (0.5 + f * (1.0 / 6 + f * (1.0 / 24 + f * (1.0 / 120 + f / 720)))));
    const double v = x * (static_cast<double>(sh.pow[2 * threadIdx.x]) * 0x1p-43);
    const float h = static_cast<float>(v);
    sh.pow16[threadIdx.x] = make_float2(h, static_cast<float>(v - static_cast<double>(h)));
    sh.mh = mh;
    if (threadIdx.x == 0) {                                   // the least logit that min-p keeps, rounded up
      const double least = mp > 0.0f ? static_cast<double>(top) + sh.low64 : -INFINITY;
      sh.low = __double2float_ru(least);
    }
  }
  if (threadIdx.x < NW) sh.above[threadIdx.x] = 0;
  __syncthreads();
  // ---- the cut: min-p, top-k, top-p
  Cut cut{Key<T>::of(ninf) + 1, ALL};
  if (mp > 0.0f) {
    const float low = fminf(sh.low, top) + 0.0f;
    const uint32_t key = Key<T>::of(low);
    cut.key = max(cut.key, Key<T>::value(key) < low ? key + 1 : key);
  }
  if (k > 0 || mp > 0.0f) {
    const uint32_t lo = k > 0 && k < a.vocab ? r.bound_k(cut.key, khi, lane_top, least_top, k) : cut.key;
    r.make_list(cut, Key<T>::value(lo), top);
    if (k > 0 && k < a.vocab) {
      // (fewer than k: all of them)
      Cut to{};
      if (r.template narrow<false>(cut, lo, khi, 0, k, &to)) cut = to;
    }
  }
  if (p < 1.0f) {
    if (r.listed) {
      r.sums_kept(cut);
      const uint64_t mass = r.pick(0.0f, [](float, int) { return 0ull; }, [](uint64_t) { return 0ull; }, nullptr, nullptr);
      const uint64_t target = max(static_cast<uint64_t>(1), static_cast<uint64_t>(ceil(static_cast<double>(p) * static_cast<double>(mass))));
      Cut to{};
      if (r.template narrow<true>(cut, cut.key, khi, 0, min(target, mass), &to)) cut = to;
    } else {
      cut = r.nucleus(cut, p, a.vocab);
    }
  }
  // ---- the draw
  uint64_t value = 0;
  r.sums_kept(cut);
  const uint64_t mass = r.pick(Key<T>::value(cut.key), [&](float l, int i) { return r.kept(cut, Key<T>::of(l), i) ? r.w(l) : 0ull; },
                               [&](uint64_t all) {
    const double u = u0 > 0.0f ? static_cast<double>(u0) : 0.0;
    const double x = u * static_cast<double>(all);
    return x >= static_cast<double>(all) ? all - 1 : min(all - 1, static_cast<uint64_t>(x));
  }, &id, &value);
  if (writer) {
    a.tok[row] = id;
    if (a.prob) a.prob[row] = static_cast<float>(static_cast<double>(value) / static_cast<double>(mass));
  }
  r.sync();                                                   // no block leaves while another reads its memory
}

template <class T, int CS>
cudaError_t launch(const SampleArgs& a, int rows, size_t smem, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  static PerDevice ready;
  int dev = 0;
  cudaGetDevice(&dev);
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(sample_kernel<T, CS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * CS);
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CS, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, CS>, a);
}

}  // namespace

const char* sample_rows(const SampleCall& c, cudaStream_t s) {
  int dev = 0;
  const int sms = current_sms(&dev), es = c.bf16 ? 2 : 4, chunk = 32 * (16 / es);
  // Blocks of a row: as few as let two of them share an SM (one loads while the other searches), and more while SMs would
  // stay idle and every warp still has a few loads of its own.
  auto seg_of = [&](int cs) { return (c.vocab + cs * NW * chunk - 1) / (cs * NW * chunk) * chunk; };
  int cs = 1;
  while (cs < MAXC && static_cast<int64_t>(seg_of(cs)) * NW * es > 90 * 1024) cs *= 2;
  while (cs < MAXC && static_cast<int64_t>(c.rows) * cs * 2 <= sms && seg_of(cs) > 2 * chunk) cs *= 2;
  const SampleArgs a{c.logits, c.ld, c.vocab, c.mask_id, seg_of(cs), c.temperature, c.top_k, c.top_p, c.min_p, c.u, c.tok, c.prob};
  const size_t smem = (sizeof(Shared) + 15) / 16 * 16 + static_cast<size_t>(a.seg) * NW * es;
  cudaError_t e;
  if (c.bf16) {
    e = cs == 1 ? launch<bf16, 1>(a, c.rows, smem, s) : cs == 2 ? launch<bf16, 2>(a, c.rows, smem, s)
      : cs == 4 ? launch<bf16, 4>(a, c.rows, smem, s) : launch<bf16, 8>(a, c.rows, smem, s);
  } else {
    e = cs == 1 ? launch<float, 1>(a, c.rows, smem, s) : cs == 2 ? launch<float, 2>(a, c.rows, smem, s)
      : cs == 4 ? launch<float, 4>(a, c.rows, smem, s) : launch<float, 8>(a, c.rows, smem, s);
  }
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
