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
// ids, warp w of it the w-th segment of that part.  A cut is narrowed down by
// histograms of 512 bins, first over the value, then over the key, until 128
// elements or one key are left.  What the blocks know together goes through
// distributed shared memory; every block reads all parts and comes to the same
// decisions.
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

struct Shared {
  uint64_t pow[32];
  uint64_t mass[2][NB];                    // histograms, two in turn
  uint32_t count[2][NB];
  uint64_t sums[2][NW];                    // per warp
  uint64_t scan_mass[NW];
  uint32_t scan_count[NW];
  uint32_t found_id[2];                    // what pick() found
  uint64_t found_w[2];
  float2 top;                              // maximum and, of the finite ones, minimum of the block
  uint32_t list_n[2];
  uint32_t list_key[2][LIST], list_id[2][LIST];
  uint64_t all_w[LIST];
  uint32_t all_key[LIST], all_id[LIST];
  uint64_t part[NW];
  float wmax[NW];
  float fhi, flo;
  // what one thread decides for its block
  uint64_t d_mass;
  uint32_t d_bin, d_count, d_key, d_id;
  uint64_t d_above;
  uint32_t d_above_n;
};

static_assert((sizeof(Shared) + 15) / 16 * 16 + (kSampleMaxVocab + MAXC * NW * 128 - 1) / (MAXC * NW * 128) * 128 * NW * 4 <= 232448, "shared memory");

struct Cut {
  uint32_t key;
  int id;                                  // ids of that key up to this one are kept
};

template <class T, int CS>
struct Row {
  using V = Vec<T>;
  Shared& sh;
  const uint4* data;                       // this block's part
  int first, seg, rank;                    // id of the part's first element
  Scale s;
  int turn;                                // of the arrays that pick() uses in turn: a sync lies between two uses of one

  __device__ __forceinline__ uint64_t w(float l) const { return weight(s, sh.pow, l); }
  __device__ __forceinline__ static bool kept(const Cut& c, uint32_t key, int id) { return key > c.key || (key == c.key && id <= c.id); }
  __device__ __forceinline__ void sync() const {
    if constexpr (CS > 1) cluster_sync();
    else __syncthreads();
  }
  // f(logit, id) of this warp's elements whose logit is at least `least`
  template <class F>
  __device__ __forceinline__ void each(float least, F&& f) const {
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
  // Sum of f over the elements with a logit of at least `least`; with `id`, also the first element in the order of ids with
  // which the sum exceeds target(whole sum), and its f.
  template <class F, class G>
  __device__ uint64_t pick(float least, F&& f, G&& target, int* id, uint64_t* value) {
    turn ^= 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t mine = 0;
    each(least, [&](float l, int i) { mine += f(l, i); });
    mine = warp_sum_u64(mine);
    if (lane == 0) sh.sums[turn][warp] = mine;
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
    if (!id) return total;
    const uint64_t t = target(total);
    const unsigned past = __ballot_sync(0xffffffffu, incl > t);
    if (!past) {                                              // (t is below a sum that is not zero)
      *id = -1;
      return total;
    }
    const int src = __ffs(past) - 1;
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
      const uint64_t x = lane < NW ? sh.part[lane] : 0, inc = warp_scan_u64(x);
      const int who = __ffs(__ballot_sync(0xffffffffu, inc > left)) - 1;
      if (who == warp) {
        left -= __shfl_sync(0xffffffffu, inc - x, who);
        for (int c = c0; c < c1; ++c) {
          const uint64_t mine2 = lane_sum(c), in = warp_scan_u64(mine2);
          const unsigned hit = __ballot_sync(0xffffffffu, in > left);
          if (hit) {
            if (lane == __ffs(hit) - 1) {
              uint64_t rem = left - (in - mine2);
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
    return total;
  }

  // The cut that keeps, of the elements that `from` keeps, the first ones of the order: `target` of them (BY_MASS: as many
  // as have less than `target` of mass in front of them).  At least one element is kept by `from`, target >= 1 and at most
  // all of them (their mass).  lo: a key below which nothing needs to be looked at.
  template <bool BY_MASS>
  __device__ Cut narrow(Cut from, uint32_t lo, uint32_t hi, uint64_t target) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t above = 0;                    // what lies above the window counts: elements or mass
    uint32_t inside = 0xffffffffu;         // elements in the window
    for (int level = 0; lo < hi && inside > LIST; ++level) {
      const int buf = level & 1;
      sh.count[buf][threadIdx.x] = 0;
      sh.mass[buf][threadIdx.x] = 0;
      __syncthreads();
      // first by value, in steps of equal ratios of weights; then by key
      const float range = s.max - Key<T>::value(lo);
      const bool by_value = level == 0 && range < 3e38f;
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
      const uint64_t own = BY_MASS ? m : n;
      uint64_t incl = warp_scan_u64(own);
      if (lane == 31) sh.scan_mass[warp] = incl;
      __syncthreads();
      const uint64_t x = warp_scan_u64(lane < NW ? sh.scan_mass[lane] : 0);
      if (warp > 0) incl += __shfl_sync(0xffffffffu, x, warp - 1);
      if (above + incl >= target && above + incl - own < target) {
        sh.d_bin = threadIdx.x;
        sh.d_count = n;
        sh.d_above = above + incl - own;
      }
      __syncthreads();
      const uint32_t bin = sh.d_bin;
      inside = sh.d_count;
      above = sh.d_above;
      if (by_value) {
        const int b = static_cast<int>(bin);
        const uint32_t lo2 = first_key(lo, hi, [&](uint32_t k) { return value_bin(Key<T>::value(k)) <= b; });
        if (b > 0) hi = first_key(lo2, hi, [&](uint32_t k) { return value_bin(Key<T>::value(k)) <= b - 1; }) - 1;
        lo = lo2;
      } else {
        const uint32_t top = hi - (bin << shift);
        lo = max(lo, top - min(top, (1u << shift) - 1));
        hi = top;
      }
      __syncthreads();                                        // (d_bin is written again)
    }
    const float least = Key<T>::value(lo), most = Key<T>::value(hi);
    if (lo >= hi) {
      // one key: of its ids the first ones, in the order of ids
      uint64_t need = target - above;
      if (BY_MASS) {
        const uint64_t each_w = w(least);
        need = (need + each_w - 1) / each_w;
      }
      int id;
      pick(least, [&](float l, int i) { return l == least && kept(from, Key<T>::of(l), i) ? 1ull : 0ull; },
           [&](uint64_t) { return need - 1; }, &id, nullptr);
      return {lo, id};
    }
    // a few elements: each of them finds what is in front of it
    if (threadIdx.x == 0) sh.list_n[0] = 0;
    __syncthreads();
    each(least, [&](float l, int id) {
      const uint32_t key = Key<T>::of(l);
      if (l > most || !kept(from, key, id)) return;
      const uint32_t at = atomicAdd(&sh.list_n[0], 1u);
      sh.list_key[0][at] = key;
      sh.list_id[0][at] = id;
    });
    sync();
    uint32_t before = 0, n_all = 0, off = 0;
    int src = -1;
#pragma unroll
    for (int r = 0; r < CS; ++r) {
      const uint32_t n = remote_u32(cluster_addr(&sh.list_n[0], r));
      if (threadIdx.x >= before && threadIdx.x < before + n) {
        src = r;
        off = threadIdx.x - before;
      }
      before += n;
    }
    n_all = before;
    if (src >= 0) {
      const uint32_t key = remote_u32(cluster_addr(&sh.list_key[0][off], src));
      sh.all_key[threadIdx.x] = key;
      sh.all_id[threadIdx.x] = remote_u32(cluster_addr(&sh.list_id[0][off], src));
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
    sync();                                                   // (the lists have been read by all)
    return {sh.d_key, static_cast<int>(sh.d_id)};
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
  float top = ninf;
  if (threadIdx.x == 0) {
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    const double c = 1.4426950408889634074 / static_cast<double>(t);
    sh.fhi = static_cast<float>(c);
    sh.flo = static_cast<float>(c - static_cast<double>(sh.fhi));
  }
  {
    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    const int base = first + warp * a.seg, n = a.seg / V::N;
    uint4* dst = data + warp * n;
    auto take = [&](int i, const uint4& q) {
      float v[V::N];
      V::get(q, v);
#pragma unroll
      for (int e = 0; e < V::N; ++e) {
        const int id = base + i * V::N + e;
        v[e] = v[e] != v[e] || id == a.mask_id || id >= a.vocab ? ninf : v[e] + 0.0f;
        top = fmaxf(top, v[e]);
      }
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
  top = warp_max(top);
  if (lane == 0) sh.wmax[warp] = top;
  __syncthreads();
  top = warp_max(lane < NW ? sh.wmax[lane] : ninf);
  if (threadIdx.x == 0) sh.top.x = top;
  Row<T, CS> r{sh, data, first, a.seg, rank, {}, 0};
  r.sync();
#pragma unroll
  for (int k = 0; k < CS; ++k) top = fmaxf(top, __uint_as_float(remote_u32(cluster_addr(&sh.top, k))));
  const bool writer = rank == 0 && threadIdx.x == 0;
  if (top == ninf) {                                          // nothing to draw from
    if (writer) {
      a.tok[row] = -1;
      if (a.prob) a.prob[row] = 0.0f;
    }
    r.sync();
    return;
  }
  r.s = {top, sh.fhi, sh.flo};
  const uint32_t khi = Key<T>::of(top);
  const float t = a.temperature ? a.temperature[row] : 1.0f;
  const int k = !(t > 0x1p-100f) ? 1 : a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.0f, mp = a.min_p ? a.min_p[row] : 0.0f;
  int id = -1;
  if (k == 1 || p <= 0.0f) {
    // the first of the order: the lowest id of the maximum
    r.pick(top, [&](float, int) { return 1ull; }, [](uint64_t) { return 0ull; }, &id, nullptr);
    if (writer) {
      a.tok[row] = id;
      if (a.prob) a.prob[row] = 1.0f;
    }
    r.sync();
    return;
  }
  // ---- the cut: weights that count at all, min-p, top-k, top-p
  uint64_t least_w = 1;
  if (mp > 0.0f) least_w = mp >= 1.0f ? ONE : max(static_cast<uint64_t>(1), static_cast<uint64_t>(ceil(static_cast<double>(mp) * static_cast<double>(ONE))));
  const uint32_t kinf = Key<T>::of(ninf) + 1;
  Cut cut{first_key(kinf, khi, [&](uint32_t key) { return r.w(Key<T>::value(key)) >= least_w; }), 0x7fffffff};
  if (k > 0 && k < a.vocab) {
    const uint64_t n = r.pick(Key<T>::value(cut.key), [&](float, int) { return 1ull; }, [](uint64_t) { return 0ull; }, nullptr, nullptr);
    if (n > static_cast<uint64_t>(k)) cut = r.template narrow<false>(cut, cut.key, khi, k);
  }
  auto kept_w = [&](float l, int i) { return r.kept(cut, Key<T>::of(l), i) ? r.w(l) : 0ull; };
  if (p < 1.0f) {
    const uint64_t mass = r.pick(Key<T>::value(cut.key), kept_w, [](uint64_t) { return 0ull; }, nullptr, nullptr);
    const uint64_t target = max(static_cast<uint64_t>(1), static_cast<uint64_t>(ceil(static_cast<double>(p) * static_cast<double>(mass))));
    cut = r.template narrow<true>(cut, cut.key, khi, min(target, mass));
  }
  // ---- the draw
  uint64_t value = 0;
  const float u0 = a.u[row];
  const uint64_t mass = r.pick(Key<T>::value(cut.key), kept_w, [&](uint64_t all) {
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
