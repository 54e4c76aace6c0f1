// Attention of packed bf16 rows over the paged 8-bit cache, tcgen05.
//
//   S^T = K Q^T,  O^T = V^T P^T      (keys and head dims on the 128 MMA rows)
//
// The rows that read one KV head (query heads of its group x rows of a block
// step or a single token) are few: 2 to 64 virtual rows.  They are the N of
// both products here, so the tensor work follows their number (16, 32 or 64)
// instead of being padded to 128, and a key is one TMEM lane = one thread,
// whose page scales are two registers.
//
// K enters the tensor cores as the e4m3 bytes that the page holds; Q is the sum
// of an e4m3 and an e5m2 term, both multiplied with K into the same fp32 scores.  V^T is
// widened to f16, because the probabilities need more than 8 bits.
//
// A tile is 128 keys, two pages.  Roles of a CTA (12, 16 or 24 warps for 16, 32 or 64 rows):
//   warp 0       streams the pages with TMA (one 4-D map for K, one for V^T)
//                and leaves their scales beside them;
//   warps 2, 3   stage Q of the next work item while this one runs;
//   warps 4-7    convert V^T: e4m3 -> f16, exact, from shared memory into the
//                TMEM A operand (a dim per lane); keys that no row
//                of the item sees become zeros here;
//   warp 1       S^T(i) = K Q^T, then O^T += V^T P^T of tile i - 1;
//   warps 8-     softmax: a key per thread, the values of 16 rows in
//                registers.  The running maximum of a row is a reference that
//                moves only when a tile exceeds it by 2^8, so a tile costs
//                one vote of the four warps that share rows and no reduction
//                over the keys; the sums of a row stay one partial per thread
//                until the end of the work item.
// Precision: each row of Q is scaled by a power of four of its own (with one factor
// per tile, a large row took the bits of the others); the two terms hold a bf16
// value exactly if it is within 2^-12 of its row's largest, and to 2^-20 of that
// below (e5m2, because its steps go down to 2^-16, e4m3's to 2^-9).  K and V are
// exact.  A key's weight, its probability times its page's V scale, is rounded to
// f16 (11 bits) with the row's largest weight at 2^7 to 2^15, so that a weight of
// 2^-21 of the largest still has all of them and one below 2^-32 is lost: with
// equal probabilities, a page whose V scale is that far below another page's.
// Scores, sums and O are fp32.
//
// Bound: the bytes of the cache.  Measured: 4 tokens over 386,544 cached ones (8
// KV heads of 128) 135 us, 5.9 TB/s; with 64 virtual rows a tile takes 1.1 us
// per SM for 0.73 us of bytes, paced by the softmax warps' chain of waits (8 x
// 32 rows over 99,641 tokens, 16 KV heads: 103 us, 4.0 TB/s).  There, in the order
// of their making: K and V both widened to f16 157 us; K multiplied as it is
// stored, 142 with Q in three terms and 121 in two; fewer instructions around
// the items 109; 16 rows per softmax thread where 32 were 100;
// 98 with one factor of Q per tile.  A factor per row, read by the softmax with
// every tile, took 107 as fp32, 106 as bf16 and 103 as a byte.
//
// Work: the tiles of all (sequence, KV head, row tile) items lie on one line,
// each item followed by what its start and end cost, and the line is cut
// evenly over the SMs, whatever the lengths; an item that a cut splits leaves
// fp32 partials, which a second small kernel merges in order.  Where the cuts
// fall follows from all lengths of a call, and with them a row's last bits.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "ragged.cuh"
#include "serve.h"
#include "softmax_rows.cuh"
#include "tensor_map.h"
#include "umma_tiles.cuh"

namespace tadm {
namespace {

constexpr int PT = TADM_PAGE_TOKENS;
constexpr int TK = 2 * PT;                 // keys of a tile

struct PagedArgs {
  const bf16* q;
  bf16* o;
  const float *sk, *sv;                    // this layer's scales
  const int32_t *cu, *lens, *table;
  int batch, total, max_rows, max_len, ld_table, pages;
  int group, n_kv;
  uint32_t group_inv;                      // floor((2^32 - 1) / group)
  int64_t ldq, ldo;
  int causal, window;
  float scale_log2;                        // log2(e) / sqrt(hd)
  float* part_o;                           // [2 * CTAs][N][HD]
  float2* part_ml;                         // [2 * CTAs][N]: (reference in log2 units, sum)
  struct Place* place;                     // [CTAs] where each CTA's units begin
  int* status;
};

// ------------------------------------------------------------------ work items
struct SeqInfo {
  int first, n_virt, len, pos0, n_rt;      // first row, virtual rows, tokens, position of row 0, row tiles
};
// v / group for 0 <= v < 2^31: the product is the quotient or one less
__device__ __forceinline__ int by_group(const PagedArgs& a, int v) {
  const uint32_t q = __umulhi(static_cast<uint32_t>(v), a.group_inv);
  return static_cast<int>(q + (static_cast<uint32_t>(v) - q * a.group >= static_cast<uint32_t>(a.group)));
}
template <int N>
__device__ __forceinline__ SeqInfo seq_info(const PagedArgs& a, int b) {
  const SeqRows r = seq_rows(a.cu, b, a.total, a.max_rows);
  const int len = min(max(a.lens[b], 0), a.max_len);
  return {r.first, r.n * a.group, len, len - r.n, (r.n * a.group + N - 1) / N};
}
// The keys that any row of row tile rt sees: from .x to before .y.
template <int N>
__device__ __forceinline__ int2 key_range(const PagedArgs& a, const SeqInfo& s, int rt) {
  const int r_lo = by_group(a, rt * N), r_hi = by_group(a, min((rt + 1) * N, s.n_virt) - 1);
  return make_int2(a.window > 0 ? max(0, s.pos0 + r_lo - a.window + 1) : 0,
                   a.causal ? max(0, min(s.len, s.pos0 + r_hi + 1)) : s.len);
}
// Their tiles: first tile and how many (maybe none).
__device__ __forceinline__ int2 tiles_of(int2 keys) {
  const int t0 = keys.x / TK, t1 = (keys.y + TK - 1) / TK;
  return make_int2(t0, keys.x < keys.y ? t1 - t0 : 0);
}
template <int N>
__device__ __forceinline__ int2 tile_range(const PagedArgs& a, const SeqInfo& s, int rt) {
  return tiles_of(key_range<N>(a, s, rt));
}
// An item's units: its tiles, then kItemUnits for its start and end (Q, the
// first references, the sums, O), measured in tiles (32 block steps of 32 rows over
// 1 to 2000 tokens / 8 over 3000 to 30,000: 46.4 / 105 us with 3, 43.1 / 102.7
// with 5, 43.3 / 103.2 with 6, 43.3 / 104.4 with 8, 44.2 / 106 with 10; the middle
// of what serves both); a row tile that sees nothing has zeros to write there.
constexpr int kItemUnits = 6;
// Units of a sequence and KV head.
template <int N>
__device__ __forceinline__ int64_t seq_units(const PagedArgs& a, int b) {
  const SeqInfo s = seq_info<N>(a, b);
  if (s.n_virt <= 0) return 0;
  if (!a.causal && a.window == 0) return static_cast<int64_t>(s.n_rt) * (tile_range<N>(a, s, 0).y + kItemUnits);
  int64_t u = 0;
  for (int rt = 0; rt < s.n_rt; ++rt) u += tile_range<N>(a, s, rt).y + kItemUnits;
  return u;
}
// where CTA `cta` of `ctas` begins (64-bit divisions only for more units than 2^32 / ctas)
__device__ __forceinline__ int64_t cut(int64_t total, int cta, int ctas) {
  const int64_t x = total * cta;
  return x >> 32 ? x / ctas : static_cast<uint32_t>(x) / static_cast<uint32_t>(ctas);
}
struct Item {
  int b, hk, rt, off;                      // off: units of the item before the place asked for
};
struct Place {
  int64_t total, unit;                     // units of the call, of this CTA's start
  Item it;
  SeqInfo s;                               // of the item's sequence
  int nt;                                  // the item's tiles
};
// The units of the call, and where CTA `cta` of `ctas` begins.  Warp-collective; the lanes keep the units of the first
// 32 sequences between the sum and the search.
template <int N>
__device__ __forceinline__ Place locate(const PagedArgs& a, int cta, int ctas) {
  const int lane = threadIdx.x & 31;
  const int64_t own = lane < a.batch ? seq_units<N>(a, lane) : 0;
  int64_t sum = own;
  for (int b = lane + 32; b < a.batch; b += 32) sum += seq_units<N>(a, b);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  Place pl{sum * a.n_kv, 0, Item{0, 0, 0, 0}, SeqInfo{0, 0, 0, 0, 0}, 0};
  pl.unit = cut(pl.total, cta, ctas);
  if (pl.unit >= pl.total) return pl;
  int64_t before = 0;
  for (int base = 0; base < a.batch; base += 32) {
    const int b = base + lane;
    const int64_t mine = base == 0 ? own : b < a.batch ? seq_units<N>(a, b) : 0;
    int64_t x = mine * a.n_kv;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + x > pl.unit);
    if (past) {
      const int src = __ffs(past) - 1;
      const int64_t per = __shfl_sync(0xffffffffu, mine, src);
      int64_t in = pl.unit - before - (__shfl_sync(0xffffffffu, x, src) - per * a.n_kv);
      pl.it.b = base + src;
      while (in >= per) {                                     // (fewer steps than KV heads)
        in -= per;
        ++pl.it.hk;
      }
      pl.s = seq_info<N>(a, pl.it.b);
      for (int rt = 0; rt < pl.s.n_rt; ++rt) {
        pl.nt = tile_range<N>(a, pl.s, rt).y;
        if (in < pl.nt + kItemUnits) {
          pl.it.rt = rt;
          pl.it.off = static_cast<int>(in);
          break;
        }
        in -= pl.nt + kItemUnits;
      }
      return pl;
    }
    before += __shfl_sync(0xffffffffu, x, 31);
  }
  return pl;
}

// A warp's walk over its CTA's units: one segment = consecutive tiles of one
// item.  It lies in shared memory and lane 0 moves it: a segment's fields are
// read where they are needed instead of filling registers.
template <int N>
struct Walk {
  Item it;
  SeqInfo s;
  int64_t left;            // units behind the segment
  int t0, nt;              // tiles of the segment; none: the item sees nothing and has zeros to write
  int from_start, to_end;  // it begins / ends with its item's tiles
  int started;
  int begin;               // the first key that a row of the item sees
  __device__ __forceinline__ bool next(const PagedArgs& a) {   // false: no segment left.  Warp-collective.
    __syncwarp();
    if ((threadIdx.x & 31) == 0) move(a);
    __syncwarp();
    return nt >= 0;
  }
  // one copy for all roles: code that runs once per segment costs its instruction fetches
  __device__ __noinline__ void move(const PagedArgs& a) {
    for (;;) {
      if (started) step(a);
      started = 1;
      if (left <= 0) {
        nt = -1;
        return;
      }
      const int2 keys = key_range<N>(a, s, it.rt), r = tiles_of(keys);
      begin = keys.x;
      const int units = r.y + kItemUnits, off = it.off;
      const int take = static_cast<int>(min(left, static_cast<int64_t>(units - off)));
      const int lo = min(off, r.y), hi = min(off + take, r.y);
      left -= take;
      if (hi > lo || (r.y == 0 && off == 0)) {
        t0 = r.x + lo;
        nt = hi - lo;
        from_start = lo == 0;
        to_end = hi == r.y;
        return;
      }
    }
  }
  __device__ __forceinline__ void step(const PagedArgs& a) {   // to the next item
    it.off = 0;
    if (++it.rt < s.n_rt) return;
    it.rt = 0;
    if (++it.hk < a.n_kv) return;
    it.hk = 0;
    if (left <= 0) return;
    do {
      s = seq_info<N>(a, ++it.b);
    } while (s.n_virt <= 0 && it.b + 1 < a.batch);
  }
};

// Zeroes what line `row` of a staged V^T tile (two pages of PB bytes) holds of its first `lo` keys.  Out of line: it runs
// once per item, and the loop that calls it is short of registers.
template <int PB>
__device__ __noinline__ void hide_front(uint8_t* v, int row, int lo) {
#pragma unroll 1
  for (int n = 0; n < lo; n += 4) {
    uint32_t* word = reinterpret_cast<uint32_t*>(v + (n >> 6) * PB + row * PT + ((((n >> 4) & 3) ^ ((row >> 1) & 3)) << 4) + (n & 15));
    *word = lo - n >= 4 ? 0u : *word & ~((1u << (8 * (lo - n))) - 1u);
  }
  fence_proxy_async_smem();                                   // the next page arrives there
}

// ------------------------------------------------------------------ the kernel
template <int HD_, int N_>
struct PagedCfg {
  static constexpr int HD = HD_, N = N_;
  static constexpr int PAGE_BYTES = PT * HD;                 // of K or V^T, one head
  static constexpr int STAGE_BYTES = 4 * PAGE_BYTES;         // two pages of K, two of V^T
  static constexpr int STAGES = HD == 64 ? 8 : N == 64 ? 4 : 5;
  static constexpr int QT_BYTES = N * HD, Q_BYTES = 2 * QT_BYTES;   // two terms of N rows; two buffers
  static constexpr int RAW_BYTES = N * HD * 2;               // Q as it is in memory
  static constexpr int P_BYTES = TK * 128;                   // a 128-byte line of up to 64 rows per key, f16
  static constexpr int RN = 16, GROUPS = N / RN;   // rows per softmax thread (its loads from TMEM have 16 columns), groups of four softmax warps
  static constexpr int SM_THREADS = 128 * GROUPS;
  static constexpr int THREADS = 256 + SM_THREADS;
  static constexpr int MISC = 3328 + N * 44;
  static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + 2 * Q_BYTES + 2 * P_BYTES + RAW_BYTES + MISC;
  static constexpr int V_COL = 0, S_COL = 128, O_COL = 256;  // TMEM columns: two V^T, two S, one O
  static_assert(SMEM <= 232448, "shared memory");
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
// A and B: f16, B K-major or MN-major
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool b_mn_major) {
  return (1u << 4) | (b_mn_major ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}
// A: e4m3, B: e4m3 or e5m2, both K-major
__host__ __device__ constexpr uint32_t idesc_f8_f32(int M, int N, bool b_e5m2) {
  return (1u << 4) | (b_e5m2 ? 1u << 10 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// High word of the descriptor of a K-major 8-bit operand whose rows are HD bytes, swizzled over the row's width (the low
// word is desc_k's).
template <int HD>
constexpr uint32_t kRows8Hi = (8u * HD >> 4) | 1u << 14 | (HD == 128 ? 2u : 4u) << 29;
// 16-byte chunk `c` of row `r` in that layout
template <int HD>
__device__ __forceinline__ int chunk_at(int r, int c) {
  return r * HD + ((HD == 128 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)) << 4);
}
// `bytes` (a multiple of 16) of global memory into shared memory, counted on the mbarrier
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// the largest of the warp's 32 values (NaN left out)
__device__ __forceinline__ float warp_top(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// v[r] of 32 lanes -> lanes r and r + 16 get the sum of row r
__device__ __forceinline__ float sum_rows(float (&v)[16]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float send = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
  return v[0];
}
// four e4m3 -> two pairs of f16 (exact)
__device__ __forceinline__ void e4m3x4_f16x4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]),
      "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}

template <int HD_, int N_>
__global__ void __launch_bounds__(PagedCfg<HD_, N_>::THREADS, 1)
    attn_paged_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const PagedArgs a) {
  using C = PagedCfg<HD_, N_>;
  constexpr int HD = C::HD, N = C::N, NST = C::STAGES, PB = C::PAGE_BYTES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sKV = smem;
  uint8_t* sQ = sKV + NST * C::STAGE_BYTES;
  uint8_t* sP = sQ + 2 * C::Q_BYTES;
  uint8_t* sRaw = sP + 2 * C::P_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sRaw + C::RAW_BYTES);
  uint64_t *kv_full = bars, *kv_empty = bars + 8;             // [NST]
  uint64_t *vt_full = bars + 20, *vt_empty = bars + 22;       // [2] converted V^T
  uint64_t *s_full = bars + 24, *p_full = bars + 26;          // [2]
  uint64_t *q_full = bars + 28, *q_empty = bars + 30;         // [2]
  uint64_t *o_full = bars + 32, *drain = bars + 33;           // o_full: a completion per PV
  uint64_t* o_done = bars + 35;                               // a completion per segment, its last PV
  uint64_t* raw_full = bars + 43;                             // a completion per segment, its rows of Q
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 34);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  Place* s_place = reinterpret_cast<Place*>(bars + 44);
  static_assert(sizeof(Place) <= 160, "place");
  // [16][2] of the pages of tile t at t % 16: K scale, V scale * 128, log2(V scale)
  float4* s_scale = reinterpret_cast<float4*>(bars + 64);
  Walk<N>* s_walk = reinterpret_cast<Walk<N>*>(reinterpret_cast<uint8_t*>(bars) + 1024);   // one per warp
  static_assert(sizeof(Walk<N>) * (C::THREADS / 32) <= 2304, "walks");
  // per virtual row
  float* s_negm = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + 3328);   // minus the reference
  float* s_fac = s_negm + N;
  float* s_red = s_fac + N;                                   // [4][N]
  int2* s_see = reinterpret_cast<int2*>(s_red + 4 * N);       // visible keys [x, y)
  int64_t* s_row = reinterpret_cast<int64_t*>(s_see + N);     // element offset of the output row, -1: none
  // [4][N] what a score of a row of segment i counts, 1 / the row's factor, at i % 4 (the softmax reads it later than the
  // MMAs read Q): b stands for 2^(2 b - 126), whose fp32 bits are b, then 0x80, then zeros
  uint8_t* s_unit = reinterpret_cast<uint8_t*>(s_row + N);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(&kv_full[i], 1);
      mbar_init(&kv_empty[i], 5);          // four converting warps, the MMAs that read K
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&vt_full[i], 4);
      mbar_init(&vt_empty[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 4 * C::GROUPS);
      mbar_init(&q_full[i], 2);
      mbar_init(&q_empty[i], 1);
    }
    mbar_init(o_full, 1);
    mbar_init(o_done, 1);
    mbar_init(raw_full, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  pdl_enter();
  if (warp == 0) {
    // what the merge reads of a part that a CTA which gave up a wait did not finish
    for (int i = lane; i < 2 * N; i += 32) a.part_ml[2LL * blockIdx.x * N + i] = make_float2(NAN, NAN);
    const Place pl = locate<N>(a, blockIdx.x, gridDim.x);
    if (lane == 0) {
      *s_place = pl;
      a.place[blockIdx.x] = pl;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = 0;                                    // all 512 columns: the allocation starts at 0
  Walk<N>& w = s_walk[warp];
  if (lane == 0) {
    w.it = s_place->it;
    w.left = cut(s_place->total, blockIdx.x + 1, gridDim.x) - s_place->unit;
    w.started = 0;
    w.s = s_place->s;
  }

  if (warp == 0) {
    // --------------------------------------------------------------- producer
    // Batches of up to 16 tiles of a segment: a lane per page.  The ids of a
    // batch are asked for two batches ahead, the scales one batch ahead.
    struct Batch {
      int hk, tile, n, n_pages;            // n = 0: no batch left
      int id;
      float4 sc;
    };
    int at = 0;                            // tiles of w's segment that are in a batch
    bool more = w.next(a);
    auto take = [&]() {
      while (more && at >= w.nt) {
        more = w.next(a);
        at = 0;
      }
      Batch b{0, 0, 0, 0, -1, make_float4(0.0f, 128.0f, 0.0f, 0.0f)};
      if (!more) return b;
      b.hk = w.it.hk;
      b.tile = w.t0 + at;
      b.n = min(16, w.nt - at);
      b.n_pages = (w.s.len + PT - 1) / PT;
      at += b.n;
      const int page = 2 * b.tile + lane;
      // (a page in front of the window is not there)
      if (lane < 2 * b.n && page >= w.begin / PT && page < b.n_pages) b.id = a.table[static_cast<int64_t>(w.it.b) * a.ld_table + page];
      return b;
    };
    auto scales = [&](Batch& b) {          // a page that is not there: K = V = 0
      if (b.id < 0 || b.id >= a.pages) return;
      const int64_t p = static_cast<int64_t>(b.id) * a.n_kv + b.hk;
      const float v = a.sv[p];
      b.sc = make_float4(a.sk[p], v * 128.0f, v > 0.0f ? log2f(v) : 0.0f, 0.0f);   // (a page of zeros may have a scale of 0)
    };
    Batch now = take();
    scales(now);
    Batch next = take();
    int g = 0;
    bool ok = true;
    while (ok && now.n > 0) {
      scales(next);
      const Batch after = take();
      for (int i = 0; i < now.n; ++i, ++g) {
        const int p0 = __shfl_sync(0xffffffffu, now.id, 2 * i), p1 = __shfl_sync(0xffffffffu, now.id, 2 * i + 1);
        const int st = g % NST;
        if (!warp_wait_bounded(&kv_empty[st], ((g / NST) & 1) ^ 1, abort_flag, a.status)) { ok = false; break; }
        // the converters are done with tile g - NST, so the softmax is with tile g - 16
        if ((lane >> 1) == i) s_scale[(g & 15) * 2 + (lane & 1)] = now.sc;
        __syncwarp();
        if (lane == 0) {
          const bool two = 2 * (now.tile + i) + 1 < now.n_pages;   // an id out of range lies outside the map: zeros arrive
          uint8_t* dst = sKV + st * C::STAGE_BYTES;
          mbar_arrive_expect_tx(&kv_full[st], two ? 4 * PB : 2 * PB);
          tma_load_4d(dst, &tmK, &kv_full[st], 0, 0, now.hk, p0);
          tma_load_4d(dst + 2 * PB, &tmV, &kv_full[st], 0, 0, now.hk, p0);
          if (two) {
            tma_load_4d(dst + PB, &tmK, &kv_full[st], 0, 0, now.hk, p1);
            tma_load_4d(dst + 3 * PB, &tmV, &kv_full[st], 0, 0, now.hk, p1);
          }
        }
        __syncwarp();
      }
      now = next;
      next = after;
    }
    // every copy started here has landed before the CTA may exit (g tiles were issued in ring order)
    volatile int never = 0;
    for (int i = max(0, g - NST); i < g; ++i) mbar_wait_bounded(&kv_full[i % NST], (i / NST) & 1, &never, a.status);
  } else if (warp == 1) {
    // --------------------------------------------------------------- MMA issuer
    constexpr uint32_t idesc_hi = idesc_f8_f32(128, N, false), idesc_lo = idesc_f8_f32(128, N, true), idesc_o = idesc_f16_f32(128, N, true);
    const uint32_t q_lo = desc_k(smem_u32(sQ)), k_lo = desc_k(smem_u32(sKV)), p_lo = desc_mn(smem_u32(sP));
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || warp_wait_bounded(bar, parity, abort_flag, a.status);
    };
    uint32_t st = 0, turn = 0, tile = 0;                      // ring place and its parity; tiles so far
    int seg = 0;
    bool ok = true;
    while (ok && w.next(a)) {
      const int nt = uniform(w.nt);
      if (nt == 0) continue;
      const int qb = seg & 1;
      if (!wait(&q_full[qb], (seg >> 1) & 1)) break;
      ++seg;
      const uint32_t q0 = q_lo + qb * (C::Q_BYTES >> 4);
      for (int i = 0; i <= nt; ++i, ++tile) {
        if (i < nt) {
          // S^T of this tile; its buffer was read before p_full of two tiles ago, which PV has waited for
          const uint32_t sb = tile & 1, s = tmem + C::S_COL + sb * 64, k0 = k_lo + st * (C::STAGE_BYTES >> 4);
          if (!wait(&kv_full[st], turn)) { ok = false; break; }
          tc_fence_after();
          umma_f8_ss<HD / 32>(s, k0, q0, kRows8Hi<HD>, idesc_hi, 0);
          umma_f8_ss<HD / 32>(s, k0, q0 + (C::QT_BYTES >> 4), kRows8Hi<HD>, idesc_lo, 1);
          umma_commit(&s_full[sb]);
          umma_commit(&kv_empty[st]);
          if (i == nt - 1) umma_commit(&q_empty[qb]);
          if (++st == NST) st = 0, turn ^= 1;
        }
        if (i >= 1) {
          const uint32_t t = tile - 1, pb = t & 1, parity = (t >> 1) & 1;
          const uint32_t v = tmem + C::V_COL + pb * 64, p0 = p_lo + pb * (C::P_BYTES >> 4);
          if (!wait(&vt_full[pb], parity) || !wait(&p_full[pb], parity)) { ok = false; break; }
          tc_fence_after();
          umma4_ts_mn(tmem + C::O_COL, v, p0, idesc_o, i != 1);
          umma4_ts_mn(tmem + C::O_COL, v + 32, p0 + 512, idesc_o, 1);
          umma_commit(o_full);
          umma_commit(&vt_empty[pb]);
          if (i == nt) umma_commit(o_done);
        }
      }
      --tile;                                                 // the last round of a segment has no tile of its own
    }
    umma_commit(drain);
    volatile int never = 0;
    warp_wait_bounded(drain, 0, &never, a.status);
  } else if (warp >= 4 && warp < 8) {
    // --------------------------------------------------------------- converters
    const int row = (warp & 3) * 32 + lane;                   // dim of V^T
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    int g = 0;
    bool ok = true;
    while (ok && w.next(a)) {
      const int nt = w.nt, keys = w.s.len - w.t0 * TK;        // keys from the segment's start on
      for (int i = 0; i < nt; ++i, ++g) {
        const int st = g % NST, sb = g & 1;
        const uint32_t again = ((g >> 1) & 1) ^ 1;
        const uint8_t* base = sKV + st * C::STAGE_BYTES;
        if (!warp_wait_bounded(&kv_full[st], (g / NST) & 1, abort_flag, a.status)) { ok = false; break; }
        {
          if (!warp_wait_bounded(&vt_empty[sb], again, abort_flag, a.status)) { ok = false; break; }
          tc_fence_after();
          if (HD == 128 || row < 64) {                        // hd 64: lanes 64 .. 127 of V^T stay as they are, unread
            const int valid = keys - i * TK;                  // keys of this tile that exist
            if (a.window > 0 && i == 0) hide_front<PB>(sKV + st * C::STAGE_BYTES + 2 * PB, row, w.begin - w.t0 * TK);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const uint8_t* line = base + (2 + c) * PB + row * PT;
              uint32_t out[32];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint4 x = *reinterpret_cast<const uint4*>(line + ((j ^ ((row >> 1) & 3)) << 4));
                uint32_t v[4] = {x.x, x.y, x.z, x.w};
                if (valid < TK) {
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const int n = valid - (64 * c + 16 * j + 4 * e);
                    v[e] &= n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
                  }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) e4m3x4_f16x4(v[e], out[8 * j + 2 * e], out[8 * j + 2 * e + 1]);
              }
              tmem_st32(tmem + lane_off + C::V_COL + sb * 64 + 32 * c, out);
            }
          }
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(&vt_full[sb]);
        }
        warp_arrive(&kv_empty[st]);
      }
    }
  } else if (warp < 4) {
    // --------------------------------------------------------------- Q
    // N rows, each scaled by a power of four so that its largest value is in 2^6 .. 2^8, in an e4m3 and an e5m2 term
    // (rolled loops: this runs once per item, straight-line code would wait for its instructions)
    constexpr int CPR = HD / 8, QV = N * CPR / 64;            // groups of 8 dims per row, per thread
    const int tid = threadIdx.x - 64;
    int seg = 0;
    bool more = w.next(a);
    while (more && w.nt == 0) more = w.next(a);
    // the rows of an item: one box where its tiles hold whole rows of the sequence (what lies behind the sequence's end
    // comes along and is not used), else row by row
    auto fetch = [&]() {
      const int v0 = w.it.rt * N, rows = min(N, w.s.n_virt - v0);
      if (warp == 2 && N % a.group == 0) {
        if (lane == 0) {
          mbar_arrive_expect_tx(raw_full, N * HD * 2);
          tma_load_3d(sRaw, &tmQ, raw_full, 0, w.it.hk * a.group, w.s.first + by_group(a, v0));
        }
        __syncwarp();
      } else if (warp == 2) {
        if (lane == 0) mbar_arrive_expect_tx(raw_full, rows * HD * 2);
        __syncwarp();
        for (int r = lane; r < rows; r += 32) {
          const int t = by_group(a, v0 + r);
          bulk_load(sRaw + r * HD * 2, a.q + (w.s.first + t) * a.ldq + static_cast<int64_t>(w.it.hk * a.group + v0 + r - t * a.group) * HD,
                    HD * 2, raw_full);
        }
      }
      return rows;
    };
    while (more) {
      const int qb = seg & 1, rows = fetch();
      bool ok = warp_wait_bounded(raw_full, seg & 1, abort_flag, a.status);
      // the largest magnitude of each row, infinities and NaN (an exponent of ones) aside: 64 / N threads per row, which
      // begin at different groups (and banks)
      constexpr int TPR = 64 / N;
      const int own = tid / TPR;
      uint32_t m = 0;
#pragma unroll 4
      for (int i = 0; i < QV; ++i) {
        uint4 q = reinterpret_cast<const uint4*>(sRaw)[own * CPR + (TPR * (i + own) + tid % TPR) % CPR];
        if (own >= rows) q = make_uint4(0, 0, 0, 0);
        auto finite = [](uint32_t w) { return w & 0x7fff7fffu & ~__vcmpgeu2(w & 0x7fff7fffu, 0x7f807f80u); };
        m = __vmaxu2(m, __vmaxu2(__vmaxu2(finite(q.x), finite(q.y)), __vmaxu2(finite(q.z), finite(q.w))));
      }
      uint32_t top = max(m & 0xffff0000u, m << 16);
#pragma unroll
      for (int o = 1; o < TPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int e_max = max(static_cast<int>(top >> 23), 40) - 127;      // 2^e_max <= the largest
      s_unit[(seg & 3) * N + own] = static_cast<uint8_t>((e_max - 7 + 127) >> 1);
      asm volatile("barrier.cta.sync 8, 64;" ::: "memory");
      ok = warp_wait_bounded(&q_empty[qb], ((seg >> 1) & 1) ^ 1, abort_flag, a.status) && ok;
#pragma unroll 4
      for (int i = 0; i < QV; ++i) {
        const int c = i * 64 + tid, r = c / CPR, ch = c % CPR;
        uint4 q = reinterpret_cast<const uint4*>(sRaw)[c];
        if (r >= rows) q = make_uint4(0, 0, 0, 0);
        const float q_up = __int_as_float((253 - 2 * s_unit[(seg & 3) * N + r]) << 23);
        const uint64_t up2 = f2_pack(q_up, q_up);
        const uint32_t x[4] = {q.x, q.y, q.z, q.w};
        uint32_t term[2][2] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // each value rounded to four significant bits, then the rest: at most 8 times the last place of the value's
          // eight bits, which has three (and 0 v, a NaN where v is infinite: the conversions would saturate)
          const uint64_t v = f2_mul(f2_pack(__uint_as_float(x[e] << 16), __uint_as_float(x[e] & 0xffff0000u)), up2);
          float2 f;
          f2_unpack(v, f.x, f.y);
          const uint32_t p = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
          f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(p), __NV_E4M3)));
          f2_unpack(f2_fma(v, f2_pack(0.0f, 0.0f), f2_fma(f2_pack(f.x, f.y), f2_pack(-1.0f, -1.0f), v)), f.x, f.y);
          const uint32_t l = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E5M2);
          term[0][e >> 1] |= p << (16 * (e & 1));
          term[1][e >> 1] |= l << (16 * (e & 1));
        }
        uint8_t* dst = sQ + qb * C::Q_BYTES + chunk_at<HD>(r, ch >> 1) + (ch & 1) * 8;
#pragma unroll
        for (int k = 0; k < 2; ++k) *reinterpret_cast<uint2*>(dst + k * C::QT_BYTES) = make_uint2(term[k][0], term[k][1]);
      }
      fence_proxy_async_smem();
      warp_arrive(&q_full[qb]);
      ++seg;
      // both warps have read the exponents and the rows, and they go on or leave together
      uint32_t leave;
      asm volatile(
          "{\n\t.reg .pred a, b;\n\t"
          "setp.ne.u32 a, %1, 0;\n\t"
          "barrier.cta.red.or.pred b, 8, 64, a;\n\t"
          "selp.u32 %0, 1, 0, b;\n\t}"
          : "=r"(leave)
          : "r"(static_cast<uint32_t>(!ok))
          : "memory");
      if (leave) break;
      more = w.next(a);
      while (more && w.nt == 0) more = w.next(a);
    }
    volatile int never = 0;                                   // the rows have landed (a warp that gave up)
    if (seg > 0) mbar_wait_bounded(raw_full, (seg - 1) & 1, &never, a.status);
  } else {
    // --------------------------------------------------------------- softmax
    constexpr int RN = C::RN;
    const int tid = (threadIdx.x - 256) & 127, sw = warp - 8;  // of the group of four warps that share rows
    const int key_lane = (warp & 3) * 32 + lane;              // this thread's key in a tile = its TMEM lane
    const int grp = sw >> 2, row0 = grp * RN;                 // its rows: row0 .. row0 + RN - 1
    const int own = row0 + tid;                               // thread tid < RN keeps row `own`'s reference
    float* my_red = s_red + (sw & 3) * N + row0;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    int g = 0, seg = 0;
    bool ok = true;
    while (ok && w.next(a)) {
      const int v0 = w.it.rt * N;
      if (tid < RN) {
        const int v = v0 + own;
        const bool in = v < w.s.n_virt;
        const int r = by_group(a, v), pos = w.s.pos0 + r;
        s_row[own] = in ? (w.s.first + r) * a.ldo + static_cast<int64_t>(w.it.hk * a.group + v - r * a.group) * HD : -1;
        s_see[own] = make_int2(in && a.window > 0 ? pos - a.window + 1 : 0,
                               in && a.causal ? min(w.s.len, pos + 1) : w.s.len);
        s_negm[own] = 0.0f;
      }
      if (w.nt == 0) {                                        // no key: zeros
        bar_group<128>(1 + grp);
        for (int r = row0; r < row0 + RN; ++r)
          if (s_row[r] >= 0 && tid < HD) a.o[s_row[r] + tid] = __float2bfloat16_rn(0.0f);
        bar_group<128>(1 + grp);
        continue;
      }
      bar_group<128>(1 + grp);
      // rows whose bounds cut a tile: every key below `all_lo` or from `all_hi` on is hidden from some row
      const int last_v = min(v0 + N, w.s.n_virt) - 1;
      const int all_hi = a.causal ? min(w.s.len, w.s.pos0 + by_group(a, v0) + 1) : w.s.len;
      const int all_lo = a.window > 0 ? w.s.pos0 + by_group(a, last_v) - a.window + 1 : 0;

      float l[RN];
#pragma unroll
      for (int r = 0; r < RN; ++r) l[r] = 0.0f;
      bool has_ref = false;                                   // of row `own`
      bool unset = true;                                      // some row has no reference yet (the warps agree)
      const int nt = w.nt, t0 = w.t0;
      for (int i = 0; i < nt; ++i) {
        const int t = g + i, sb = t & 1, tile = t0 + i;
        if (!warp_wait_bounded(&s_full[sb], (t >> 1) & 1, abort_flag, a.status)) { ok = false; }
        // the warps vote below: all of them leave together
        tc_fence_after();
        const float4 sc = s_scale[(t & 15) * 2 + (key_lane >> 6)];
        const float lv = sc.z;
        const int key = tile * TK + key_lane;
        const bool masked = tile * TK < all_lo || (tile + 1) * TK > all_hi;
        float x[RN], mx = -INFINITY;
        tmem_ld16(tmem + lane_off + C::S_COL + sb * 64 + row0, x);
        const float ks = sc.x * a.scale_log2;
        const uint64_t ks2 = f2_pack(ks, ks);
#pragma unroll
        for (int r = 0; r < RN; r += 4) {
          const ulonglong2 nm = *reinterpret_cast<const ulonglong2*>(s_negm + row0 + r);
          const uint32_t un = *reinterpret_cast<const uint32_t*>(s_unit + (seg & 3) * N + row0 + r);
          auto unit = [&](int k) { return __uint_as_float(__byte_perm(un, 0x00800000u, 0x0644 | k << 12)); };
          f2_unpack(f2_fma(f2_pack(x[r], x[r + 1]), f2_mul(f2_pack(unit(0), unit(1)), ks2), nm.x), x[r], x[r + 1]);
          f2_unpack(f2_fma(f2_pack(x[r + 2], x[r + 3]), f2_mul(f2_pack(unit(2), unit(3)), ks2), nm.y), x[r + 2], x[r + 3]);
        }
        if (masked) {
#pragma unroll
          for (int r = 0; r < RN; ++r) {
            const int2 see = s_see[row0 + r];
            x[r] = key >= see.x && key < see.y ? x[r] : -INFINITY;
          }
        }
#pragma unroll
        for (int r = 0; r < RN; r += 2) mx = fmax3(mx, x[r], x[r + 1]);
        if (vote_group<128>(1 + grp, unset || mx + lv > 8.0f || !ok)) {
          // ---- some row exceeds its reference (or has none): new references, O and the sums follow
          if (*abort_flag) ok = false;
          float m = -INFINITY;
#pragma unroll
          for (int r = 0; r < RN; ++r) {
            const float top = warp_top(x[r] + lv);
            m = lane == r ? top : m;
          }
          if (lane < RN) my_red[lane] = m;
          bar_group<128>(1 + grp);
          bool none = false;
          if (tid < RN) {
            const float rel = fmaxf(fmaxf(s_red[own], s_red[N + own]), fmaxf(s_red[2 * N + own], s_red[3 * N + own]));
            float f = 1.0f, d = 0.0f;                         // factor of O and l, step of the reference
            if (!has_ref) {                                   // O and l of the row are still zero
              none = rel == -INFINITY;
              has_ref = !none;
              d = none ? 0.0f : rel;
            } else if (rel > 8.0f) {
              d = rel;
              f = ex2_approx(-rel);
            }
            s_negm[own] -= d;
            s_fac[own] = f;
            s_red[own] = d;                                   // its four inputs have been read by this thread alone
          }
          unset = vote_group<128>(1 + grp, none);
#pragma unroll
          for (int r = 0; r < RN; ++r) x[r] -= s_red[row0 + r];
          if (i > 0) {
            // O holds the segment's tiles up to i - 1 once their PV is complete (all but the last are: S of this tile
            // was issued behind them)
            if (!warp_wait_bounded(o_full, (t - 1) & 1, abort_flag, a.status)) ok = false;
            tc_fence_after();
            float y[RN];
            tmem_ld16(tmem + lane_off + C::O_COL + row0, y);
#pragma unroll
            for (int r = 0; r < RN; ++r) y[r] *= s_fac[row0 + r];
            tmem_st16(tmem + lane_off + C::O_COL + row0, y);
            tmem_wait_st();
#pragma unroll
            for (int r = 0; r < RN; ++r) l[r] *= s_fac[row0 + r];
          }
          if (vote_group<128>(1 + grp, !ok)) { ok = false; break; }       // also: s_fac and s_red may be written again
        }
        // ---- P = 2^x times the page's V scale, f16, a 128-byte line per key
        const uint64_t vs2 = f2_pack(sc.y, sc.y);
        uint8_t* line = sP + sb * C::P_BYTES + key_lane * 128;
#pragma unroll
        for (int r = 0; r < RN; r += 8) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p0 = ex2_approx(x[r + 2 * e]), p1 = ex2_approx(x[r + 2 * e + 1]);
            f2_unpack(f2_add(f2_pack(l[r + 2 * e], l[r + 2 * e + 1]), f2_pack(p0, p1)), l[r + 2 * e], l[r + 2 * e + 1]);
            float y0, y1;
            f2_unpack(f2_mul(f2_pack(p0, p1), vs2), y0, y1);
            const __half2 q = __floats2half2_rn(y0, y1);
            h[e] = *reinterpret_cast<const uint32_t*>(&q);
          }
          *reinterpret_cast<uint4*>(line + ((((row0 + r) >> 3) ^ (key_lane & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        warp_arrive(&p_full[sb]);
      }
      if (!ok) break;
      g += nt;
      // ---- the rows' sums, then O
      const float l_row = sum_rows(l);
      if (lane < RN) my_red[lane] = l_row;
      bar_group<128>(1 + grp);
      if (tid < RN) {
        const float s = (s_red[own] + s_red[N + own]) + (s_red[2 * N + own] + s_red[3 * N + own]);
        if (w.from_start && w.to_end) {
          s_fac[own] = s == 0.0f ? 0.0f : 1.0f / (s * 128.0f);
        } else {
          const int64_t slot = 2LL * blockIdx.x + w.from_start;   // at most one part of each kind per CTA
          a.part_ml[slot * N + own] = make_float2(s == 0.0f ? -INFINITY : -s_negm[own], s * 128.0f);
        }
      }
      // o_done, not o_full: the PV ahead of the last one may still be running as well
      ok = warp_wait_bounded(o_done, seg & 1, abort_flag, a.status);
      ++seg;
      tc_fence_after();
      bar_group<128>(1 + grp);
      if (ok && (HD == 128 || key_lane < HD)) {               // warp-uniform: a dim per thread
        const bool direct = w.from_start && w.to_end;
        float* part = a.part_o + ((2LL * blockIdx.x + w.from_start) * N + row0) * HD + key_lane;
#pragma unroll 1
        for (int c = 0; c < RN; c += 8) {
          float y[8];
          tmem_ld8(tmem + lane_off + C::O_COL + row0 + c, y);
          if (direct) {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const int64_t at = s_row[row0 + c + r];
              const float f = s_fac[row0 + c + r];
              if (at >= 0) a.o[at + key_lane] = __float2bfloat16_rn(y[r] * f);
            }
          } else {
#pragma unroll
            for (int r = 0; r < 8; ++r) part[(c + r) * HD] = y[r];
          }
        }
      }
      tc_fence_before();
      if (vote_group<128>(1 + grp, !ok)) {                            // also: s_row, s_see, s_negm and s_fac may be written again
        ok = false;
        break;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Merges the partials of an item that the cut between two CTAs splits first:
// m* = max m_s, O = sum 2^(m_s - m*) O_s / sum 2^(m_s - m*) l_s, in the order
// of the CTAs.  Block (c - 1, y) has the cut ahead of CTA c and takes four of
// the item's rows, a warp each.  6 to 8 us by itself, which are latency (places,
// sums, partials); part of it passes while the last CTAs end.
template <int HD, int N>
__global__ void __launch_bounds__(128) merge_paged_kernel(const PagedArgs a, int ctas) {
  pdl_enter();
  const int c = blockIdx.x + 1, lane = threadIdx.x & 31, r = blockIdx.y * 4 + (threadIdx.x >> 5);
  const Place pl = a.place[c];
  const Item it = pl.it;
  if (it.off == 0 || cut(pl.total, c + 1, ctas) == pl.unit) return;   // no item is split here, or CTA c has no units
  const int64_t first = pl.unit - it.off;                     // the item's first unit
  int k = c - 1;                                              // the CTA that ends at this cut
  while (k > 0 && cut(pl.total, k, ctas) == pl.unit) --k;
  if (cut(pl.total, k, ctas) > first) return;                 // an earlier cut splits the item first
  const SeqInfo s = pl.s;
  const int v = it.rt * N + r, row = by_group(a, v);
  if (v >= s.n_virt) return;
  const int64_t nt = pl.nt;
  if (it.off >= nt) return;                                   // its tiles end ahead of the cut
  constexpr int PL = HD / 32;
  float m = -INFINITY, l = 0.0f, acc[PL] = {};
  // four parts are asked for at a time; a CTA without units has none
  int64_t k0 = cut(pl.total, k, ctas);
  while (k < ctas && k0 < first + nt) {
    float2 ml[4];
    float x[4][PL];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      ml[u] = make_float2(-INFINITY, 0.0f);
      if (k >= ctas || k0 >= first + nt) continue;
      const int64_t k1 = cut(pl.total, k + 1, ctas);
      if (k0 < k1) {
        const int64_t slot = 2LL * k + (k0 <= first);
        ml[u] = a.part_ml[slot * N + r];
        const float* p = a.part_o + (slot * N + r) * HD + lane * PL;
#pragma unroll
        for (int d = 0; d < PL; ++d) x[u][d] = p[d];
      }
      k0 = k1;
      ++k;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (ml[u].x == -INFINITY) continue;                     // it saw no key
      const float mn = fmaxf(m, ml[u].x), f = ex2_approx(m - mn), h = ex2_approx(ml[u].x - mn);
      l = l * f + ml[u].y * h;
#pragma unroll
      for (int d = 0; d < PL; ++d) acc[d] = acc[d] * f + x[u][d] * h;
      m = mn;
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16* o = a.o + (s.first + row) * a.ldo + static_cast<int64_t>(it.hk * a.group + v - row * a.group) * HD + lane * PL;
#pragma unroll
  for (int d = 0; d < PL; d += 2) *reinterpret_cast<__nv_bfloat162*>(o + d) = __floats2bfloat162_rn(acc[d] * inv, acc[d + 1] * inv);
}

// uint8 map {d0, d1, n_kv, pages}, dense, box {d0, d1, 1, 1}, swizzled by its row
bool page_map(CUtensorMap* m, const void* ptr, uint32_t d0, uint32_t d1, uint64_t n_kv, uint64_t pages) {
  const cuuint64_t dims[4] = {d0, d1, n_kv, pages};
  const cuuint64_t strides[3] = {d0, static_cast<uint64_t>(d0) * d1, static_cast<uint64_t>(d0) * d1 * n_kv};
  const cuuint32_t box[4] = {d0, d1, 1, 1}, estr[4] = {1, 1, 1, 1};
  return tensor_map_encoder()(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(ptr), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, d0 == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// bf16 map {hd, heads, rows}, box {hd, group, n / group}, not swizzled
bool q_map(CUtensorMap* m, const void* ptr, int hd, int heads, int total, int64_t ld, int group, int n) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(total)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(hd) * 2, static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(hd), static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(n / group)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return tensor_map_encoder()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Virtual rows of a tile: the least of 16, 32, 64 that holds a sequence's rows of one KV head (64: several tiles).  Single
// tokens of 16 / 8 heads, 4 over 60,000 cached ones each and 32 over 4000: 109 and 72 us with 16, 111 and 74 with 32, 118 and
// 83 with 64; 8 x 16 rows over 8000: 46 with 32, 53 with 64.
int tile_rows(int max_rows, int group) {
  const int64_t v = static_cast<int64_t>(max_rows) * group;
  return v <= 16 ? 16 : v <= 32 ? 32 : 64;
}

template <int HD, int N>
const char* launch(const RaggedCall& c, cudaStream_t s) {
  using C = PagedCfg<HD, N>;
  if (!tensor_map_encoder()) return "cuTensorMapEncodeTiled is unavailable";
  int dev = 0;
  const int ctas = current_sms(&dev);
  static PerDevice ready;
  if (ready.get(dev, [] {
        return cudaFuncSetAttribute(attn_paged_kernel<HD, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) ==
                       cudaSuccess ? 1 : 0;
      }) <= 0)
    return "attention smem attribute failed";
  const tadm_page_pool& p = *c.pool;
  const int64_t at = static_cast<int64_t>(c.layer) * p.pages * p.n_kv_heads;
  const int group = c.n_heads / c.n_kv;
  CUtensorMap mq{}, mk, mv;
  if ((N % group == 0 && !q_map(&mq, c.q, HD, c.n_heads, c.total, c.ldq, group, N)) ||
      !page_map(&mk, static_cast<const uint8_t*>(p.k) + at * PT * HD, HD, PT, p.n_kv_heads, p.pages) ||
      !page_map(&mv, static_cast<const uint8_t*>(p.v) + at * PT * HD, PT, HD, p.n_kv_heads, p.pages))
    return "page tensor map encode failed";
  float* part = static_cast<float*>(c.scratch);
  const PagedArgs a{static_cast<const bf16*>(c.q), static_cast<bf16*>(c.o), p.k_scale + at, p.v_scale + at,
                    c.cu, c.lens, c.table, c.batch, c.total, c.max_rows, c.max_len, c.ld_table, p.pages,
                    group, c.n_kv, 0xffffffffu / static_cast<uint32_t>(group),
                    c.ldq, c.ldo, c.causal, c.window,
                    1.4426950408889634f / sqrtf(static_cast<float>(HD)), part,
                    reinterpret_cast<float2*>(part + 2LL * ctas * N * HD),
                    reinterpret_cast<Place*>(part + 2LL * ctas * N * (HD + 2)), c.status};
  cudaError_t e = launch_pdl(attn_paged_kernel<HD, N>, ctas, C::THREADS, C::SMEM, s, mq, mk, mv, a);
  if (e == cudaSuccess && ctas > 1)
    e = launch_pdl(merge_paged_kernel<HD, N>, dim3(ctas - 1, N / 4), 128, 0, s, a, ctas);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace

size_t attention_paged_scratch(int max_rows, int group, int head_dim) {
  int dev = 0;
  return static_cast<size_t>(current_sms(&dev)) *
         (2ull * tile_rows(max_rows, group) * (head_dim + 2) * sizeof(float) + sizeof(Place));
}

const char* attention_paged(const RaggedCall& c, cudaStream_t s) {
  auto hd = [&](auto n) {
    constexpr int N = decltype(n)::value;
    return c.head_dim == 128 ? launch<128, N>(c, s) : launch<64, N>(c, s);
  };
  switch (tile_rows(c.max_rows, c.n_heads / c.n_kv)) {
    case 16: return hd(std::integral_constant<int, 16>{});
    case 32: return hd(std::integral_constant<int, 32>{});
    default: return hd(std::integral_constant<int, 64>{});
  }
}

}  // namespace tadm
