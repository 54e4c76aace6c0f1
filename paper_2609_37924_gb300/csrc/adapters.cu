// Projections with an adapter per request, bf16, tcgen05:
//
//   y[t] = W x[t] + B_a h[t],   h[t] = scale_a A_a x[t],   a: the adapter of row t's sequence
//
// One GEMM whose K goes on behind n_in: a tile of 256 rows has the adapters
// of its rows (few of them for prompts, one per row for single tokens), and
// behind the k-blocks of x and W come blocks of h and B.  A block's columns
// of h belong to one adapter and are zero in the rows of the others, so that
// any mix of adapters in a tile is the same dense product:
//
//   y_tile = [x | h_a1 | h_a2 ...] [W | B_a1 | B_a2 ...]^T
//
// h is carried as three bf16 terms, each the rounding of what the ones before
// leave of it, that multiply the same 16 columns of B: 24 bits, h as fp32 has
// it, for 3 x 16 more steps of K per 16 ranks.  (With two, 16 bits, y was off by
// up to 2^-18 of an adapter's part: of the bf16 outputs of prompts 1.55 in 1000
// were not the nearest to the exact value instead of 1.16, which are as many as
// of rows without an adapter, from the matrix unit's sums, which truncate.)
// The terms of four groups of 16 ranks lie one behind the other in three blocks.
//
// Two launches:
//   lora_down_kernel    each cluster finds the adapters of its tile's rows, then x A^T for
//                       128 rows and eight groups of 16 ranks of the tile's
//                       list (M = 128, N = 128), K split over the blocks of the
//                       cluster, whose partial sums are added in the order of K
//                       through distributed shared memory; scale, mask, hi, lo;
//   lora_gemm_kernel    the product, CTA pairs (M = 256): persistent over tiles,
//                       or, where there are few, K (and the blocks of h and B)
//                       split over the two pairs of a cluster likewise.
// lora_gemm_kernel needs of its predecessor only h and the lists: its blocks of
// x and W run ahead of the grid dependency (when it starts, every block of
// its predecessor has waited for what came before, so x and W are there).
//
// Bound: of prompts the tensor pipe (24 prompts, 5874 rows, 2048 -> 4096, 6
// adapters of rank 16: 74 us, of which the product 63 at 83 % of the pipe; the
// FLOP alone are 52); of few rows the chain of the two kernels: h
// after 10 us (lists 2, x A^T 2 to 5, sums 3), then its blocks (64 tokens, 40 adapters:
// 24.6 us; 256 rows, 5376 -> 8192, rank 64: 38.3, of which W's 88 MB are 13).  Blocks of
// h and B cost 0.4 us each against 0.25 of x and W: B comes in rows of 32 bytes.
// Tried, with h in two terms: tiles of 192 columns (prompts 77 us where 256 took 64), of 128 (100); K over the four pairs of a cluster of 8 (only 15 of those run at once,
// 36 us for the tokens); h as the first units of the product's own kernel, with a
// counter per tile that the others wait for (tokens 21, prompts 68, 256 rows 34 us: no
// gain that is worth a wait between blocks).
#include <algorithm>
#include <cstdint>

#include "ragged.cuh"
#include "requests.h"
#include "tensor_map.h"

namespace tadm {

namespace {

constexpr int TR = 256;                    // rows of a tile
constexpr int BK = 64;
constexpr int G = 16;                      // ranks of a group
constexpr int TERMS = 3;                   // of h
constexpr int PLACES = BK / G;             // of a block of h: term i of group g is at place TERMS g + i of the tile's blocks
constexpr int KB_BYTES = TR * BK * 2;      // a block of h
__host__ __device__ constexpr int blocks_of(int groups) { return (TERMS * groups + PLACES - 1) / PLACES; }
__host__ __device__ constexpr int first_group(int block) { return PLACES * block / TERMS; }
__host__ __device__ constexpr int last_group(int block, int groups) {
  const int last = (PLACES * block + PLACES - 1) / TERMS;
  return last < groups ? last : groups - 1;
}
static_assert(PLACES <= TERMS + 1, "a block has terms of two groups at most");

// What the first kernel leaves for the second, and its place in the scratch memory.
struct Plan {
  int32_t* n_ad;                           // [tiles] adapters of the tile
  int32_t* base;                           // [tiles] first block of h
  int32_t* list;                           // [tiles][cap]
  bf16* h;                                 // [slots][TR][64]
  int tiles, cap, slots, groups;           // cap: most adapters of a tile; groups: of 16 ranks per adapter
  int by_seq, step;                        // where a tile's blocks of h begin: `step` for each sequence in front, or for each tile
};
size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }
Plan make_plan(int batch, int total, int n_adapters, int rank, uint8_t* scratch, size_t* bytes) {
  Plan p{};
  p.tiles = (total + TR - 1) / TR;
  p.groups = (rank + G - 1) / G;
  p.cap = std::max(1, std::min(std::min(TR, batch), n_adapters));
  // blocks of h: a tile has at most cap adapters; all tiles together at most as many as there are sequences and tiles
  const int per_tile = blocks_of(p.cap * p.groups), per_seq = blocks_of(p.groups);
  const int64_t by_tile = static_cast<int64_t>(p.tiles) * per_tile, by_seq = (static_cast<int64_t>(batch) + p.tiles) * per_seq;
  p.by_seq = by_seq < by_tile;
  p.step = p.by_seq ? per_seq : per_tile;
  const int64_t slots = std::min(by_tile, by_seq);
  p.slots = static_cast<int>(std::min<int64_t>(slots, INT32_MAX / TR));   // (more of them are refused: kLoraMaxScratch)
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at = up(at + n, 1024);
    return scratch + here;
  };
  p.n_ad = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * p.tiles));
  p.base = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * p.tiles));
  p.list = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * p.tiles * static_cast<size_t>(p.cap)));
  p.h = reinterpret_cast<bf16*>(take(static_cast<size_t>(slots) * KB_BYTES));
  if (bytes) *bytes = at + 1024;           // the blocks start on 1024 bytes, scratch on 16
  return p;
}

// ------------------------------------------------------------------ shared pieces
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* map, uint32_t cluster_bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(cluster_bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ float4 remote_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// Waits for the kernel before this one, without letting the next one start.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// K-major bf16 tile with rows of 16 elements, 32-byte swizzle: 256 bytes from one 8-row group to the next
__device__ __forceinline__ uint64_t sdesc_rows32(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | 1ull << 16 | static_cast<uint64_t>(256 >> 4) << 32 | 1ull << 46 | 6ull << 61;
}

// ------------------------------------------------------------------ h = scale A x
constexpr int D_STAGES = 4, D_GROUPS = 8, D_N = D_GROUPS * G;
constexpr int D_X_BYTES = 128 * BK * 2, D_A_BYTES = D_N * BK * 2, D_STAGE_BYTES = D_X_BYTES + D_A_BYTES;
constexpr int D_THREADS = 192, TABLE = 4096, CACHE = 4096;
static_assert((TABLE + 2 * CACHE + 1) * 4 <= 128 * D_N * 4, "the lists are made where the sums come later");
constexpr int D_SMEM = 1024 + D_STAGES * D_STAGE_BYTES + 128 * D_N * 4 + 2 * TR * 4 + 256;

struct DownArgs {
  Plan p;
  const int32_t *cu, *adapter;
  const float* scale;
  int batch, total, n_adapters, kblocks;
  int* status;
};

// The adapters of tile `tile`'s rows (s_row: -1 none) and the list of them in the order of their first rows (s_list); returns
// how many.  Block-collective; `room`: scratch of TABLE + 2 CACHE + 1 words.
__device__ __forceinline__ int make_lists(const DownArgs& a, int tile, int32_t* room, int32_t* s_row, int32_t* s_list, int* first_seq) {
  int32_t *s_first = room, *s_ad = room + TABLE, *s_cu = s_ad + CACHE;
  const bool cached = a.batch <= CACHE, table = a.n_adapters <= TABLE;
  if (table)
    for (int j = threadIdx.x; j < a.n_adapters; j += D_THREADS) s_first[j] = TR;
  if (cached)
    for (int j = threadIdx.x; j <= a.batch; j += D_THREADS) {
      s_cu[j] = a.cu[j];
      if (j < a.batch) s_ad[j] = a.adapter[j];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < TR; i += D_THREADS) {
    const int row = tile * TR + i;
    const int32_t* cu = cached ? s_cu : a.cu;
    int lo = 0, hi = a.batch + 1;          // boundaries <= row: in lo .. hi
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      if (cu[mid] <= row) lo = mid + 1;
      else hi = mid;
    }
    const int b = lo - 1;
    int ad = -1;
    if (row < a.total && b >= 0 && b < a.batch) {
      ad = cached ? s_ad[b] : a.adapter[b];
      if (ad < 0 || ad >= a.n_adapters) ad = -1;
    }
    if (i == 0) *first_seq = max(b, 0);
    s_row[i] = ad;
    if (table && ad >= 0) atomicMin(&s_first[ad], i);
  }
  __syncthreads();
  // every warp counts all, the first one writes the list
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int n = 0;
  for (int i = lane; i < TR; i += 32) {
    const int ad = s_row[i];
    bool first = ad >= 0;
    if (table) {
      first = first && s_first[ad] == i;
    } else {
      for (int j = 0; j < i && first; ++j) first = s_row[j] != ad;
    }
    const unsigned have = __ballot_sync(0xffffffffu, first);
    const int at = n + __popc(have & ((1u << lane) - 1));
    if (warp == 0 && first) s_list[at] = ad;
    n += __popc(have);
  }
  __syncthreads();
  return min(n, a.p.cap);
}

// A cluster has a half of a tile (128 rows) and every so many of its eights of groups.
template <int CS>
__global__ void __launch_bounds__(D_THREADS, 1)
    lora_down_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmA, const DownArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float4* s_d = reinterpret_cast<float4*>(smem + D_STAGES * D_STAGE_BYTES);   // [D_N / 4][128 rows]
  int32_t *s_row = reinterpret_cast<int32_t*>(s_d + 128 * D_N / 4), *s_list = s_row + TR;
  uint64_t* full = reinterpret_cast<uint64_t*>(s_list + TR);
  uint64_t *empty = full + D_STAGES, *done = empty + D_STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_seq = reinterpret_cast<int*>(tmem_slot + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CS > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < D_STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(done, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmA);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, D_N);
    tmem_relinquish();
  }
  pdl_enter();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int kb0 = a.kblocks * rank / CS, kb1 = a.kblocks * (rank + 1) / CS;
  int stage = 0, loads = 0;
  uint32_t phase = 0, done_phase = 0;
  bool any = false;
  const int clusters = gridDim.x / CS, halves = (a.total + 127) / 128, per = max(1, clusters / halves);   // clusters of a half
  for (int th = blockIdx.x / CS % (per * halves) % halves, c0 = blockIdx.x / CS / halves; th < halves && c0 < per; th += clusters) {
    const int t = th >> 1, half = th & 1, row0 = th * 128;
    const int n_list = make_lists(a, t, reinterpret_cast<int32_t*>(s_d), s_row, s_list, s_seq);
    const int base = min((a.p.by_seq ? *s_seq + t : t) * a.p.step, a.p.slots);
    // (sequences that overlap or run backwards may ask for more blocks of h than there are: none past the last is touched)
    const int n_ad = min(n_list, PLACES * (a.p.slots - base) / (TERMS * a.p.groups)), all = n_ad * a.p.groups;
    if (half == 0 && c0 == 0 && rank == 0) {
      if (threadIdx.x == 0) {
        a.p.n_ad[t] = n_ad;
        a.p.base[t] = base;
      }
      for (int i = threadIdx.x; i < n_ad; i += D_THREADS) a.p.list[static_cast<int64_t>(t) * a.p.cap + i] = s_list[i];
    }
    for (int g0 = c0 * D_GROUPS; g0 < all; g0 += per * D_GROUPS) {
      const int ng = min(D_GROUPS, all - g0);
      float scale = 0.0f;                  // lane i of the summing warps: of group i
      if (warp == 0) {
        // (lane i: group i)
        const int ad = lane < ng ? s_list[(g0 + lane) / a.p.groups] : 0, at = (g0 + lane) % a.p.groups * G;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!warp_wait_bounded(&empty[stage], phase ^ 1, abort_flag, a.status)) break;
          uint8_t* sx = smem + stage * D_STAGE_BYTES;
          if (lane == 0) {
            mbar_arrive_expect_tx(&full[stage], D_X_BYTES + ng * G * BK * 2);
            tma_load_2d(sx, &tmX, &full[stage], kb * BK, row0);
          }
          __syncwarp();
          if (lane < ng) tma_load_3d(sx + D_X_BYTES + lane * G * BK * 2, &tmA, &full[stage], kb * BK, at, ad);
          loads = min(loads + 1, D_STAGES);
          if (++stage == D_STAGES) { stage = 0; phase ^= 1; }
        }
      } else if (warp == 1) {
        const uint32_t idesc = idesc_bf16_f32(128, ng * G);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!warp_wait_bounded(&full[stage], phase, abort_flag, a.status)) break;
          tc_fence_after();
          const uint64_t x0 = sdesc_kmajor_sw128(smem_u32(smem + stage * D_STAGE_BYTES));
          const uint64_t a0 = sdesc_kmajor_sw128(smem_u32(smem + stage * D_STAGE_BYTES + D_X_BYTES));
#pragma unroll
          for (int k = 0; k < BK / 16; ++k) umma_bf16(tmem, x0 + 2 * k, a0 + 2 * k, idesc, kb != kb0 || k != 0);
          umma_commit(&empty[stage]);
          if (++stage == D_STAGES) { stage = 0; phase ^= 1; }
        }
        umma_commit(done);
      } else {
        const int quad = warp & 3;
        if (lane < ng) scale = a.scale[s_list[(g0 + lane) / a.p.groups]];
        const bool ok = warp_wait_bounded(done, done_phase, abort_flag, a.status) && !*abort_flag;
        tc_fence_after();
        for (int c = 0; c < ng; ++c) {
          float v[16];
          __syncwarp();
          if (ok && kb1 > kb0) {
            tmem_ld16(tmem + c * G + (static_cast<uint32_t>(quad * 32) << 16), v);
          } else {
            for (int e = 0; e < 16; ++e) v[e] = ok ? 0.0f : NAN;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q)
            s_d[(c * 4 + q) * 128 + quad * 32 + lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
        tc_fence_before();
      }
      done_phase ^= 1;
      any = true;
      __syncwarp();
      if constexpr (CS > 1) cluster_sync();
      else __syncthreads();
      if (warp >= 2) {
        // this block's share of the groups: the sum in the order of K, then a row's 32 bytes of each term
        const int r = (warp - 2) * 32 + lane, mine = s_row[half * 128 + r];
        for (int c = rank; c < ng; c += CS) {
          float v[16];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int p = 0; p < CS; ++p) {
              const float4 x = CS > 1 ? remote_f4(cluster_addr(&s_d[(c * 4 + q) * 128 + r], p)) : s_d[(c * 4 + q) * 128 + r];
              s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
            }
            v[4 * q] = s.x, v[4 * q + 1] = s.y, v[4 * q + 2] = s.z, v[4 * q + 3] = s.w;
          }
          const int ad = s_list[(g0 + c) / a.p.groups];
          const float by = __shfl_sync(0xffffffffu, scale, c);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = mine == ad ? v[e] * by : 0.0f;
#pragma unroll
          for (int i = 0; i < TERMS; ++i) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
              v[2 * e] -= __low2float(h), v[2 * e + 1] -= __high2float(h);
              w[e] = *reinterpret_cast<const uint32_t*>(&h);
            }
            const int place = TERMS * (g0 + c) + i;
            uint4* out = reinterpret_cast<uint4*>(a.p.h + (static_cast<int64_t>(base + place / PLACES) * TR + half * 128 + r) * BK + place % PLACES * G);
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
            out[1] = make_uint4(w[4], w[5], w[6], w[7]);
          }
        }
      }
      __syncwarp();
      if constexpr (CS > 1) cluster_sync();                   // the partial sums may be written again, blocks may leave
      else __syncthreads();
    }
    __syncthreads();                                          // (the lists are read no more)
  }
  // (after a wait that gave up: the copies have landed and the MMAs are through before the block ends)
  volatile int never = 0;
  if (warp == 0) {
    for (; loads > 0; --loads) {
      if (stage == 0) { stage = D_STAGES; phase ^= 1; }
      --stage;
      warp_wait_bounded(&full[stage], phase, &never, a.status);
    }
  } else if (warp == 1) {
    if (any) warp_wait_bounded(done, done_phase ^ 1, &never, a.status);
    tc_fence_after();
    tmem_dealloc(tmem, D_N);
  }
}

// ------------------------------------------------------------------ the product
constexpr int E_WARPS = 8, BOX_BYTES = 32 * 128, G_THREADS = 64 + 32 * E_WARPS;

template <int BN>
struct GemmCfg {
  static constexpr int A_BYTES = 128 * BK * 2, B_BYTES = BN / 2 * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int EXT_BYTES = BN / 2 * G * 2;            // 16 columns of B for this CTA's half of the tile's columns
  static constexpr int STAGES = BN == 128 ? 8 : 6;
  static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + E_WARPS * BOX_BYTES + 256;
  static_assert(SMEM <= 232448 && STAGES * STAGE_BYTES >= 128 * BN * 4 && 2 * EXT_BYTES <= B_BYTES, "shared memory");
};

struct GemmArgs {
  Plan p;
  const int32_t* cu;
  void* y;
  int64_t ldy;
  int batch, total, n_out, kblocks, n_tiles_n, m_fast, y_bf16, y_vec;
  int* status;
};

// 32 rows and 32 columns (n0 on) of the warp: v, a lane's row, through its box to y; whole 16-byte pieces where rows and columns
// allow them, else element by element.  Rows r_lo .. r_hi - 1 of all are written.
template <class YT>
__device__ __forceinline__ void store32x32(const GemmArgs& a, uint8_t* box, const float (&v)[32], int row0, int n0, int r_lo, int r_hi) {
  constexpr int PER = 16 / sizeof(YT), PIECES = 32 / PER, ROW = 32 * sizeof(YT);
  const int lane = threadIdx.x & 31;
  // piece q of row r lies at q ^ swz(r): eight lanes that write 16 bytes, or read them, meet all banks
  auto swz = [](int r) { return PIECES == 8 ? r & 7 : (r >> 1) & 3; };
  __syncwarp();
#pragma unroll
  for (int q = 0; q < PIECES; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(YT) == 4) {
        w[e] = __float_as_uint(v[4 * q + e]);
      } else {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[8 * q + 2 * e], v[8 * q + 2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&t);
      }
    }
    *reinterpret_cast<uint4*>(box + lane * ROW + ((q ^ swz(lane)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __syncwarp();
  YT* y = static_cast<YT*>(a.y);
  if (a.y_vec && n0 + 32 <= a.n_out) {
    constexpr int ROWS = 32 / PIECES;                          // of one store instruction
    const int q = lane % PIECES;
#pragma unroll
    for (int i = 0; i < 32 / ROWS; ++i) {
      const int r = i * ROWS + lane / PIECES, m = row0 + r;
      const uint4 t = *reinterpret_cast<const uint4*>(box + r * ROW + ((q ^ swz(r)) << 4));
      if (m >= r_lo && m < r_hi) *reinterpret_cast<uint4*>(y + m * a.ldy + n0 + q * PER) = t;
    }
  } else if (n0 + lane < a.n_out) {
    for (int r = 0; r < 32; ++r) {
      const int m = row0 + r;
      if (m >= r_lo && m < r_hi)
        y[m * a.ldy + n0 + lane] = *reinterpret_cast<const YT*>(box + r * ROW + (((lane / PER) ^ swz(r)) << 4) + lane % PER * sizeof(YT));
    }
  }
}

// KS: pairs of a cluster, which share a tile's k-blocks.
template <int BN, int KS>
__global__ void __launch_bounds__(G_THREADS, 1)
    lora_gemm_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
                     const __grid_constant__ CUtensorMap tmH, const __grid_constant__ CUtensorMap tmB, const GemmArgs a) {
  using C = GemmCfg<BN>;
  constexpr int NST = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *sA = smem, *sB = smem + NST * C::A_BYTES, *boxes = smem + NST * C::STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(boxes + E_WARPS * BOX_BYTES);
  uint64_t *empty = full + NST, *tfull = empty + NST, *tempty = tfull + 2, *drain = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int crank = static_cast<int>(cluster_ctarank()), half = crank & 1, pair = crank >> 1;
  const uint32_t lead = static_cast<uint32_t>(crank & ~1);    // the pair's even block
  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], 2 * E_WARPS);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmW);
  }
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // tiles with rows of a sequence (buffers may be longer)
  const int r_lo = max(a.cu[0], 0), r_hi = min(a.cu[a.batch], a.total), t0 = r_lo / TR;
  const int tiles = r_hi > r_lo ? (r_hi + TR - 1) / TR - t0 : 0;
  const int units = tiles * a.n_tiles_n, u0 = blockIdx.x / (2 * KS), ustep = gridDim.x / (2 * KS);
  auto place = [&](int u, int& mt, int& nt) {
    if (a.m_fast) {
      nt = u / tiles;
      mt = t0 + u - nt * tiles;
    } else {
      mt = u / a.n_tiles_n;
      nt = u - mt * a.n_tiles_n;
      mt += t0;
    }
  };
  const int k0 = a.kblocks * pair / KS, k1 = a.kblocks * (pair + 1) / KS;   // this pair's blocks of x and W (at least one)
  auto share = [&](int mt, int& e0, int& e1) {                // and of h and B; returns the tile's groups
    const int groups = a.p.n_ad[mt] * a.p.groups, blocks = blocks_of(groups);
    e0 = blocks * pair / KS;
    e1 = blocks * (pair + 1) / KS;
    return groups;
  };

  if (warp == 0) {
    const uint32_t full_l = cluster_addr(full, lead);
    int stage = 0;
    uint32_t phase = 0;
    bool waited = false;
    for (int u = u0; u < units && !*abort_flag; u += ustep) {
      int mt, nt;
      place(u, mt, nt);
      const int n0 = nt * BN + half * (BN / 2);
      bool ok = true;
      for (int kb = k0; kb < k1; ++kb) {
        if (!(ok = warp_wait_bounded(&empty[stage], phase ^ 1, abort_flag, a.status))) break;
        if (lane == 0) {
          const uint32_t bar = full_l + 8u * stage;
          if (!half) mbar_arrive_expect_tx(&full[stage], 2 * C::STAGE_BYTES);
          tma_load_2d_pair(sB + stage * C::B_BYTES, &tmW, bar, kb * BK, n0);
          tma_load_2d_pair(sA + stage * C::A_BYTES, &tmX, bar, kb * BK, mt * TR + half * 128);
        }
        if (++stage == NST) { stage = 0; phase ^= 1; }
      }
      if (!ok) break;
      if (!waited) {                       // h and the lists come from the kernel before
        pdl_enter();
        waited = true;
      }
      int e0, e1;
      const int groups = share(mt, e0, e1), base = a.p.base[mt];
      const int32_t* list = a.p.list + static_cast<int64_t>(mt) * a.p.cap;
      int ad = 0, g32 = -32;               // lane i: the adapter of group g32 + i
      for (int kb = e0; kb < e1; ++kb) {
        const int g = first_group(kb), ng = last_group(kb, groups) - g + 1;
        if (g + 1 >= g32 + 32) {
          g32 = g;
          ad = g + lane < groups ? list[(g + lane) / a.p.groups] : 0;
        }
        const int mine = __shfl_sync(0xffffffffu, ad, g - g32 + (lane & 1));
        if (!(ok = warp_wait_bounded(&empty[stage], phase ^ 1, abort_flag, a.status))) break;
        const uint32_t bar = full_l + 8u * stage;
        if (lane == 0) {
          if (!half) mbar_arrive_expect_tx(&full[stage], 2 * (C::A_BYTES + ng * C::EXT_BYTES));
          tma_load_2d_pair(sA + stage * C::A_BYTES, &tmH, bar, 0, (base + kb) * TR + half * 128);
        }
        __syncwarp();
        if (lane < ng)
          tma_load_3d_pair(sB + stage * C::B_BYTES + lane * C::EXT_BYTES, &tmB, bar, (g + lane) % a.p.groups * G, n0, mine);
        if (++stage == NST) { stage = 0; phase ^= 1; }
      }
      if (!ok) break;
    }
    if (!waited) pdl_enter();              // (every block waits before it lets the next kernel start)
    // every stage released: all copies into this block's memory have landed and been read
    for (int i = 0; i < NST; ++i) {
      warp_wait_bounded(&empty[stage], phase ^ 1, abort_flag, a.status);
      if (++stage == NST) { stage = 0; phase ^= 1; }
    }
  } else if (warp == 1) {
    if (!half) {
      constexpr uint32_t idesc = idesc_bf16_f32(2 * 128, BN);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      for (int u = u0; u < units; u += ustep) {
        int mt, nt;
        place(u, mt, nt);
        if (!warp_wait_bounded(&tempty[acc], acc_phase ^ 1, abort_flag, a.status)) break;
        tc_fence_after();
        const uint32_t d = tmem + acc * BN;
        bool ok = true;
        for (int kb = k0; kb < k1; ++kb) {
          if (!warp_wait_bounded(&full[stage], phase, abort_flag, a.status)) { ok = false; break; }
          tc_fence_after();
          const uint64_t a0 = sdesc_kmajor_sw128(smem_u32(sA + stage * C::A_BYTES));
          const uint64_t b0 = sdesc_kmajor_sw128(smem_u32(sB + stage * C::B_BYTES));
#pragma unroll
          for (int k = 0; k < BK / 16; ++k) umma_bf16_pair(d, a0 + 2 * k, b0 + 2 * k, idesc, kb != k0 || k != 0);
          umma_commit_pair_mc(&empty[stage], 0x3 << lead);
          if (++stage == NST) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        grid_wait();
        int e0, e1;
        const int groups = share(mt, e0, e1);
        for (int kb = e0; kb < e1; ++kb) {
          if (!warp_wait_bounded(&full[stage], phase, abort_flag, a.status)) { ok = false; break; }
          tc_fence_after();
          const uint64_t a0 = sdesc_kmajor_sw128(smem_u32(sA + stage * C::A_BYTES));
          for (int i = 0, place = PLACES * kb; i < PLACES && place < TERMS * groups; ++i, ++place)
            umma_bf16_pair(d, a0 + 2 * i, sdesc_rows32(smem_u32(sB + stage * C::B_BYTES + (place / TERMS - first_group(kb)) * C::EXT_BYTES)), idesc, 1);
          umma_commit_pair_mc(&empty[stage], 0x3 << lead);
          if (++stage == NST) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        umma_commit_pair_mc(&tfull[acc], 0x3 << lead);
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
      umma_commit_pair_mc(drain, 0x1 << lead);
      volatile int never = 0;
      warp_wait_bounded(drain, 0, &never, a.status);
    }
  } else {
    const int quad = warp & 3, part = (warp - 2) / 4;         // 32 rows, half of the columns
    uint8_t* box = boxes + (warp - 2) * BOX_BYTES;
    const uint32_t tempty_l = cluster_addr(tempty, lead), lanes = static_cast<uint32_t>(quad * 32) << 16;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int u = u0; u < units; u += ustep) {
      int mt, nt;
      place(u, mt, nt);
      const int row0 = mt * TR + half * 128 + quad * 32;
      const bool ok = warp_wait_bounded(&tfull[acc], acc_phase, abort_flag, a.status);
      tc_fence_after();
      const uint32_t d = tmem + acc * BN + lanes;
      float v[32];
      if constexpr (KS == 1) {
        if (!ok) break;
        if (row0 < r_hi && row0 + 32 > r_lo) {
          for (int c = part * (BN / 64); c < (part + 1) * (BN / 64); ++c) {
            if (nt * BN + 32 * c >= a.n_out) break;
            __syncwarp();
            tmem_ld32(d + 32 * c, v);
            if (a.y_bf16) store32x32<bf16>(a, box, v, row0, nt * BN + 32 * c, r_lo, r_hi);
            else store32x32<float>(a, box, v, row0, nt * BN + 32 * c, r_lo, r_hi);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(tempty_l + 8u * acc);
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      } else {
        // this pair's share of the sum, for the others: [columns / 4][128 rows] over the stages, which all have been read
        float4* s_d = reinterpret_cast<float4*>(smem);
        if (row0 < r_hi && row0 + 32 > r_lo) {
          for (int c = part * (BN / 64); c < (part + 1) * (BN / 64); ++c) {
            __syncwarp();
            if (ok) {
              tmem_ld32(d + 32 * c, v);
            } else {
              for (int e = 0; e < 32; ++e) v[e] = NAN;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q)
              s_d[(c * 8 + q) * 128 + quad * 32 + lane] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          }
        }
        break;                             // (a cluster has one tile)
      }
    }
  }
  if constexpr (KS > 1) {
    tc_fence_before();
    __syncwarp();
    cluster_sync();
    if (warp >= 2 && u0 < units) {
      // this block's share of the columns, summed over the pairs in the order of K
      constexpr int COLS = BN / KS;
      int mt, nt;
      place(u0, mt, nt);
      const int quad = warp & 3, part = (warp - 2) / 4, row0 = mt * TR + half * 128 + quad * 32;
      uint8_t* box = boxes + (warp - 2) * BOX_BYTES;
      const float4* s_d = reinterpret_cast<const float4*>(smem);
      if (row0 < r_hi && row0 + 32 > r_lo) {
        for (int c = part; c < COLS / 32; c += 2) {
          const int col = pair * COLS + 32 * c;
          if (nt * BN + col >= a.n_out) break;
          float v[32];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int p = 0; p < KS; ++p) {
              const float4 x = remote_f4(cluster_addr(&s_d[(col / 4 + q) * 128 + quad * 32 + lane], 2 * p + half));
              s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
            }
            v[4 * q] = s.x, v[4 * q + 1] = s.y, v[4 * q + 2] = s.z, v[4 * q + 3] = s.w;
          }
          if (a.y_bf16) store32x32<bf16>(a, box, v, row0, nt * BN + col, r_lo, r_hi);
          else store32x32<float>(a, box, v, row0, nt * BN + col, r_lo, r_hi);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                          // no block frees TMEM or leaves while others may still reach it
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// ------------------------------------------------------------------ host
bool make_map(CUtensorMap* m, const void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
              CUtensorMapSwizzle swizzle) {
  const auto encode = tensor_map_encoder();
  const cuuint32_t step[3] = {1, 1, 1};
  return encode && encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(p), dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool rows_map(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld * 2)};
  const cuuint32_t box[2] = {BK, static_cast<cuuint32_t>(box_rows)};
  return make_map(m, p, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// [n][rows][cols] dense, a box of box_cols x box_rows of one of the n
bool adapter_map(CUtensorMap* m, const void* p, int n, int64_t rows, int64_t cols, int box_cols, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(n)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(cols * 2), static_cast<cuuint64_t>(rows * cols * 2)};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 1};
  return make_map(m, p, 3, dims, strides, box, box_cols == BK ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_32B);
}

template <class... KArgs, class... Args>
cudaError_t launch_cluster(void (*kernel)(KArgs...), int blocks, int cluster, int threads, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <int CS>
cudaError_t launch_down(const CUtensorMap& x, const CUtensorMap& w, const DownArgs& a, int clusters, int dev, cudaStream_t s) {
  static PerDevice ready;
  cudaError_t e = cudaSuccess;
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(lora_down_kernel<CS>, cudaFuncAttributeMaxDynamicSharedMemorySize, D_SMEM);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return e;
  return launch_cluster(lora_down_kernel<CS>, clusters * CS, CS, D_THREADS, D_SMEM, s, x, w, a);
}

// Clusters of the GEMM that run at once on the current device; <= 0: its shared memory cannot be had.
template <int BN, int KS>
int gemm_clusters(int dev, int sms, cudaError_t* e) {
  static PerDevice fit;
  return fit.get(dev, [&] {
    *e = cudaFuncSetAttribute(lora_gemm_kernel<BN, KS>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmCfg<BN>::SMEM);
    if (*e != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(sms / (2 * KS) * 2 * KS);
    cfg.blockDim = dim3(G_THREADS);
    cfg.dynamicSmemBytes = GemmCfg<BN>::SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 * KS, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, lora_gemm_kernel<BN, KS>, &cfg) != cudaSuccess || n <= 0) {
      cudaGetLastError();
      n = sms / (2 * KS);
    }
    return n;
  });
}

struct Maps {
  CUtensorMap x, w, h, b;
};
template <int BN, int KS>
cudaError_t launch_gemm(const LoraCall& c, Maps& m, GemmArgs a, int dev, int sms, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  const int fit = gemm_clusters<BN, KS>(dev, sms, &e);
  if (fit <= 0) return e;
  if (!rows_map(&m.w, c.w, c.n_out, c.n_in, c.ldw, BN / 2) ||
      !(c.n_adapters > 0 ? adapter_map(&m.b, c.b, c.n_adapters, c.n_out, c.rank, G, BN / 2) : rows_map(&m.b, c.x, c.total, c.n_in, c.ldx, 128)))
    return cudaErrorInvalidValue;
  a.n_tiles_n = (c.n_out + BN - 1) / BN;
  const int64_t units = static_cast<int64_t>(a.p.tiles) * a.n_tiles_n;
  const int clusters = static_cast<int>(KS > 1 ? units : std::min<int64_t>(units, fit));
  return launch_cluster(lora_gemm_kernel<BN, KS>, clusters * 2 * KS, 2 * KS, G_THREADS, GemmCfg<BN>::SMEM, s, m.x, m.w, m.h, m.b, a);
}

}  // namespace

size_t lora_scratch(int batch, int total, int n_in, int n_out, int n_adapters, int rank, int bf16) {
  if (!bf16) return lora_rows_scratch(total, rank);
  size_t bytes = 0;
  make_plan(batch, total, n_adapters, rank, nullptr, &bytes);
  return bytes;
}

const char* lora_project(const LoraCall& c, cudaStream_t s) {
  if (!c.bf16) return lora_rows(c, s);
  int dev = 0;
  const int sms = current_sms(&dev);
  uint8_t* scratch = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(c.scratch) + 1023) & ~uintptr_t(1023));
  const Plan p = make_plan(c.batch, c.total, c.n_adapters, c.rank, scratch, nullptr);
  const int kblocks = (c.n_in + BK - 1) / BK;
  Maps m;
  CUtensorMap ta;
  if (!rows_map(&m.x, c.x, c.total, c.n_in, c.ldx, 128) || !rows_map(&m.h, p.h, static_cast<int64_t>(p.slots) * TR, BK, BK, 128) ||
      !(c.n_adapters > 0 ? adapter_map(&ta, c.a, c.n_adapters, c.rank, c.n_in, BK, G) : rows_map(&ta, c.x, c.total, c.n_in, c.ldx, 128)))
    return "tensor map encode failed";
  // h: at most so many products of 128 rows and 128 ranks; K is split over a cluster's blocks while SMs would stay idle
  const int halves = (c.total + 127) / 128;
  const int64_t most = halves * ((static_cast<int64_t>(c.n_adapters > 0 ? p.cap : 0) * p.groups + D_GROUPS - 1) / D_GROUPS);
  int cs = 1;
  while (cs < 8 && most * cs * 2 <= sms && kblocks >= 4 * cs) cs *= 2;
  const int clusters = static_cast<int>(std::min<int64_t>(std::max<int64_t>(most, halves), sms / cs));
  const DownArgs d{p, c.cu, c.adapter, c.scale, c.batch, c.total, c.n_adapters, kblocks, c.status};
  cudaError_t e = cs == 1 ? launch_down<1>(m.x, ta, d, clusters, dev, s) : cs == 2 ? launch_down<2>(m.x, ta, d, clusters, dev, s)
                : cs == 4 ? launch_down<4>(m.x, ta, d, clusters, dev, s) : launch_down<8>(m.x, ta, d, clusters, dev, s);
  if (e != cudaSuccess) return cudaGetErrorString(e);
  GemmArgs a{};
  a.p = p, a.cu = c.cu, a.y = c.y, a.ldy = c.ldy, a.batch = c.batch, a.total = c.total, a.n_out = c.n_out, a.kblocks = kblocks;
  a.y_bf16 = c.y_bf16, a.status = c.status;
  a.y_vec = (reinterpret_cast<uintptr_t>(c.y) & 15) == 0 && c.ldy * (c.y_bf16 ? 2 : 4) % 16 == 0;
  a.m_fast = static_cast<int64_t>(c.n_out) > c.total;         // the larger operand's tiles are shared through L2
  const int64_t t256 = static_cast<int64_t>(p.tiles) * ((c.n_out + 255) / 256), t128 = static_cast<int64_t>(p.tiles) * ((c.n_out + 127) / 128);
  const bool split = kblocks >= 8;
  if (split && t128 <= gemm_clusters<128, 2>(dev, sms, &e)) e = launch_gemm<128, 2>(c, m, a, dev, sms, s);
  else if (split && t256 <= gemm_clusters<256, 2>(dev, sms, &e)) e = launch_gemm<256, 2>(c, m, a, dev, sms, s);
  else e = launch_gemm<256, 1>(c, m, a, dev, sms, s);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
