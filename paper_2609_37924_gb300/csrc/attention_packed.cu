// Attention of packed bf16 prompts, tcgen05.
//
// A CTA takes one or two tiles of up to 128 virtual rows (as many whole rows of
// one sequence as fit, row-major, then the query heads of one KV head) and
// walks the key tiles that they see, 128 keys each.  Two tiles both use a K or V
// tile while it is in shared memory, and their softmaxes alternate with the
// tensor pipe.  A CTA that is through takes the work of a block of the grid that
// has not started (the hardware hands it out, longest work first), so that the
// next Q, K and first scores come while the last O leaves:
//   warp 0       finds the work and streams Q, K and V tiles with TMA, these
//                into a ring of four slots;
//   warp 1       O_A += P_A V(j), S_A = Q_A K(j+1)^T, then the same for B: one
//                tile's softmax runs while the tensor pipe works on the other,
//                and P V of a tile's first 64 keys while it is at the others;
//   warps 4-7    softmax of tile A, warps 8-11 of tile B: a row per thread.
// P (bf16) lies in TMEM over the scores that it was made from, V is read as it
// lies in memory (a key per line, an MN-major operand).  The reference maximum
// of a row moves only when a tile exceeds it by 2^8; O is rescaled then.
// Key tiles that the mask cuts keep P in two bf16 terms, whose 128 columns are
// those of the scores: a row that sees few keys, or weighs most those next to it,
// does not feel the rounding of single probabilities to 8 bits, 2^-8 of each (one
// term where every row sees 256 keys or more: 129 us instead of 133 under a window
// of 1024, and a row that is all on its own key off by 1.3 times 2^-8).
// What a tile holds behind the sequence's end belongs to its neighbour: those
// scores are masked, and those lines of V are zeroed in shared memory.
//
// Bound: the tensor pipe, 1024 cycles per 128 x 128 tile at hd 128 (the
// exponentials take 512).  Measured: about 1450 per tile, 1.34 PFLOP/s over an
// 8111-token prompt of 32 / 16 heads (450 us with its neighbours; 461 where
// each block starts and ends by itself, and a window of 1024 over 8900 rows 133
// and 157; with 64-key tiles and two S per row tile 587 and 155); prompts of a few hundred tokens are bound by the latency of
// cut tiles and of the first pair, whose code and rows come from memory (24
// prompts, 6400 tokens, 16 / 8 heads: 32 us; 43 with the code of cut tiles
// unrolled over the 128 columns, 36 with the sequences' work in their order).
#include "ragged.cuh"
#include "serve.h"
#include "softmax_rows.cuh"
#include "tensor_map.h"
#include "umma_tiles.cuh"

namespace tadm {
namespace {

constexpr int TQ = 128, TK = 128;

// NT row tiles per CTA
template <int HD_, int NT_>
struct PackedCfg {
  static constexpr int HD = HD_, NT = NT_;
  static constexpr int TILE_BYTES = HD / 64 * 16384;          // HD/64 atoms of 128 rows x 64 dims: a tile of Q, K or V
  static constexpr int SLOTS = 4;
  static constexpr int STAGE_BYTES = 16384;                   // 64 dims of a tile's O on their way out
  static constexpr int MIN_BLOCKS = 3 - NT;
  static constexpr int SMEM = 1024 + (NT + SLOTS) * TILE_BYTES + NT * STAGE_BYTES + 512;
  static constexpr int S_COL = 0, O_COL = NT * TK, TMEM_COLS = NT * 256;   // NT tiles of 128 columns, then of HD
  static constexpr int THREADS = 128 + NT * 128;
  static constexpr int REGS = NT == 2 ? 224 : 200;            // of a softmax thread; the other warps keep 56
  static_assert(56 + NT * REGS <= (NT + 1) * (NT == 2 ? 168 : 128), "registers at launch");
};

struct PackedArgs {
  bf16* o;
  const int32_t* cu;
  int batch, total, max_rows, group, n_kv;
  int tq, rows;            // rows of a sequence in a tile, virtual rows (tq * group <= 128)
  uint32_t group_inv;      // row / group = row * group_inv >> 16 for rows below 128
  int64_t ldo;
  int causal, window;
  float scale_log2;
  int* status;
};

// A pair of row tiles: KV head, first row and row count of the sequence (0: no pair is left), first row of the pair in it.
struct Work {
  int hk, first, n, tok0;
};
// Asks for the index of a block of this grid that has not started, which then never starts: 16 bytes arrive at `resp`,
// counted on the mbarrier.  One thread; not again after next_block() has said that there is none.
__device__ __forceinline__ void ask_block(void* resp, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(resp)),
               "r"(smem_u32(bar))
               : "memory");
}
// The index (blockIdx.x), -1: none is left.
__device__ __forceinline__ int next_block(const void* resp) {
  int x;
  asm volatile(
      "{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t"
      "ld.shared.b128 h, [%1];\n\t"
      "mov.u32 %0, -1;\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, h;\n\t}"
      : "=r"(x)
      : "r"(smem_u32(resp))
      : "memory");
  return x;
}
// P = 2^(s * scale - m) of 32 columns as 16 packed pairs, added to the sums.
__device__ __forceinline__ void exp32_pack(const uint32_t (&r)[32], uint64_t sc2, uint64_t negm2, uint64_t (&ps2)[2],
                                           uint32_t (&pk)[16]) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    float x0, x1;
    f2_unpack(f2_fma(f2_pack(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), sc2, negm2), x0, x1);
    const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
    ps2[j & 1] = f2_add(ps2[j & 1], f2_pack(p0, p1));
    __nv_bfloat162 t = __floats2bfloat162_rn(p0, p1);
    pk[j] = *reinterpret_cast<uint32_t*>(&t);
  }
}
// Columns lo .. lim - 1 of 32, a bit each
__device__ __forceinline__ uint32_t columns(int lo, int lim) {
  const uint32_t below = lim >= 32 ? 0xffffffffu : lim <= 0 ? 0u : (1u << lim) - 1u;
  return below & ~(lo >= 32 ? 0xffffffffu : lo <= 0 ? 0u : (1u << lo) - 1u);
}
// exp32_pack() where only the columns of `see` are visible (else P = 0), with the remainders P - bf16(P) as bf16 pairs.
__device__ __forceinline__ void exp32_masked(const uint32_t (&r)[32], uint64_t sc2, uint64_t negm2, uint32_t see, uint64_t (&ps2)[2],
                                             uint32_t (&pk)[16], uint32_t (&rest)[16]) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    float x0, x1;
    f2_unpack(f2_fma(f2_pack(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), sc2, negm2), x0, x1);
    const float p0 = see >> 2 * j & 1 ? ex2_approx(x0) : 0.0f;
    const float p1 = see >> (2 * j + 1) & 1 ? ex2_approx(x1) : 0.0f;
    ps2[j & 1] = f2_add(ps2[j & 1], f2_pack(p0, p1));
    __nv_bfloat162 t = __floats2bfloat162_rn(p0, p1);
    pk[j] = *reinterpret_cast<uint32_t*>(&t);
    t = __floats2bfloat162_rn(p0 - __uint_as_float(pk[j] << 16), p1 - __uint_as_float(pk[j] & 0xffff0000u));
    rest[j] = *reinterpret_cast<uint32_t*>(&t);
  }
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
      "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

template <int HD_, int NT_>
__global__ void __launch_bounds__(PackedCfg<HD_, NT_>::THREADS, PackedCfg<HD_, NT_>::MIN_BLOCKS)
    attn_packed_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO, const PackedArgs a) {
  using C = PackedCfg<HD_, NT_>;
  constexpr int HD = C::HD, NT = C::NT, NS = C::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                                         // NT tiles
  uint8_t* sKV = sQ + NT * C::TILE_BYTES;                     // ring: K and V tiles in turn
  uint8_t* sO = sKV + NS * C::TILE_BYTES;                     // O of each tile on its way out
  uint64_t* bars = reinterpret_cast<uint64_t*>(sO + NT * C::STAGE_BYTES);
  uint64_t *full = bars, *empty = bars + NS;                  // [NS]
  uint64_t *q_full = bars + 2 * NS, *s_full = q_full + 2, *o_done = q_full + 4;   // [2] by tile
  uint64_t* p_full = q_full + 6;                              // [2][2] by tile, keys 0 .. 63 and 64 .. 127
  uint64_t *drain = q_full + 10, *asked = drain + 1;
  uint64_t* q_empty = drain + 2;                              // [2] by tile
  uint64_t *w_full = drain + 4, *w_empty = drain + 6;         // [2] the pairs of row tiles in turn
  Work* s_work = reinterpret_cast<Work*>(bars + 40);          // [2]
  uint4* s_asked = reinterpret_cast<uint4*>(bars + 44);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 46);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[2 * i], 4);
      mbar_init(&p_full[2 * i + 1], 4);
      mbar_init(&o_done[i], 1);
      mbar_init(&q_empty[i], 1);
      mbar_init(&w_full[i], 1);
      mbar_init(&w_empty[i], 1 + 4 * NT);
    }
    mbar_init(drain, 1);
    mbar_init(asked, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  pdl_enter();
  // the blocks of a pair of row tiles are its KV heads; the pairs that see most keys come first
  auto find = [&](int block) {
    int at;
    const int b = find_largest(a.batch, block / a.n_kv,
                               [&](int i) { return (seq_rows(a.cu, i, a.total, a.max_rows).n + NT * a.tq - 1) / (NT * a.tq); }, &at);
    if (b < 0) return Work{0, 0, 0, 0};
    const SeqRows rows = seq_rows(a.cu, b, a.total, a.max_rows);
    return Work{block % a.n_kv, rows.first, rows.n, at * NT * a.tq};
  };
  const Work first = find(blockIdx.x);
  if (first.n == 0) return;                                   // uniform; nothing allocated or in flight
  if (warp == 1) {
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(static_cast<int>(*tmem_slot));
  // the key tiles of tile h, whose rows of the sequence are tok0 + h tq and on: first and end
  auto range = [&](const Work& w, int h) {
    const int lo = w.tok0 + h * a.tq, hi = min(lo + a.tq, w.n) - 1;
    if (h >= NT || lo >= w.n) return make_int2(0, 0);
    const int end = a.causal ? hi + 1 : w.n;
    const int begin = a.window > 0 ? max(0, lo - a.window + 1) : 0;
    return make_int2(begin / TK, (end + TK - 1) / TK);
  };
  // the keys that every row of tile h sees: [x, y); a key tile that is not inside them is cut by the mask
  auto common = [&](const Work& w, int h) {
    const int lo = w.tok0 + h * a.tq, hi = min(lo + a.tq, w.n) - 1;
    return make_int2(a.window > 0 ? hi - a.window + 1 : 0, a.causal ? lo + 1 : w.n);
  };
  auto partial = [](int2 c, int j) { return (j + 1) * TK > c.y || j * TK < c.x; };
  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == 0) {
    // --------------------------------------------------------------- producer
    // Also finds the pairs: the block's own first, then those of blocks that have not started, so that the loads and first
    // scores of a pair hide behind the end of the one before it and all CTAs end together.
    Work w = first;
    int t = 0, g = 0, qn[2] = {0, 0};                         // pairs; loads into the ring and of each Q (lane 0)
    bool ok = true, asking = false;
    volatile int never = 0;
    for (;; ++t) {
      if (!warp_wait_bounded(&w_empty[t & 1], ((t >> 1) & 1) ^ 1, abort_flag, a.status)) break;
      if (lane == 0) s_work[t & 1] = w;
      warp_arrive(&w_full[t & 1]);
      if (w.n == 0) break;
      const int2 rA = range(w, 0), rB = range(w, 1);
      const bool two = rB.y > 0;
      if (lane == 0) {
        for (int h = 0; ok && h < (two ? 2 : 1); ++h) {       // rows behind the sequence's end are other rows, unused
          ok = mbar_wait_bounded(&q_empty[h], (qn[h] & 1) ^ 1, abort_flag, a.status);
          if (!ok) break;
          ++qn[h];
          mbar_arrive_expect_tx(&q_full[h], HD / 64 * a.rows * 128);
          for (int s = 0; s < HD / 64; ++s)
            tma_load_3d(sQ + h * C::TILE_BYTES + s * 16384, &tmQ, &q_full[h], 64 * s, w.hk * a.group, w.first + w.tok0 + h * a.tq);
        }
        for (int j = rA.x; ok && j < (two ? rB.y : rA.y); ++j)
          for (int m = 0; m < 2; ++m, ++g) {
            const int sl = g % NS;
            if (!mbar_wait_bounded(&empty[sl], ((g / NS) & 1) ^ 1, abort_flag, a.status)) { ok = false; break; }
            mbar_arrive_expect_tx(&full[sl], C::TILE_BYTES);
            for (int s = 0; s < HD / 64; ++s)
              tma_load_3d(sKV + sl * C::TILE_BYTES + s * 16384, m ? &tmV : &tmK, &full[sl], 64 * s, w.hk, w.first + j * TK);
          }
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      // two key tiles before the pair's end: late, so that no CTA keeps a pair waiting that another one could begin
      if (lane == 0) {
        mbar_arrive_expect_tx(asked, 16);
        ask_block(s_asked, asked);
      }
      asking = true;
      if (!warp_wait_bounded(asked, t & 1, abort_flag, a.status)) break;
      asking = false;
      const int block = next_block(s_asked);
      fence_proxy_async_smem();                               // the next answer is written there
      __syncwarp();
      w = block < 0 ? Work{0, 0, 0, 0} : find(block);         // (blocks past the last pair are the grid's last)
    }
    // every copy started here has landed before the CTA may exit
    if (lane == 0) {
      if (asking) mbar_wait_bounded(asked, t & 1, &never, a.status);
      for (int h = 0; h < 2; ++h)
        if (qn[h] > 0) mbar_wait_bounded(&q_full[h], (qn[h] - 1) & 1, &never, a.status);
      for (int i = max(0, g - NS); i < g; ++i) mbar_wait_bounded(&full[i % NS], (i / NS) & 1, &never, a.status);
    }
  } else if (warp == 1) {
    // --------------------------------------------------------------- MMA issuer
    constexpr uint32_t idesc_s = idesc_bf16_f32(TQ, TK), idesc_o = idesc_bf16_f32(TQ, HD) | 1u << 16;   // V: MN-major
    struct Slot {                                             // a place of the ring and the parity of its phase
      uint32_t at, parity;
    };
    auto after = [](Slot s) { return s.at + 1 == NS ? Slot{0, s.parity ^ 1} : Slot{s.at + 1, s.parity}; };
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || warp_wait_bounded(bar, parity, abort_flag, a.status);
    };
    const uint32_t q_lo = desc_k(smem_u32(sQ)), kv_lo = smem_u32(sKV);
    auto scores = [&](int h, Slot s, bool last) {             // S_h = Q_h K^T, the pair's last ones release Q_h
      const uint32_t q0 = q_lo + h * (C::TILE_BYTES >> 4), k0 = desc_k(kv_lo + s.at * C::TILE_BYTES);
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) umma4_ss(tmem + C::S_COL + h * TK, q0 + c * 1024, k0 + c * 1024, idesc_s, c);
      umma_commit(&s_full[h]);
      if (last) umma_commit(&q_empty[h]);
    };
    auto values = [&](int h, Slot s, int n, bool first, bool split) {   // O_h += P_h V, the tile's n-th P
      const uint32_t vd = desc_mn(kv_lo + s.at * C::TILE_BYTES), o = tmem + C::O_COL + h * HD, p = tmem + C::S_COL + h * TK;
      if (!wait(&p_full[2 * h], n & 1)) return false;
      if (split) {
        if (!wait(&p_full[2 * h + 1], n & 1)) return false;
        tc_fence_after();
        for (int c = 0; c < 4; ++c) umma4_ts_two(o, p + 32 * c, vd + 256 * c, idesc_o, c > 0 || !first);
        return true;
      }
      tc_fence_after();
      umma4_ts_mn(o, p, vd, idesc_o, !first);
      if (!wait(&p_full[2 * h + 1], n & 1)) return false;
      tc_fence_after();
      umma4_ts_mn(o, p + 32, vd + 512, idesc_o, 1);
      return true;
    };
    Slot sk{0, 0};                                            // K(j0) of the pair
    bool early = false;                                       // the pair's first scores of tile 0 are issued
    int nA = 0, nB = 0, uB = 0;                               // P's of tiles 0 and 1 ahead of the pair, pairs with a tile 1
    for (int t = 0;; ++t) {
      if (!wait(&w_full[t & 1], (t >> 1) & 1)) break;
      const Work w = s_work[t & 1];
      warp_arrive(&w_empty[t & 1]);
      const int n_keys = uniform(w.n);
      if (n_keys == 0) break;
      const int2 rA = uniform(range(w, 0)), rB = uniform(range(w, 1)), cA = uniform(common(w, 0)), cB = uniform(common(w, 1));
      const bool two = rB.y > 0;
      const int j0 = rA.x, j1 = two ? rB.y : rA.y;            // A's keys begin and end no later than B's
      bool ok = early || (wait(&q_full[0], t & 1) && wait(&full[sk.at], sk.parity));
      if (!ok) break;
      tc_fence_after();
      if (!early) scores(0, sk, j0 + 1 == rA.y);
      early = false;
      if (two) {
        if (!wait(&q_full[1], uB & 1)) break;
        ++uB;
        tc_fence_after();
        if (rB.x == j0) scores(1, sk, j0 + 1 == rB.y);
      }
      umma_commit(&empty[sk.at]);
      for (int j = j0; j < j1; ++j) {
        const Slot sv = after(sk);                            // V(j), then K(j + 1)
        sk = after(sv);
        ok = wait(&full[sv.at], sv.parity) && (j + 1 >= j1 || wait(&full[sk.at], sk.parity));
        if (!ok) break;
        const int valid = n_keys - j * TK;
        if (valid < TK) {                                     // the lines of V behind the sequence's end
          uint8_t* sV = sKV + sv.at * C::TILE_BYTES;
          for (int i = lane; i < (TK - valid) * 8; i += 32)
#pragma unroll
            for (int s = 0; s < HD / 64; ++s) *reinterpret_cast<uint4*>(sV + s * 16384 + valid * 128 + i * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after();
        if (j < rA.y) {
          ok = values(0, sv, nA + j - j0, j == j0, partial(cA, j));
          if (!ok) break;
          if (j == rA.y - 1) umma_commit(&o_done[0]);
        }
        if (!two) umma_commit(&empty[sv.at]);
        if (j + 1 < rA.y) scores(0, sk, j + 2 == rA.y);
        if (two) {
          if (j + 1 == j1) {                                  // tile 0 of the next pair, if its Q and K are here, ahead of tile 1's last P
            const uint32_t u = t + 1;
            const Slot next = after(sv);
            early = __all_sync(0xffffffffu, mbar_test(&w_full[u & 1], (u >> 1) & 1) && s_work[u & 1].n > 0 &&
                                                mbar_test(&q_full[0], u & 1) && mbar_test(&full[next.at], next.parity));
            if (early) {
              tc_fence_after();
              const int2 r = uniform(range(s_work[u & 1], 0));
              scores(0, next, r.x + 1 == r.y);
            }
          }
          if (j >= rB.x) {                                    // (j < rB.y: B's keys end last)
            ok = values(1, sv, nB + j - rB.x, j == rB.x, partial(cB, j));
            if (!ok) break;
            if (j == rB.y - 1) umma_commit(&o_done[1]);
          }
          umma_commit(&empty[sv.at]);
          if (j + 1 >= rB.x && j + 1 < rB.y) scores(1, sk, j + 2 == rB.y);
        }
        if (j + 1 < j1) umma_commit(&empty[sk.at]);
      }
      if (!ok) break;
      nA += rA.y - rA.x;
      nB += rB.y - rB.x;
    }
    umma_commit(drain);
    volatile int never = 0;
    warp_wait_bounded(drain, 0, &never, a.status);
  } else if (warp >= 4) {
    // --------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS));
    const int h = (warp >> 2) - 1, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(quad * 32) << 16;
    const int in_tile = static_cast<int>(row * a.group_inv >> 16);
    const uint32_t t_s = tmem + lane_off + C::S_COL + h * TK, t_o = tmem + lane_off + C::O_COL + h * HD;
    const uint64_t sc2 = f2_pack(a.scale_log2, a.scale_log2);
    uint8_t* stage = sO + h * C::STAGE_BYTES;
    int n = 0, used = 0;                                      // scores so far, pairs with this tile
    for (int t = 0;; ++t) {
      bool ok = warp_wait_bounded(&w_full[t & 1], (t >> 1) & 1, abort_flag, a.status);
      if (vote_group<128>(1 + h, !ok)) break;                   // the four warps of a tile leave together
      const Work w = s_work[t & 1];
      warp_arrive(&w_empty[t & 1]);
      if (w.n == 0) break;
      const int2 r = range(w, h);
      if (r.y == 0) continue;
      const int tok = w.tok0 + h * a.tq + in_tile;
      const bool v_ok = row < a.rows && tok < w.n;
      const int pos = v_ok ? tok : 0;
      const int see_hi = !v_ok ? 0 : a.causal ? pos + 1 : w.n, see_lo = a.window > 0 ? pos - a.window + 1 : 0;
      // O of a row is scaled by `factor` (and its sum): the tiles before this one are complete, their PV was issued ahead
      // of this tile's S
      float m_ref = -INFINITY, l_run = 0.0f;
      auto rescale = [&](float factor) {
#pragma unroll
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t ro[32];
          tmem_ld32_nowait(t_o + 32 * c, ro);
          tmem_wait_ld(ro);
#pragma unroll
          for (int k = 0; k < 32; ++k) ro[k] = __float_as_uint(__uint_as_float(ro[k]) * factor);
          tmem_st32(t_o + 32 * c, ro);
        }
        l_run *= factor;
      };
      const int2 all = common(w, h);
      for (int j = r.x; j < r.y; ++j, ++n) {
        if (!warp_wait_bounded(&s_full[h], n & 1, abort_flag, a.status)) { ok = false; break; }
        tc_fence_after();
        uint64_t ps2[2] = {0, 0};
        // the new reference, from the tile's largest score; O and the sum follow
        auto refer = [&](float m_tile) {
          float factor = 1.0f;
          if (m_ref == -INFINITY) {
            m_ref = m_tile;                                   // every earlier exponential was 0
          } else if (m_tile > m_ref + 8.0f) {
            factor = ex2_approx(m_ref - m_tile);
            m_ref = m_tile;
          }
          if (__any_sync(0xffffffffu, factor != 1.0f)) rescale(factor);
          const float negm = m_ref == -INFINITY ? 0.0f : -m_ref;   // (scores of minus infinity alone weigh nothing)
          return f2_pack(negm, negm);
        };
        if (partial(all, j)) {
          // A cut tile: 32 columns at a time, twice (the maximum, the exponentials), and those that no row of the warp sees
          // are left out.  Rolled, because it runs once or twice per tile of rows and would wait for its instructions.
          // P goes over the scores that it was made from: two terms of 16 columns for 32.
          const int lim = see_hi - j * TK, lo = see_lo - j * TK;   // visible columns of this tile: [lo, lim)
          uint32_t s[32], pk[16], rest[16];
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            const uint32_t see = columns(lo - 32 * c, lim - 32 * c);
            if (!__any_sync(0xffffffffu, see != 0)) continue;
            tmem_ld32_nowait(t_s + 32 * c, s);
            tmem_wait_ld(s);
#pragma unroll
            for (int k = 0; k < 32; k += 2)
              top[(k >> 1) & 3] = fmax3(top[(k >> 1) & 3], see >> k & 1 ? __uint_as_float(s[k]) : -INFINITY,
                                        see >> (k + 1) & 1 ? __uint_as_float(s[k + 1]) : -INFINITY);
          }
          const uint64_t negm2 = refer(fmax3(fmaxf(top[0], top[1]), top[2], top[3]) * a.scale_log2);
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            const uint32_t see = columns(lo - 32 * c, lim - 32 * c);
            if (__any_sync(0xffffffffu, see != 0)) {
              tmem_ld32_nowait(t_s + 32 * c, s);
              tmem_wait_ld(s);
              exp32_masked(s, sc2, negm2, see, ps2, pk, rest);
            } else {
#pragma unroll
              for (int k = 0; k < 16; ++k) pk[k] = rest[k] = 0;
            }
            tmem_st16(t_s + 32 * c, pk);
            tmem_st16(t_s + 32 * c + 16, rest);
          }
        } else {
          // the row's scores stay in registers: P is written over them in TMEM
          uint32_t s[4][32], pk[16];
          tmem_ld32_nowait(t_s, s[0]);
          tmem_ld32_nowait(t_s + 32, s[1]);
          tmem_wait_ld(s[0]);
          tmem_bind(s[1]);
          tmem_ld32_nowait(t_s + 64, s[2]);
          tmem_ld32_nowait(t_s + 96, s[3]);
          float mxa[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          max64<false>(s[0], s[1], 0, 64, mxa);
          tmem_wait_ld(s[2]);
          tmem_bind(s[3]);
          max64<false>(s[2], s[3], 0, 64, mxa);
          const uint64_t negm2 = refer(fmax3(fmaxf(mxa[0], mxa[1]), mxa[2], mxa[3]) * a.scale_log2);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            exp32_pack(s[c], sc2, negm2, ps2, pk);
            tmem_st16(t_s + 16 * c, pk);
            if (c == 1) {                                       // P V of the first 64 keys may start
              tmem_wait_st();
              tc_fence_before();
              warp_arrive(&p_full[2 * h]);
            }
          }
        }
        float a0, a1, b0, b1;
        f2_unpack(ps2[0], a0, a1);
        f2_unpack(ps2[1], b0, b1);
        l_run += (a0 + a1) + (b0 + b1);
        tmem_wait_st();
        tc_fence_before();
        if (partial(all, j)) warp_arrive(&p_full[2 * h]);
        warp_arrive(&p_full[2 * h + 1]);
      }
      ok = ok && warp_wait_bounded(&o_done[h], used & 1, abort_flag, a.status);
      if (vote_group<128>(1 + h, !ok)) break;
      ++used;
      // O leaves 64 dims at a time.  A tile of whole rows of the sequence is one tensor store, else its rows are copied
      tc_fence_after();
      const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
      const int tile_tok = w.tok0 + h * a.tq;
      const bool full_tile = tile_tok + a.tq <= w.n;
#pragma unroll 1
      for (int c = 0; c < HD / 64; ++c) {
        uint32_t ro[32], rp[32];
        tmem_ld32_nowait(t_o + 64 * c, ro);
        tmem_ld32_nowait(t_o + 64 * c + 32, rp);
        tmem_wait_ld(ro);
        tmem_bind(rp);
        if (row == 0) bulk_wait_read0();
        bar_group<128>(1 + h);                                  // the memory is free again
#pragma unroll
        for (int k = 0; k < 64; k += 8) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = __uint_as_float(k < 32 ? ro[(k + 2 * e) & 31] : rp[(k + 2 * e) & 31]);
            const float y = __uint_as_float(k < 32 ? ro[(k + 2 * e + 1) & 31] : rp[(k + 2 * e + 1) & 31]);
            __nv_bfloat162 b = __floats2bfloat162_rn(x * inv, y * inv);
            v[e] = *reinterpret_cast<uint32_t*>(&b);
          }
          *reinterpret_cast<uint4*>(stage + row * 128 + (((k >> 3) ^ (row & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        if (full_tile) {
          fence_proxy_async_smem();
          bar_group<128>(1 + h);
          if (row == 0) {
            tma_store_3d(&tmO, stage, 64 * c, w.hk * a.group, w.first + tile_tok);
            bulk_commit();
          }
        } else {
          __syncwarp();                                         // a warp copies its own 32 rows, 8 lanes each
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            const int rr = quad * 32 + 4 * i + (lane >> 3), it = static_cast<int>(rr * a.group_inv >> 16);
            if (rr < a.rows && tile_tok + it < w.n)
              *reinterpret_cast<uint4*>(a.o + (w.first + tile_tok + it) * a.ldo + static_cast<int64_t>(w.hk * a.group + rr - it * a.group) * HD +
                                        64 * c + 8 * (lane & 7)) =
                  *reinterpret_cast<const uint4*>(stage + rr * 128 + (((lane & 7) ^ (rr & 7)) << 4));
          }
        }
      }
    }
    if (row == 0) bulk_wait0();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// bf16 map {HD, heads, rows}, box {64, box_heads, box_rows}, 128-byte swizzle
bool rows_map(CUtensorMap* m, const void* ptr, int hd, int heads, int total, int64_t ld, int box_heads, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(total)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(hd) * 2, static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_rows)}, estr[3] = {1, 1, 1};
  return tensor_map_encoder()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, int NT>
const char* launch(const RaggedCall& c, cudaStream_t s) {
  using C = PackedCfg<HD, NT>;
  if (!tensor_map_encoder()) return "cuTensorMapEncodeTiled is unavailable";
  int dev = 0;
  current_sms(&dev);
  static PerDevice ready;
  if (ready.get(dev, [] {
        return cudaFuncSetAttribute(attn_packed_kernel<HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) == cudaSuccess ? 1 : 0;
      }) <= 0)
    return "attention smem attribute failed";
  const int group = c.n_heads / c.n_kv, tq = TQ / group;
  CUtensorMap mq, mk, mv, mo;
  if (!rows_map(&mq, c.q, HD, c.n_heads, c.total, c.ldq, group, tq) || !rows_map(&mo, c.o, HD, c.n_heads, c.total, c.ldo, group, tq) ||
      !rows_map(&mk, c.k, HD, c.n_kv, c.total, c.ldk, 1, TK) || !rows_map(&mv, c.v, HD, c.n_kv, c.total, c.ldv, 1, TK))
    return "attention tensor map encode failed";
  const PackedArgs a{static_cast<bf16*>(c.o), c.cu, c.batch, c.total, c.max_rows, group, c.n_kv, tq, tq * group, 65536u / group + 1,
                     c.ldo, c.causal, c.window, 1.4426950408889634f / sqrtf(static_cast<float>(HD)), c.status};
  // at most one CTA per NT tiles of rows and one more per sequence
  const int64_t blocks = (static_cast<int64_t>(c.total) / (NT * tq) + c.batch) * c.n_kv;
  const cudaError_t e = launch_pdl(attn_packed_kernel<HD, NT>, dim3(static_cast<unsigned>(blocks)), C::THREADS, C::SMEM, s, mq, mk, mv, mo, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace

const char* attention_packed(const RaggedCall& c, cudaStream_t s) {
  // Heads of 128: two tiles share K and V in one CTA per SM (one 8192-token prompt, 32 / 16 heads: 377 us; one tile and two
  // CTAs per SM, whose rings then hold one K and one V, 734.  24 prompts of 512, 16 / 8 heads: 54 and 79).  Heads of 64
  // leave shared memory and tensor memory for two CTAs with whole rings, whose starts and ends overlap (12 prompts of 1024,
  // 12 heads: 48 us, 54 with two tiles; 64 of 64: 25 and 29; one of 8192, 32 / 16 heads: 341 and 331).
  return c.head_dim == 128 ? launch<128, 2>(c, s) : launch<64, 1>(c, s);
}

}  // namespace tadm
