// Attention of packed fp32 rows on the CUDA cores: over the rows of their own
// sequence, or over a sequence's pages of the 8-bit cache.
//
// A block takes 16 virtual rows (row-major, then the query heads of one KV
// head, so that a key tile serves all of them) of one sequence and walks its
// visible keys in tiles of 64: K and V as fp32 in shared memory, a warp per
// two virtual rows (eight apart, so that a single token's rows are on warps of
// their own), two keys per lane for the scores, four or two dims per lane for
// P V.  Everything is fp32: scores, running maximum and sum (online softmax),
// accumulators.  It serves fp32 rows, those of the small models, whose calls
// are a launch (9 us with the host's part for a few hundred rows of 4 heads).
// Longer ones are bound by a tile's latency, about 3 us: the next tile's loads
// wait in registers meanwhile, 16 bytes each (a row over 600 tokens of the cache
// 27 us, 72 with loads of single elements between the barriers; four prompts of
// 500 rows 54 and 70; with tiles of 32 rows 26 and 60, and four blocks of 32
// rows over 600 tokens 58 instead of 42).
#include <cuda_fp8.h>

#include <type_traits>

#include "ragged.cuh"
#include "serve.h"

namespace tadm {
namespace {

constexpr int RT = 16, KT = 64, NT = 256;     // virtual rows and keys of a tile, threads
constexpr int WR = RT * 32 / NT;              // rows of a warp: its index and every eighth on
static_assert(KT == TADM_PAGE_TOKENS, "a key tile is a page");

struct RowsAttnArgs {
  const float *q, *k, *v;
  float* o;
  const uint8_t *pk, *pv;
  const float *sk, *sv;
  const int32_t *cu, *lens, *table;
  int batch, total, max_rows, max_len, ld_table, pages;
  int n_heads, n_kv;
  int64_t ldq, ldk, ldv, ldo;
  int causal, window;
  float scale;
};

template <bool PAGED, int HD>
__global__ void __launch_bounds__(NT) attn_rows_kernel(const RowsAttnArgs a) {
  pdl_enter();
  constexpr int LD = HD + 4, PL = HD / 32;
  extern __shared__ __align__(16) float sm[];
  float* sK = sm;                      // [KT][LD]
  float* sV = sK + KT * LD;            // [KT][LD]
  float* sQ = sV + KT * LD;            // [RT][HD]
  float* sP = sQ + RT * HD;            // [RT][KT]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = a.n_heads / a.n_kv, hk = blockIdx.y;
  int t;
  const int b = find_tile(a.batch, blockIdx.x, [&](int i) {
    return (static_cast<int64_t>(seq_rows(a.cu, i, a.total, a.max_rows).n) * group + RT - 1) / RT;
  }, &t);
  if (b < 0) return;
  const SeqRows rows = seq_rows(a.cu, b, a.total, a.max_rows);
  const int n_virt = rows.n * group, v0 = t * RT;
  const int len = PAGED ? min(max(a.lens[b], 0), a.max_len) : rows.n;
  const int pos0 = len - rows.n;                       // position of row 0
  // keys that any row of the tile sees
  const int r_lo = v0 / group, r_hi = (min(v0 + RT, n_virt) - 1) / group;
  const int k_end = a.causal ? max(0, min(len, pos0 + r_hi + 1)) : len;
  const int k_begin = a.window > 0 ? max(0, pos0 + r_lo - a.window + 1) : 0;
  for (int i = tid; i < RT * HD; i += NT) {
    const int v = v0 + i / HD;
    sQ[i] = v < n_virt ? a.q[(rows.first + v / group) * a.ldq + static_cast<int64_t>(hk * group + v % group) * HD + i % HD] : 0.0f;
  }
  float m[WR], l[WR], acc[WR][PL];
#pragma unroll
  for (int i = 0; i < WR; ++i) {
    m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
    for (int d = 0; d < PL; ++d) acc[i][d] = 0.0f;
  }
  // a thread's part of the next key tile waits in registers while this one is computed
  constexpr int NF = PAGED ? HD / 64 : HD / 16;               // 16-byte loads per thread of K, of V
  int4 rk[NF], rv[NF];
  float ks = 0.0f, vs = 0.0f;
  auto fetch = [&](int k0) {
    if (PAGED) {
      const int slot = k0 / KT;
      const int page = slot < a.ld_table ? a.table[static_cast<int64_t>(b) * a.ld_table + slot] : -1;
      const bool ok = page >= 0 && page < a.pages;
      const int64_t ph = static_cast<int64_t>(ok ? page : 0) * a.n_kv + hk;
      ks = ok ? a.sk[ph] : 0.0f, vs = ok ? a.sv[ph] : 0.0f;
#pragma unroll
      for (int u = 0; u < NF; ++u) {
        const int64_t at = ph * KT * HD + (u * NT + tid) * 16;
        rk[u] = ok ? *reinterpret_cast<const int4*>(a.pk + at) : make_int4(0, 0, 0, 0);
        rv[u] = ok ? *reinterpret_cast<const int4*>(a.pv + at) : make_int4(0, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int u = 0; u < NF; ++u) {
        const int i = (u * NT + tid) * 4, r = i / HD;
        const int64_t row = rows.first + k0 + r, c = static_cast<int64_t>(hk) * HD + i % HD;
        const bool in = k0 + r < len;
        rk[u] = in ? *reinterpret_cast<const int4*>(a.k + row * a.ldk + c) : make_int4(0, 0, 0, 0);
        rv[u] = in ? *reinterpret_cast<const int4*>(a.v + row * a.ldv + c) : make_int4(0, 0, 0, 0);
      }
    }
  };
  auto stage = [&](int k0) {
#pragma unroll
    for (int u = 0; u < NF; ++u) {
      if (PAGED) {
        // K: 16 dims of a key, V: 16 keys of a dim; what no row of the tile sees may hold anything
        const int i = (u * NT + tid) * 16, kr = i / HD, kc = i % HD, vt = i % KT, vd = i / KT;
        const uint32_t wk[4] = {static_cast<uint32_t>(rk[u].x), static_cast<uint32_t>(rk[u].y), static_cast<uint32_t>(rk[u].z),
                                static_cast<uint32_t>(rk[u].w)};
        const uint32_t wv[4] = {static_cast<uint32_t>(rv[u].x), static_cast<uint32_t>(rv[u].y), static_cast<uint32_t>(rv[u].z),
                                static_cast<uint32_t>(rv[u].w)};
        auto dec = [](uint32_t w, int e) {
          return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<uint8_t>(w >> (8 * (e & 3))), __NV_E4M3)));
        };
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          sK[kr * LD + kc + e] = k0 + kr < k_end ? dec(wk[e >> 2], e) * ks : 0.0f;
          const int key = k0 + vt + e;
          sV[(vt + e) * LD + vd] = key >= k_begin && key < k_end ? dec(wv[e >> 2], e) * vs : 0.0f;
        }
      } else {
        const int i = (u * NT + tid) * 4, at = i / HD * LD + i % HD;
        *reinterpret_cast<int4*>(sK + at) = rk[u];
        *reinterpret_cast<int4*>(sV + at) = rv[u];
      }
    }
  };
  if (k_begin < k_end) fetch(k_begin / KT * KT);
  for (int k0 = k_begin / KT * KT; k0 < k_end; k0 += KT) {
    __syncthreads();
    stage(k0);
    __syncthreads();
    if (k0 + KT < k_end) fetch(k0 + KT);
    // the first R rows of the warp
    auto tile = [&](auto count) {
      constexpr int R = decltype(count)::value;
      float s[R][2] = {};                              // [row][key half]
#pragma unroll 4
      for (int c = 0; c < HD; c += 4) {
        const float4 ka = *reinterpret_cast<const float4*>(sK + lane * LD + c);
        const float4 kb = *reinterpret_cast<const float4*>(sK + (lane + 32) * LD + c);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(sQ + (warp + 8 * i) * HD + c);
          s[i][0] = fmaf(q.x, ka.x, fmaf(q.y, ka.y, fmaf(q.z, ka.z, fmaf(q.w, ka.w, s[i][0]))));
          s[i][1] = fmaf(q.x, kb.x, fmaf(q.y, kb.y, fmaf(q.z, kb.z, fmaf(q.w, kb.w, s[i][1]))));
        }
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int v = v0 + warp + 8 * i, pos = pos0 + v / group;
        const int hi = a.causal ? min(len, pos + 1) : len, lo = a.window > 0 ? pos - a.window + 1 : 0;
        const bool see0 = v < n_virt && k0 + lane >= lo && k0 + lane < hi;
        const bool see1 = v < n_virt && k0 + lane + 32 >= lo && k0 + lane + 32 < hi;
        const float x0 = see0 ? s[i][0] * a.scale : -INFINITY, x1 = see1 ? s[i][1] * a.scale : -INFINITY;
        const float mn = fmaxf(m[i], warp_max(fmaxf(x0, x1)));
        const float ref = mn == -INFINITY ? 0.0f : mn;  // (scores of minus infinity alone weigh nothing)
        const float f = m[i] == -INFINITY ? 0.0f : expf(m[i] - ref);
        const float p0 = see0 ? expf(x0 - ref) : 0.0f, p1 = see1 ? expf(x1 - ref) : 0.0f;
        sP[(warp + 8 * i) * KT + lane] = p0;
        sP[(warp + 8 * i) * KT + lane + 32] = p1;
        l[i] = l[i] * f + p0 + p1;                     // this lane's keys; the lanes' sums meet at the end
#pragma unroll
        for (int d = 0; d < PL; ++d) acc[i][d] *= f;
        m[i] = mn;
      }
      __syncwarp();
#pragma unroll 4
      for (int j = 0; j < KT; j += 4) {
        float p[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(sP + (warp + 8 * i) * KT + j);
          p[i][0] = q.x, p[i][1] = q.y, p[i][2] = q.z, p[i][3] = q.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < PL; ++d) {
            const float x = sV[(j + e) * LD + 32 * d + lane];
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i][d] = fmaf(p[i][e], x, acc[i][d]);
          }
      }
    };
    const int left = n_virt - v0 - warp;               // > 8 i: the warp has row i
    if (left > 8) tile(std::integral_constant<int, WR>{});
    else if (left > 0) tile(std::integral_constant<int, 1>{});
  }
#pragma unroll
  for (int i = 0; i < WR; ++i) {
    const int v = v0 + warp + 8 * i;
    const float sum = warp_sum(l[i]);
    if (v >= n_virt) continue;
    float* o = a.o + (rows.first + v / group) * a.ldo + static_cast<int64_t>(hk * group + v % group) * HD;
#pragma unroll
    for (int d = 0; d < PL; ++d) o[32 * d + lane] = sum == 0.0f ? 0.0f : acc[i][d] / sum;
  }
}

template <bool PAGED, int HD>
const char* launch(const RaggedCall& c, cudaStream_t s) {
  constexpr int smem = (2 * KT * (HD + 4) + RT * HD + RT * KT) * 4;
  int dev = 0;
  current_sms(&dev);
  static PerDevice ready;
  if (ready.get(dev, [] {
        return cudaFuncSetAttribute(attn_rows_kernel<PAGED, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) ==
                       cudaSuccess ? 1 : 0;
      }) <= 0)
    return "attention smem attribute failed";
  RowsAttnArgs a{static_cast<const float*>(c.q), static_cast<const float*>(c.k), static_cast<const float*>(c.v),
                 static_cast<float*>(c.o), nullptr, nullptr, nullptr, nullptr, c.cu, c.lens, c.table, c.batch, c.total,
                 c.max_rows, c.max_len, c.ld_table, 0, c.n_heads, c.n_kv, c.ldq, c.ldk, c.ldv, c.ldo, c.causal, c.window,
                 1.0f / sqrtf(static_cast<float>(HD))};
  if (PAGED) {
    const tadm_page_pool& p = *c.pool;
    const int64_t at = static_cast<int64_t>(c.layer) * p.pages * p.n_kv_heads;
    a.pk = static_cast<const uint8_t*>(p.k) + at * KT * HD;
    a.pv = static_cast<const uint8_t*>(p.v) + at * KT * HD;
    a.sk = p.k_scale + at;
    a.sv = p.v_scale + at;
    a.pages = p.pages;
  }
  const int group = c.n_heads / c.n_kv;
  // at most one tile per RT virtual rows and one more per sequence
  const int64_t tiles = static_cast<int64_t>(c.total) * group / RT + c.batch;
  const cudaError_t e = launch_pdl(attn_rows_kernel<PAGED, HD>, dim3(static_cast<unsigned>(tiles), c.n_kv), NT, smem, s, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace

const char* attention_rows(const RaggedCall& c, cudaStream_t s) {
  if (c.batch == 0 || c.total == 0 || c.max_rows == 0) return nullptr;
  if (c.pool) return c.head_dim == 128 ? launch<true, 128>(c, s) : launch<true, 64>(c, s);
  return c.head_dim == 128 ? launch<false, 128>(c, s) : launch<false, 64>(c, s);
}

}  // namespace tadm
