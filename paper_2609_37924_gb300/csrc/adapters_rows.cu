// Projections with an adapter per request on CUDA cores (fp32):
//
//   h[t]  = scale_a A_a x[t]           a: the adapter of row t's sequence
//   y[t]  = W x[t] + B_a h[t]
//
// The second product runs in the tile of the first: after the k-blocks of W
// come, for each adapter that a row of the tile has, k-blocks of B_a against
// h with the other rows' h taken as zero.  W's blocks run while h is made: the
// kernel waits for its predecessor before the first block of h (x, W and the
// sequences were there when that one had waited for what came before it).
// Bound: the latency of the steps in front of the first products (where the
// rows lie, their adapters, the first blocks), then shared-memory reads of the
// 2 x 2 products per thread (four prompts of 228 rows, 256 -> 768, rank 8: 10.9
// us; blocks fetched one ahead into registers, a warp per row for its adapter and
// no overlap, 15.8; tiles of 64 x 64, 48 blocks of them, 57).
#include <cstdint>

#include "ragged.cuh"
#include "requests.h"

namespace tadm {
namespace {

struct LoraRowsArgs {
  const float *x, *w, *a, *b;
  float* y;
  const int32_t *cu, *adapter;
  const float* scale;
  float* h;                          // [total][rank]
  int batch, total, n_in, n_out, n_adapters, rank;
  int64_t ldx, ldw, ldy;
};

// adapter of row `row`: -1 none, -2 the row is in no sequence.  Warp-collective.
__device__ __forceinline__ int adapter_of(const LoraRowsArgs& a, int row) {
  const int b = row < a.total ? seq_of_row(a.cu, a.batch, row) : -1;
  if (b < 0) return -2;
  const int ad = a.adapter[b];
  return ad >= 0 && ad < a.n_adapters ? ad : -1;
}

// A warp per row and 8 of the adapter's ranks, four elements a lane.
__global__ void __launch_bounds__(256) lora_down_kernel(const LoraRowsArgs a) {
  pdl_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, eights = a.rank / 8;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 8 + warp;
  const int row = static_cast<int>(item / eights), r0 = static_cast<int>(item % eights) * 8;
  if (row >= a.total) return;
  const int ad = adapter_of(a, row);
  if (ad < 0) return;
  const float4* x = reinterpret_cast<const float4*>(a.x + row * a.ldx);
  const float4* p = reinterpret_cast<const float4*>(a.a + (static_cast<int64_t>(ad) * a.rank + r0) * a.n_in);
  const int n4 = a.n_in / 4;
  const float by = a.scale[ad];
  float s[8] = {};
#pragma unroll 2
  for (int k = lane; k < n4; k += 32) {
    const float4 v = x[k];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float4 t = p[static_cast<int64_t>(r) * n4 + k];
      s[r] = fmaf(v.w, t.w, fmaf(v.z, t.z, fmaf(v.y, t.y, fmaf(v.x, t.x, s[r]))));
    }
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) s[r] = warp_sum(s[r]);
  if (lane < 8) {
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) mine = lane == r ? s[r] : mine;
    a.h[static_cast<int64_t>(row) * a.rank + r0 + lane] = mine * by;
  }
}

// Tiles of 32 x 32 outputs (a few short prompts give many of them), K in blocks of 64 that come in a ring of asynchronous
// copies: 256 threads with 2 x 2 outputs and two 16-byte pieces of each operand per block.
constexpr int TM = 32, TN = 32, TKB = 64, RING = 3, LD = TKB + 4;
constexpr int R_SMEM = RING * (TM + TN) * LD * 4;

// 16 bytes into shared memory, zeros where not `in`
__device__ __forceinline__ void copy16(float* to, const float* from, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(in ? 16 : 0) : "memory");
}

__global__ void __launch_bounds__(256) lora_rows_kernel(const LoraRowsArgs a) {
  extern __shared__ __align__(16) float smem[];
  float(*sx)[TM][LD] = reinterpret_cast<float(*)[TM][LD]>(smem);
  float(*sw)[TN][LD] = reinterpret_cast<float(*)[TN][LD]>(smem + RING * TM * LD);
  __shared__ int s_ad[TM], s_list[TM], s_n;
  const int m0 = blockIdx.y * TM, n0 = blockIdx.x * TN, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lr = threadIdx.x >> 3, lk = (threadIdx.x & 7) * 4;   // a row of either operand, its elements lk .. and 32 + lk ..
  const bool x_in = m0 + lr < a.total, w_in = n0 + lr < a.n_out;
  const float* px = a.x + static_cast<int64_t>(x_in ? m0 + lr : 0) * a.ldx;
  const float* pw = a.w + static_cast<int64_t>(w_in ? n0 + lr : 0) * a.ldw;
  const int main = (a.n_in + TKB - 1) / TKB, per = (a.rank + TKB - 1) / TKB;   // blocks of x and W; of h and B, per adapter
  bool waited = false;
  int blocks = main;
  // block i of K into its place of the ring; past the last one nothing
  auto ask = [&](int i) {
    if (i >= main && !waited) {            // h comes from the kernel before; x, W and the sequences were there when that one ran
      pdl_enter();
      waited = true;
    }
    if (i < blocks) {
      const bool ext = i >= main;
      const int e = i - main, ad = ext ? s_list[e / per] : 0, k0 = (ext ? e % per : i) * TKB, width = ext ? a.rank : a.n_in;
      const float* x = ext ? a.h + static_cast<int64_t>(x_in ? m0 + lr : 0) * a.rank : px;
      const float* w = ext ? a.b + (static_cast<int64_t>(ad) * a.n_out + (w_in ? n0 + lr : 0)) * a.rank : pw;
      const bool x_on = ext ? s_ad[lr] == ad : x_in;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int k = k0 + 32 * p + lk;
        copy16(&sx[i % RING][lr][32 * p + lk], k < width ? x + k : x, x_on && k < width);
        copy16(&sw[i % RING][lr][32 * p + lk], k < width ? w + k : w, w_in && k < width);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  static_assert(RING == 3, "two blocks ahead");
  ask(0);
  if (main > 1) ask(1);
  if (warp == 0) {
    // a row per lane: its adapter (-1 none, -2: it is in no sequence), and the list of them in the order of their first rows
    const int row = m0 + lane;
    int lo = 0, hi = a.batch + 1;                // boundaries <= row: in lo .. hi
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      if (a.cu[mid] <= row) lo = mid + 1;
      else hi = mid;
    }
    int ad = -2;
    if (row < a.total && lo >= 1 && lo <= a.batch) {
      ad = a.adapter[lo - 1];
      if (ad < 0 || ad >= a.n_adapters) ad = -1;
    }
    s_ad[lane] = ad;
    const unsigned same = __match_any_sync(0xffffffffu, ad);    // (every lane calls it)
    const bool first = ad >= 0 && __ffs(same) - 1 == lane;
    const unsigned have = __ballot_sync(0xffffffffu, first);
    if (first) s_list[__popc(have & ((1u << lane) - 1))] = ad;
    const unsigned rows = __ballot_sync(0xffffffffu, ad > -2);
    if (lane == 0) s_n = rows ? __popc(have) : -1;
  }
  __syncthreads();
  if (s_n < 0) {                                 // rows of no sequence (buffers may be longer than what is in use)
    asm volatile("cp.async.wait_all;" ::: "memory");
    pdl_enter();                                 // (no block is through before the kernel in front)
    return;
  }
  blocks = main + s_n * per;
  if (main == 1) ask(1);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[2][2] = {};
  for (int i = 0; i < blocks; ++i) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();                             // (the block is there; the one before has been read)
    ask(i + 2);
    const auto &x = sx[i % RING], &w = sw[i % RING];
    auto step = [&](int k) {
      const float4 x0 = *reinterpret_cast<const float4*>(&x[ty][k]), x1 = *reinterpret_cast<const float4*>(&x[ty + 16][k]);
      const float4 w0 = *reinterpret_cast<const float4*>(&w[tx][k]), w1 = *reinterpret_cast<const float4*>(&w[tx + 16][k]);
      auto dot = [](const float4& p, const float4& q, float s) { return fmaf(p.w, q.w, fmaf(p.z, q.z, fmaf(p.y, q.y, fmaf(p.x, q.x, s)))); };
      acc[0][0] = dot(x0, w0, acc[0][0]);
      acc[0][1] = dot(x0, w1, acc[0][1]);
      acc[1][0] = dot(x1, w0, acc[1][0]);
      acc[1][1] = dot(x1, w1, acc[1][1]);
    };
    const int left = i < main ? TKB : a.rank - (i - main) % per * TKB;   // (ranks come in eights)
    if (left >= TKB) {
#pragma unroll
      for (int k = 0; k < TKB; k += 4) step(k);
    } else {
      for (int k = 0; k < left; k += 8) step(k), step(k + 4);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + ty + 16 * i;
    if (s_ad[ty + 16 * i] == -2) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (n0 + tx + 16 * j < a.n_out) a.y[m * a.ldy + n0 + tx + 16 * j] = acc[i][j];
  }
}

}  // namespace

size_t lora_rows_scratch(int total, int rank) { return static_cast<size_t>(total) * rank * sizeof(float); }

const char* lora_rows(const LoraCall& c, cudaStream_t s) {
  auto f = [](const void* p) { return static_cast<const float*>(p); };
  const LoraRowsArgs a{f(c.x), f(c.w), f(c.a), f(c.b), static_cast<float*>(c.y), c.cu, c.adapter, c.scale, static_cast<float*>(c.scratch),
                       c.batch, c.total, c.n_in, c.n_out, c.n_adapters, c.rank, c.ldx, c.ldw, c.ldy};
  const int64_t items = static_cast<int64_t>(c.total) * (c.rank / 8);
  static PerDevice ready;
  int dev = 0;
  cudaGetDevice(&dev);
  cudaError_t e = cudaSuccess;
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(lora_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R_SMEM);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return cudaGetErrorString(e);
  e = launch_pdl(lora_down_kernel, static_cast<unsigned>((items + 7) / 8), 256, 0, s, a);
  if (e == cudaSuccess) e = launch_pdl(lora_rows_kernel, dim3((c.n_out + TN - 1) / TN, (c.total + TM - 1) / TM), 256, R_SMEM, s, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
