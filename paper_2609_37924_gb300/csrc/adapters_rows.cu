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
// Bound: of few rows the latency of the steps in front of the first products
// (where the rows lie, their adapters, the first blocks) and the 2 x 2 products
// per thread between reads of shared memory (four prompts of 228 rows, 256 ->
// 768, rank 8: 10.9 us; blocks fetched one ahead into registers, a warp per row
// for its adapter and no overlap, 15.8); of many the FMA and shared-memory
// pipes (2020 rows, 768 -> 2304: 204 us with rank 16, 35 TFLOP/s; 222 with rank
// 64, 251 with 128).
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

// Tiles of 16 R x 16 R outputs, K in blocks of 64 that come in a ring of asynchronous copies: 256 threads with R x R outputs
// and R 16-byte pieces of each operand per block.  R = 2 gives the many tiles that few rows need, R = 4 reads half as much
// shared memory per product.
constexpr int TKB = 64, RING = 3, LD = TKB + 4;
constexpr int ring_bytes(int R) { return RING * 2 * 16 * R * LD * 4; }

// 16 bytes into shared memory, zeros where not `in`
__device__ __forceinline__ void copy16(float* to, const float* from, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(in ? 16 : 0) : "memory");
}

template <int R>
__global__ void __launch_bounds__(256, R == 2 ? 4 : 2) lora_rows_kernel(const LoraRowsArgs a) {
  constexpr int TM = 16 * R;
  extern __shared__ __align__(16) float smem[];
  float(*sx)[TM][LD] = reinterpret_cast<float(*)[TM][LD]>(smem);
  float(*sw)[TM][LD] = reinterpret_cast<float(*)[TM][LD]>(smem + RING * TM * LD);
  __shared__ int s_ad[TM], s_list[TM], s_n;
  const int m0 = blockIdx.y * TM, n0 = blockIdx.x * TM, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lr = threadIdx.x >> 4, lk = (threadIdx.x & 15) * 4;   // rows lr, lr + 16 .. of either operand, their elements lk ..
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
      const int e = i - main, ad = ext ? s_list[e / per] : 0, k = (ext ? e % per : i) * TKB + lk;
      const bool k_in = k < (ext ? a.rank : a.n_in);
#pragma unroll
      for (int p = 0; p < R; ++p) {
        const int r = lr + 16 * p, m = m0 + r, n = n0 + r;
        const bool x_on = k_in && m < a.total && (!ext || s_ad[r] == ad), w_on = k_in && n < a.n_out;
        const float* x = ext ? a.h + static_cast<int64_t>(m) * a.rank : a.x + m * a.ldx;
        const float* w = ext ? a.b + (static_cast<int64_t>(ad) * a.n_out + n) * a.rank : a.w + n * a.ldw;
        copy16(&sx[i % RING][r][lk], x_on ? x + k : a.x, x_on);
        copy16(&sw[i % RING][r][lk], w_on ? w + k : a.w, w_on);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  static_assert(RING == 3, "two blocks ahead");
  ask(0);
  if (main > 1) ask(1);
  if (warp == 0) {
    // a row per lane: its adapter (-1 none, -2: it is in no sequence), and the list of them in the order of their first rows
    auto adapter_at = [&](int row) {
      int lo = 0, hi = a.batch + 1;              // boundaries <= row: in lo .. hi
      while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (a.cu[mid] <= row) lo = mid + 1;
        else hi = mid;
      }
      if (row >= a.total || lo < 1 || lo > a.batch) return -2;
      const int ad = a.adapter[lo - 1];
      return ad >= 0 && ad < a.n_adapters ? ad : -1;
    };
    int n = 0;
    bool any = false;
    for (int r = 0; r < TM; r += 32) {
      const int ad = adapter_at(m0 + r + lane);
      s_ad[r + lane] = ad;
      const unsigned same = __match_any_sync(0xffffffffu, ad);  // (every lane calls it)
      bool first = ad >= 0 && __ffs(same) - 1 == lane;
      for (int j = 0; j < n; ++j) first = first && s_list[j] != ad;
      const unsigned have = __ballot_sync(0xffffffffu, first);
      any = any || __any_sync(0xffffffffu, ad > -2);
      if (first) s_list[n + __popc(have & ((1u << lane) - 1))] = ad;
      n += __popc(have);
      __syncwarp();
    }
    if (lane == 0) s_n = any ? n : -1;
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
  float acc[R][R] = {};
  for (int i = 0; i < blocks; ++i) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();                             // (the block is there; the one before has been read)
    ask(i + 2);
    const auto &x = sx[i % RING], &w = sw[i % RING];
    auto step = [&](int k) {
      float4 p[R], q[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        p[r] = *reinterpret_cast<const float4*>(&x[ty + 16 * r][k]);
        q[r] = *reinterpret_cast<const float4*>(&w[tx + 16 * r][k]);
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < R; ++c) acc[r][c] = fmaf(p[r].w, q[c].w, fmaf(p[r].z, q[c].z, fmaf(p[r].y, q[c].y, fmaf(p[r].x, q[c].x, acc[r][c]))));
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
  for (int i = 0; i < R; ++i) {
    const int m = m0 + ty + 16 * i;
    if (s_ad[ty + 16 * i] == -2) continue;
#pragma unroll
    for (int j = 0; j < R; ++j)
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
  const int sms = current_sms(&dev);
  cudaError_t e = cudaSuccess;
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(lora_rows_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(2));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_rows_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(4));
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return cudaGetErrorString(e);
  e = launch_pdl(lora_down_kernel, static_cast<unsigned>((items + 7) / 8), 256, 0, s, a);
  auto grid = [&](int tile) { return dim3((c.n_out + tile - 1) / tile, (c.total + tile - 1) / tile); };
  const dim3 wide = grid(64);
  // 64 x 64 from a tile for every other SM on (84 tiles, 768 -> 768: 32 us instead of 45; 96 tiles, 256 -> 768: 24.5 instead of
  // 22; 1152 tiles, 768 -> 2304: 200 instead of 318); fewer are quicker as 32 x 32 (48 tiles, 768 -> 768: 25 instead of 30)
  if (e == cudaSuccess)
    e = 2 * static_cast<int64_t>(wide.x) * wide.y >= sms ? launch_pdl(lora_rows_kernel<4>, wide, 256, ring_bytes(4), s, a)
                                                         : launch_pdl(lora_rows_kernel<2>, grid(32), 256, ring_bytes(2), s, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
