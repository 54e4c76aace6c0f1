// Projections with an adapter per request on CUDA cores (fp32):
//
//   h[t]  = scale_a A_a x[t]           a: the adapter of row t's sequence
//   y[t]  = W x[t] + B_a h[t]
//
// The second product runs in the tile of the first: after the k-blocks of W
// come, for each adapter that a row of the tile has, k-blocks of B_a against
// h with the other rows' h taken as zero.  Bound: shared-memory reads of the
// 2 x 2 products per thread, and for few rows the latency of a k-block (four
// prompts of 228 rows, 256 -> 768, rank 8: 16 us; tiles of 64 x 64, 48 blocks
// of them, 57).
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
    a.h[static_cast<int64_t>(row) * a.rank + r0 + lane] = mine * a.scale[ad];
  }
}

// Tiles of 32 x 32 outputs (a few short prompts give many of them), K in blocks of 64 that are fetched one ahead: 256
// threads with 2 x 2 outputs and a float4 of each operand for each half of the block.
constexpr int TM = 32, TN = 32, TKB = 64;

__global__ void __launch_bounds__(256) lora_rows_kernel(const LoraRowsArgs a) {
  __shared__ __align__(16) float sx[2][TM][TKB + 4], sw[2][TN][TKB + 4];
  __shared__ int s_ad[TM], s_list[TM], s_n;
  const int m0 = blockIdx.y * TM, n0 = blockIdx.x * TN, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_enter();
  const int lr = threadIdx.x >> 3, lk = (threadIdx.x & 7) * 4;   // a row of either operand, its elements lk .. and 32 + lk ..
  const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float* px = a.x + (m0 + lr) * a.ldx;
  const float* pw = a.w + (n0 + lr) * a.ldw;
  const bool x_in = m0 + lr < a.total, w_in = n0 + lr < a.n_out;
  float4 fx[2], fw[2];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = k0 + 32 * i + lk;
      fx[i] = x_in && k < a.n_in ? *reinterpret_cast<const float4*>(px + k) : zero;
      fw[i] = w_in && k < a.n_in ? *reinterpret_cast<const float4*>(pw + k) : zero;
    }
  };
  fetch(0);
  for (int i = warp; i < TM; i += 8) {
    const int ad = adapter_of(a, m0 + i);
    if (lane == 0) s_ad[i] = ad;
  }
  __syncthreads();
  if (warp == 0) {                               // the tile's adapters, in the order of their first rows
    const int ad = s_ad[lane];
    bool first = ad >= 0;
    for (int j = 0; j < lane; ++j) first = first && s_ad[j] != ad;
    const unsigned have = __ballot_sync(0xffffffffu, first);
    if (first) s_list[__popc(have & ((1u << lane) - 1))] = ad;
    if (lane == 0) s_n = __popc(have);
  }
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[2][2] = {};
  int buf = 0;
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *reinterpret_cast<float4*>(&sx[buf][lr][32 * i + lk]) = fx[i];
      *reinterpret_cast<float4*>(&sw[buf][lr][32 * i + lk]) = fw[i];
    }
    __syncthreads();
  };
  auto multiply = [&]() {
#pragma unroll
    for (int k = 0; k < TKB; k += 4) {
      const float4 x0 = *reinterpret_cast<const float4*>(&sx[buf][ty][k]), x1 = *reinterpret_cast<const float4*>(&sx[buf][ty + 16][k]);
      const float4 w0 = *reinterpret_cast<const float4*>(&sw[buf][tx][k]), w1 = *reinterpret_cast<const float4*>(&sw[buf][tx + 16][k]);
      auto dot = [](const float4& p, const float4& q, float s) { return fmaf(p.w, q.w, fmaf(p.z, q.z, fmaf(p.y, q.y, fmaf(p.x, q.x, s)))); };
      acc[0][0] = dot(x0, w0, acc[0][0]);
      acc[0][1] = dot(x0, w1, acc[0][1]);
      acc[1][0] = dot(x1, w0, acc[1][0]);
      acc[1][1] = dot(x1, w1, acc[1][1]);
    }
    buf ^= 1;                                    // (the other buffer's readers have passed the barrier in put())
  };
  for (int k0 = 0; k0 < a.n_in; k0 += TKB) {
    put();
    if (k0 + TKB < a.n_in) fetch(k0 + TKB);
    multiply();
  }
  __syncthreads();
  for (int i = 0; i < s_n; ++i) {
    const int ad = s_list[i];
    const bool mine = s_ad[lr] == ad;
    const float* ph = a.h + static_cast<int64_t>(m0 + lr) * a.rank;
    const float* pb = a.b + (static_cast<int64_t>(ad) * a.n_out + n0 + lr) * a.rank;
    for (int k0 = 0; k0 < a.rank; k0 += TKB) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + 32 * h + lk;
        fx[h] = mine && k < a.rank ? *reinterpret_cast<const float4*>(ph + k) : zero;
        fw[h] = w_in && k < a.rank ? *reinterpret_cast<const float4*>(pb + k) : zero;
      }
      put();
      multiply();
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
  cudaError_t e = launch_pdl(lora_down_kernel, static_cast<unsigned>((items + 7) / 8), 256, 0, s, a);
  if (e == cudaSuccess) e = launch_pdl(lora_rows_kernel, dim3((c.n_out + TN - 1) / TN, (c.total + TM - 1) / TM), 256, 0, s, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
