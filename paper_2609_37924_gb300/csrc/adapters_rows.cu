// Projections with an adapter per request on CUDA cores (fp32):
//
//   h[t]  = scale_a A_a x[t]           a: the adapter of row t's sequence
//   y[t]  = W x[t] + B_a h[t]
//
// The second product runs in the tile of the first: after the k-blocks of W
// come, for each adapter that a row of the tile has, k-blocks of B_a against
// h with the other rows' h taken as zero.  Bound: shared-memory reads of the
// 4 x 4 products per thread, and for few rows the latency of a k-block.
#include <cstdint>

#include "ragged.cuh"
#include "requests.h"

namespace tadm {
namespace {

struct LoraRowsArgs {
  const void *x, *w, *a, *b;
  void* y;
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

// A warp per row and 8 of the adapter's dims.
template <class T>
__global__ void __launch_bounds__(256) lora_down_kernel(const LoraRowsArgs a) {
  pdl_enter();
  const int row = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ad = adapter_of(a, row);
  if (ad < 0) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  for (int r0 = 8 * warp; r0 < a.rank; r0 += 8 * (blockDim.x >> 5)) {
    const T* p = static_cast<const T*>(a.a) + (static_cast<int64_t>(ad) * a.rank + r0) * a.n_in;
    float s[8] = {};
    for (int k = lane; k < a.n_in; k += 32) {
      const float v = to_f32(x[k]);
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = fmaf(v, to_f32(p[static_cast<int64_t>(r) * a.n_in + k]), s[r]);
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) s[r] = warp_sum(s[r]);
    if (lane == 0)
      for (int r = 0; r < 8; ++r) a.h[static_cast<int64_t>(row) * a.rank + r0 + r] = s[r] * a.scale[ad];
  }
}

constexpr int TM = 64, TN = 64, TKB = 16;

template <class T, class YT>
__global__ void __launch_bounds__(256) lora_rows_kernel(const LoraRowsArgs a) {
  __shared__ float sx[TKB][TM + 4], sw[TKB][TN + 4];
  __shared__ int s_ad[TM], s_list[TM], s_n;
  pdl_enter();
  const int m0 = blockIdx.y * TM, n0 = blockIdx.x * TN, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = warp; i < TM; i += 8) {
    const int ad = adapter_of(a, m0 + i);
    if (lane == 0) s_ad[i] = ad;
  }
  __syncthreads();
  if (warp == 0) {                               // the tile's adapters, in the order of their first rows
    int n = 0;
    for (int half = 0; half < TM; half += 32) {
      const int i = half + lane, ad = s_ad[i];
      bool is_first = ad >= 0;
      for (int j = 0; j < i; ++j) is_first = is_first && s_ad[j] != ad;
      const unsigned have = __ballot_sync(0xffffffffu, is_first);
      if (is_first) s_list[n + __popc(have & ((1u << lane) - 1))] = ad;
      n += __popc(have);
    }
    if (lane == 0) s_n = n;
  }
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  auto multiply = [&]() {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < TKB; ++k) {
      const float4 xv = *reinterpret_cast<const float4*>(&sx[k][4 * ty]), wv = *reinterpret_cast<const float4*>(&sw[k][4 * tx]);
      const float xa[4] = {xv.x, xv.y, xv.z, xv.w}, wa[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xa[i], wa[j], acc[i][j]);
    }
    __syncthreads();
  };
  const int lr = threadIdx.x >> 2, lk = (threadIdx.x & 3) * 4;   // a row and four of its elements per thread
  for (int k0 = 0; k0 < a.n_in; k0 += TKB) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = k0 + lk + e;
      const bool in = k < a.n_in;
      sx[lk + e][lr] = in && m0 + lr < a.total ? to_f32(static_cast<const T*>(a.x)[(m0 + lr) * a.ldx + k]) : 0.0f;
      sw[lk + e][lr] = in && n0 + lr < a.n_out ? to_f32(static_cast<const T*>(a.w)[(n0 + lr) * a.ldw + k]) : 0.0f;
    }
    multiply();
  }
  __syncthreads();
  for (int i = 0; i < s_n; ++i) {
    const int ad = s_list[i];
    for (int k0 = 0; k0 < a.rank; k0 += TKB) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int k = k0 + lk + e;
        const bool in = k < a.rank;
        sx[lk + e][lr] = in && s_ad[lr] == ad ? a.h[static_cast<int64_t>(m0 + lr) * a.rank + k] : 0.0f;
        sw[lk + e][lr] = in && n0 + lr < a.n_out
                             ? to_f32(static_cast<const T*>(a.b)[(static_cast<int64_t>(ad) * a.n_out + n0 + lr) * a.rank + k]) : 0.0f;
      }
      multiply();
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 4 * ty + i;
    if (s_ad[4 * ty + i] == -2) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + 4 * tx + j < a.n_out) static_cast<YT*>(a.y)[m * a.ldy + n0 + 4 * tx + j] = from_f32<YT>(acc[i][j]);
  }
}

template <class T, class YT>
cudaError_t launch(const LoraRowsArgs& a, cudaStream_t s) {
  if (cudaError_t e = launch_pdl(lora_down_kernel<T>, a.total, 256, 0, s, a)) return e;
  return launch_pdl(lora_rows_kernel<T, YT>, dim3((a.n_out + TN - 1) / TN, (a.total + TM - 1) / TM), 256, 0, s, a);
}

}  // namespace

size_t lora_rows_scratch(int total, int rank) { return static_cast<size_t>(total) * rank * sizeof(float); }

const char* lora_rows(const LoraCall& c, cudaStream_t s) {
  const LoraRowsArgs a{c.x, c.w, c.a, c.b, c.y, c.cu, c.adapter, c.scale, static_cast<float*>(c.scratch),
                       c.batch, c.total, c.n_in, c.n_out, c.n_adapters, c.rank, c.ldx, c.ldw, c.ldy};
  const cudaError_t e = launch<float, float>(a, s);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
