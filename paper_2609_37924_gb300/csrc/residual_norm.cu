// The norms between two blocks of a layer, in one pass over the residual
// stream: for a row of sequence b
//
//   u  = y * rsqrt(mean(y^2) + eps) * g_post        (without g_post: u = y)
//   x' = alpha x + gate_b * u                       (without a gate: alpha x + u)
//   n  = x' * rsqrt(mean(x'^2) + eps) * g_pre       (without g_pre: no gain)
//
// x and y are read once, x' and n written once, everything between is fp32 in
// registers; n is made from x' before it is rounded to its own type.
//
// Bound: HBM, (2 es_x + es_y + es_n) bytes per element.
#include <cstdint>

#include "ragged.cuh"
#include "requests.h"

namespace tadm {
namespace {

struct NormArgs {
  const void *x, *y;
  void *xo, *no;
  const int32_t* cu;
  int batch, total, d;
  int64_t ldx, ldy, ldxo, ldn, ldg;
  const void *post, *gate, *pre;
  float alpha, eps;
};

// eight consecutive elements, 16-byte aligned
__device__ __forceinline__ void ld8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void ld8(const bf16* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void st8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void st8(bf16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Sum over the threads that share a row: a warp (WARPS 1) or the block.
template <bool BLOCK>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = warp_sum(v);
  if constexpr (BLOCK) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
    if (lane == 0) red[warp] = v;
    __syncthreads();
    v = warp_sum(lane < n ? red[lane] : 0.0f);
  }
  return v;
}

// Rows of 16-byte vectors held in registers: NV vectors of eight elements per
// thread.  BLOCK: a row per block, else a row per warp.
template <class XT, class YT, class T, int NV, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? 1024 : 256) norm_reg_kernel(const NormArgs a) {
  __shared__ float red[2][32];
  const int row = BLOCK ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int me = BLOCK ? threadIdx.x : threadIdx.x & 31, step = BLOCK ? blockDim.x : 32, nvec = a.d / 8;
  pdl_enter();
  if (row >= a.total) return;
  const int b = a.cu ? seq_of_row(a.cu, a.batch, row) : 0;
  if (b < 0) return;
  const XT* x = static_cast<const XT*>(a.x) + row * a.ldx;
  const YT* y = static_cast<const YT*>(a.y) + row * a.ldy;
  const T *post = static_cast<const T*>(a.post), *pre = static_cast<const T*>(a.pre), *gate = static_cast<const T*>(a.gate);
  float u[NV][8], v[NV][8], w[8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = me + i * step;
    if (c < nvec) {
      ld8(y + 8 * c, u[i]);
      ld8(x + 8 * c, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i][e] = v[i][e] = 0.0f;
    }
  }
  if (post) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(u[i][e], u[i][e], s);
    const float r = rsqrtf(row_sum<BLOCK>(s, red[0]) / static_cast<float>(a.d) + a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = me + i * step;
      if (c < nvec) {
        ld8(post + 8 * c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i][e] = u[i][e] * r * w[e];
      }
    }
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = me + i * step;
    if (c < nvec) {
      if (gate) {
        ld8(gate + b * a.ldg + 8 * c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i][e] *= w[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] = fmaf(a.alpha, v[i][e], u[i][e]);
        s = fmaf(v[i][e], v[i][e], s);
      }
      st8(static_cast<XT*>(a.xo) + row * a.ldxo + 8 * c, v[i]);
    }
  }
  if (!a.no) return;
  const float r = rsqrtf(row_sum<BLOCK>(s, red[1]) / static_cast<float>(a.d) + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = me + i * step;
    if (c < nvec) {
      if (pre) ld8(pre + 8 * c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = pre ? v[i][e] * r * w[e] : v[i][e] * r;
      st8(static_cast<T*>(a.no) + row * a.ldn + 8 * c, v[i]);
    }
  }
}

// Any width, stride and alignment: a row per block, x' in shared memory.
template <class XT, class YT, class T>
__global__ void __launch_bounds__(512) norm_any_kernel(const NormArgs a) {
  extern __shared__ float xs[];
  __shared__ float red[2][32];
  const int row = blockIdx.x;
  pdl_enter();
  const int b = a.cu ? seq_of_row(a.cu, a.batch, row) : 0;
  if (b < 0) return;
  const XT* x = static_cast<const XT*>(a.x) + row * a.ldx;
  const YT* y = static_cast<const YT*>(a.y) + row * a.ldy;
  const T *post = static_cast<const T*>(a.post), *pre = static_cast<const T*>(a.pre), *gate = static_cast<const T*>(a.gate);
  float s = 0.0f, r = 0.0f;
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    const float v = to_f32(y[c]);
    xs[c] = v;
    s = fmaf(v, v, s);
  }
  if (post) r = rsqrtf(row_sum<true>(s, red[0]) / static_cast<float>(a.d) + a.eps);
  s = 0.0f;
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {       // (each thread reads what it wrote)
    float u = xs[c];
    if (post) u = u * r * to_f32(post[c]);
    if (gate) u *= to_f32(gate[b * a.ldg + c]);
    const float v = fmaf(a.alpha, to_f32(x[c]), u);
    s = fmaf(v, v, s);
    xs[c] = v;
    static_cast<XT*>(a.xo)[row * a.ldxo + c] = from_f32<XT>(v);
  }
  if (!a.no) return;
  r = rsqrtf(row_sum<true>(s, red[1]) / static_cast<float>(a.d) + a.eps);
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    const float v = xs[c] * r;
    static_cast<T*>(a.no)[row * a.ldn + c] = from_f32<T>(pre ? v * to_f32(pre[c]) : v);
  }
}

template <class XT, class YT, class T>
cudaError_t launch(const NormArgs& a, bool vec, cudaStream_t s) {
  const int nvec = a.d / 8;
  if (vec && nvec <= 128) {
    const int rows = 8, grid = (a.total + rows - 1) / rows;
    if (nvec <= 32) return launch_pdl(norm_reg_kernel<XT, YT, T, 1, false>, grid, 32 * rows, 0, s, a);
    if (nvec <= 64) return launch_pdl(norm_reg_kernel<XT, YT, T, 2, false>, grid, 32 * rows, 0, s, a);
    return launch_pdl(norm_reg_kernel<XT, YT, T, 4, false>, grid, 32 * rows, 0, s, a);
  }
  if (vec && nvec <= 2048) {
    const int one = (nvec + 31) / 32 * 32, two = ((nvec + 1) / 2 + 31) / 32 * 32;
    if (one <= 512) return launch_pdl(norm_reg_kernel<XT, YT, T, 1, true>, a.total, one, 0, s, a);
    return launch_pdl(norm_reg_kernel<XT, YT, T, 2, true>, a.total, two, 0, s, a);
  }
  static PerDevice ready;
  int dev = 0;
  cudaGetDevice(&dev);
  cudaError_t e = cudaSuccess;
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(norm_any_kernel<XT, YT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormMaxWidth * 4);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return e;
  return launch_pdl(norm_any_kernel<XT, YT, T>, a.total, a.d >= 512 ? 512 : (a.d + 31) / 32 * 32, a.d * 4, s, a);
}

template <class XT, class YT>
cudaError_t launch_out(const NormArgs& a, bool vec, bool bf, cudaStream_t s) {
  return bf ? launch<XT, YT, bf16>(a, vec, s) : launch<XT, YT, float>(a, vec, s);
}

}  // namespace

const char* residual_norm(const NormCall& c, cudaStream_t s) {
  const NormArgs a{c.x, c.y, c.x_out, c.n_out, c.cu, c.batch, c.total, c.d, c.ldx, c.ldy, c.ldxo, c.ldn, c.ldg,
                   c.post, c.gate, c.pre, c.residual_scale, c.eps};
  // 16-byte vectors of eight elements: widths, row strides and bases that allow them
  auto ok = [](const void* p, int64_t ld, int bf) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * (bf ? 2 : 4) % 16 == 0;
  };
  const bool vec = c.d % 8 == 0 && ok(c.x, c.ldx, c.x_bf16) && ok(c.x_out, c.ldxo, c.x_bf16) && ok(c.y, c.ldy, c.y_bf16) &&
                   ok(c.n_out, c.n_out ? c.ldn : 0, c.bf16) && ok(c.gate, c.gate ? c.ldg : 0, c.bf16) && ok(c.post, 0, 1) &&
                   ok(c.pre, 0, 1);
  const cudaError_t e = c.x_bf16 ? (c.y_bf16 ? launch_out<bf16, bf16>(a, vec, c.bf16, s) : launch_out<bf16, float>(a, vec, c.bf16, s))
                                 : (c.y_bf16 ? launch_out<float, bf16>(a, vec, c.bf16, s) : launch_out<float, float>(a, vec, c.bf16, s));
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
