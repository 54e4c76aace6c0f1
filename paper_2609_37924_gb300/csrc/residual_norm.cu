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
// Bound: HBM, (2 es_x + es_y + es_n) bytes per element: 11512 rows of 5376 (fp32 x, bf16 y) 123 us, 6.0 TB/s, 89 % of a
// plain copy's rate; 1024 rows of 2048 in bf16 4.4 us out of L2; one row 3.5 us, the launch.
// Past the ring, a block per row: 11512 rows of 5376, fp32 x and y, 144 us (128 at a copy's rate), of 8192, bf16 y, 200 (167), 4096
// of 16384 168 (119).  Other widths, element by element: 11512 rows of 5377 284 us (110), 1024 of 49152 760 (89).
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
  int* status;
};

// `bytes` (a multiple of 16) of global memory into shared memory, counted on the mbarrier
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
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

// four consecutive elements: what 32 lanes store at once are whole lines
__device__ __forceinline__ void ld4(const float* p, float (&v)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
}
__device__ __forceinline__ void ld4(const bf16* p, float (&v)[4]) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void st4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void st4(bf16* p, const float (&v)[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
// four parameters as they lie in memory
template <class T>
struct Raw4 {
  alignas(sizeof(T) * 4) uint32_t q[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(q) = *reinterpret_cast<const uint4*>(p);
    else *reinterpret_cast<uint2*>(q) = *reinterpret_cast<const uint2*>(p);
  }
  __device__ __forceinline__ void get(float (&v)[4]) const { ld4(reinterpret_cast<const T*>(q), v); }
};

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

// Many rows: blocks that stay, each with the rows of its next RING turns on the way into shared memory by bulk copies, so
// that the loads go on while a row waits for its sums.  (11512 rows of 5376, fp32 x and bf16 y: a block per row, which loads,
// sums, and stores one after the other, 157 us; blocks of 256 threads 153; gains read for every row, 149; eight elements a
// thread instead of four, whose 16-byte stores of fp32 fill half sectors, 134; 123 as it is.)
constexpr int RT = 512, RING = 3, kRingBytes = 112 * 1024;   // two blocks an SM
template <class XT, class YT>
__host__ __device__ constexpr int ring_stage(int d) { return d * static_cast<int>(sizeof(XT) + sizeof(YT)); }

template <class XT, class YT, class T, int NV>
__global__ void __launch_bounds__(RT, 2) norm_ring_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float red[2][32];
  __shared__ __align__(8) uint64_t full[RING];
  __shared__ int abort_flag;
  const int nvec = a.d / 4, stage_bytes = ring_stage<XT, YT>(a.d), step = gridDim.x;
  const uint32_t xb = a.d * sizeof(XT), yb = a.d * sizeof(YT);
  if (threadIdx.x == 0) {
    for (int i = 0; i < RING; ++i) mbar_init(&full[i], 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();
  pdl_enter();
  auto ask = [&](int row, int i) {         // thread 0
    uint8_t* to = smem + i * stage_bytes;
    mbar_arrive_expect_tx(&full[i], xb + yb);
    bulk_load(to, static_cast<const XT*>(a.x) + row * a.ldx, xb, &full[i]);
    bulk_load(to + xb, static_cast<const YT*>(a.y) + row * a.ldy, yb, &full[i]);
  };
  if (threadIdx.x == 0)
    for (int i = 0; i < RING; ++i)
      if (static_cast<int>(blockIdx.x) + i * step < a.total) ask(blockIdx.x + i * step, i);
  const T *post = static_cast<const T*>(a.post), *pre = static_cast<const T*>(a.pre), *gate = static_cast<const T*>(a.gate);
  Raw4<T> g_post[NV], g_pre[NV];           // the same for every row
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = threadIdx.x + i * RT;
    if (c < nvec && post) g_post[i].load(post + 4 * c);
    if (c < nvec && pre) g_pre[i].load(pre + 4 * c);
  }
  int stage = 0;
  uint32_t phase = 0;
  for (int row = blockIdx.x; row < a.total; row += step) {
    const int b = a.cu ? seq_of_row(a.cu, a.batch, row) : 0;
    if (__syncthreads_or(!mbar_wait_bounded(&full[stage], phase, &abort_flag, a.status))) break;
    const XT* x = reinterpret_cast<const XT*>(smem + stage * stage_bytes);
    const YT* y = reinterpret_cast<const YT*>(smem + stage * stage_bytes + xb);
    float v[NV][4], w[4];
    float r = 1.0f, s = 0.0f;
    if (post) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = threadIdx.x + i * RT;
        if (c < nvec) {
          ld4(y + 4 * c, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) s = fmaf(w[e], w[e], s);
        }
      }
      r = rsqrtf(row_sum<true>(s, red[0]) / static_cast<float>(a.d) + a.eps);
      s = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = threadIdx.x + i * RT;
      if (c < nvec) {
        float u[4];
        ld4(y + 4 * c, u);
        ld4(x + 4 * c, v[i]);
        if (post) {
          g_post[i].get(w);
#pragma unroll
          for (int e = 0; e < 4; ++e) u[e] = u[e] * r * w[e];
        }
        if (gate && b >= 0) {
          ld4(gate + b * a.ldg + 4 * c, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) u[e] *= w[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[i][e] = fmaf(a.alpha, v[i][e], u[e]);
          s = fmaf(v[i][e], v[i][e], s);
        }
      }
    }
    const float q = rsqrtf(row_sum<true>(s, red[1]) / static_cast<float>(a.d) + a.eps);   // (its barrier: the stage has been read)
    if (threadIdx.x == 0 && row + RING * step < a.total) ask(row + RING * step, stage);
    if (++stage == RING) { stage = 0; phase ^= 1; }
    if (b < 0) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = threadIdx.x + i * RT;
      if (c < nvec) {
        st4(static_cast<XT*>(a.xo) + row * a.ldxo + 4 * c, v[i]);
        if (!a.no) continue;
        if (pre) g_pre[i].get(w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = pre ? v[i][e] * q * w[e] : v[i][e] * q;
        st4(static_cast<T*>(a.no) + row * a.ldn + 4 * c, v[i]);
      }
    }
  }
  if (abort_flag && threadIdx.x == 0) {    // (a wait gave up: no copy is left in flight)
    volatile int never = 0;
    for (int i = 0; i < RING; ++i) {
      mbar_wait_bounded(&full[stage], phase, &never, a.status);
      if (++stage == RING) { stage = 0; phase ^= 1; }
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

template <class XT, class YT, class T, int NV>
cudaError_t launch_ring(const NormArgs& a, int dev, int sms, cudaStream_t s) {
  static PerDevice ready;
  cudaError_t e = cudaSuccess;
  if (ready.get(dev, [&] {
        e = cudaFuncSetAttribute(norm_ring_kernel<XT, YT, T, NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
        return e == cudaSuccess ? 1 : 0;
      }) <= 0)
    return e;
  return launch_pdl(norm_ring_kernel<XT, YT, T, NV>, 2 * sms, RT, RING * ring_stage<XT, YT>(a.d), s, a);
}

template <class XT, class YT, class T>
cudaError_t launch(const NormArgs& a, bool vec, cudaStream_t s) {
  const int nvec = a.d / 8;
  int dev = 0;
  const int sms = current_sms(&dev);
  // The ring for rows of more than 4096, two turns of every block or more.  Instead of a block per row, fp32 and bf16 x, bf16 y:
  //   of 5376   304 rows 6.1 for 6.2 us and 5.5 for 5.1; 608 9.6 for 11.0 and 8.7 for 9.1; 4864 57 for 69 and 45 for 58
  //   of 4096   1216 rows 12.2 for 12.8 and 11.3 for 9.8; 11512 101 for 85 and 78 for 65
  //   of 2048   1216 rows 8.6 for 7.0 and 8.3 for 5.5; 11512 55 for 44 and 56 for 32
  // (of narrow rows many are in flight at once as it is, and a turn of the ring ends in its barriers).
  if (vec && nvec > RT && nvec <= 2 * RT && a.total >= 4 * sms && RING * ring_stage<XT, YT>(a.d) <= kRingBytes)
    return a.d <= 3 * 4 * RT ? launch_ring<XT, YT, T, 3>(a, dev, sms, s) : launch_ring<XT, YT, T, 4>(a, dev, sms, s);
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
                   c.post, c.gate, c.pre, c.residual_scale, c.eps, c.status};
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
