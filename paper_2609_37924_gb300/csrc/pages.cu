// The paged 8-bit KV cache: rows into pages and back, and the pages' bookkeeping.
//
// A page holds 64 tokens of every KV head: K as [64, hd] and V transposed as
// [hd, 64] e4m3 bytes (the operand layouts that attention reads), with one
// fp32 scale for K and one for V per page and head.  Scales that this file
// writes are powers of two: dividing by one and multiplying by it are exact,
// e4m3 has an exponent of its own, so nothing is lost against a free scale
// but at most one bit of its range, and a page's earlier tokens survive a
// growing scale unchanged unless they fall below the smallest e4m3 step.
#include <cuda_fp8.h>

#include <algorithm>
#include <cstring>

#include "serve.h"

namespace tadm {
namespace {

constexpr int PT = TADM_PAGE_TOKENS;

// ------------------------------------------------------------ rows <-> pages
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }

// The least power of two s in 2^-60 .. 2^60 with amax <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ float needed_scale(float amax) {
  const int bits = __float_as_int(amax);
  const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return pow2f(min(60, max(-60, e)));
}

__device__ __forceinline__ uint32_t enc8(float x) {
  const uint32_t q = __nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
  return fabsf(x) <= 3.402823466e38f ? q : 0x7fu;     // infinities too become NaN
}
// four finite values at a time, the first in the low byte
__device__ __forceinline__ uint32_t enc8x4(const float* x, float s) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[0] * s, x[1] * s), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[2] * s, x[3] * s), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}
__device__ __forceinline__ void dec8x4(uint32_t w, float s, float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * h)), __NV_E4M3)));
    x[2 * h] = f.x * s, x[2 * h + 1] = f.y * s;
  }
}
// four words of four bytes, transposed
__device__ __forceinline__ void transpose4(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  const uint32_t p = __byte_perm(a, b, 0x5140), q = __byte_perm(c, d, 0x5140);
  const uint32_t r = __byte_perm(a, b, 0x7362), s = __byte_perm(c, d, 0x7362);
  a = __byte_perm(p, q, 0x5410), b = __byte_perm(p, q, 0x7632);
  c = __byte_perm(r, s, 0x5410), d = __byte_perm(r, s, 0x7632);
}

// 8 consecutive elements as they are in memory, and as floats
template <class T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <class T> __device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
// the largest magnitude as fp32 bits, infinities and NaN (0x7f800000 and above) included
__device__ __forceinline__ uint32_t top8(const Raw8<float>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    m = max(max(max(m, r.v[i].x & 0x7fffffffu), r.v[i].y & 0x7fffffffu), max(r.v[i].z & 0x7fffffffu, r.v[i].w & 0x7fffffffu));
  return m;
}
__device__ __forceinline__ uint32_t top8(const Raw8<bf16>& r) {
  const uint32_t m = __vmaxu2(__vmaxu2(r.v[0].x & 0x7fff7fffu, r.v[0].y & 0x7fff7fffu),
                              __vmaxu2(r.v[0].z & 0x7fff7fffu, r.v[0].w & 0x7fff7fffu));
  return max(m & 0xffff0000u, m << 16);
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(r.v[i].x), x[4 * i + 1] = __uint_as_float(r.v[i].y);
    x[4 * i + 2] = __uint_as_float(r.v[i].z), x[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
__device__ __forceinline__ void widen8(const Raw8<bf16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <class T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<bf16>(bf16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

struct RowsArgs {
  uint8_t *pk, *pv;            // this layer's pages
  float *sk, *sv;
  void *k, *v;                 // rows (read by the write, written by the read)
  const int32_t *cu, *start, *table;
  int64_t ldk, ldv;
  int total, max_rows, ld_table, pages, n_kv;
};

// What block (i, y, b) works on: the i-th 64-token range that sequence b
// touches, slots lo .. hi - 1 of it, which are rows row0 + lo .. of the operand,
// and the place of its page in the table (at most 2^20 wide: tokens fit 27 bits).
struct Part {
  int64_t entry;
  int row0, lo, hi;
};
__device__ __forceinline__ bool find_part(const RowsArgs& a, Part* p) {
  const int b = blockIdx.z, s = a.start[b];
  const int c0 = min(max(a.cu[b], 0), a.total), c1 = min(max(a.cu[b + 1], c0), a.total);
  const int n = min(min(c1 - c0, a.max_rows), 1 << 27);
  const int slot = s / PT + static_cast<int>(blockIdx.x);
  if (n <= 0 || s < 0 || slot >= a.ld_table) return false;
  const int first = slot * PT;
  if (first >= s + n) return false;
  p->entry = static_cast<int64_t>(b) * a.ld_table + slot;
  p->lo = max(s, first) - first;
  p->hi = min(s + n - first, PT);
  p->row0 = c0 + first - s;
  return true;
}

// V's tile in shared memory: 16 words of four slots per dim, the words of dim d
// in the order w ^ (d / 8), which spreads the 8-dim groups of a warp over the banks.
__device__ __forceinline__ int tile_word(int dim, int w) { return dim * 16 + (w ^ ((dim >> 3) & 15)); }

// One block per (page, head, K or V), 16 groups of HD / 8 threads: a thread
// takes 8 dims of four slots, which stay in registers between the maximum and
// the conversion, so the rows are read once.  V is transposed four slots (a
// word) at a time through shared memory.
// 6212 rows of 8 x 128 bf16 (K and V): 10.0 us for 38 MB, issue-bound (68 % of
// the slots); reading them back 7.5 us.  Single bytes of V into pages that keep
// tokens took 14.5 us: 8192 sector writes for such a page and head.
template <class T, int HD>
__global__ void __launch_bounds__(2 * HD, sizeof(T) == 2 ? 1024 / HD : 512 / HD) page_write_kernel(const RowsArgs a) {
  pdl_enter();
  constexpr int TPR = HD / 8, NT = 2 * HD;
  __shared__ uint32_t tile[HD * 16];
  __shared__ uint32_t red[NT / 32];
  Part p;
  if (!find_part(a, &p)) return;
  const int page = a.table[p.entry];
  const int head = blockIdx.y >> 1, is_v = blockIdx.y & 1;
  const int tid = threadIdx.x, w = tid / TPR, d = (tid % TPR) * 8;
  const int64_t ld = is_v ? a.ldv : a.ldk;
  const T* src = static_cast<const T*>(is_v ? a.v : a.k) + p.row0 * ld + static_cast<int64_t>(head) * HD + d;
  Raw8<T> raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * w + i;
    if (slot >= p.lo && slot < p.hi) raw[i] = load8<T>(src + slot * ld);
    else raw[i] = Raw8<T>{};
  }
  if (page < 0 || page >= a.pages) return;                    // uniform: not followed
  const int64_t ph = static_cast<int64_t>(page) * a.n_kv + head;
  float* sp = (is_v ? a.sv : a.sk) + ph;
  uint8_t* data = (is_v ? a.pv : a.pk) + ph * (PT * HD);
  const float had = p.lo > 0 ? *sp : 0.0f;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, top8(raw[i]));
  top = __reduce_max_sync(0xffffffffu, top);
  if ((tid & 31) == 0) red[tid >> 5] = top;
  __syncthreads();                                            // also: every thread has read the old scale
#pragma unroll
  for (int k = 0; k < NT / 32; ++k) top = max(top, red[k]);
  const bool odd = top >= 0x7f800000u;                        // an infinity or NaN among the rows: the largest finite value
  if (odd) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[8];
      widen8(raw[i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m = __float_as_uint(x[e]) & 0x7fffffffu;
        if (m < 0x7f800000u) top = max(top, m);
      }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    __syncthreads();
    if ((tid & 31) == 0) red[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NT / 32; ++k) top = max(top, red[k]);
  }
  const float amax = __uint_as_float(top);
  const float scale = fmaxf(needed_scale(amax), had);
  const float again = had >= 0.0f ? had / scale : 1.0f;       // what becomes of the tokens that stay (of scale 0: zeros)
  if (tid == 0 && scale != had) *sp = scale;
  const float inv = 1.0f / scale;
  const bool fresh = p.lo == 0;                               // slots past the rows become zeros
  uint32_t q[4][2];                                           // a slot's 8 dims
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[8];
    widen8(raw[i], x);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      q[i][h] = enc8x4(x + 4 * h, inv);
      if (odd) {
        q[i][h] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[i][h] |= enc8(x[4 * h + e] * inv) << (8 * e);
      }
    }
  }
  auto encode_again = [&](uint32_t word) {                    // four values in the new scale (a NaN stays one)
    float x[4];
    dec8x4(word, again, x);
    return enc8x4(x, 1.0f);
  };
  if (!is_v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * w + i;
      uint2* at = reinterpret_cast<uint2*>(data + slot * HD + d);
      if (fresh || (slot >= p.lo && slot < p.hi)) {
        *at = make_uint2(q[i][0], q[i][1]);
      } else if (slot < p.lo && again != 1.0f) {
        const uint2 old = *at;
        *at = make_uint2(encode_again(old.x), encode_again(old.y));
      }
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) transpose4(q[0][h], q[1][h], q[2][h], q[3][h]);   // now four slots of dim d + 4 h + e in q[e][h]
  if (fresh) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[tile_word(d + 4 * h + e, w)] = q[e][h];
    __syncthreads();
    for (int c = tid; c < HD * 4; c += NT) {
      const int dim = c >> 2, at = (c & 3) * 4;
      *reinterpret_cast<uint4*>(data + dim * PT + 4 * at) = make_uint4(tile[tile_word(dim, at)], tile[tile_word(dim, at + 1)],
                                                                       tile[tile_word(dim, at + 2)], tile[tile_word(dim, at + 3)]);
    }
  } else if (4 * w < p.hi && (4 * w + 4 > p.lo || again != 1.0f)) {
    // words of a page that keeps tokens: read, merged, written
    uint32_t mine = 0, before = 0;                            // bytes of the new rows, of the tokens that stay
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * w + i < p.lo) before |= 0xffu << (8 * i);
      else if (4 * w + i < p.hi) mine |= 0xffu << (8 * i);
    }
    uint32_t old[4][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) old[e][h] = *reinterpret_cast<const uint32_t*>(data + (d + 4 * h + e) * PT + 4 * w);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t o = old[e][h];
        if (again != 1.0f) o = (o & ~before) | (encode_again(o) & before);
        *reinterpret_cast<uint32_t*>(data + (d + 4 * h + e) * PT + 4 * w) = (o & ~mine) | (q[e][h] & mine);
      }
  }
}

// The same blocks and threads; rows of a page that the table does not hold read as zeros.
template <class T, int HD>
__global__ void __launch_bounds__(2 * HD) page_read_kernel(const RowsArgs a) {
  pdl_enter();
  constexpr int TPR = HD / 8, NT = 2 * HD;
  __shared__ uint32_t tile[HD * 16];
  Part p;
  if (!find_part(a, &p)) return;
  const int page = a.table[p.entry];
  const bool ok = page >= 0 && page < a.pages;
  const int head = blockIdx.y >> 1, is_v = blockIdx.y & 1;
  const int tid = threadIdx.x, w = tid / TPR, d = (tid % TPR) * 8;
  const int64_t ph = static_cast<int64_t>(ok ? page : 0) * a.n_kv + head;
  const float scale = ok ? (is_v ? a.sv : a.sk)[ph] : 0.0f;
  const uint8_t* data = (is_v ? a.pv : a.pk) + ph * (PT * HD);
  const int64_t ld = is_v ? a.ldv : a.ldk;
  T* dst = static_cast<T*>(is_v ? a.v : a.k) + p.row0 * ld + static_cast<int64_t>(head) * HD + d;
  uint32_t q[4][2];                                           // a slot's 8 dims
  if (is_v) {
    for (int c = tid; c < HD * 4; c += NT) {
      const int dim = c >> 2, at = (c & 3) * 4;
      const uint4 t = ok ? *reinterpret_cast<const uint4*>(data + dim * PT + 4 * at) : make_uint4(0, 0, 0, 0);
      tile[tile_word(dim, at)] = t.x, tile[tile_word(dim, at + 1)] = t.y;
      tile[tile_word(dim, at + 2)] = t.z, tile[tile_word(dim, at + 3)] = t.w;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e][h] = tile[tile_word(d + 4 * h + e, w)];
      transpose4(q[0][h], q[1][h], q[2][h], q[3][h]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * w + i;
      const uint2 t = ok && slot >= p.lo && slot < p.hi ? *reinterpret_cast<const uint2*>(data + slot * HD + d) : make_uint2(0, 0);
      q[i][0] = t.x, q[i][1] = t.y;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * w + i;
    if (slot < p.lo || slot >= p.hi) continue;
    float x[8];
    dec8x4(q[i][0], scale, x);
    dec8x4(q[i][1], scale, x + 4);
    store8<T>(dst + slot * ld, x);
  }
}

template <class T, int HD>
cudaError_t launch_rows(const RowsArgs& a, int batch, bool write, cudaStream_t s) {
  const dim3 grid((a.max_rows + PT - 2) / PT + 1, 2 * a.n_kv, batch);
  return write ? launch_pdl(page_write_kernel<T, HD>, grid, 2 * HD, 0, s, a) : launch_pdl(page_read_kernel<T, HD>, grid, 2 * HD, 0, s, a);
}

// ------------------------------------------------------------- bookkeeping
// Every call is two launches: one block plans (checks, counts, prefix sums in
// list order, the free list lowest id first), then a grid applies the plan to
// the tables and moves the pages.  The plan lives in the caller's scratch.
constexpr int PB = 1024;      // threads of the planning block

struct Plan {
  int status, n_copies, pad[2];
};
struct Scratch {
  Plan* plan;
  int *mark;                        // [n_seqs] 1 + list index of a listed (target) sequence, 0 for the others
  int *first, *count, *offset;      // [n_seqs] per list entry: first slot that gets a new page, how many, where in fresh
  int *fresh;                       // [pages] free pages taken, in order
  int *from, *to;                   // [pages] page copies
  int *map;                         // [pages] new id of a page
};
size_t scratch_layout(int pages, int n_seqs, char* base, Scratch* s) {
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (4 * n + 15) / 16 * 16;
    return reinterpret_cast<int*>(base + o);
  };
  Scratch t;
  t.plan = reinterpret_cast<Plan*>(take(4));
  t.mark = take(n_seqs), t.first = take(n_seqs), t.count = take(n_seqs), t.offset = take(n_seqs);
  t.fresh = take(pages), t.from = take(pages), t.to = take(pages), t.map = take(pages);
  if (s) *s = t;
  return at;
}

// Exclusive prefix sum of v over the block; *total is the block's sum.  Every thread calls it.
__device__ __forceinline__ int block_scan(int v, int* total) {
  __shared__ int ws[PB / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) ws[warp] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < PB / 32; ++w) {
    const int y = ws[w];
    if (w < warp) before += y;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// The first `want` pages without a reference, ascending, into fresh; returns how many there are (at most want).
__device__ int take_free(const int32_t* refs, int pages, int want, int* fresh) {
  int have = 0;
  for (int base = 0; base < pages && have < want; base += 4 * PB) {
    int free4 = 0, n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = base + 4 * static_cast<int>(threadIdx.x) + e;
      if (p < pages && refs[p] == 0) free4 |= 1 << e, ++n;
    }
    int total;
    int at = have + block_scan(n, &total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (free4 >> e & 1) {
        if (at < want) fresh[at] = base + 4 * static_cast<int>(threadIdx.x) + e;
        ++at;
      }
    have += total;
  }
  return min(have, want);
}

__device__ __forceinline__ int pages_of(int tokens) { return tokens / PT + (tokens % PT != 0); }

struct SeqArgs {
  const int32_t *tables, *lens, *refs, *list, *list2;
  int32_t *tables_out, *lens_out, *refs_out, *status;
  int pages, n_seqs, ld, n;
  Scratch sc;
};

// Marks the listed sequences; false where one is out of range or listed twice.
__device__ bool mark_list(const SeqArgs& a, const int32_t* list) {
  for (int i = threadIdx.x; i < a.n_seqs; i += PB) a.sc.mark[i] = 0;
  __syncthreads();
  bool ok = true;
  for (int i = threadIdx.x; i < a.n; i += PB) {
    const int s = list[i];
    if (s < 0 || s >= a.n_seqs || atomicCAS(a.sc.mark + s, 0, i + 1) != 0) ok = false;
  }
  return __syncthreads_and(ok);
}

__device__ __forceinline__ void copy_refs(const SeqArgs& a) {
  if (a.refs_out != a.refs)
    for (int i = threadIdx.x; i < a.pages; i += PB) a.refs_out[i] = a.refs[i];
}

__device__ __forceinline__ void finish(const SeqArgs& a, int status, int copies) {
  if (threadIdx.x == 0) {
    a.sc.plan->status = status;
    a.sc.plan->n_copies = status ? 0 : copies;
    *a.status = status;
  }
}

// How many pages sequence s holds (its row's entries before the first -1), by one warp.
__device__ __forceinline__ int held(const SeqArgs& a, int s) {
  const int32_t* row = a.tables + static_cast<int64_t>(s) * a.ld;
  for (int i = 0; i < a.ld; i += 32) {
    const int j = i + (threadIdx.x & 31);
    const unsigned none = __ballot_sync(0xffffffffu, j >= a.ld || row[j] < 0);
    if (none) return i + __ffs(none) - 1;
  }
  return a.ld;
}

__global__ void __launch_bounds__(PB) plan_reserve_kernel(const SeqArgs a) {
  pdl_enter();
  int status = mark_list(a, a.list) ? 0 : TADM_PAGES_BAD;
  bool ok = true;
  if (!status)
    for (int i = threadIdx.x >> 5; i < a.n; i += PB / 32) {
      const int have = held(a, a.list[i]), want = a.list2[i];
      if (want < 0 || pages_of(want) > a.ld) ok = false;
      // a page that it holds and that counts as free would be handed out a second time
      const int32_t* row = a.tables + static_cast<int64_t>(a.list[i]) * a.ld;
      for (int j = threadIdx.x & 31; j < have; j += 32)
        if (row[j] >= a.pages || a.refs[row[j]] <= 0) ok = false;
      if ((threadIdx.x & 31) == 0) {
        a.sc.first[i] = have;
        a.sc.count[i] = max(0, pages_of(max(want, 0)) - have);
      }
    }
  if (!__syncthreads_and(ok)) status = TADM_PAGES_BAD;
  int need = 0;
  for (int base = 0; !status && base < a.n; base += PB) {
    const int i = base + threadIdx.x;
    int total;
    // a sum past the pool saturates (each term and the pool are below 2^31 / PB after the clamp)
    const int at = block_scan(i < a.n ? min(a.sc.count[i], min(a.pages, (1 << 20)) + 1) : 0, &total);
    if (i < a.n) a.sc.offset[i] = need + at;
    need = total > a.pages - need ? a.pages + 1 : need + total;
    if (need > a.pages) status = TADM_PAGES_SHORT;
  }
  __syncthreads();
  if (!status && take_free(a.refs, a.pages, need, a.sc.fresh) < need) status = TADM_PAGES_SHORT;
  __syncthreads();
  copy_refs(a);
  __syncthreads();
  if (!status)
    for (int k = threadIdx.x; k < need; k += PB) a.refs_out[a.sc.fresh[k]] = 1;
  finish(a, status, 0);
}

// (Each step is a chain of dependent reads of about 0.7 us each: what does not
// need the list comes first, and the steps share their barriers.)
__global__ void __launch_bounds__(PB) plan_fork_kernel(const SeqArgs a) {
  pdl_enter();
  copy_refs(a);
  const int have = take_free(a.refs, a.pages, min(a.n, a.pages), a.sc.fresh);   // an entry takes one page at most
  int status = mark_list(a, a.list2) ? 0 : TADM_PAGES_BAD;
  bool ok = true;
  int need = 0;
  for (int base = 0; !status && base < a.n; base += PB) {
    const int i = base + threadIdx.x;
    int c = 0;
    if (i < a.n) {
      const int s = a.list[i];
      const bool in = s >= 0 && s < a.n_seqs && a.sc.mark[s] == 0;
      const int len = in ? a.lens[s] : -1;
      if (len < 0 || pages_of(len) > a.ld || a.tables[static_cast<int64_t>(a.list2[i]) * a.ld] >= 0) ok = false;
      else c = len % PT != 0;
      a.sc.count[i] = c;
      a.sc.first[i] = max(len, 0) / PT;
    }
    int total;
    const int at = block_scan(c, &total);
    if (i < a.n) a.sc.offset[i] = need + at;
    need += total;
  }
  if (!__syncthreads_and(ok)) status = TADM_PAGES_BAD;
  if (!status)
    for (int i = threadIdx.x >> 4; i < a.n; i += PB / 16) {     // the pages that are shared or copied, 16 threads per entry
      const int32_t* row = a.tables + static_cast<int64_t>(a.list[i]) * a.ld;
      const int np = a.sc.first[i] + a.sc.count[i];
      for (int j = threadIdx.x & 15; j < np; j += 16) {
        const int p = row[j];
        if (p < 0 || p >= a.pages || a.refs[p] <= 0) ok = false;
      }
    }
  if (!__syncthreads_and(ok)) status = TADM_PAGES_BAD;
  if (!status && need > have) status = TADM_PAGES_SHORT;
  if (!status)
    for (int i = threadIdx.x; i < a.n; i += PB)
      if (a.sc.count[i]) {
        const int k = a.sc.offset[i], page = a.sc.fresh[k];
        a.refs_out[page] = 1;
        a.sc.from[k] = a.tables[static_cast<int64_t>(a.list[i]) * a.ld + a.sc.first[i]];
        a.sc.to[k] = page;
      }
  finish(a, status, need);
}

__global__ void __launch_bounds__(PB) plan_free_kernel(const SeqArgs a) {
  pdl_enter();
  int status = mark_list(a, a.list) ? 0 : TADM_PAGES_BAD;
  copy_refs(a);
  __syncthreads();
  if (!status) {
    // references go down; one that falls below 0 (or an id out of range) takes all of them back
    auto each = [&](auto f) {
      for (int i = threadIdx.x >> 5; i < a.n; i += PB / 32) {
        const int32_t* row = a.tables + static_cast<int64_t>(a.list[i]) * a.ld;
        const int n = held(a, a.list[i]);
        for (int j = threadIdx.x & 31; j < n; j += 32) f(row[j]);
      }
    };
    bool ok = true;
    each([&](int p) {
      if (p >= a.pages) ok = false;
      else if (atomicSub(a.refs_out + p, 1) <= 0) ok = false;
    });
    if (!__syncthreads_and(ok)) {
      status = TADM_PAGES_BAD;
      each([&](int p) { if (p < a.pages) atomicAdd(a.refs_out + p, 1); });
    }
  }
  finish(a, status, 0);
}

__global__ void __launch_bounds__(PB) plan_compact_kernel(const SeqArgs a) {
  pdl_enter();
  int live = 0;
  for (int base = 0; base < a.pages; base += PB) {
    const int p = base + threadIdx.x;
    live += __syncthreads_count(p < a.pages && a.refs[p] > 0);
  }
  // the i-th hole below `live` and the i-th page in use from there on
  int holes = 0, movers = 0;
  for (int base = 0; base < a.pages; base += PB) {
    const int p = base + threadIdx.x;
    const bool used = p < a.pages && a.refs[p] > 0;
    const bool hole = p < live && !used, mover = used && p >= live;
    int total;
    const int at = block_scan((hole ? 1 : 0) | (mover ? 1 << 16 : 0), &total);   // at most 1024 of each
    if (hole) a.sc.to[holes + (at & 0xffff)] = p;
    if (mover) a.sc.from[movers + (at >> 16)] = p;
    holes += total & 0xffff;
    movers += total >> 16;
    if (p < a.pages) a.sc.map[p] = p;
  }
  __syncthreads();
  copy_refs(a);
  __syncthreads();
  for (int k = threadIdx.x; k < movers; k += PB) {
    const int from = a.sc.from[k], to = a.sc.to[k];
    a.refs_out[to] = a.refs[from];
    a.sc.map[from] = to;
  }
  __syncthreads();                       // in place: every mover's count has been read
  for (int k = threadIdx.x; k < movers; k += PB) a.refs_out[a.sc.from[k]] = 0;
  if (threadIdx.x == 0) {
    a.sc.plan->status = 0;
    a.sc.plan->n_copies = movers;
    *a.status = live;
  }
}

// Copies pages from[i] -> to[i], i < *n (n_max where n is null), in every layer: 16-byte vectors in chunks of 4 KB,
// four chunks of a block in flight.
struct CopyArgs {
  uint4 *k, *v;
  float *sk, *sv;
  const int *from, *to, *n;
  int n_max, layers, pages, n_kv;
  int page_chunks;                 // chunks of 256 vectors per page and layer
};
__device__ __forceinline__ bool pair_ok(const CopyArgs& c, int from, int to) {
  return from >= 0 && from < c.pages && to >= 0 && to < c.pages;
}
__device__ void copy_pages(const CopyArgs& c, int block, int blocks) {
  const int n = c.n ? *c.n : c.n_max;
  const int64_t per = static_cast<int64_t>(c.layers) * 2 * c.page_chunks, total = n * per;
  constexpr int U = 4;
  for (int64_t base = static_cast<int64_t>(block) * U; base < total; base += static_cast<int64_t>(blocks) * U) {
    uint4 x[U];
    uint4* dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      dst[u] = nullptr;
      const int64_t id = base + u;
      if (id >= total) continue;
      const int in = static_cast<int>(id / n), i = static_cast<int>(id - static_cast<int64_t>(in) * n);
      const int unit = in / c.page_chunks, chunk = in - unit * c.page_chunks;
      const int from = c.from[i], to = c.to[i];
      if (!pair_ok(c, from, to)) continue;
      uint4* base_p = (unit & 1) ? c.v : c.k;
      const int64_t layer = static_cast<int64_t>(unit >> 1) * c.pages;
      const int64_t at = static_cast<int64_t>(chunk) * 256 + threadIdx.x;
      x[u] = base_p[(layer + from) * c.page_chunks * 256 + at];
      dst[u] = base_p + (layer + to) * c.page_chunks * 256 + at;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (dst[u]) *dst[u] = x[u];
  }
  const int64_t ns = static_cast<int64_t>(n) * c.layers * c.n_kv;
  for (int64_t e = static_cast<int64_t>(block) * 256 + threadIdx.x; e < ns; e += static_cast<int64_t>(blocks) * 256) {
    const int i = static_cast<int>(e / (c.layers * c.n_kv));
    const int in = static_cast<int>(e - static_cast<int64_t>(i) * c.layers * c.n_kv), l = in / c.n_kv, h = in - l * c.n_kv;
    const int from = c.from[i], to = c.to[i];
    if (!pair_ok(c, from, to)) continue;
    const int64_t src = (static_cast<int64_t>(l) * c.pages + from) * c.n_kv + h;
    const int64_t dst = (static_cast<int64_t>(l) * c.pages + to) * c.n_kv + h;
    c.sk[dst] = c.sk[src];
    c.sv[dst] = c.sv[src];
  }
}

// The same copies, from the caller's lists.
__global__ void __launch_bounds__(256) copy_pages_kernel(const CopyArgs c) {
  pdl_enter();
  copy_pages(c, blockIdx.x, gridDim.x);
}

enum { OP_RESERVE, OP_FORK, OP_FREE, OP_COMPACT };

// The planned tables, and the page copies.  Bound by memory: 48 last pages of 22
// layers (46 MB, each written three times, 138 MB) 41 us, at the rate of plain
// writes; 96 pages moved to the front (277 MB) 89 us, near a plain copy's.  The
// plans ahead take 10 and 5 us, chains of dependent reads.
template <int OP>
__global__ void __launch_bounds__(256) apply_kernel(const SeqArgs a, const CopyArgs c) {
  pdl_enter();
  const bool ok = a.sc.plan->status == 0, same = a.tables_out == a.tables;
  const int64_t entries = static_cast<int64_t>(a.n_seqs) * a.ld;
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < entries; e += static_cast<int64_t>(gridDim.x) * 256) {
    const int row = static_cast<int>(e / a.ld), slot = static_cast<int>(e - static_cast<int64_t>(row) * a.ld);
    if (OP == OP_COMPACT) {
      const int p = a.tables[e];
      a.tables_out[e] = p >= 0 && p < a.pages ? a.sc.map[p] : p;
      continue;
    }
    const int i = ok ? a.sc.mark[row] - 1 : -1;
    if (i < 0) {
      if (!same) a.tables_out[e] = a.tables[e];
    } else if (OP == OP_FREE) {
      a.tables_out[e] = -1;
    } else if (OP == OP_RESERVE) {
      const int k = slot - a.sc.first[i];
      if (k >= 0 && k < a.sc.count[i]) a.tables_out[e] = a.sc.fresh[a.sc.offset[i] + k];
      else if (!same) a.tables_out[e] = a.tables[e];
    } else {
      int p = -1;
      if (slot < a.sc.first[i]) {                               // a page that the source's tokens fill
        p = a.tables[static_cast<int64_t>(a.list[i]) * a.ld + slot];
        atomicAdd(a.refs_out + p, 1);
      } else if (slot == a.sc.first[i] && a.sc.count[i]) {
        p = a.sc.fresh[a.sc.offset[i]];
      }
      a.tables_out[e] = p;
    }
  }
  if (OP == OP_FORK || OP == OP_FREE)
    for (int row = blockIdx.x * 256 + threadIdx.x; row < a.n_seqs; row += gridDim.x * 256) {
      const int i = ok ? a.sc.mark[row] - 1 : -1;
      if (i >= 0) a.lens_out[row] = OP == OP_FREE ? 0 : a.lens[a.list[i]];
      else if (a.lens_out != a.lens) a.lens_out[row] = a.lens[row];
    }
  if (OP == OP_FORK || OP == OP_COMPACT) copy_pages(c, blockIdx.x, gridDim.x);
}

CopyArgs copy_args(const tadm_page_pool& p, const int* from, const int* to, const int* n, int n_max) {
  return CopyArgs{static_cast<uint4*>(p.k), static_cast<uint4*>(p.v), p.k_scale, p.v_scale, from, to, n, n_max,
                  p.layers, p.pages, p.n_kv_heads, p.n_kv_heads * PT * p.head_dim / 4096};
}

// Blocks for `bytes` of copying and `entries` of tables: 16 KB or 256 entries each, at most eight per SM.
int apply_grid(int64_t bytes, int64_t entries) {
  int dev = 0;
  const int64_t most = 8LL * current_sms(&dev);
  return static_cast<int>(std::max<int64_t>(1, std::min(most, std::max(bytes / 16384, entries / 256) + 1)));
}

template <int OP>
const char* run_pages(const PagesCall& c, cudaStream_t s, void (*plan)(SeqArgs)) {
  Scratch sc;
  scratch_layout(c.pages, c.n_seqs, static_cast<char*>(c.scratch), &sc);
  const SeqArgs a{c.tables, c.lens, c.refs, c.list, c.list2, c.tables_out, c.lens_out, c.refs_out, c.status,
                  c.pages, c.n_seqs, c.ld_table, c.n, sc};
  CopyArgs cp{};
  int64_t bytes = 0;
  if (c.pool) {
    cp = copy_args(*c.pool, sc.from, sc.to, &sc.plan->n_copies, 0);
    const int64_t most = OP == OP_FORK ? c.n : c.pages / 2;
    bytes = most * 2 * c.pool->layers * cp.page_chunks * 4096;
  }
  cudaError_t e = launch_pdl(plan, 1, PB, 0, s, a);
  if (e == cudaSuccess)
    e = launch_pdl(apply_kernel<OP>, apply_grid(bytes, static_cast<int64_t>(c.n_seqs) * c.ld_table), 256, 0, s, a, cp);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace

const char* page_rows(const PageRowsCall& c, bool write, cudaStream_t s) {
  if (c.batch == 0 || c.max_rows == 0) return nullptr;
  const tadm_page_pool& p = *c.pool;
  const int64_t page = static_cast<int64_t>(p.pages) * p.n_kv_heads;
  RowsArgs a{static_cast<uint8_t*>(p.k) + c.layer * page * PT * p.head_dim,
             static_cast<uint8_t*>(p.v) + c.layer * page * PT * p.head_dim,
             p.k_scale + c.layer * page, p.v_scale + c.layer * page, c.k, c.v, c.cu, c.start, c.table, c.ldk, c.ldv,
             c.total, c.max_rows, c.ld_table, p.pages, p.n_kv_heads};
  cudaError_t e;
  if (p.head_dim == 128) e = c.bf16 ? launch_rows<bf16, 128>(a, c.batch, write, s) : launch_rows<float, 128>(a, c.batch, write, s);
  else e = c.bf16 ? launch_rows<bf16, 64>(a, c.batch, write, s) : launch_rows<float, 64>(a, c.batch, write, s);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

size_t pages_scratch(int pages, int n_seqs) { return scratch_layout(pages, n_seqs, nullptr, nullptr); }
const char* pages_reserve(const PagesCall& c, cudaStream_t s) { return run_pages<OP_RESERVE>(c, s, plan_reserve_kernel); }
const char* pages_fork(const PagesCall& c, cudaStream_t s) { return run_pages<OP_FORK>(c, s, plan_fork_kernel); }
const char* pages_free(const PagesCall& c, cudaStream_t s) { return run_pages<OP_FREE>(c, s, plan_free_kernel); }
const char* pages_compact(const PagesCall& c, cudaStream_t s) { return run_pages<OP_COMPACT>(c, s, plan_compact_kernel); }
const char* pages_copy(const tadm_page_pool& p, const int32_t* src, const int32_t* dst, int n, cudaStream_t s) {
  if (n == 0) return nullptr;
  const CopyArgs c = copy_args(p, src, dst, nullptr, n);
  const cudaError_t e = launch_pdl(copy_pages_kernel, apply_grid(2LL * n * p.layers * c.page_chunks * 4096, 0), 256, 0, s, c);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace tadm
