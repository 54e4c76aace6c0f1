// C entry points of the operators for sequences of different lengths: the
// checks of their arguments (all on the host, before anything is enqueued)
// and the choice of kernel.
#include <cstdint>

#include "per_device.h"
#include "serve.h"

using namespace tadm;

// Set by an attention kernel that gave up a bounded wait, cleared by tadm_ragged_sync_status().
__device__ int g_ragged_status;

namespace tadm {
int* ragged_status() {
  struct Word {
    int* at[PerDevice::kMax] = {};
  };
  static Word word;
  static PerDevice ready;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= PerDevice::kMax) return nullptr;
  const int ok = ready.get(dev, [&] {
    // (no work on a stream: allowed while one is captured)
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) return 0;
    void* p = nullptr;
    const bool got = cudaGetSymbolAddress(&p, g_ragged_status) == cudaSuccess;
    cudaThreadExchangeStreamCaptureMode(&mode);
    word.at[dev] = static_cast<int*>(p);
    return got ? 1 : 0;
  });
  return ok > 0 ? word.at[dev] : nullptr;
}
}  // namespace tadm

namespace {

bool aligned(const void* p, size_t n = 16) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int es(int dtype) { return dtype ? 2 : 4; }

// rows of an operand: 16-byte aligned, wide enough
bool rows_ok(const void* p, int64_t ld, int64_t width, int dtype) {
  return p && aligned(p) && ld >= width && (ld * es(dtype)) % 16 == 0;
}
bool packed_ok(const int32_t* cu, int batch, int total, int max_rows) {
  return batch >= 0 && total >= 0 && max_rows >= 0 && (cu || batch == 0);
}
bool pool_ok(const tadm_page_pool* p) {
  return p && p->layers > 0 && p->pages > 0 && p->n_kv_heads > 0 && p->n_kv_heads <= 16384 &&
         (p->head_dim == 64 || p->head_dim == 128) &&
         p->k && p->v && p->k_scale && p->v_scale && aligned(p->k) && aligned(p->v) && aligned(p->k_scale, 4) &&
         aligned(p->v_scale, 4);
}
// ld_table * 64 tokens have to be an int32; grids cover batch * touched pages
bool table_ok(const int32_t* table, int ld_table, int rows) {
  return ld_table >= 0 && ld_table <= (1 << 20) && (table || ld_table == 0 || rows == 0);
}

tadm_status page_rows_call(const tadm_page_pool* pool, int layer, const void* k, const void* v, const int32_t* cu,
                           const int32_t* start, int batch, int total, int max_rows, int64_t ldk, int64_t ldv,
                           const int32_t* table, int ld_table, int dtype, bool write, cudaStream_t s) {
  if (!pool_ok(pool) || layer < 0 || layer >= pool->layers || (dtype != 0 && dtype != 1) ||
      !packed_ok(cu, batch, total, max_rows) || (!start && batch > 0) || !table_ok(table, ld_table, batch))
    return TADM_ERR_INVALID_ARG;
  if (batch == 0 || total == 0 || max_rows == 0) return TADM_OK;
  const int64_t width = static_cast<int64_t>(pool->n_kv_heads) * pool->head_dim;
  if (!rows_ok(k, ldk, width, dtype) || !rows_ok(v, ldv, width, dtype)) return TADM_ERR_INVALID_ARG;
  const int rows = max_rows < total ? max_rows : total;      // no sequence has more
  if (batch > 65535) return TADM_ERR_UNSUPPORTED;            // a grid dimension
  const PageRowsCall c{pool, layer, const_cast<void*>(k), const_cast<void*>(v), cu, start, table, batch, total, rows,
                       ld_table, ldk, ldv, dtype};
  return page_rows(c, write, s) ? TADM_ERR_CUDA : TADM_OK;
}

bool heads_ok(int n_heads, int n_kv, int head_dim) {
  return n_heads > 0 && n_kv > 0 && n_heads % n_kv == 0 && n_kv <= 16384 && (head_dim == 64 || head_dim == 128);
}

// query heads x rows of one sequence and KV head, and tiles of 16 of them over the call, are int32
bool grid_ok(int batch, int total, int rows, int group) {
  return static_cast<int64_t>(rows) * group <= INT32_MAX - 512 &&
         static_cast<int64_t>(total) * group / 16 + batch <= INT32_MAX;
}

bool seqs_ok(const int32_t* tables, const int32_t* refs, int pages, int n_seqs, int ld_table, const int32_t* list, int n,
             const int32_t* tables_out, const int32_t* refs_out, const int32_t* status, const void* scratch,
             size_t scratch_bytes) {
  if (pages < 0 || n_seqs < 0 || !table_ok(tables, ld_table, n_seqs) || !table_ok(tables_out, ld_table, n_seqs) ||
      (pages > 0 && (!refs || !refs_out)) || n < 0 || n > n_seqs || (n > 0 && !list) || !status)
    return false;
  return scratch && aligned(scratch) && scratch_bytes >= pages_scratch(pages, n_seqs);
}

}  // namespace

extern "C" {

tadm_status tadm_attention_packed(const void* q, const void* k, const void* v, void* o, const int32_t* cu_rows, int batch,
                                  int total_rows, int max_rows, int n_heads, int n_kv_heads, int head_dim, int64_t ldq,
                                  int64_t ldk, int64_t ldv, int64_t ldo, int causal, int window, int dtype,
                                  tadm_stream stream) {
  if (!packed_ok(cu_rows, batch, total_rows, max_rows) || !heads_ok(n_heads, n_kv_heads, head_dim) || window < 0 ||
      (dtype != 0 && dtype != 1) || (causal != 0 && causal != 1))
    return TADM_ERR_INVALID_ARG;
  if (batch == 0 || total_rows == 0 || max_rows == 0) return TADM_OK;
  const int64_t wq = static_cast<int64_t>(n_heads) * head_dim, wk = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (!rows_ok(q, ldq, wq, dtype) || !rows_ok(k, ldk, wk, dtype) || !rows_ok(v, ldv, wk, dtype) ||
      !rows_ok(o, ldo, wq, dtype))
    return TADM_ERR_INVALID_ARG;
  if (!grid_ok(batch, total_rows, max_rows < total_rows ? max_rows : total_rows, n_heads / n_kv_heads)) return TADM_ERR_UNSUPPORTED;
  // a tile of the tensor-core kernel holds whole rows, all query heads of a KV head; its grid is one-dimensional
  if (dtype && (n_heads / n_kv_heads > 128 ||
                (static_cast<int64_t>(total_rows) / (128 / (n_heads / n_kv_heads)) + batch) * n_kv_heads > INT32_MAX))
    return TADM_ERR_UNSUPPORTED;
  RaggedCall c{};
  c.q = q, c.k = k, c.v = v, c.o = o;
  c.cu = cu_rows, c.batch = batch, c.total = total_rows, c.max_rows = max_rows < total_rows ? max_rows : total_rows;
  c.n_heads = n_heads, c.n_kv = n_kv_heads, c.head_dim = head_dim;
  c.ldq = ldq, c.ldk = ldk, c.ldv = ldv, c.ldo = ldo;
  c.causal = causal, c.window = window < c.max_rows ? window : 0, c.bf16 = dtype;   // none where no distance reaches it
  if (dtype && !(c.status = ragged_status())) return TADM_ERR_CUDA;
  return (dtype ? attention_packed(c, stream) : attention_rows(c, stream)) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_page_write(const tadm_page_pool* pool, int layer, const void* k, const void* v, const int32_t* cu_rows,
                            const int32_t* start, int batch, int total_rows, int max_rows, int64_t ldk, int64_t ldv,
                            const int32_t* table, int ld_table, int dtype, tadm_stream stream) {
  return page_rows_call(pool, layer, k, v, cu_rows, start, batch, total_rows, max_rows, ldk, ldv, table, ld_table, dtype,
                        true, stream);
}

tadm_status tadm_page_read(const tadm_page_pool* pool, int layer, void* k, void* v, const int32_t* cu_rows,
                           const int32_t* start, int batch, int total_rows, int max_rows, int64_t ldk, int64_t ldv,
                           const int32_t* table, int ld_table, int dtype, tadm_stream stream) {
  return page_rows_call(pool, layer, k, v, cu_rows, start, batch, total_rows, max_rows, ldk, ldv, table, ld_table, dtype,
                        false, stream);
}

tadm_status tadm_page_attention_scratch_size(int batch, int total_rows, int max_rows, int max_len, int n_heads,
                                             int n_kv_heads, int head_dim, int dtype, size_t* bytes) {
  if (batch < 0 || total_rows < 0 || max_rows < 0 || max_len < 0 || !heads_ok(n_heads, n_kv_heads, head_dim) ||
      (dtype != 0 && dtype != 1) || !bytes)
    return TADM_ERR_INVALID_ARG;
  const int rows = max_rows < total_rows ? max_rows : total_rows;
  *bytes = dtype ? attention_paged_scratch(rows, n_heads / n_kv_heads, head_dim) : 0;
  return TADM_OK;
}

tadm_status tadm_page_attention(const void* q, const tadm_page_pool* pool, int layer, void* o, const int32_t* cu_rows,
                                const int32_t* lens, int batch, int total_rows, int max_rows, int max_len, int n_heads,
                                int64_t ldq, int64_t ldo, const int32_t* table, int ld_table, int causal, int window,
                                int dtype, void* scratch, size_t scratch_bytes, tadm_stream stream) {
  if (!pool_ok(pool) || layer < 0 || layer >= pool->layers || !packed_ok(cu_rows, batch, total_rows, max_rows) ||
      !heads_ok(n_heads, pool->n_kv_heads, pool->head_dim) || window < 0 || (dtype != 0 && dtype != 1) ||
      (causal != 0 && causal != 1) || max_len < 0 || !table_ok(table, ld_table, batch) ||
      max_len > static_cast<int64_t>(ld_table) * TADM_PAGE_TOKENS || (!lens && batch > 0))
    return TADM_ERR_INVALID_ARG;
  if (batch == 0 || total_rows == 0 || max_rows == 0) return TADM_OK;
  const int64_t wq = static_cast<int64_t>(n_heads) * pool->head_dim;
  if (!rows_ok(q, ldq, wq, dtype) || !rows_ok(o, ldo, wq, dtype)) return TADM_ERR_INVALID_ARG;
  if (!grid_ok(batch, total_rows, max_rows < total_rows ? max_rows : total_rows, n_heads / pool->n_kv_heads))
    return TADM_ERR_UNSUPPORTED;
  size_t need = 0;
  tadm_page_attention_scratch_size(batch, total_rows, max_rows, max_len, n_heads, pool->n_kv_heads, pool->head_dim, dtype, &need);
  if (need > 0 && (!scratch || !aligned(scratch) || scratch_bytes < need)) return TADM_ERR_INVALID_ARG;
  RaggedCall c{};
  c.q = q, c.o = o, c.pool = pool, c.layer = layer;
  c.cu = cu_rows, c.lens = lens, c.table = table, c.batch = batch, c.total = total_rows;
  c.max_rows = max_rows < total_rows ? max_rows : total_rows, c.max_len = max_len, c.ld_table = ld_table;
  c.n_heads = n_heads, c.n_kv = pool->n_kv_heads, c.head_dim = pool->head_dim;
  c.ldq = ldq, c.ldo = ldo, c.causal = causal, c.bf16 = dtype, c.scratch = scratch;
  c.window = window < max_len ? window : 0;                   // none where no distance reaches it
  if (dtype && !(c.status = ragged_status())) return TADM_ERR_CUDA;
  return (dtype ? attention_paged(c, stream) : attention_rows(c, stream)) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_ragged_sync_status(tadm_stream stream) {
  int* word = ragged_status();
  int st = 0;
  if (!word || cudaStreamSynchronize(stream) != cudaSuccess ||
      cudaMemcpy(&st, word, sizeof st, cudaMemcpyDeviceToHost) != cudaSuccess || (st && cudaMemset(word, 0, sizeof st) != cudaSuccess))
    return TADM_ERR_CUDA;
  return st ? TADM_ERR_TIMEOUT : TADM_OK;
}

tadm_status tadm_pages_scratch_size(int pages, int n_seqs, size_t* bytes) {
  if (pages < 0 || n_seqs < 0 || !bytes) return TADM_ERR_INVALID_ARG;
  *bytes = pages_scratch(pages, n_seqs);
  return TADM_OK;
}

tadm_status tadm_pages_reserve(const int32_t* tables, const int32_t* refs, int pages, int n_seqs, int ld_table,
                               const int32_t* seqs, const int32_t* new_len, int n, int32_t* tables_out, int32_t* refs_out,
                               int32_t* status, void* scratch, size_t scratch_bytes, tadm_stream stream) {
  if (!seqs_ok(tables, refs, pages, n_seqs, ld_table, seqs, n, tables_out, refs_out, status, scratch, scratch_bytes) ||
      (n > 0 && !new_len))
    return TADM_ERR_INVALID_ARG;
  const PagesCall c{nullptr, tables, nullptr, refs, seqs, new_len, tables_out, nullptr, refs_out, status,
                    pages, n_seqs, ld_table, n, scratch};
  return pages_reserve(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_pages_fork(const tadm_page_pool* pool, const int32_t* tables, const int32_t* lens, const int32_t* refs,
                            int n_seqs, int ld_table, const int32_t* src, const int32_t* dst, int n, int32_t* tables_out,
                            int32_t* lens_out, int32_t* refs_out, int32_t* status, void* scratch, size_t scratch_bytes,
                            tadm_stream stream) {
  if (!pool_ok(pool) || (n_seqs > 0 && (!lens || !lens_out)) || (n > 0 && (!dst || ld_table == 0)) ||
      !seqs_ok(tables, refs, pool->pages, n_seqs, ld_table, src, n, tables_out, refs_out, status, scratch, scratch_bytes))
    return TADM_ERR_INVALID_ARG;
  const PagesCall c{pool, tables, lens, refs, src, dst, tables_out, lens_out, refs_out, status,
                    pool->pages, n_seqs, ld_table, n, scratch};
  return pages_fork(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_pages_free(const int32_t* tables, const int32_t* lens, const int32_t* refs, int pages, int n_seqs,
                            int ld_table, const int32_t* seqs, int n, int32_t* tables_out, int32_t* lens_out,
                            int32_t* refs_out, int32_t* status, void* scratch, size_t scratch_bytes, tadm_stream stream) {
  if ((n_seqs > 0 && (!lens || !lens_out)) ||
      !seqs_ok(tables, refs, pages, n_seqs, ld_table, seqs, n, tables_out, refs_out, status, scratch, scratch_bytes))
    return TADM_ERR_INVALID_ARG;
  const PagesCall c{nullptr, tables, lens, refs, seqs, nullptr, tables_out, lens_out, refs_out, status,
                    pages, n_seqs, ld_table, n, scratch};
  return pages_free(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_pages_compact(const tadm_page_pool* pool, const int32_t* tables, const int32_t* refs, int n_seqs,
                               int ld_table, int32_t* tables_out, int32_t* refs_out, int32_t* n_live, void* scratch,
                               size_t scratch_bytes, tadm_stream stream) {
  if (!pool_ok(pool) ||
      !seqs_ok(tables, refs, pool->pages, n_seqs, ld_table, nullptr, 0, tables_out, refs_out, n_live, scratch, scratch_bytes))
    return TADM_ERR_INVALID_ARG;
  const PagesCall c{pool, tables, nullptr, refs, nullptr, nullptr, tables_out, nullptr, refs_out, n_live,
                    pool->pages, n_seqs, ld_table, 0, scratch};
  return pages_compact(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_pages_copy(const tadm_page_pool* pool, const int32_t* src, const int32_t* dst, int n, tadm_stream stream) {
  if (!pool_ok(pool) || n < 0 || (n > 0 && (!src || !dst))) return TADM_ERR_INVALID_ARG;
  return pages_copy(*pool, src, dst, n, stream) ? TADM_ERR_CUDA : TADM_OK;
}

}  // extern "C"
