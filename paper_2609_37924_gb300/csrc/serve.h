// Host-side launchers of the operators for sequences of different lengths
// (packed prompts, the paged 8-bit cache); each returns nullptr on success or
// a static error string.  Arguments have been checked by the C entry points.
#pragma once
#include "../../include/tadm.h"
#include "kernels.h"

namespace tadm {

struct PageRowsCall {
  const tadm_page_pool* pool;
  int layer;
  void *k, *v;
  const int32_t *cu, *start, *table;
  int batch, total, max_rows, ld_table;
  int64_t ldk, ldv;
  int bf16;
};
const char* page_rows(const PageRowsCall& c, bool write, cudaStream_t s);

struct PagesCall {
  const tadm_page_pool* pool;      // null: no page is moved
  const int32_t *tables, *lens, *refs, *list, *list2;
  int32_t *tables_out, *lens_out, *refs_out, *status;
  int pages, n_seqs, ld_table, n;
  void* scratch;
};
size_t pages_scratch(int pages, int n_seqs);
const char* pages_reserve(const PagesCall& c, cudaStream_t s);
const char* pages_fork(const PagesCall& c, cudaStream_t s);
const char* pages_free(const PagesCall& c, cudaStream_t s);
const char* pages_compact(const PagesCall& c, cudaStream_t s);
const char* pages_copy(const tadm_page_pool& p, const int32_t* src, const int32_t* dst, int n, cudaStream_t s);

// Attention of packed rows over packed keys (pool null) or over a page pool.
struct RaggedCall {
  const void *q, *k, *v;
  void* o;
  const tadm_page_pool* pool;
  int layer;
  const int32_t *cu, *lens, *table;
  int batch, total, max_rows, max_len, ld_table;
  int n_heads, n_kv, head_dim;
  int64_t ldq, ldk, ldv, ldo;
  int causal, window, bf16;
  void* scratch;
  int* status;           // this device's status word
};
const char* attention_rows(const RaggedCall& c, cudaStream_t s);      // CUDA cores, fp32
const char* attention_packed(const RaggedCall& c, cudaStream_t s);    // tcgen05, bf16 rows over themselves
const char* attention_paged(const RaggedCall& c, cudaStream_t s);     // tcgen05, bf16 rows over a pool
size_t attention_paged_scratch(int max_rows, int group, int head_dim);
int* ragged_status();                                                 // of the current device; null: it cannot be had

}  // namespace tadm
