// C entry points of the operators for requests with settings of their own:
// the checks of their arguments, all on the host, before anything is enqueued.
#include <cmath>
#include <cstdint>

#include "requests.h"
#include "serve.h"

using namespace tadm;

namespace {
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool is_type(int dtype) { return dtype == 0 || dtype == 1; }
int es(int dtype) { return dtype ? 2 : 4; }
}  // namespace

extern "C" {

tadm_status tadm_sample_scratch_size(int rows, int vocab, size_t* bytes) {
  if (rows < 0 || vocab < 1 || !bytes) return TADM_ERR_INVALID_ARG;
  *bytes = vocab > kSampleMaxVocab ? 0 : sample_scratch(rows, vocab);
  return TADM_OK;
}

tadm_status tadm_sample(const void* logits, int64_t ld, int rows, int vocab, int mask_id, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* tok,
                        float* prob, int dtype, void* scratch, size_t scratch_bytes, tadm_stream stream) {
  if (!is_type(dtype) || rows < 0 || vocab < 1 || ld < vocab || mask_id < -1 || mask_id >= vocab) return TADM_ERR_INVALID_ARG;
  if (rows == 0) return TADM_OK;
  if (!logits || !u || !tok || !aligned(logits, es(dtype)) || !aligned(u, 4) || !aligned(tok, 4) || !aligned(temperature, 4) ||
      !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(prob, 4))
    return TADM_ERR_INVALID_ARG;
  if (vocab > kSampleMaxVocab || rows > (1 << 24)) return TADM_ERR_UNSUPPORTED;   // a row's parts, a grid of up to 64 blocks a row
  const size_t need = sample_scratch(rows, vocab);
  if (need > 0 && (!scratch || !aligned(scratch, 256) || scratch_bytes < need)) return TADM_ERR_INVALID_ARG;
  const SampleCall c{logits, ld, rows, vocab, mask_id, dtype, temperature, top_k, top_p, min_p, u, tok, prob, scratch};
  return sample_rows(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_lora_scratch_size(int batch, int total_rows, int n_in, int n_out, int n_adapters, int rank, int dtype,
                                   size_t* bytes) {
  if (batch < 0 || total_rows < 0 || n_in < 1 || n_out < 1 || n_adapters < 0 || rank < 8 || rank % 8 || rank > kLoraMaxRank ||
      !is_type(dtype) || !bytes)
    return TADM_ERR_INVALID_ARG;
  *bytes = lora_scratch(batch, total_rows, n_in, n_out, n_adapters, rank, dtype);
  return TADM_OK;
}

tadm_status tadm_lora_project(const void* x, const void* w, void* y, const int32_t* cu_rows, const int32_t* adapter,
                              int batch, int total_rows, int n_in, int n_out, int64_t ldx, int64_t ldw, int64_t ldy,
                              const void* lora_a, const void* lora_b, const float* lora_scale, int n_adapters, int rank,
                              int dtype, int y_dtype, void* scratch, size_t scratch_bytes, tadm_stream stream) {
  size_t need = 0;
  if (tadm_lora_scratch_size(batch, total_rows, n_in, n_out, n_adapters, rank, dtype, &need) != TADM_OK || !is_type(y_dtype) ||
      (!dtype && y_dtype) || ldx < n_in || ldw < n_in || ldy < n_out ||
      static_cast<int64_t>(n_in) * es(dtype) % 16 || ldx * es(dtype) % 16 || ldw * es(dtype) % 16)
    return TADM_ERR_INVALID_ARG;
  if (batch == 0 || total_rows == 0) return TADM_OK;
  if (!x || !w || !y || !cu_rows || !adapter || !aligned(x, 16) || !aligned(w, 16) || !aligned(y, es(y_dtype)) ||
      !aligned(cu_rows, 4) || !aligned(adapter, 4))
    return TADM_ERR_INVALID_ARG;
  if (n_adapters > 0 && (!lora_a || !lora_b || !lora_scale || !aligned(lora_a, 16) || !aligned(lora_b, 16) || !aligned(lora_scale, 4)))
    return TADM_ERR_INVALID_ARG;
  if (dtype && need > kLoraMaxScratch) return TADM_ERR_UNSUPPORTED;
  if (need > 0 && (!scratch || !aligned(scratch, 16) || scratch_bytes < need)) return TADM_ERR_INVALID_ARG;
  if (total_rows > kLoraMaxRows || n_out > kLoraMaxRows || batch > kMaxSequences) return TADM_ERR_UNSUPPORTED;   // grids, counts of tiles
  LoraCall c{};
  c.x = x, c.w = w, c.y = y, c.cu = cu_rows, c.adapter = adapter;
  c.batch = batch, c.total = total_rows, c.n_in = n_in, c.n_out = n_out, c.ldx = ldx, c.ldw = ldw, c.ldy = ldy;
  c.a = lora_a, c.b = lora_b, c.scale = lora_scale, c.n_adapters = n_adapters, c.rank = rank;
  c.bf16 = dtype, c.y_bf16 = y_dtype, c.scratch = scratch;
  if (dtype && !(c.status = ragged_status())) return TADM_ERR_CUDA;
  return lora_project(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

tadm_status tadm_residual_norm(const void* x, const void* y, void* x_out, void* n_out, const int32_t* cu_rows, int batch,
                               int total_rows, int d, int64_t ldx, int64_t ldy, int64_t ldxo, int64_t ldn,
                               const void* post_gain, const void* gate, int64_t ldg, const void* pre_gain,
                               float residual_scale, float eps, int x_dtype, int y_dtype, int dtype, tadm_stream stream) {
  if (!is_type(x_dtype) || !is_type(y_dtype) || !is_type(dtype) || batch < 0 || total_rows < 0 || d < 1 || ldx < d || ldy < d ||
      ldxo < d || (n_out && ldn < d) || (gate && ldg < d) || (!cu_rows && batch != 1) || !(eps >= 0.0f) || std::isinf(eps) || std::isnan(residual_scale))
    return TADM_ERR_INVALID_ARG;
  if (batch == 0 || total_rows == 0) return TADM_OK;
  if (!x || !y || !x_out || !aligned(x, es(x_dtype)) || !aligned(x_out, es(x_dtype)) || !aligned(y, es(y_dtype)) ||
      !aligned(n_out, es(dtype)) || !aligned(post_gain, es(dtype)) || !aligned(gate, es(dtype)) || !aligned(pre_gain, es(dtype)) ||
      !aligned(cu_rows, 4))
    return TADM_ERR_INVALID_ARG;
  if (d > kNormMaxWidth || total_rows > kNormMaxRows || batch > kMaxSequences) return TADM_ERR_UNSUPPORTED;
  const NormCall c{x, y, x_out, n_out, cu_rows, batch, total_rows, d, ldx, ldy, ldxo, ldn, ldg,
                   post_gain, gate, pre_gain, residual_scale, eps, x_dtype, y_dtype, dtype, ragged_status()};
  if (!c.status) return TADM_ERR_CUDA;
  return residual_norm(c, stream) ? TADM_ERR_CUDA : TADM_OK;
}

}  // extern "C"
