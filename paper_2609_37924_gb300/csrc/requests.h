// Host-side launchers of the operators around attention in a serving step:
// sampling with settings per row, projections with an adapter per request,
// norms with gate and residual scale.  Each returns nullptr on success or a
// static error string.  Arguments have been checked by the C entry points.
#pragma once
#include "kernels.h"

namespace tadm {

struct SampleCall {
  const void* logits;
  int64_t ld;
  int rows, vocab, mask_id, bf16;
  const float* temperature;        // null: 1
  const int32_t* top_k;            // null: all
  const float *top_p, *min_p;      // null: off
  const float* u;
  int32_t* tok;
  float* prob;                     // null: not wanted
  void* scratch;
};
constexpr int kSampleMaxVocab = 1 << 19;
size_t sample_scratch(int rows, int vocab);
const char* sample_rows(const SampleCall& c, cudaStream_t s);

struct LoraCall {
  const void *x, *w;
  void* y;
  const int32_t *cu, *adapter;
  int batch, total, n_in, n_out;
  int64_t ldx, ldw, ldy;
  const void *a, *b;
  const float* scale;
  int n_adapters, rank, bf16, y_bf16;
  void* scratch;
  int* status;                     // this device's status word
};
constexpr int kLoraMaxRank = 256, kLoraMaxRows = 1 << 20;
constexpr size_t kLoraMaxScratch = size_t{1} << 38;   // bf16: rows of 128 bytes, which tensor maps count in 31 bits
size_t lora_scratch(int batch, int total, int n_in, int n_out, int n_adapters, int rank, int bf16);
const char* lora_project(const LoraCall& c, cudaStream_t s);          // tcgen05 (bf16), or
size_t lora_rows_scratch(int total, int rank);
const char* lora_rows(const LoraCall& c, cudaStream_t s);             // CUDA cores (fp32)

struct NormCall {
  const void *x, *y;
  void *x_out, *n_out;             // n_out null: not wanted
  const int32_t* cu;               // null: every row, one gate
  int batch, total, d;
  int64_t ldx, ldy, ldxo, ldn, ldg;
  const void *post, *gate, *pre;
  float residual_scale, eps;
  int x_bf16, y_bf16, bf16;
  int* status;                     // this device's status word
};
constexpr int kNormMaxWidth = 49152, kNormMaxRows = 1 << 30;
constexpr int kMaxSequences = 1 << 30;      // of adapters and norms
const char* residual_norm(const NormCall& c, cudaStream_t s);

}  // namespace tadm
