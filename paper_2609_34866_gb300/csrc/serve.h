// Host-side launchers of the serving kernels (internal to libjab): quantised projection, quantised
// paged cache, attention over it.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/jab.h"

namespace jab {

// kv_cache.cu
struct KvWriteArgs {
  jab_kv_cache cache;
  const void* x;
  jab_dtype type;
  int64_t ldx, n_tokens;
  int n_q_heads;
  const int64_t* slots;
  const int32_t* positions;  // null: no rotation
  const float *cos_t, *sin_t;
  int rope_len;
  void* q_out;  // null: Q is not wanted
  int* status;
};
cudaError_t launch_kv_write(const KvWriteArgs& a, int sms, cudaStream_t st);

struct KvReadArgs {
  jab_kv_cache cache;
  int n_seqs, max_pages, T;
  const int32_t *pages, *starts, *counts;
  void *k, *v;
  jab_dtype type;
  int* status;
};
cudaError_t launch_kv_read(const KvReadArgs& a, int sms, cudaStream_t st);

// kv_attn.cu
struct KvAttnArgs {
  jab_kv_cache cache;
  int n_seqs;
  int64_t n_tokens;
  int n_q_heads;
  const void* q;
  jab_dtype type;
  int64_t ldq;
  const int32_t *q_start, *pages, *lens;
  int max_pages, max_q, max_len, shared, window;
  float scale;
  void* out;
  int64_t ldo;
  float* lse;  // null: not wanted
  void* ws;    // kv_attention_scratch bytes
  int* status;
};
size_t kv_attention_scratch(int n_kv, int dh, int n_seqs, int64_t n_tokens, int n_q_heads, int max_q, int shared);
int kv_attention_kernels(const KvAttnArgs& a);  // how many launch_kv_attention launches
cudaError_t launch_kv_attention(const KvAttnArgs& a, int sms, cudaStream_t st);

// qlinear.cu
struct QLinearArgs {
  int64_t M;
  int N, K;
  const void* x;
  jab_dtype x_type;
  int64_t ldx;
  const int8_t* codes;
  const float* w_scales;
  void* y;
  jab_dtype y_type;
  int64_t ldy;
  void* ws;  // quantized_linear_scratch bytes
  int* status;
};
size_t quantized_linear_scratch(int64_t M, int N, int K);
cudaError_t launch_quantized_linear(const QLinearArgs& a, int sms, cudaStream_t st);

}  // namespace jab
