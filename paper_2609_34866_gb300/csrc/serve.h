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
  const jab_norm_rope* how;  // null: the rotation above; else what takes its place
};
cudaError_t launch_kv_write(const KvWriteArgs& a, int sms, cudaStream_t st);

struct NormRopeArgs {
  int64_t n_tokens;
  int n_q, n_k, head_dim;
  const void* x;
  jab_dtype type;
  int64_t ldx;
  jab_norm_rope how;
  void *q, *k;
  int64_t ldq, ldk;
  int* status;
};
cudaError_t launch_norm_rope(const NormRopeArgs& a, int sms, cudaStream_t st);

struct KvReadArgs {
  jab_kv_cache cache;
  int n_seqs, max_pages, T;
  const int32_t *pages, *starts, *counts;
  void *k, *v;
  jab_dtype type;
  int* status;
};
cudaError_t launch_kv_read(const KvReadArgs& a, int sms, cudaStream_t st);

// norm_rope.cu
struct NormRopeBackArgs {
  int64_t n_tokens;
  int n_q, n_k, head_dim;
  const void* x;
  jab_dtype type;
  int64_t ldx;
  jab_norm_rope how;
  const void *dq, *dk;
  int64_t lddq, lddk;
  void* dx;
  int64_t lddx;
  float *dwq, *dwk;  // null: not wanted
  void* ws;          // norm_rope_scratch bytes
  int* status;
};
size_t norm_rope_scratch(int n_heads, int dh);
int norm_rope_back_kernels(const NormRopeBackArgs& a);
cudaError_t launch_norm_rope_back(const NormRopeBackArgs& a, int sms, cudaStream_t st);
struct RopeTableArgs {
  int length, rotary;
  float theta;
  jab_rope_scaling scaling;
  float *cos_t, *sin_t;
};
cudaError_t launch_rope_table(const RopeTableArgs& a, cudaStream_t st);

// kv_plan.cu
struct KvPlanArgs {
  int n_seqs, page, max_pages, free_capacity, shared;
  int64_t n_pages, n_tokens;
  const int32_t *lens, *counts;  // counts: of new tokens, or whether a sequence has ended
  int32_t *pages, *free_pages;
  const int32_t* n_free;
  int32_t *new_lens, *new_free, *q_start, *positions;
  int64_t* slots;
  int* status;
};
int kv_plan_kernels(const KvPlanArgs& a);  // how many launch_kv_plan launches
cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st);
cudaError_t launch_kv_release(const KvPlanArgs& a, cudaStream_t st);

// fp8.cu
struct Fp8QuantArgs {
  int64_t M;
  int K;
  const void* x;
  jab_dtype type;
  int64_t ldx;
  int block_rows;
  void* codes;              // [M, K]
  float* scales;            // at row * row_pitch + block * block_pitch
  int64_t row_pitch, block_pitch;
  int* status;
};
cudaError_t launch_fp8_quantize(const Fp8QuantArgs& a, int sms, cudaStream_t st);
struct Fp8LinearArgs {
  int64_t M;
  int N, K;
  const void* x;
  jab_dtype x_type;
  int64_t ldx;
  const void* codes;
  const float* w_scales;
  int block_rows;
  void* y;
  jab_dtype y_type;
  int64_t ldy;
  void* ws;  // fp8_linear_scratch bytes
  int* status;
};
size_t fp8_linear_scratch(int64_t M, int K);
cudaError_t launch_fp8_linear(const Fp8LinearArgs& a, int sms, cudaStream_t st);

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
