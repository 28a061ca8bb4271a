// C entry points that run a fitted block on new tokens (include/jab.h): argument checks and launches.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"
#include "timing.h"

namespace jab {
jab_status device_status_ptr(int** status);

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int size_of(jab_dtype t) { return t == JAB_FP32 ? 4 : 2; }
bool is_dtype(jab_dtype t) { return t == JAB_FP16 || t == JAB_BF16 || t == JAB_FP32; }

jab_status device(int** status, int* sms) {
  const jab_status s = device_status_ptr(status);
  if (s != JAB_OK) return s;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return JAB_ERR_CUDA;
  return JAB_OK;
}

// Geometry alone (no pointers): what the workspace size needs too.
jab_status check_cache_shape(const jab_kv_cache* c) {
  if (c == nullptr || c->n_kv_heads < 1 || c->page_tokens < 1 || c->n_pages < 1) return JAB_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || (c->bits != 8 && c->bits != 4)) return JAB_ERR_UNSUPPORTED;
  if (c->page_tokens % 16 != 0 || c->page_tokens > 4096 || c->n_pages > INT32_MAX || c->n_kv_heads > 65535)
    return JAB_ERR_UNSUPPORTED;
  return JAB_OK;
}

jab_status check_cache(const jab_kv_cache* c) {
  const jab_status s = check_cache_shape(c);
  if (s != JAB_OK) return s;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return JAB_ERR_INVALID_ARG;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 16) || !aligned(c->v_scales, 16))
    return JAB_ERR_INVALID_ARG;
  return JAB_OK;
}

// Rows of `width` elements with pitch ld, each starting on 16 bytes.
bool rows_ok(const void* p, int64_t ld, int64_t width, jab_dtype t) {
  return p != nullptr && aligned(p, 16) && ld >= width && (ld * size_of(t)) % 16 == 0;
}

#define JAB_LAUNCH(name, nk, expr)                      \
  do {                                                  \
    TimedSite site_(name, st, nk);                      \
    if ((expr) != cudaSuccess) return JAB_ERR_CUDA;     \
  } while (0)

jab_status check_linear(int64_t M, int32_t N, int32_t K) {
  if (M < 0 || N < 1 || K < 1) return JAB_ERR_INVALID_ARG;
  if (K % 16 != 0 || K > 131072 || N > (1 << 24) || M > (int64_t)1 << 31) return JAB_ERR_UNSUPPORTED;
  return JAB_OK;
}

jab_status check_attention(const jab_kv_cache* c, int32_t n_seqs, int64_t n_tokens, int32_t n_q_heads, int32_t max_q_len,
                           int32_t max_seq_len, int32_t shared_len) {
  const jab_status s = check_cache_shape(c);
  if (s != JAB_OK) return s;
  if (n_seqs < 1 || n_tokens < 0 || n_q_heads < 1 || max_q_len < 1 || max_seq_len < 0 || shared_len < 0) return JAB_ERR_INVALID_ARG;
  if (n_q_heads % c->n_kv_heads != 0 || n_seqs > 2048 || n_tokens >= (int64_t)1 << 30 || n_tokens * n_q_heads >= (int64_t)1 << 30)
    return JAB_ERR_UNSUPPORTED;
  if (shared_len % c->page_tokens != 0) return JAB_ERR_UNSUPPORTED;
  return JAB_OK;
}

}  // namespace
}  // namespace jab

using namespace jab;

extern "C" {

size_t jab_quantized_linear_workspace_size(int64_t M, int32_t N, int32_t K) {
  if (check_linear(M, N, K) != JAB_OK) return 0;
  return quantized_linear_scratch(M > 0 ? M : 1, N, K);
}

jab_status jab_quantized_linear(int64_t M, int32_t N, int32_t K, const void* X_dev, jab_dtype x_type, int64_t ldx,
                                const int8_t* codes_dev, const float* w_scales_dev, void* Y_dev, jab_dtype y_type, int64_t ldy,
                                void* ws, size_t ws_bytes, jab_stream_t stream) {
  jab_status s = check_linear(M, N, K);
  if (s != JAB_OK) return s;
  if (!is_dtype(x_type) || !is_dtype(y_type)) return JAB_ERR_INVALID_ARG;
  if (x_type == JAB_FP32) return JAB_ERR_UNSUPPORTED;
  if (M == 0) return JAB_OK;
  if (!rows_ok(X_dev, ldx, K, x_type) || !codes_dev || !aligned(codes_dev, 16) || !w_scales_dev || !aligned(w_scales_dev, 4) ||
      !Y_dev || !aligned(Y_dev, size_of(y_type)) || ldy < N || !ws || !aligned(ws, 256) || ws_bytes < quantized_linear_scratch(M, N, K))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  QLinearArgs a{};
  a.M = M, a.N = N, a.K = K;
  a.x = X_dev, a.x_type = x_type, a.ldx = ldx;
  a.codes = codes_dev, a.w_scales = w_scales_dev;
  a.y = Y_dev, a.y_type = y_type, a.ldy = ldy;
  a.ws = ws, a.status = status;
  JAB_LAUNCH("quantized_linear", 2, launch_quantized_linear(a, sms, st));
  return JAB_OK;
}

jab_status jab_rope_table(int32_t length, int32_t head_dim, float theta, float* cos_dev, float* sin_dev, jab_stream_t stream) {
  if (length < 1 || !(theta > 0.f) || !isfinite(theta) || !cos_dev || !sin_dev || !aligned(cos_dev, 16) || !aligned(sin_dev, 16))
    return JAB_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return JAB_ERR_UNSUPPORTED;
  int *status, sms;
  const jab_status s = device(&status, &sms);
  if (s != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  PrepInputs in{};
  in.cos_t = cos_dev;
  in.sin_t = sin_dev;
  in.T = length;
  in.dh = head_dim;
  in.theta = theta;
  JAB_LAUNCH("rope_table", 1, launch_prep(in, status, sms, st));
  return JAB_OK;
}

jab_status jab_kv_write(const jab_kv_cache* cache, int64_t n_tokens, int32_t n_q_heads, const void* X_dev, jab_dtype type, int64_t ldx,
                        const int64_t* slots_dev, const int32_t* positions_dev, const float* cos_dev, const float* sin_dev,
                        int32_t rope_len, void* Q_dev, jab_stream_t stream) {
  jab_status s = check_cache(cache);
  if (s != JAB_OK) return s;
  if (n_tokens < 0 || n_q_heads < 0 || !is_dtype(type)) return JAB_ERR_INVALID_ARG;
  const int64_t heads = (int64_t)n_q_heads + 2 * (int64_t)cache->n_kv_heads;
  if (heads > 1 << 20 || n_tokens > (int64_t)1 << 31) return JAB_ERR_UNSUPPORTED;
  const bool turn = positions_dev || cos_dev || sin_dev;
  if (turn && (!positions_dev || !cos_dev || !sin_dev || rope_len < 1 || !aligned(positions_dev, 4) || !aligned(cos_dev, 16) ||
               !aligned(sin_dev, 16)))
    return JAB_ERR_INVALID_ARG;
  if (n_tokens == 0) return JAB_OK;
  if (!rows_ok(X_dev, ldx, heads * cache->head_dim, type) || !slots_dev || !aligned(slots_dev, 8) || (Q_dev && !aligned(Q_dev, 16)))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvWriteArgs a{};
  a.cache = *cache;
  a.x = X_dev, a.type = type, a.ldx = ldx, a.n_tokens = n_tokens, a.n_q_heads = n_q_heads;
  a.slots = slots_dev, a.positions = positions_dev, a.cos_t = cos_dev, a.sin_t = sin_dev, a.rope_len = rope_len;
  a.q_out = Q_dev;
  a.status = status;
  JAB_LAUNCH("kv_write", 1, launch_kv_write(a, sms, st));
  return JAB_OK;
}

jab_status jab_kv_read(const jab_kv_cache* cache, int32_t n_seqs, const int32_t* pages_dev, int32_t max_pages, const int32_t* starts_dev,
                       const int32_t* counts_dev, int32_t T, void* K_dev, void* V_dev, jab_dtype type, jab_stream_t stream) {
  jab_status s = check_cache(cache);
  if (s != JAB_OK) return s;
  if (n_seqs < 0 || T < 0 || max_pages < 1 || !is_dtype(type)) return JAB_ERR_INVALID_ARG;
  if (n_seqs == 0 || T == 0) return JAB_OK;
  if (!pages_dev || !aligned(pages_dev, 4) || !counts_dev || !aligned(counts_dev, 4) || !aligned(starts_dev, 4) || !K_dev || !V_dev ||
      !aligned(K_dev, 16) || !aligned(V_dev, 16))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvReadArgs a{};
  a.cache = *cache;
  a.n_seqs = n_seqs, a.max_pages = max_pages, a.T = T;
  a.pages = pages_dev, a.starts = starts_dev, a.counts = counts_dev;
  a.k = K_dev, a.v = V_dev, a.type = type;
  a.status = status;
  JAB_LAUNCH("kv_read", 1, launch_kv_read(a, sms, st));
  return JAB_OK;
}

size_t jab_kv_attention_workspace_size(const jab_kv_cache* cache, int32_t n_seqs, int64_t n_tokens, int32_t n_q_heads, int32_t max_q_len,
                                       int32_t max_seq_len, int32_t shared_len) {
  if (check_attention(cache, n_seqs, n_tokens, n_q_heads, max_q_len, max_seq_len, shared_len) != JAB_OK) return 0;
  return kv_attention_scratch(cache->n_kv_heads, cache->head_dim, n_seqs, n_tokens, n_q_heads, max_q_len, shared_len);
}

jab_status jab_kv_attention(const jab_kv_cache* cache, int32_t n_seqs, int64_t n_tokens, int32_t n_q_heads, const void* Q_dev,
                            jab_dtype type, int64_t ldq, const int32_t* q_start_dev, const int32_t* pages_dev, int32_t max_pages,
                            const int32_t* seq_lens_dev, int32_t max_q_len, int32_t max_seq_len, int32_t shared_len, int32_t window,
                            float softmax_scale, void* O_dev, int64_t ldo, float* lse_dev, void* ws, size_t ws_bytes,
                            jab_stream_t stream) {
  jab_status s = check_cache(cache);
  if (s != JAB_OK) return s;
  if ((s = check_attention(cache, n_seqs, n_tokens, n_q_heads, max_q_len, max_seq_len, shared_len)) != JAB_OK) return s;
  if (!is_dtype(type) || max_pages < 1 || window < 0 || !isfinite(softmax_scale)) return JAB_ERR_INVALID_ARG;
  if (type == JAB_FP32 || (int64_t)max_pages * cache->page_tokens >= (int64_t)1 << 30) return JAB_ERR_UNSUPPORTED;
  if (shared_len > (int64_t)max_pages * cache->page_tokens) return JAB_ERR_INVALID_ARG;
  if (n_tokens == 0) return JAB_OK;
  const int64_t width = (int64_t)n_q_heads * cache->head_dim;
  if (!rows_ok(Q_dev, ldq, width, type) || !rows_ok(O_dev, ldo, width, type) || !q_start_dev || !aligned(q_start_dev, 4) || !pages_dev ||
      !aligned(pages_dev, 4) || !seq_lens_dev || !aligned(seq_lens_dev, 4) || !aligned(lse_dev, 4) || !ws || !aligned(ws, 256) ||
      ws_bytes < kv_attention_scratch(cache->n_kv_heads, cache->head_dim, n_seqs, n_tokens, n_q_heads, max_q_len, shared_len))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvAttnArgs a{};
  a.cache = *cache;
  a.n_seqs = n_seqs, a.n_tokens = n_tokens, a.n_q_heads = n_q_heads;
  a.q = Q_dev, a.type = type, a.ldq = ldq;
  a.q_start = q_start_dev, a.pages = pages_dev, a.lens = seq_lens_dev;
  a.max_pages = max_pages, a.max_q = max_q_len, a.max_len = max_seq_len, a.shared = shared_len, a.window = window;
  a.scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)cache->head_dim));
  a.out = O_dev, a.ldo = ldo, a.lse = lse_dev;
  a.ws = ws, a.status = status;
  JAB_LAUNCH("kv_attention", kv_attention_kernels(a), launch_kv_attention(a, sms, st));
  return JAB_OK;
}

}  // extern "C"
