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

// Norm and rotation of heads of head_dim: kinds, sizes and pointers.
jab_status check_how(const jab_norm_rope* h, int32_t head_dim) {
  if (h == nullptr) return JAB_ERR_INVALID_ARG;
  if (h->norm && !(h->eps >= 1e-30f && h->eps <= 1e30f)) return JAB_ERR_INVALID_ARG;
  if (!aligned(h->q_weight_dev, 16) || !aligned(h->k_weight_dev, 16)) return JAB_ERR_INVALID_ARG;
  const bool turn = h->positions_dev || h->cos_dev || h->sin_dev;
  if (!turn) return JAB_OK;
  if (!h->positions_dev || !h->cos_dev || !h->sin_dev || h->rope_len < 1 || !aligned(h->positions_dev, 4) || !aligned(h->cos_dev, 16) ||
      !aligned(h->sin_dev, 16) || h->rotary_dim < 1 || h->rotary_dim > head_dim)
    return JAB_ERR_INVALID_ARG;
  return h->rotary_dim % 16 == 0 ? JAB_OK : JAB_ERR_UNSUPPORTED;
}
jab_status check_heads(int64_t n_tokens, int32_t n_q, int32_t n_k, int32_t head_dim) {
  if (n_tokens < 0 || n_q < 0 || n_k < 0 || (int64_t)n_q + n_k < 1) return JAB_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || (int64_t)n_q + n_k > 4096 || n_tokens > (int64_t)1 << 31) return JAB_ERR_UNSUPPORTED;
  return JAB_OK;
}

jab_status check_plan(const jab_kv_cache* c, int32_t n_seqs, int32_t max_pages, int32_t free_capacity) {
  if (c == nullptr || c->page_tokens < 1 || c->n_pages < 1 || n_seqs < 1 || max_pages < 1 || free_capacity < 0) return JAB_ERR_INVALID_ARG;
  if (c->page_tokens % 16 != 0 || c->page_tokens > 4096 || c->n_pages > INT32_MAX || n_seqs > 8192 ||
      (int64_t)max_pages * c->page_tokens >= (int64_t)1 << 30)
    return JAB_ERR_UNSUPPORTED;
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

jab_status jab_fp8_quantize(int64_t M, int32_t K, const void* X_dev, jab_dtype type, int64_t ldx, int32_t block_rows, void* codes_dev,
                            float* scales_dev, jab_stream_t stream) {
  jab_status s = check_linear(M, 1, K);
  if (s != JAB_OK) return s;
  if (!is_dtype(type) || (block_rows != 1 && block_rows != 128)) return JAB_ERR_INVALID_ARG;
  if (M == 0) return JAB_OK;
  if (!rows_ok(X_dev, ldx, K, type) || !codes_dev || !aligned(codes_dev, 16) || !scales_dev || !aligned(scales_dev, 4)) return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  Fp8QuantArgs a{};
  a.M = M, a.K = K, a.x = X_dev, a.type = type, a.ldx = ldx, a.block_rows = block_rows;
  a.codes = codes_dev, a.scales = scales_dev, a.row_pitch = (K + 127) / 128, a.block_pitch = 1;
  a.status = status;
  JAB_LAUNCH("fp8_quantize", 1, launch_fp8_quantize(a, sms, st));
  return JAB_OK;
}

size_t jab_fp8_linear_workspace_size(int64_t M, int32_t N, int32_t K) {
  if (check_linear(M, N, K) != JAB_OK) return 0;
  return fp8_linear_scratch(M > 0 ? M : 1, K);
}

jab_status jab_fp8_linear(int64_t M, int32_t N, int32_t K, const void* X_dev, jab_dtype x_type, int64_t ldx, const void* codes_dev,
                          const float* w_scales_dev, int32_t block_rows, void* Y_dev, jab_dtype y_type, int64_t ldy, void* ws,
                          size_t ws_bytes, jab_stream_t stream) {
  jab_status s = check_linear(M, N, K);
  if (s != JAB_OK) return s;
  if (!is_dtype(x_type) || !is_dtype(y_type) || (block_rows != 1 && block_rows != 128)) return JAB_ERR_INVALID_ARG;
  if (M == 0) return JAB_OK;
  if (!rows_ok(X_dev, ldx, K, x_type) || !codes_dev || !aligned(codes_dev, 16) || !w_scales_dev || !aligned(w_scales_dev, 4) || !Y_dev ||
      !aligned(Y_dev, size_of(y_type)) || ldy < N || !ws || !aligned(ws, 256) || ws_bytes < fp8_linear_scratch(M, K))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  Fp8LinearArgs a{};
  a.M = M, a.N = N, a.K = K;
  a.x = X_dev, a.x_type = x_type, a.ldx = ldx;
  a.codes = codes_dev, a.w_scales = w_scales_dev, a.block_rows = block_rows;
  a.y = Y_dev, a.y_type = y_type, a.ldy = ldy;
  a.ws = ws, a.status = status;
  JAB_LAUNCH("fp8_linear", 2, launch_fp8_linear(a, sms, st));
  return JAB_OK;
}

jab_status jab_rope_table_scaled(int32_t length, int32_t rotary_dim, float theta, const jab_rope_scaling* scaling, float* cos_dev,
                                 float* sin_dev, jab_stream_t stream) {
  if (length < 1 || rotary_dim < 1 || !(theta > 0.f) || !isfinite(theta) || !cos_dev || !sin_dev || !aligned(cos_dev, 16) ||
      !aligned(sin_dev, 16))
    return JAB_ERR_INVALID_ARG;
  if (rotary_dim % 16 != 0 || rotary_dim > 128) return JAB_ERR_UNSUPPORTED;
  RopeTableArgs a{};
  a.scaling = scaling != nullptr ? *scaling : jab_rope_scaling{JAB_ROPE_PLAIN, 1.f, 0.f, 0.f, 0.f, 1.f};
  const jab_rope_scaling& c = a.scaling;
  if (c.kind != JAB_ROPE_PLAIN && c.kind != JAB_ROPE_LINEAR && c.kind != JAB_ROPE_BY_PARTS) return JAB_ERR_INVALID_ARG;
  if (!(c.attention > 0.f) || !isfinite(c.attention)) return JAB_ERR_INVALID_ARG;
  if (c.kind != JAB_ROPE_PLAIN && (!(c.factor >= 1.f) || !isfinite(c.factor))) return JAB_ERR_INVALID_ARG;
  if (c.kind == JAB_ROPE_BY_PARTS && (!(c.original_length > 0.f) || !isfinite(c.original_length) || !(c.low_turns >= 0.f) ||
                                      !(c.high_turns > c.low_turns) || !isfinite(c.high_turns)))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  const jab_status s = device(&status, &sms);
  if (s != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  a.length = length, a.rotary = rotary_dim, a.theta = theta, a.cos_t = cos_dev, a.sin_t = sin_dev;
  JAB_LAUNCH("rope_table", 1, launch_rope_table(a, st));
  return JAB_OK;
}

jab_status jab_kv_write_norm_rope(const jab_kv_cache* cache, int64_t n_tokens, int32_t n_q_heads, const void* X_dev, jab_dtype type,
                                  int64_t ldx, const int64_t* slots_dev, const jab_norm_rope* how, void* Q_dev, jab_stream_t stream) {
  jab_status s = check_cache(cache);
  if (s != JAB_OK) return s;
  if (n_tokens < 0 || n_q_heads < 0 || !is_dtype(type)) return JAB_ERR_INVALID_ARG;
  const int64_t heads = (int64_t)n_q_heads + 2 * (int64_t)cache->n_kv_heads;
  if (heads > 1 << 20 || n_tokens > (int64_t)1 << 31) return JAB_ERR_UNSUPPORTED;
  if ((s = check_how(how, cache->head_dim)) != JAB_OK) return s;
  if (n_tokens == 0) return JAB_OK;
  if (!rows_ok(X_dev, ldx, heads * cache->head_dim, type) || !slots_dev || !aligned(slots_dev, 8) || (Q_dev && !aligned(Q_dev, 16)))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvWriteArgs a{};
  a.cache = *cache;
  a.x = X_dev, a.type = type, a.ldx = ldx, a.n_tokens = n_tokens, a.n_q_heads = n_q_heads;
  a.slots = slots_dev, a.how = how;
  a.q_out = Q_dev;
  a.status = status;
  JAB_LAUNCH("kv_write_norm_rope", 1, launch_kv_write(a, sms, st));
  return JAB_OK;
}

jab_status jab_qk_norm_rope(int64_t n_tokens, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, const void* X_dev, jab_dtype type,
                            int64_t ldx, const jab_norm_rope* how, void* Q_dev, int64_t ldq, void* K_dev, int64_t ldk,
                            jab_stream_t stream) {
  jab_status s = check_heads(n_tokens, n_q_heads, n_k_heads, head_dim);
  if (s != JAB_OK) return s;
  if (!is_dtype(type)) return JAB_ERR_INVALID_ARG;
  if ((s = check_how(how, head_dim)) != JAB_OK) return s;
  if (n_tokens == 0) return JAB_OK;
  const int64_t wq = (int64_t)n_q_heads * head_dim, wk = (int64_t)n_k_heads * head_dim;
  if (!rows_ok(X_dev, ldx, wq + wk, type) || (wq > 0 && !rows_ok(Q_dev, ldq, wq, type)) || (wk > 0 && !rows_ok(K_dev, ldk, wk, type)))
    return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  NormRopeArgs a{};
  a.n_tokens = n_tokens, a.n_q = n_q_heads, a.n_k = n_k_heads, a.head_dim = head_dim;
  a.x = X_dev, a.type = type, a.ldx = ldx, a.how = *how;
  // (heads without an output of their own are not there: a null Q_dev would mean that Q is not wanted)
  a.q = wq > 0 ? Q_dev : K_dev, a.k = K_dev, a.ldq = ldq, a.ldk = ldk;
  a.status = status;
  JAB_LAUNCH("qk_norm_rope", 1, launch_norm_rope(a, sms, st));
  return JAB_OK;
}

size_t jab_qk_norm_rope_backward_workspace_size(int64_t n_tokens, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim) {
  if (check_heads(n_tokens, n_q_heads, n_k_heads, head_dim) != JAB_OK) return 0;
  return norm_rope_scratch(n_q_heads + n_k_heads, head_dim);
}

jab_status jab_qk_norm_rope_backward(int64_t n_tokens, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, const void* X_dev,
                                     jab_dtype type, int64_t ldx, const jab_norm_rope* how, const void* dQ_dev, int64_t lddq,
                                     const void* dK_dev, int64_t lddk, void* dX_dev, int64_t lddx, float* dq_weight_dev,
                                     float* dk_weight_dev, void* ws, size_t ws_bytes, jab_stream_t stream) {
  jab_status s = check_heads(n_tokens, n_q_heads, n_k_heads, head_dim);
  if (s != JAB_OK) return s;
  if (!is_dtype(type)) return JAB_ERR_INVALID_ARG;
  if ((s = check_how(how, head_dim)) != JAB_OK) return s;
  const bool weights = dq_weight_dev || dk_weight_dev;
  if ((weights && !how->norm) || !aligned(dq_weight_dev, 4) || !aligned(dk_weight_dev, 4)) return JAB_ERR_INVALID_ARG;
  if (n_tokens == 0 && !weights) return JAB_OK;
  const int64_t wq = (int64_t)n_q_heads * head_dim, wk = (int64_t)n_k_heads * head_dim;
  if (n_tokens > 0 && (!rows_ok(X_dev, ldx, wq + wk, type) || !rows_ok(dX_dev, lddx, wq + wk, type) ||
                       (wq > 0 && !rows_ok(dQ_dev, lddq, wq, type)) || (wk > 0 && !rows_ok(dK_dev, lddk, wk, type))))
    return JAB_ERR_INVALID_ARG;
  if (weights && (!ws || !aligned(ws, 256) || ws_bytes < norm_rope_scratch(n_q_heads + n_k_heads, head_dim))) return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  NormRopeBackArgs a{};
  a.n_tokens = n_tokens, a.n_q = n_q_heads, a.n_k = n_k_heads, a.head_dim = head_dim;
  a.x = X_dev, a.type = type, a.ldx = ldx, a.how = *how;
  a.dq = dQ_dev, a.dk = dK_dev, a.lddq = lddq, a.lddk = lddk;
  a.dx = dX_dev, a.lddx = lddx, a.dwq = dq_weight_dev, a.dwk = dk_weight_dev;
  a.ws = ws, a.status = status;
  JAB_LAUNCH("qk_norm_rope_backward", norm_rope_back_kernels(a), launch_norm_rope_back(a, sms, st));
  return JAB_OK;
}

jab_status jab_kv_release(const jab_kv_cache* cache, int32_t n_seqs, const int32_t* lens_dev, const int32_t* ended_dev,
                          const int32_t* pages_dev, int32_t max_pages, int32_t shared_len, int32_t* free_dev, int32_t free_capacity,
                          const int32_t* n_free_dev, int32_t* new_lens_dev, int32_t* new_free_dev, jab_stream_t stream) {
  jab_status s = check_plan(cache, n_seqs, max_pages, free_capacity);
  if (s != JAB_OK) return s;
  if (shared_len < 0 || shared_len > (int64_t)max_pages * cache->page_tokens) return JAB_ERR_INVALID_ARG;
  if (shared_len % cache->page_tokens != 0) return JAB_ERR_UNSUPPORTED;
  const void* all[] = {lens_dev, ended_dev, pages_dev, n_free_dev, new_lens_dev, new_free_dev};
  for (const void* q : all)
    if (!q || !aligned(q, 4)) return JAB_ERR_INVALID_ARG;
  if ((!free_dev && free_capacity > 0) || !aligned(free_dev, 4)) return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvPlanArgs a{};
  a.n_seqs = n_seqs, a.page = cache->page_tokens, a.max_pages = max_pages, a.free_capacity = free_capacity, a.shared = shared_len;
  a.n_pages = cache->n_pages;
  a.lens = lens_dev, a.counts = ended_dev, a.pages = const_cast<int32_t*>(pages_dev), a.free_pages = free_dev, a.n_free = n_free_dev;
  a.new_lens = new_lens_dev, a.new_free = new_free_dev;
  a.status = status;
  JAB_LAUNCH("kv_release", 1, launch_kv_release(a, st));
  return JAB_OK;
}

jab_status jab_kv_plan(const jab_kv_cache* cache, int32_t n_seqs, int64_t n_tokens, const int32_t* lens_dev, const int32_t* counts_dev,
                       int32_t* pages_dev, int32_t max_pages, const int32_t* free_dev, int32_t free_capacity, const int32_t* n_free_dev,
                       int32_t* new_lens_dev, int32_t* new_free_dev, int32_t* q_start_dev, int64_t* slots_dev, int32_t* positions_dev,
                       jab_stream_t stream) {
  jab_status s = check_plan(cache, n_seqs, max_pages, free_capacity);
  if (s != JAB_OK) return s;
  if (n_tokens < 0) return JAB_ERR_INVALID_ARG;
  if (n_tokens >= (int64_t)1 << 30) return JAB_ERR_UNSUPPORTED;
  const void* all[] = {lens_dev, counts_dev, pages_dev, n_free_dev, new_lens_dev, new_free_dev, q_start_dev};
  for (const void* q : all)
    if (!q || !aligned(q, 4)) return JAB_ERR_INVALID_ARG;
  if ((!free_dev && free_capacity > 0) || !aligned(free_dev, 4)) return JAB_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!slots_dev || !aligned(slots_dev, 8) || !positions_dev || !aligned(positions_dev, 4))) return JAB_ERR_INVALID_ARG;
  int *status, sms;
  if ((s = device(&status, &sms)) != JAB_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KvPlanArgs a{};
  a.n_seqs = n_seqs, a.page = cache->page_tokens, a.max_pages = max_pages, a.free_capacity = free_capacity;
  a.n_pages = cache->n_pages, a.n_tokens = n_tokens;
  a.lens = lens_dev, a.counts = counts_dev, a.pages = pages_dev, a.free_pages = const_cast<int32_t*>(free_dev), a.n_free = n_free_dev;
  a.new_lens = new_lens_dev, a.new_free = new_free_dev, a.q_start = q_start_dev, a.slots = slots_dev, a.positions = positions_dev;
  a.status = status;
  JAB_LAUNCH("kv_plan", kv_plan_kernels(a), launch_kv_plan(a, st));
  return JAB_OK;
}

}  // extern "C"
