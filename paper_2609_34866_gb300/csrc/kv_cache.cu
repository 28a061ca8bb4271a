// The quantised paged cache: tokens are rotated, quantised and written as they come from the projection,
// and read back as numbers. Both kernels move each byte once and are bound by memory on long inputs, by
// their launch on short ones.
//
//   write   per (token, head) row x: s = fl32(max|x| / qmax), q = clip(rint(fl32(x / s)), +-qmax);
//           rotate-half first on Q and K: (a cos - b sin, b cos + a sin), each product and sum rounded
//           to fp32 (no fused multiply-add: the codes are then a function of the inputs that any
//           implementation can reproduce bit by bit)
//   read    q * s, rounded to the type asked for
#include <algorithm>

#include "common.cuh"
#include "serve.h"

namespace jab {
namespace {

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<half_t>(const half_t* p, float (&v)[8]) {
  const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}

__device__ __forceinline__ uint32_t pack2(float a, float b, half_t) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bf16_t) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T, int N>
__device__ __forceinline__ void store(T* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 8)
    *reinterpret_cast<uint4*>(p + i) = make_uint4(pack2(v[i], v[i + 1], T()), pack2(v[i + 2], v[i + 3], T()),
                                                  pack2(v[i + 4], v[i + 5], T()), pack2(v[i + 6], v[i + 7], T()));
}
template <int N>
__device__ __forceinline__ void store(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}

struct WriteParams {
  const void* x;
  int64_t ldx, units, n_slots;
  int n_heads, n_q, n_kv, page;
  const int64_t* slots;
  const int32_t* positions;
  const float *cos_t, *sin_t;
  int rope_len;
  void* q_out;
  uint8_t *k_codes, *v_codes;
  float *k_scales, *v_scales;
  int* status;
};

// A row of DH elements by DH / 16 threads, each with elements [8t, 8t + 8) of either half: the rotation's
// partners are in the same thread, all loads and stores of Q are 16 bytes.
template <class T, int DH, int BITS>
__global__ void __launch_bounds__(256) kv_write_kernel(const __grid_constant__ WriteParams p) {
  constexpr int LANES = DH / 16, QMAX = (1 << (BITS - 1)) - 1;
  stream_order();
  const int t = threadIdx.x % LANES;
  const int64_t step = (int64_t)gridDim.x * (256 / LANES);
  const int64_t first = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  // whole warps go round together: the rows' maxima are exchanged by shuffles
  const int64_t rounds = (p.units + step - 1) / step;
  for (int64_t it = 0; it < rounds; ++it) {
    const int64_t unit = first + it * step;
    bool live = unit < p.units;
    const int64_t token = live ? unit / p.n_heads : 0;
    const int head = live ? (int)(unit - token * p.n_heads) : 0;
    const int64_t slot = live ? __ldg(p.slots + token) : -1;
    live = slot >= 0;
    const bool is_q = head < p.n_q, turn = p.positions != nullptr && head < p.n_q + p.n_kv;
    if (live && slot >= p.n_slots) {
      report(p.status, JAB_ERR_INVALID_ARG);
      live = false;
    }
    int pos = 0;
    if (live && turn) {
      pos = __ldg(p.positions + token);
      if (pos < 0 || pos >= p.rope_len) {
        report(p.status, JAB_ERR_INVALID_ARG);
        live = false;
      }
    }
    if (is_q && p.q_out == nullptr) live = false;
    float a[8] = {}, b[8] = {};
    if (live) {
      const T* row = static_cast<const T*>(p.x) + token * p.ldx + (int64_t)head * DH + 8 * t;
      load8(row, a);
      load8(row + DH / 2, b);
      if (turn) {
        float c[8], s[8];
        load8(p.cos_t + (int64_t)pos * (DH / 2) + 8 * t, c);
        load8(p.sin_t + (int64_t)pos * (DH / 2) + 8 * t, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = __fsub_rn(__fmul_rn(a[i], c[i]), __fmul_rn(b[i], s[i]));
          b[i] = __fadd_rn(__fmul_rn(b[i], c[i]), __fmul_rn(a[i], s[i]));
          a[i] = u;
        }
      }
    }
    uint32_t big = 0;  // magnitude bits of the row's largest (an infinity or a NaN is larger than all others)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      big = max(big, max(__float_as_uint(a[i]) & 0x7fffffffu, __float_as_uint(b[i]) & 0x7fffffffu));
    if (is_q) {
      if (live) {
        T* out = static_cast<T*>(p.q_out) + (token * p.n_q + head) * DH + 8 * t;
        store(out, a);
        store(out + DH / 2, b);
        // finite, but not in Q's type: from halfway past the largest fp16 (65504) on
        if (sizeof(T) == 2 && std::is_same<T, half_t>::value && big >= 0x477ff000u) report(p.status, JAB_ERR_RANGE);
      }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
    if (is_q || !live) continue;
    const bool fine = big < 0x7f800000u;
    if (!fine) report(p.status, JAB_ERR_NONFINITE);
    const float s = fine ? __fdiv_rn(__uint_as_float(big), (float)QMAX) : __uint_as_float(0x7fc00000u);
    int q[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = i < 8 ? a[i] : b[i - 8];
      const float r = fminf(fmaxf(rintf(__fdiv_rn(x, s)), (float)-QMAX), (float)QMAX);
      q[i] = (fine && s > 0.f ? (int)r : 0) + QMAX + 1;
    }
    const bool is_k = head < p.n_q + p.n_kv;
    const int h = head - p.n_q - (is_k ? 0 : p.n_kv);
    const int64_t pg = slot / p.page;
    const int64_t r = (pg * p.n_kv + h) * p.page + (slot - pg * p.page);
    uint8_t* codes = (is_k ? p.k_codes : p.v_codes) + r * (DH * BITS / 8);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int* c = q + 8 * half;
      if (BITS == 8) {
        uint2 w;
        w.x = c[0] | c[1] << 8 | c[2] << 16 | (uint32_t)c[3] << 24;
        w.y = c[4] | c[5] << 8 | c[6] << 16 | (uint32_t)c[7] << 24;
        *reinterpret_cast<uint2*>(codes + half * (DH / 2) + 8 * t) = w;
      } else {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint32_t)c[i] << (4 * i);
        *reinterpret_cast<uint32_t*>(codes + half * (DH / 4) + 4 * t) = w;
      }
    }
    if (t == 0) (is_k ? p.k_scales : p.v_scales)[r] = s;
  }
}

struct ReadParams {
  const uint8_t *k_codes, *v_codes;
  const float *k_scales, *v_scales;
  int64_t rows;  // n_seqs * T * n_kv
  int64_t n_pages;
  int n_kv, page, T, max_pages;
  const int32_t *pages, *starts, *counts;
  void *k, *v;
  int* status;
};

// N codes (N * BITS / 8 bytes at p) as numbers.
template <int BITS, int N>
__device__ __forceinline__ void decode(const uint8_t* p, float s, float (&v)[N]) {
  constexpr int BYTES = N * BITS / 8;
  uint8_t raw[BYTES];
  if (BYTES == 8)
    *reinterpret_cast<uint2*>(raw) = __ldg(reinterpret_cast<const uint2*>(p));
  else if (BYTES == 4)
    *reinterpret_cast<uint32_t*>(raw) = __ldg(reinterpret_cast<const uint32_t*>(p));
  else
    *reinterpret_cast<uint16_t*>(raw) = __ldg(reinterpret_cast<const uint16_t*>(p));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = BITS == 8 ? raw[i] : (raw[i / 2] >> (4 * (i & 1))) & 15;
    v[i] = __fmul_rn((float)(u - (1 << (BITS - 1))), s);
  }
}

// A thread stores 16 bytes of K and 16 of V.
template <class T, int DH, int BITS>
__global__ void __launch_bounds__(256) kv_read_kernel(const __grid_constant__ ReadParams p) {
  constexpr int N = 16 / sizeof(T), LANES = DH / N;
  stream_order();
  const int t = threadIdx.x % LANES;
  const int64_t step = (int64_t)gridDim.x * (256 / LANES);
  for (int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; row < p.rows; row += step) {
    const int64_t bt = row / p.n_kv;
    const int h = (int)(row - bt * p.n_kv);
    const int b = (int)(bt / p.T), j = (int)(bt - (int64_t)b * p.T);
    float k[N] = {}, v[N] = {};
    if (j < __ldg(p.counts + b)) {
      const int64_t at = (int64_t)j + (p.starts != nullptr ? __ldg(p.starts + b) : 0);
      const int64_t pg = at / p.page;
      const int id = at >= 0 && pg < p.max_pages ? __ldg(p.pages + (int64_t)b * p.max_pages + pg) : -1;
      if (id >= 0 && id < p.n_pages) {
        const int64_t r = ((int64_t)id * p.n_kv + h) * p.page + (at - pg * p.page);
        const int64_t c = r * (DH * BITS / 8) + t * (N * BITS / 8);
        decode<BITS>(p.k_codes + c, __ldg(p.k_scales + r), k);
        decode<BITS>(p.v_codes + c, __ldg(p.v_scales + r), v);
      } else {
        report(p.status, JAB_ERR_INVALID_ARG);
      }
    }
    store(static_cast<T*>(p.k) + row * DH + t * N, k);
    store(static_cast<T*>(p.v) + row * DH + t * N, v);
  }
}

template <class T, int DH, int BITS>
cudaError_t write_as(const WriteParams& p, int sms, cudaStream_t st) {
  const int64_t blocks = (p.units + 256 / (DH / 16) - 1) / (256 / (DH / 16));
  return launch_after(kv_write_kernel<T, DH, BITS>, (unsigned)std::min<int64_t>(blocks, (int64_t)sms * 32), 256, 0, st, p);
}
template <class T>
cudaError_t write_type(const WriteParams& p, int dh, int bits, int sms, cudaStream_t st) {
  if (dh == 128) return bits == 8 ? write_as<T, 128, 8>(p, sms, st) : write_as<T, 128, 4>(p, sms, st);
  return bits == 8 ? write_as<T, 64, 8>(p, sms, st) : write_as<T, 64, 4>(p, sms, st);
}

template <class T, int DH, int BITS>
cudaError_t read_as(const ReadParams& p, int sms, cudaStream_t st) {
  constexpr int ROWS = 256 / (DH * (int)sizeof(T) / 16);
  return launch_after(kv_read_kernel<T, DH, BITS>, (unsigned)std::min<int64_t>((p.rows + ROWS - 1) / ROWS, (int64_t)sms * 32),
                      256, 0, st, p);
}
template <class T>
cudaError_t read_type(const ReadParams& p, int dh, int bits, int sms, cudaStream_t st) {
  if (dh == 128) return bits == 8 ? read_as<T, 128, 8>(p, sms, st) : read_as<T, 128, 4>(p, sms, st);
  return bits == 8 ? read_as<T, 64, 8>(p, sms, st) : read_as<T, 64, 4>(p, sms, st);
}

}  // namespace

cudaError_t launch_kv_write(const KvWriteArgs& a, int sms, cudaStream_t st) {
  const jab_kv_cache& c = a.cache;
  WriteParams p{};
  p.x = a.x;
  p.ldx = a.ldx;
  p.n_q = a.n_q_heads;
  p.n_kv = c.n_kv_heads;
  p.n_heads = p.n_q + 2 * p.n_kv;
  p.units = a.n_tokens * p.n_heads;
  p.page = c.page_tokens;
  p.n_slots = c.n_pages * c.page_tokens;
  p.slots = a.slots;
  p.positions = a.positions;
  p.cos_t = a.cos_t;
  p.sin_t = a.sin_t;
  p.rope_len = a.rope_len;
  p.q_out = a.q_out;
  p.k_codes = static_cast<uint8_t*>(c.k_codes);
  p.v_codes = static_cast<uint8_t*>(c.v_codes);
  p.k_scales = c.k_scales;
  p.v_scales = c.v_scales;
  p.status = a.status;
  if (a.type == JAB_FP16) return write_type<half_t>(p, c.head_dim, c.bits, sms, st);
  if (a.type == JAB_BF16) return write_type<bf16_t>(p, c.head_dim, c.bits, sms, st);
  return write_type<float>(p, c.head_dim, c.bits, sms, st);
}

cudaError_t launch_kv_read(const KvReadArgs& a, int sms, cudaStream_t st) {
  const jab_kv_cache& c = a.cache;
  ReadParams p{};
  p.k_codes = static_cast<const uint8_t*>(c.k_codes);
  p.v_codes = static_cast<const uint8_t*>(c.v_codes);
  p.k_scales = c.k_scales;
  p.v_scales = c.v_scales;
  p.rows = (int64_t)a.n_seqs * a.T * c.n_kv_heads;
  p.n_pages = c.n_pages;
  p.n_kv = c.n_kv_heads;
  p.page = c.page_tokens;
  p.T = a.T;
  p.max_pages = a.max_pages;
  p.pages = a.pages;
  p.starts = a.starts;
  p.counts = a.counts;
  p.k = a.k;
  p.v = a.v;
  p.status = a.status;
  if (a.type == JAB_FP16) return read_type<half_t>(p, c.head_dim, c.bits, sms, st);
  if (a.type == JAB_BF16) return read_type<bf16_t>(p, c.head_dim, c.bits, sms, st);
  return read_type<float>(p, c.head_dim, c.bits, sms, st);
}

}  // namespace jab
