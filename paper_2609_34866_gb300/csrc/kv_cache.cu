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
#include "quotient.cuh"
#include "serve.h"

namespace jab {
namespace {

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
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
  int64_t ldx, n_tokens, n_slots;
  int n_heads, n_q, n_kv, page, page_shift;  // page_shift: log2 of page, or -1
  const int64_t* slots;
  const int32_t* positions;
  const float *cos_t, *sin_t;
  int rope_len;
  void* q_out;
  uint8_t *k_codes, *v_codes;
  float *k_scales, *v_scales;
  int* status;
};

// Codes of 8 elements of a row with scale s (> 0), offset by 2^(BITS - 1): bytes, or halves of bytes.
template <int BITS>
__device__ __forceinline__ void codes8(const float (&x)[8], float s, uint32_t (&w)[BITS / 4]) {
  constexpr float OFFSET = BITS == 8 ? 128.f : 8.f;
  uint32_t u[8];
  if (usual_scale(s)) {
    const float r1 = __frcp_rn(s);
    const float2 r = make_float2(r1, r1), ms = make_float2(-s, -s);
    const float2 magic = make_float2(kToWhole, kToWhole), off = make_float2(OFFSET, OFFSET);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 q = tc::add2(tc::add2(quotients(make_float2(x[i], x[i + 1]), r, ms), magic), off);
      u[i] = __float_as_uint(q.x), u[i + 1] = __float_as_uint(q.y);  // (the low bits are the number)
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = (uint32_t)((int)fminf(fmaxf(rintf(__fdiv_rn(x[i], s)), 1.f - OFFSET), OFFSET - 1.f) + (int)OFFSET);
  }
  if constexpr (BITS == 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = __byte_perm(__byte_perm(u[4 * i], u[4 * i + 1], 0x0040), __byte_perm(u[4 * i + 2], u[4 * i + 3], 0x0040), 0x5410);
  } else {
    const uint32_t even = __byte_perm(__byte_perm(u[0], u[2], 0x0040), __byte_perm(u[4], u[6], 0x0040), 0x5410);
    const uint32_t odd = __byte_perm(__byte_perm(u[1], u[3], 0x0040), __byte_perm(u[5], u[7], 0x0040), 0x5410);
    w[0] = (even & 0x0f0f0f0fu) | (odd & 0x0f0f0f0fu) << 4;
  }
}

// Eight elements of a row as they lie in memory.
template <class T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void numbers(float (&x)[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        x[4 * i] = __uint_as_float(w[i].x), x[4 * i + 1] = __uint_as_float(w[i].y), x[4 * i + 2] = __uint_as_float(w[i].z), x[4 * i + 3] = __uint_as_float(w[i].w);
    } else {
      const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<T, half_t>::value) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
          x[2 * i] = f.x, x[2 * i + 1] = f.y;
        } else {
          x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
      }
    }
  }
};

// The largest magnitude of three, or NaN if one is NaN.
__device__ __forceinline__ float largest(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Blocks go over the tokens and a token's heads, a row of DH elements by DH / 16 threads, each with elements [8t, 8t + 8)
// of either half: the rotation's partners are in the same thread, all loads and stores of Q are 16 bytes. The next row,
// the next token's angles and the slot and position of the one after are under way while a row is worked on. Long inputs
// are bound by instructions as much as by bytes: with a grid-stride loop over rows, its 64-bit divisions and a division of
// every element, 8 x 2048 tokens of 48 heads of 128 (370 MB) took 108 us, with a token a block and no row ahead 90, like this 67 (5.5 TB/s).
constexpr int kWriteThreads = 384;  // of a block, at most
template <class T, int DH, int BITS>
__global__ void __launch_bounds__(kWriteThreads, sizeof(T) == 2 ? 2 : 1) kv_write_kernel(const __grid_constant__ WriteParams p) {
  constexpr int LANES = DH / 16;
  stream_order();
  const int t = threadIdx.x % LANES, head0 = threadIdx.x / LANES, heads = blockDim.x / LANES;
  Raw8<T> lo, hi;
  float c[8], s[8];
  int64_t slot = -1, next_slot = -1;
  int pos = 0, next_pos = 0;
  auto place = [&](int64_t token) {
    next_slot = __ldg(p.slots + token);
    if (p.positions != nullptr) next_pos = __ldg(p.positions + token);
  };
  auto angles = [&] {
    slot = next_slot, pos = next_pos;
    if (p.positions != nullptr && pos >= 0 && pos < p.rope_len) {
      load8(p.cos_t + (int64_t)pos * (DH / 2) + 8 * t, c);
      load8(p.sin_t + (int64_t)pos * (DH / 2) + 8 * t, s);
    }
  };
  auto fetch = [&](int64_t token, int head) {
    if (head < p.n_heads && (head >= p.n_q || p.q_out != nullptr)) {
      const T* row = static_cast<const T*>(p.x) + token * p.ldx + (int64_t)head * DH + 8 * t;
      lo.load(row), hi.load(row + DH / 2);
    }
  };
  int64_t token = blockIdx.x;
  int head = head0;
  place(token);
  fetch(token, head);
  angles();
  if (token + gridDim.x < p.n_tokens) place(token + gridDim.x);
  // (whole warps go round together: the rows' maxima are exchanged by shuffles)
  while (token < p.n_tokens) {
    float a[8], b[8];
    lo.numbers(a), hi.numbers(b);
    const int64_t now = token, to = slot;
    const int row = head;
    const bool is_q = row < p.n_q, is_k = row < p.n_q + p.n_kv, turn = p.positions != nullptr && is_k;
    const bool placed = to >= 0 && to < p.n_slots, turnable = p.positions == nullptr || (pos >= 0 && pos < p.rope_len);
    const bool live = placed && row < p.n_heads && (!turn || turnable) && !(is_q && p.q_out == nullptr);
    if (threadIdx.x == 0 && to >= 0 && (!placed || !turnable)) report(p.status, JAB_ERR_INVALID_ARG);
    if (live && turn) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // every product and every sum rounded: no contraction, which packed forms were seen to get
        const float x = a[i], y = b[i];
        a[i] = __fsub_rn(__fmul_rn(x, c[i]), __fmul_rn(y, s[i]));
        b[i] = __fadd_rn(__fmul_rn(y, c[i]), __fmul_rn(x, s[i]));
      }
    }
    head += heads;
    if (head - head0 >= p.n_heads) {
      head = head0, token += gridDim.x;
      if (token < p.n_tokens) angles();
      if (token + gridDim.x < p.n_tokens) place(token + gridDim.x);
    }
    if (token < p.n_tokens) fetch(token, head);
    float big = 0.f;
    if (live) {
#pragma unroll
      for (int i = 0; i < 8; ++i) big = largest(big, a[i], b[i]);
      if (is_q) {
        const int64_t at = (now * p.n_q + row) * DH + 8 * t;
        T* out = static_cast<T*>(p.q_out) + at;
        if (in_bounds(at + DH / 2 + 7, p.n_tokens * p.n_q * DH, p.status)) {
          store(out, a);
          store(out + DH / 2, b);
        }
        // finite, but not in Q's type (or neither): from halfway past the largest fp16 (65504) on
        if (std::is_same<T, half_t>::value && !(big < 65520.f)) report(p.status, JAB_ERR_RANGE);
      }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) big = largest(big, __shfl_xor_sync(0xffffffffu, big, o), 0.f);
    if (is_q || !live) continue;
    const bool fine = big < INFINITY;
    if (!fine) report(p.status, JAB_ERR_NONFINITE);
    const float scale = fine ? __fdiv_rn(big, (float)((1 << (BITS - 1)) - 1)) : __uint_as_float(0x7fc00000u);
    uint32_t w[2][BITS / 4];
    if (scale > 0.f) {
      codes8<BITS>(a, scale, w[0]);
      codes8<BITS>(b, scale, w[1]);
    } else {
#pragma unroll
      for (int i = 0; i < BITS / 4; ++i) w[0][i] = w[1][i] = BITS == 8 ? 0x80808080u : 0x88888888u;
    }
    const int h = row - p.n_q - (is_k ? 0 : p.n_kv);
    const int64_t pg = p.page_shift >= 0 ? to >> p.page_shift : to / p.page;
    const int64_t r = (pg * p.n_kv + h) * p.page + (to - pg * p.page);
    if (!in_bounds(r, p.n_slots * p.n_kv, p.status)) continue;
    uint8_t* codes = (is_k ? p.k_codes : p.v_codes) + r * (DH * BITS / 8) + t * BITS;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if constexpr (BITS == 8)
        *reinterpret_cast<uint2*>(codes + half * (DH / 2)) = make_uint2(w[half][0], w[half][1]);
      else
        *reinterpret_cast<uint32_t*>(codes + half * (DH / 4)) = w[half][0];
    }
    if (t == 0) (is_k ? p.k_scales : p.v_scales)[r] = scale;
  }
}

struct ReadParams {
  const uint8_t *k_codes, *v_codes;
  const float *k_scales, *v_scales;
  int64_t tokens;  // n_seqs * T
  int64_t n_pages;
  int n_kv, page, page_shift, T, max_pages;
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

// A thread stores 16 bytes of K and 16 of V of the block's tokens in turn.
// Bound: bytes; 16384 tokens of 8 heads of 128 in 8 bits to bf16 (34 + 67 MB) take 21 us, 0.7 of HBM's rate.
template <class T, int DH, int BITS>
__global__ void __launch_bounds__(256) kv_read_kernel(const __grid_constant__ ReadParams p, int per_block) {
  constexpr int N = 16 / sizeof(T), LANES = DH / N;
  stream_order();
  const int units = p.n_kv * LANES;
  const int64_t t0 = (int64_t)blockIdx.x * per_block;
  const int n = (int)min((int64_t)per_block, p.tokens - t0);
  int b = (int)(t0 / p.T), j = (int)(t0 - (int64_t)b * p.T);
  // places of 16 bytes of the tokens' rows: u counts over (token, head, lane)
  int token = threadIdx.x / units, u = threadIdx.x - token * units;
  j += token;
  while (token < n) {
    while (j >= p.T) j -= p.T, ++b;
    const int h = u / LANES, t = u % LANES;
    float k[N] = {}, v[N] = {};
    if (j < __ldg(p.counts + b)) {
      const int64_t at = (int64_t)j + (p.starts != nullptr ? __ldg(p.starts + b) : 0);
      const int64_t pg = p.page_shift >= 0 ? at >> p.page_shift : at / p.page;
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
    const int64_t o = ((t0 + token) * p.n_kv + h) * DH + t * N;
    if (in_bounds(o + N - 1, p.tokens * p.n_kv * DH, p.status)) {
      store(static_cast<T*>(p.k) + o, k);
      store(static_cast<T*>(p.v) + o, v);
    }
    for (u += 256; u >= units; u -= units) ++token, ++j;
  }
}

template <class T, int DH, int BITS>
cudaError_t write_as(const WriteParams& p, int sms, cudaStream_t st) {
  // A block has a token's heads, or as many of them as kWriteThreads threads take. With four tokens for every SM and more, a
  // third of the heads where that leaves no thread idle: it loads a token's angles once for its rows in turn (2048 tokens of 48
  // heads of 128: 19 us for writing and reading, 22 without; but 64 tokens 4.9 instead of 4.5).
  constexpr int PER_SM = sizeof(T) == 2 ? 768 : 512;
  const int want = p.n_heads * (DH / 16), share = p.n_tokens >= 4 * (int64_t)sms && want % 96 == 0 ? want / 3 : want;
  const int threads = (std::min(share, kWriteThreads) + 31) / 32 * 32;
  const int64_t blocks = std::min<int64_t>(p.n_tokens, (int64_t)sms * std::min(32, std::max(1, PER_SM / threads)));
  return launch_after(kv_write_kernel<T, DH, BITS>, (unsigned)blocks, threads, 0, st, p);
}
template <class T>
cudaError_t write_type(const WriteParams& p, int dh, int bits, int sms, cudaStream_t st) {
  if (dh == 128) return bits == 8 ? write_as<T, 128, 8>(p, sms, st) : write_as<T, 128, 4>(p, sms, st);
  return bits == 8 ? write_as<T, 64, 8>(p, sms, st) : write_as<T, 64, 4>(p, sms, st);
}

template <class T, int DH, int BITS>
cudaError_t read_as(const ReadParams& p, int sms, cudaStream_t st) {
  // four passes of a block's threads, fewer where the SMs would not all have one
  const int64_t places = p.tokens * p.n_kv * (DH * (int64_t)sizeof(T) / 16);
  const int64_t passes = std::max<int64_t>(1, std::min<int64_t>(4, places / (256 * (int64_t)sms)));
  const int per_block = (int)std::max<int64_t>(1, passes * 256 / (p.n_kv * (DH * (int64_t)sizeof(T) / 16)));
  return launch_after(kv_read_kernel<T, DH, BITS>, (unsigned)((p.tokens + per_block - 1) / per_block), 256, 0, st, p, per_block);
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
  p.n_tokens = a.n_tokens;
  p.page = c.page_tokens;
  p.page_shift = (p.page & (p.page - 1)) == 0 ? 31 - __builtin_clz(p.page) : -1;
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
  p.tokens = (int64_t)a.n_seqs * a.T;
  p.page_shift = (c.page_tokens & (c.page_tokens - 1)) == 0 ? 31 - __builtin_clz(c.page_tokens) : -1;
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
