// The gradient of the norm and rotation of the heads of Q and K (the forward is a mode of kv_cache.cu's writing kernel), and rotation
// tables for stretched contexts.
//
//   y = R n, n = (x r) w, r = (mean x^2 + eps)^(-1/2):   g = R^T dy, u = g w,
//   dx = r (u - x r mean(u x r)),  dw = sum over tokens and heads of g x r
//
// Bound: bytes in flight and instructions; 16384 tokens of 40 heads of 128 in bf16 (503 MB) take 108 us, 4.7 TB/s, without a norm 91.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "rows.cuh"
#include "serve.h"

namespace jab {
namespace {

struct BackParams {
  const void *x, *dq, *dk;
  int64_t ldx, lddq, lddk, lddx, n_tokens;
  void* dx;
  int n_q, n_k;
  const int32_t* positions;
  const float *cos_t, *sin_t, *wq, *wk;
  int rope_len, rotary;
  bool neighbours;
  float eps;    // 0: no norm
  float* part;  // [blocks, 2, DH] of the weights' gradients, or null
  int* status;
};

constexpr int kBackThreads = 256;
constexpr int kMostParts = 1216;  // blocks along the tokens times blocks along the heads, where the heads allow it

// A thread stays with one head's two groups of 8 (as in the writing kernel) and goes over the tokens, so that its share of the
// weights' gradient is 16 registers. The next token's rows are under way while one is worked on (two ahead: slower, registers).
template <class T, int DH>
__global__ void __launch_bounds__(kBackThreads, 2) norm_rope_back_kernel(const __grid_constant__ BackParams p) {
  constexpr int LANES = DH / 16;
  __shared__ alignas(16) float sums[kBackThreads / LANES][DH];
  __shared__ alignas(16) float weights[2][DH];
  stream_order();
  for (int i = threadIdx.x; i < 2 * DH; i += blockDim.x) {
    const float* from = i < DH ? p.wq : p.wk;
    weights[i / DH][i % DH] = from != nullptr ? __ldg(from + i % DH) : 1.f;
  }
  __syncthreads();
  const int heads = blockDim.x / LANES;
  const int t = threadIdx.x % LANES, slot = threadIdx.x / LANES, head = blockIdx.y * heads + slot;
  const bool exists = head < p.n_q + p.n_k, is_q = head < p.n_q;
  const bool turns = p.positions != nullptr && 16 * t < p.rotary, pairs = p.neighbours || 16 * t >= p.rotary;
  const int at0 = pairs ? 16 * t : 8 * t, at1 = pairs ? at0 + 8 : at0 + p.rotary / 2;
  const float2 *w0 = reinterpret_cast<const float2*>(weights[is_q ? 0 : 1] + at0), *w1 = reinterpret_cast<const float2*>(weights[is_q ? 0 : 1] + at1);
  float2 dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[i] = make_float2(0.f, 0.f);
  const T* x = static_cast<const T*>(p.x) + (int64_t)head * DH;
  const T* dy = is_q ? static_cast<const T*>(p.dq) + (int64_t)head * DH : static_cast<const T*>(p.dk) + (int64_t)(head - p.n_q) * DH;
  const int64_t lddy = is_q ? p.lddq : p.lddk;
  Raw8<T> x0 = {}, x1 = {}, g0 = {}, g1 = {};
  int next = 0;
  auto fetch = [&](int64_t token) {
    if (token >= p.n_tokens) return;
    if (p.positions != nullptr) next = __ldg(p.positions + token);
    if (!exists) return;
    x0.load(x + token * p.ldx + at0), x1.load(x + token * p.ldx + at1);
    g0.load(dy + token * lddy + at0), g1.load(dy + token * lddy + at1);
  };
  fetch(blockIdx.x);
  for (int64_t token = blockIdx.x; token < p.n_tokens; token += gridDim.x) {
    alignas(8) float a[8], b[8], g[8], h[8];
    x0.numbers(a), x1.numbers(b), g0.numbers(g), g1.numbers(h);
    const int pos = next;
    const bool fine = p.positions == nullptr || (pos >= 0 && pos < p.rope_len);
    if (threadIdx.x == 0 && !fine) report(p.status, JAB_ERR_INVALID_ARG);
    float c[8], s[8];
    if (turns && fine) {
      load8(p.cos_t + (int64_t)pos * (p.rotary / 2) + 8 * t, c);
      load8(p.sin_t + (int64_t)pos * (p.rotary / 2) + 8 * t, s);
    }
    fetch(token + gridDim.x);
    if (!fine) continue;  // (the whole block has this token)
    // (packed pairs halve the instructions; no rounding here is part of a definition)
    float2 *a2 = reinterpret_cast<float2*>(a), *b2 = reinterpret_cast<float2*>(b), *g2 = reinterpret_cast<float2*>(g), *h2 = reinterpret_cast<float2*>(h);
    if (turns) {
      if (p.neighbours) {
        auto back = [](float& y, float& z, float cs, float sn) {
          const float da = y * cs + z * sn, db = z * cs - y * sn;
          y = da, z = db;
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) back(g[2 * i], g[2 * i + 1], c[i], s[i]), back(h[2 * i], h[2 * i + 1], c[4 + i], s[4 + i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 cs = make_float2(c[2 * i], c[2 * i + 1]), sn = make_float2(s[2 * i], s[2 * i + 1]), ns = make_float2(-sn.x, -sn.y);
          const float2 y = g2[i], z = h2[i];
          g2[i] = tc::fma2(z, sn, tc::mul2(y, cs));
          h2[i] = tc::fma2(y, ns, tc::mul2(z, cs));
        }
      }
    }
    if (p.eps > 0.f) {
      // r to a few ulp does here: the two sums of a row go through the lanes together
      float2 sq2 = make_float2(0.f, 0.f), dot2 = make_float2(0.f, 0.f);
      float2 u2[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u2[i] = tc::mul2(g2[i], w0[i]), u2[4 + i] = tc::mul2(h2[i], w1[i]);
        sq2 = tc::fma2(b2[i], b2[i], tc::fma2(a2[i], a2[i], sq2));
        dot2 = tc::fma2(u2[4 + i], b2[i], tc::fma2(u2[i], a2[i], dot2));
      }
      float sq = sq2.x + sq2.y, dot = dot2.x + dot2.y;
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) {
        sq += __shfl_xor_sync(0xffffffffu, sq, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      const float mean = sq * (1.f / DH) + p.eps;
      const float r = mean < INFINITY ? rsqrtf(mean) : __uint_as_float(0x7fc00000u);
      const float k = -(r * dot) * r * (1.f / DH);  // of x: -r^2 mean(u x)
      const float2 r2 = make_float2(r, r), k2 = make_float2(k, k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dw[i] = tc::fma2(g2[i], tc::mul2(a2[i], r2), dw[i]), dw[4 + i] = tc::fma2(h2[i], tc::mul2(b2[i], r2), dw[4 + i]);
        g2[i] = tc::mul2(r2, tc::fma2(a2[i], k2, u2[i]));
        h2[i] = tc::mul2(r2, tc::fma2(b2[i], k2, u2[4 + i]));
      }
      if (exists && !(r == r)) report(p.status, JAB_ERR_NONFINITE);
    }
    if (exists) {
      if constexpr (std::is_same<T, half_t>::value) {  // finite, but not in fp16: from halfway past its largest on
        float big = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) big = largest(big, g[i], h[i]);
        if (!(big < 65520.f)) report(p.status, JAB_ERR_RANGE);
      }
      const int64_t at = token * p.lddx + (int64_t)head * DH;
      if (in_bounds(at + max(at0, at1) + 7, (p.n_tokens - 1) * p.lddx + (int64_t)(p.n_q + p.n_k) * DH, p.status)) {
        store(static_cast<T*>(p.dx) + at + at0, g);
        store(static_cast<T*>(p.dx) + at + at1, h);
      }
    }
  }
  if (p.part == nullptr) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    *reinterpret_cast<float2*>(&sums[slot][at0 + 2 * i]) = dw[i];  // (0 without a head)
    *reinterpret_cast<float2*>(&sums[slot][at1 + 2 * i]) = dw[4 + i];
  }
  __syncthreads();
  const int q_end = min(max(p.n_q - (int)blockIdx.y * heads, 0), heads);
  for (int i = threadIdx.x; i < 2 * DH; i += blockDim.x) {
    const int d = i % DH, h0 = i < DH ? 0 : q_end, h1 = i < DH ? q_end : heads;
    float v = 0.f;
    for (int h = h0; h < h1; ++h) v += sums[h][d];
    p.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * DH + i] = v;
  }
}

// The blocks' sums, in their order: eight columns a block of threads, 32 runs of blocks each, added up as pairs.
__global__ void __launch_bounds__(256) weight_sum_kernel(const float* part, int n, int dh, float* dwq, float* dwk) {
  __shared__ float hi_s[32][8], lo_s[32][8];
  stream_order();
  const int lane = threadIdx.x & 7, run = threadIdx.x >> 3, col = blockIdx.x * 8 + lane;
  float hi = 0.f, lo = 0.f;
#pragma unroll 8
  for (int i = run; i < n; i += 32) pair_add(hi, lo, part[(int64_t)i * 2 * dh + col], 0.f);
  hi_s[run][lane] = hi, lo_s[run][lane] = lo;
  __syncthreads();
  if (run != 0) return;
  for (int i = 1; i < 32; ++i) pair_add(hi, lo, hi_s[i][lane], lo_s[i][lane]);
  float* out = col < dh ? dwq : dwk;
  if (out != nullptr) out[col < dh ? col : col - dh] = fabsf(hi) < INFINITY ? hi + lo : hi;
}

// ------------------------------------------------------------------ tables
struct TableParams {
  double freq_pi[64];  // angle of a step over pi
  double by;
  float *cos_t, *sin_t;
  int length, half;
};

// Angles are position x frequency in 64 bits, reduced by the pi forms without a long division; the rounding of the product
// (2^-53 of up to 2^31 turns) is 2^-22 of a turn at the very worst and 2^-36 at 2^17 positions. A thread takes sixteen positions of its
// pair and rotates from the first, as an fp64 sincos costs some sixty instructions at two a clock and SM.
// 131072 positions of 64 pairs: 177 us (67 MB: 10; such tables are made once).
constexpr int kRun = 16;
__global__ void __launch_bounds__(64) rope_table_kernel(const __grid_constant__ TableParams p) {
  stream_order();
  const int j = threadIdx.x;
  if (j >= p.half) return;
  const double f = p.freq_pi[j];
  const int t0 = blockIdx.x * kRun, n = min(kRun, p.length - t0);
  double sn, cs, sd, cd;
  sincospi((double)t0 * f, &sn, &cs);
  sincospi(f, &sd, &cd);
  int64_t i = (int64_t)t0 * p.half + j;
  for (int k = 0; k < n; ++k, i += p.half) {
    p.cos_t[i] = (float)(cs * p.by);
    p.sin_t[i] = (float)(sn * p.by);
    const double c2 = cs * cd - sn * sd;
    sn = sn * cd + cs * sd;
    cs = c2;
  }
}

template <class T, int DH>
cudaError_t back_as(const BackParams& p, float* dwq, float* dwk, int sms, cudaStream_t st) {
  // as many heads a block as kBackThreads threads take, and as even a share of them as whole warps allow (16384 tokens of 40 heads of
  // 128 as 32 and 8: 145 us, as 20 and 20: 108)
  constexpr int MOST = kBackThreads / (DH / 16), WARP = 32 / (DH / 16);
  const int heads = p.n_q + p.n_k, blocks = (heads + MOST - 1) / MOST, share = ((heads + blocks - 1) / blocks + WARP - 1) / WARP * WARP;
  const int gy = (heads + share - 1) / share;
  // four tokens a block and more where the weights' gradients are wanted: every block has a part of them to be added up
  const int64_t at_most = p.part != nullptr ? (p.n_tokens + 3) / 4 : p.n_tokens;
  // and no more blocks than are resident at once (128 registers a thread): all have the same number of tokens, but for one
  // (three blocks an SM: 108 us, with four 142)
  const int resident = sms * std::min(16, 65536 / (128 * share * (DH / 16)));
  const int gx = (int)std::min<int64_t>(at_most, std::max(1, std::min(kMostParts, resident) / gy));
  if (gx > 0) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(gx, gy);
    cfg.blockDim = dim3(share * (DH / 16));
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, norm_rope_back_kernel<T, DH>, p);
    if (e != cudaSuccess) {
      cudaGetLastError();
      return e;
    }
  }
  if (p.part == nullptr) return cudaSuccess;
  return launch_after(weight_sum_kernel, 2 * DH / 8, 256, 0, st, (const float*)p.part, gx * gy, DH, dwq, dwk);
}
template <class T>
cudaError_t back_type(const BackParams& p, int dh, float* dwq, float* dwk, int sms, cudaStream_t st) {
  return dh == 128 ? back_as<T, 128>(p, dwq, dwk, sms, st) : back_as<T, 64>(p, dwq, dwk, sms, st);
}

bool wants_weights(const NormRopeBackArgs& a) { return a.dwq != nullptr || a.dwk != nullptr; }

}  // namespace

size_t norm_rope_scratch(int n_heads, int dh) {
  const int per = kBackThreads / (dh / 16);
  return (size_t)std::max(kMostParts, (n_heads + per - 1) / per) * 2 * dh * sizeof(float);
}

int norm_rope_back_kernels(const NormRopeBackArgs& a) { return (a.n_tokens > 0 ? 1 : 0) + (wants_weights(a) ? 1 : 0); }

cudaError_t launch_norm_rope_back(const NormRopeBackArgs& a, int sms, cudaStream_t st) {
  BackParams p{};
  p.x = a.x, p.dq = a.dq, p.dk = a.dk;
  p.ldx = a.ldx, p.lddq = a.lddq, p.lddk = a.lddk, p.lddx = a.lddx;
  p.n_tokens = a.n_tokens;
  p.dx = a.dx;
  p.n_q = a.n_q, p.n_k = a.n_k;
  p.positions = a.how.positions_dev;
  p.cos_t = a.how.cos_dev, p.sin_t = a.how.sin_dev;
  p.wq = a.how.q_weight_dev, p.wk = a.how.k_weight_dev;
  p.rope_len = a.how.rope_len;
  p.rotary = a.how.positions_dev != nullptr ? a.how.rotary_dim : 0;
  p.neighbours = a.how.interleaved != 0;
  p.eps = a.how.norm ? a.how.eps : 0.f;
  p.part = wants_weights(a) ? static_cast<float*>(a.ws) : nullptr;
  p.status = a.status;
  return a.type == JAB_FP16   ? back_type<half_t>(p, a.head_dim, a.dwq, a.dwk, sms, st)
         : a.type == JAB_BF16 ? back_type<bf16_t>(p, a.head_dim, a.dwq, a.dwk, sms, st)
                              : back_type<float>(p, a.head_dim, a.dwq, a.dwk, sms, st);
}

cudaError_t launch_rope_table(const RopeTableArgs& a, cudaStream_t st) {
  TableParams p{};
  p.cos_t = a.cos_t, p.sin_t = a.sin_t;
  p.length = a.length;
  p.half = a.rotary / 2;
  p.by = a.scaling.attention;
  const double pi = 3.14159265358979323846;
  for (int j = 0; j < p.half; ++j) {
    double f = pow((double)a.theta, -2.0 * j / a.rotary);
    if (a.scaling.kind == JAB_ROPE_LINEAR) f /= a.scaling.factor;
    if (a.scaling.kind == JAB_ROPE_BY_PARTS) {
      const double turns = a.scaling.original_length * f / (2 * pi);
      const double g = std::min(1.0, std::max(0.0, (turns - a.scaling.low_turns) / ((double)a.scaling.high_turns - a.scaling.low_turns)));
      f = g * f + (1 - g) * f / a.scaling.factor;
    }
    p.freq_pi[j] = f / pi;
  }
  return launch_after(rope_table_kernel, (unsigned)((a.length - 1) / kRun + 1), 64, 0, st, p);
}

}  // namespace jab
