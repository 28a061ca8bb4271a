// Rows of heads as the serving kernels hold them: a thread has two groups of 8 elements of a row.
#pragma once
#include "common.cuh"
#include "tc.cuh"

namespace jab {

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

// 1 / sqrt(mean x^2 + eps) of a row of 16 LANES elements, of which the lanes of a group have a[8], b[8] each, so near that it is the
// nearest fp32 but for one in 2^16 or fewer: the codes of what it multiplies are then the same from any implementation that
// rounds it right. A thread's squares are added to a power of two of 16 times their largest and more: the sum s = fl(h + x^2) is
// within a factor of two of h, so that h - s is exact and what s lost, x^2 + (h - s), is one fused operation; the losses
// add up beside it (about 2^-38 of the sum is lost; adding pairs takes twice the operations). NaN where 32 times a square leaves fp32.
// Called by whole warps.
template <int LANES>
__device__ __forceinline__ float norm_factor(const float (&a)[8], const float (&b)[8], float eps) {
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) big = largest(big, a[i], b[i]);
  const float base = __uint_as_float(__float_as_uint(32.f * big * big) & 0x7f800000u);
  float2 h = make_float2(base, base), l = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = make_float2(a[i], b[i]), s = tc::fma2(x, x, h);
    l = tc::add2(l, tc::fma2(x, x, tc::sub2(h, s)));
    h = s;
  }
  float hi = h.x - base, lo = l.x;
  pair_add(hi, lo, h.y - base, l.y);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, hi, o), v = __shfl_xor_sync(0xffffffffu, lo, o);
    pair_add(hi, lo, u, v);
  }
  constexpr float kMean = 1.f / (16 * LANES);
  float m, e;
  two_sum(hi * kMean, eps, m, e);
  e += lo * kMean;
  const float r = rsqrtf(m), y = __fmul_rn(m, r), ye = __fmaf_rn(m, r, -y);  // m + e is the mean, y + ye = m r
  const float rest = __fmaf_rn(-y, r, 1.f) - __fmaf_rn(ye, r, e * r * r);    // 1 - (m + e) r^2
  return m < INFINITY ? __fmaf_rn(r, 0.5f * rest, r) : __uint_as_float(0x7fc00000u);
}

}  // namespace jab
