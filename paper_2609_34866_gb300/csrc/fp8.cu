// Rows in 8-bit floating point (e4m3) with a scale for every block of 1 or 128 rows x 128 columns:
//
//   s = fl32(max|x| / 448),  code = e4m3(fl32(x / s))
//
// One pass: a block's elements stay in registers between the maximum and the codes. Bound: bytes.
#include <cuda_fp8.h>

#include <algorithm>

#include "common.cuh"
#include "fp8.cuh"
#include "rows.cuh"
#include "serve.h"

namespace jab {
namespace {

struct QuantParams {
  const void* x;
  int64_t ldx, M;
  int K, blocks;  // blocks of 128 columns
  uint8_t* codes;  // [M, K]
  float* scales;
  int64_t row_pitch, block_pitch;
  int* status;
};

// A half warp has a row's block, a lane 8 elements of it; four blocks of a half warp are under way together.
template <class T>
__global__ void __launch_bounds__(256) fp8_rows_kernel(const __grid_constant__ QuantParams p) {
  constexpr int AHEAD = sizeof(T) == 2 ? 4 : 2;
  stream_order();
  const int lane = threadIdx.x & 15;
  const int64_t units = p.M * p.blocks, step = (int64_t)gridDim.x * 16;
  for (int64_t u0 = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); u0 - (threadIdx.x >> 4) < units; u0 += step * AHEAD) {
    Raw8<T> raw[AHEAD];
    int64_t m[AHEAD];
    int kb[AHEAD];
    bool live[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t u = u0 + i * step;
      m[i] = u / p.blocks, kb[i] = (int)(u - m[i] * p.blocks);
      live[i] = u < units && kb[i] * 128 + lane * 8 < p.K;
      raw[i] = {};
      if (live[i]) raw[i].load(static_cast<const T*>(p.x) + m[i] * p.ldx + kb[i] * 128 + lane * 8);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      float v[8];
      raw[i].numbers(v);
      float big = 0.f;
#pragma unroll
      for (int j = 0; j < 8; j += 2) big = largest(big, v[j], v[j + 1]);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) big = largest(big, __shfl_xor_sync(0xffffffffu, big, o), 0.f);
      const float s = fp8_scale(big);
      if (u0 + i * step >= units) continue;
      if (lane == 0) {
        p.scales[m[i] * p.row_pitch + kb[i] * p.block_pitch] = s;
        if (!(s >= 0.f)) report(p.status, JAB_ERR_NONFINITE);
      }
      const int64_t at = m[i] * p.K + kb[i] * 128 + lane * 8;
      if (live[i] && in_bounds(at + 7, p.M * p.K, p.status)) *reinterpret_cast<uint2*>(p.codes + at) = fp8_codes(v, s);
    }
  }
}

// 128 rows x 128 columns by a block of threads.
template <class T>
__global__ void __launch_bounds__(256) fp8_blocks_kernel(const __grid_constant__ QuantParams p) {
  __shared__ float top[8];
  stream_order();
  const int lane = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int64_t mb = blockIdx.x / p.blocks;
  const int kb = (int)(blockIdx.x - mb * p.blocks), k = kb * 128 + lane * 8;
  Raw8<T> raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t m = mb * 128 + i * 16 + row;
    raw[i] = {};
    if (m < p.M && k < p.K) raw[i].load(static_cast<const T*>(p.x) + m * p.ldx + k);
  }
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    raw[i].numbers(v);
#pragma unroll
    for (int j = 0; j < 8; j += 2) big = largest(big, v[j], v[j + 1]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) big = largest(big, __shfl_xor_sync(0xffffffffu, big, o), 0.f);
  if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = big;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) big = largest(big, top[w], 0.f);
  const float s = fp8_scale(big);
  if (threadIdx.x == 0) {
    p.scales[mb * p.row_pitch + kb * p.block_pitch] = s;
    if (!(s >= 0.f)) report(p.status, JAB_ERR_NONFINITE);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t m = mb * 128 + i * 16 + row;
    float v[8];
    raw[i].numbers(v);
    if (m < p.M && k < p.K && in_bounds(m * p.K + k + 7, p.M * p.K, p.status))
      *reinterpret_cast<uint2*>(p.codes + m * p.K + k) = fp8_codes(v, s);
  }
}

template <class T>
cudaError_t quantize_as(const QuantParams& p, int block_rows, int sms, cudaStream_t st) {
  if (block_rows == 1) {
    const int64_t units = p.M * p.blocks;
    return launch_after(fp8_rows_kernel<T>, (unsigned)std::min<int64_t>((units + 15) / 16, (int64_t)sms * 8), 256, 0, st, p);
  }
  const int64_t blocks = (p.M + 127) / 128 * p.blocks;
  return launch_after(fp8_blocks_kernel<T>, (unsigned)blocks, 256, 0, st, p);
}

}  // namespace

cudaError_t launch_fp8_quantize(const Fp8QuantArgs& a, int sms, cudaStream_t st) {
  QuantParams p{};
  p.x = a.x, p.ldx = a.ldx, p.M = a.M, p.K = a.K;
  p.blocks = (a.K + 127) / 128;
  p.codes = static_cast<uint8_t*>(a.codes), p.scales = a.scales;
  p.row_pitch = a.row_pitch, p.block_pitch = a.block_pitch;
  p.status = a.status;
  return a.type == JAB_FP16   ? quantize_as<half_t>(p, a.block_rows, sms, st)
         : a.type == JAB_BF16 ? quantize_as<bf16_t>(p, a.block_rows, sms, st)
                              : quantize_as<float>(p, a.block_rows, sms, st);
}

}  // namespace jab
