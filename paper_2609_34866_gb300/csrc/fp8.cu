// Rows in 8-bit floating point (e4m3) with a scale for every block of 1 or 128 rows x 128 columns:
//
//   s = fl32(max|x| / 448),  code = e4m3(fl32(x / s))
//
// One pass: a block's elements stay in registers between the maximum and the codes. Bound: bytes (a scale for every row's 128: 8192 x
// 4096 of bf16 in 21 us, 4.8 TB/s).
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
  // fp8_rows_kernel
  int rows;          // of a block of threads at a time
  FastDiv by_blocks;
};

// Largest magnitude of what the thread's groups of eight hold; an infinity or a NaN counts as itself.
template <class T, int N>
__device__ __forceinline__ float largest_of(const Raw8<T> (&raw)[N]) {
  if constexpr (sizeof(T) == 2) {  // (magnitudes of 16-bit numbers are in the order of their bits)
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      top = max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(top, raw[i].w[0].x), raw[i].w[0].y), raw[i].w[0].z), raw[i].w[0].w);
    top = max(top & 0xffffu, top >> 16);
    return std::is_same<T, half_t>::value ? __half2float(__ushort_as_half((unsigned short)top)) : __uint_as_float(top << 16);
  } else {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v[8];
      raw[i].numbers(v);
#pragma unroll
      for (int j = 0; j < 8; j += 2) big = largest(big, v[j], v[j + 1]);
    }
    return big;
  }
}

// Eight lanes have a row's block, a lane 16 elements of it (with eight a lane the places, the scale and its reciprocal take
// two thirds of the instructions: 8192 x 4096 of bf16 in 29 us, here 21); several blocks of theirs are under way together. A block of threads
// goes over some rows at a time, so that the place of a unit takes one small division.
template <class T>
__global__ void __launch_bounds__(256) fp8_rows_kernel(const __grid_constant__ QuantParams p) {
  constexpr int AHEAD = sizeof(T) == 2 ? 2 : 1, UNITS = 32;
  stream_order();
  const int lane = threadIdx.x & 7, group = threadIdx.x >> 3;
  for (int64_t m0 = (int64_t)blockIdx.x * p.rows; m0 < p.M; m0 += (int64_t)gridDim.x * p.rows) {
    const int units = (int)min((int64_t)p.rows, p.M - m0) * p.blocks;
    for (int u0 = 0; u0 < units; u0 += UNITS * AHEAD) {  // (whole warps go round together)
      Raw8<T> raw[AHEAD][2];
      int m[AHEAD], kb[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int u = u0 + i * UNITS + group;
        p.by_blocks.divmod(u, m[i], kb[i]);
        raw[i][0] = raw[i][1] = {};
        const int k = kb[i] * 128 + lane * 16;
        if (u < units && k < p.K) {
          const T* x = static_cast<const T*>(p.x) + (m0 + m[i]) * p.ldx + k;
          raw[i][0].load(x), raw[i][1].load(x + 8);
        }
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        float big = largest_of(raw[i]);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) big = largest(big, __shfl_xor_sync(0xffffffffu, big, o), 0.f);
        const float s = fp8_scale(big);
        if (u0 + i * UNITS + group >= units) continue;
        if (lane == 0) {
          p.scales[(m0 + m[i]) * p.row_pitch + kb[i] * p.block_pitch] = s;
          if (!(s >= 0.f)) report(p.status, JAB_ERR_NONFINITE);
        }
        const int k = kb[i] * 128 + lane * 16;
        const int64_t at = (m0 + m[i]) * p.K + k;
        if (k >= p.K || !in_bounds(at + 15, p.M * p.K, p.status)) continue;
        float v[8], w[8];
        raw[i][0].numbers(v), raw[i][1].numbers(w);
        const uint2 c = fp8_codes(v, s), d = fp8_codes(w, s);
        *reinterpret_cast<uint4*>(p.codes + at) = make_uint4(c.x, c.y, d.x, d.y);
      }
    }
  }
}

// 128 rows x 128 columns by a block of threads, in registers. Bound: bytes in flight; 6144 x 4096 of bf16 take 16.2 us with five blocks an
// SM (48 registers and 44 bytes in local memory), 20.3 with three (74) and 31 with seven (more in local memory); 16384 x 8192 67 us, 6.0
// TB/s. fp32, three blocks an SM (80 registers, 12 bytes in local memory): 6144 x 4096 in 23 us, 5.4 TB/s.
template <class T>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 5 : 3) fp8_blocks_kernel(const __grid_constant__ QuantParams p) {
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
  float big = largest_of(raw);
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
cudaError_t quantize_as(QuantParams p, int block_rows, int sms, cudaStream_t st) {
  if (block_rows == 1) {
    // two turns of a block's threads where that leaves all SMs two blocks, else one
    const int64_t units = p.M * p.blocks;
    p.rows = std::max(1, (units >= (int64_t)sms * 128 ? 64 : 32) / p.blocks);
    p.by_blocks = FastDiv(p.blocks);
    return launch_after(fp8_rows_kernel<T>, (unsigned)std::min<int64_t>((p.M + p.rows - 1) / p.rows, (int64_t)sms * 8), 256, 0, st, p);
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
