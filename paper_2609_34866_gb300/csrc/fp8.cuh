// e4m3 codes of a block of numbers and its scale.
#pragma once
#include <cuda_fp8.h>

#include "quotient.cuh"

namespace jab {

constexpr float kFp8Top = 448.f;

// Scale of a block whose largest magnitude is `big`; NaN where that is an infinity or a NaN. The quotient by a corrected
// reciprocal is the IEEE one where nothing leaves the normal range (see `quotients`).
__device__ __forceinline__ float fp8_scale(float big) {
  if (quot_window(big)) {
    constexpr float r = 1.f / kFp8Top;
    float q = __fmul_rn(big, r);
    q = __fmaf_rn(__fmaf_rn(q, -kFp8Top, big), r, q);
    return __fmaf_rn(__fmaf_rn(q, -kFp8Top, big), r, q);
  }
  return big < INFINITY ? __fdiv_rn(big, kFp8Top) : __uint_as_float(0x7fc00000u);
}

// Codes of 8 numbers; 0 where the scale is 0 or NaN. Quotients by corrected reciprocals are the IEEE ones while nothing that
// counts leaves the normal range: scales within 2^-60 .. 2^60 (a quotient below 2^-10 has code 0 whatever its bits are, but for its sign).
// They are taken by -s, and the codes' signs turned round: zeros keep theirs that way. A quotient of -0 is corrected by +0, which makes it +0;
// by -s the quotients of -0 and +0 are +0 and -0, and the correction is -0, which changes neither.
__device__ __forceinline__ uint2 fp8_codes(const float (&v)[8], float s) {
  float2 q[4];
  uint32_t signs = 0;
  if (quot_window(s)) {
    const float r1 = __frcp_rn(s);
    const float2 r = make_float2(-r1, -r1), ms = make_float2(s, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = quotients(make_float2(v[2 * j], v[2 * j + 1]), r, ms);
    signs = 0x80808080u;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      q[j].x = s > 0.f ? __fdiv_rn(v[2 * j], s) : 0.f;
      q[j].y = s > 0.f ? __fdiv_rn(v[2 * j + 1], s) : 0.f;
    }
  }
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = __nv_cvt_float2_to_fp8x2(q[j], __NV_SATFINITE, __NV_E4M3);
  return make_uint2((w[0] | w[1] << 16) ^ signs, (w[2] | w[3] << 16) ^ signs);
}

}  // namespace jab
