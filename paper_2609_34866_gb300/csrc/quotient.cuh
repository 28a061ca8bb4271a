// IEEE quotients of many numbers by one: what the quantisers of the serving operators divide by a row's scale.
#pragma once
#include "tc.cuh"

namespace jab {

// fl32(x / s) for two x, with r = fl32(1 / s): the quotient corrected twice by its exact remainder. The first leaves it
// within a unit in the last place, from where the second gives the IEEE quotient (Markstein, "Computation of elementary
// functions on the IBM RISC System/6000 processor", 1990), as long as nothing leaves the normal range: see `usual_scale`.
__device__ __forceinline__ float2 quotients(float2 x, float2 r, float2 minus_s) {
  float2 q = tc::mul2(x, r);
  q = tc::fma2(tc::fma2(q, minus_s, x), r, q);
  return tc::fma2(tc::fma2(q, minus_s, x), r, q);
}
// s within 2^-100 .. 2^100: |x / s| is at most the largest code and a rounding, and where it is so small that a
// remainder loses bits, the code is 0 whatever they are.
__device__ __forceinline__ bool usual_scale(float s) { return s >= 7.8886091e-31f && s <= 1.2676506e30f; }
constexpr float kToWhole = 12582912.f;  // 1.5 * 2^23: added to a number below 2^22, rounds it to a whole one, half to even

}  // namespace jab
