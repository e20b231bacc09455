// Maxima and codes of runs of eight values at a factor that is theirs: the linear layer's rows, the 8-bit cache's tokens.
#pragma once
#include "q8_quant.h"
#include "q8_value.h"
#pragma clang fp contract(off)

namespace q8 {

// The codes of eight values of a row at its factor q = max * fl(1/127), packed: quant1 of each, 0 for what is no number.
// Where 1 / q is a normal number and every value is finite, |r / q| < 127.1 and r * fl(1/q) lies within 6.1e-5 of it
// (quant_near): Round agrees unless a value is that near to a tie, and only then the eight are divided.  Adding
// 1.5 * 2^23 rounds half to even and leaves the code in the low byte.
__device__ __forceinline__ uint2 row_codes(const float (&r)[8], float q, float inv_q, bool finite) {
  constexpr float kRound = 12582912.0f;
  unsigned u[8];
  float far = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = __fmul_rn(r[e], inv_q), s = __fadd_rn(t, kRound);
    u[e] = __float_as_uint(s);
    far = fmaxf(far, fabsf(__fsub_rn(t, __fsub_rn(s, kRound))));
  }
  if (!finite || far > 0.49993f || q < 1.17549435e-38f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = r[e] == r[e] ? (unsigned)quant1(r[e], q, -128.0f, 127.0f) : 0u;
  }
  const unsigned lo0 = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi0 = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
  const unsigned lo1 = __builtin_amdgcn_perm(u[5], u[4], 0x0c0c0400u), hi1 = __builtin_amdgcn_perm(u[7], u[6], 0x04000c0cu);
  return uint2{lo0 | hi0, lo1 | hi1};
}

// The largest of eight magnitudes and m as bit patterns, whose order is that of the numbers: at least kNotFinite where one
// is infinite or no number, and then the lane takes its maximum again, of the finite ones (row_max8).
constexpr unsigned kNotFinite = 0x7f800000u;
__device__ __forceinline__ unsigned row_bits8(const float (&r)[8], unsigned m) {
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(r[e]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ float row_max8(const float (&r)[8], float m) {
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(r[e]));
  return m;
}

}  // namespace q8
