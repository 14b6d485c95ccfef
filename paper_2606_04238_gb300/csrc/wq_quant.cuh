// wq_quant.cuh -- the division of the min-max quantizers.
#pragma once

namespace wq {

// rint(v / sf) as the IEEE division gives it.  p = v * rcp is within |p| 2^-22
// of the quotient (two roundings), as is the division's own result, so both
// round to the same integer unless p is that near to a half.
__device__ __forceinline__ float rint_div(float v, float sf, float rcp) {
  const float p = __fmul_rn(v, rcp), r = rintf(p);
  if (fabsf(p - r) < 0.5f - fabsf(p) * 0x1p-21f) return r;
  return rintf(__fdiv_rn(v, sf));  // also nan and infinite quotients
}

}  // namespace wq
