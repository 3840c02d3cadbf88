// Constants and small functions of every epilogue of a logit tile.
#pragma once
#include <hip/hip_runtime.h>

namespace kd {

constexpr float NEG_BIG = -1.0e30f;   // logit given to vocabulary rows beyond V: every exp of it is 0
// Running maxima start here, far below any real scaled logit and far above NEG_BIG * c (the host
// bounds tau so that c > 1e-9): a lane that has seen only masked rows keeps this maximum, so the
// exponent of a masked entry stays hugely negative instead of cancelling to a rounding residual.
constexpr float M_FLOOR = -1.0e20f;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float fexp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float flog2(float x) { return __builtin_amdgcn_logf(x); }

__device__ __forceinline__ float quad_max(float x) {          // over the lanes of a token, 16 and 32 apart
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

}  // namespace kd
