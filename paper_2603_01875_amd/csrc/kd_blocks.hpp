// Pieces of the e4m3 quantiser: largest magnitude, scale and codes of a block of 128.
#pragma once
#include "kd_unaligned.hpp"

namespace kd {

// Largest magnitude of a block, as bits: an infinity or a NaN is larger than every number.
constexpr uint32_t kLeastBlock = 0x04e00000u;        // 448 2^-126
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(uint32_t m) { return m < 0x7f800000u ? __uint_as_float(m) / 448.f : __builtin_nanf(""); }

// 448 x / m, rounded as 448 x and its quotient by m are:  m = 2^e f with 1 <= f < 2, a = (448 2^-e) x, q = a (1 / f), and then the remainder's share,
// (a - q f) (1 / f), added in one rounding, which gives the quotient that a division gives (448 x is exact for bf16; fp32: on all of the 5.4 10^8 pairs
// of significands whose quotient lies next to a border between codes).  A division for every element took
// three times as many instructions.
struct Divisor { float c, f, inv; };
__device__ __forceinline__ Divisor divisor_of(uint32_t m) {
  Divisor d;
  d.c = __uint_as_float(0x83600000u - (m & 0x7f800000u));      // 448 2^-e: normal, as e is -118 to 127
  d.f = __uint_as_float((m & 0x007fffffu) | 0x3f800000u);
  d.inv = 1.f / d.f;
  return d;
}
template <bool F32>
__device__ __forceinline__ float quotient(float x, const Divisor& d) {
  const float a = x * d.c, q = a * d.inv, y = fmaf(fmaf(-q, d.f, a), d.inv, q);
  return F32 ? __builtin_amdgcn_fmed3f(y, -448.f, 448.f) : y;      // (448 x rounded may be one step more than 448 m)
}
// codes of quotients (of a block with an infinity or a NaN: anything, its scale is NaN)
__device__ __forceinline__ uint32_t codes_of4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ uint2 codes_of(const float (&q)[8]) { return make_uint2(codes_of4(q[0], q[1], q[2], q[3]), codes_of4(q[4], q[5], q[6], q[7])); }
// The largest of 16 lanes (a row), in all of them.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, true));      // row_ror 1, 2, 4, 8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true));
}

template <bool F32>
__device__ __forceinline__ void load_row8(float (&x)[8], const void* row, int64_t c0, int64_t cols) {
  if (c0 + 8 <= cols) {
    if (F32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4_t v = load16((const float*)row + c0 + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = __uint_as_float(v[i]);
      }
    } else {
      const u32x4_t v = load16((const uint16_t*)row + c0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = c0 + i < cols ? (F32 ? ((const float*)row)[c0 + i] : bf16_float(((const uint16_t*)row)[c0 + i])) : 0.f;
  }
}

}  // namespace kd
