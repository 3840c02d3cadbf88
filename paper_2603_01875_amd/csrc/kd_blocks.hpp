// Pieces of the e4m3 quantiser: largest magnitude, scale and codes of a block of 128.
#pragma once
#include "kd_unaligned.hpp"

namespace kd {

constexpr float kLeastBlock = 448.f * 0x1p-126f;

__device__ __forceinline__ float block_max(float a, float b) { return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b); }
__device__ __forceinline__ float scale_of(float m) { return m < __builtin_inff() ? m / 448.f : __builtin_nanf(""); }

// codes of 8 values of blocks whose largest magnitudes are m[i] (a block with an infinity or a NaN: anything, its scale is NaN; 7 m / 16 is
// rounded for fp32, so that 448 may come out one step larger)
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], const float (&m)[8]) {
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    q[i] = fminf(fmaxf(x[i] * 0.4375f / m[i] * 1024.f, -448.f), 448.f);
  }
  uint2 w;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
  w.x = (uint32_t)lo;
  w.y = (uint32_t)hi;
  return w;
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
