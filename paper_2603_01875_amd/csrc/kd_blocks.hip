// e4m3 in blocks of 128 that share a scale: the quantiser (kd_quantize_e4m3_blocks).  The product: kd_product.hip.
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_blocks.hpp"

namespace kd {

// ------------------------------------------------------------------------------------------------
// quantiser:  m = max(largest |x| of the block, 448 2^-126), scale = m / 448, code = e4m3(448 x / m)
//
// A workgroup holds 128 x 128 elements in registers, 8 rows x 8 columns a thread: rows, columns and the tile each have their
// largest magnitude from there, so that both orders come from one reading.  448 = 7/16 2^10: 7 x / 16 does not overflow, and is exact for
// bf16, so that the quotient is rounded once and one that lies between two codes stays there (448 x / m for m = 1.5 .. is a multiple of 1/2 often).
// ------------------------------------------------------------------------------------------------
template <bool F32, bool TILE>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const BlocksArgs a) {
  __shared__ uint32_t lds[4][128];
  const int tid = threadIdx.x, tc = tid & 15, tr = tid >> 4, wave = tid >> 6;
  const int64_t n_cb = (a.cols + 127) / 128, n_rb = (a.rows + 127) / 128;
  const int64_t rb = blockIdx.x, cb = blockIdx.y;
  const int64_t r0 = rb * 128 + tr * 8, c0 = cb * 128 + tc * 8;
  const int64_t ldc = (a.cols + 15) / 16 * 16, ldt = (a.rows + 15) / 16 * 16;
  float x[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (r0 + i < a.rows) load_row8<F32>(x[i], (const char*)a.src + (r0 + i) * a.ld * (F32 ? 4 : 2), c0, a.cols);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
  }
  uint32_t rm[8], cm[8];            // largest magnitude of the thread's rows' and columns' blocks
#pragma unroll
  for (int i = 0; i < 8; ++i) rm[i] = cm[i] = kLeastBlock;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t u = magnitude(x[i][j]);
      rm[i] = max(rm[i], u);
      if (!TILE) cm[j] = max(cm[j], u);
    }
  Divisor one;
  if (TILE) {
    uint32_t m = rm[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max(m, rm[i]);
    m = row_max(m);
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    lds[wave][0] = m;
    __syncthreads();
    m = max(max(lds[0][0], lds[1][0]), max(lds[2][0], lds[3][0]));
    one = divisor_of(m);
    if (tid == 0) {
      if (a.scales) a.scales[rb * n_cb + cb] = scale_of(m);
      if (a.scales_t) a.scales_t[cb * n_rb + rb] = scale_of(m);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) rm[i] = row_max(rm[i]);
    if (a.scales && tc < 8 && r0 + tc < a.rows) {
      uint32_t m = rm[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) m = tc == i ? rm[i] : m;
      a.scales[(r0 + tc) * n_cb + cb] = scale_of(m);
    }
    if (a.codes_t) {
#pragma unroll
      for (int o = 16; o < 64; o <<= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j) cm[j] = max(cm[j], (uint32_t)__shfl_xor((int)cm[j], o, 64));
      if ((tid & 63) < 16)
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[wave][tc * 8 + j] = cm[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j)
        cm[j] = max(max(lds[0][tc * 8 + j], lds[1][tc * 8 + j]), max(lds[2][tc * 8 + j], lds[3][tc * 8 + j]));
      if (tr < 8 && c0 + tr < a.cols) {
        uint32_t m = cm[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = tr == j ? cm[j] : m;
        a.scales_t[(c0 + tr) * n_rb + rb] = scale_of(m);
      }
    }
  }
  if (a.codes && c0 < ldc)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Divisor d = TILE ? one : divisor_of(rm[i]);
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = quotient(x[i][j], d);
      if (r0 + i < a.rows) *(uint2*)(a.codes + (r0 + i) * ldc + c0) = codes_of(q);
    }
  if (a.codes_t && r0 < ldt)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Divisor d = TILE ? one : divisor_of(cm[j]);
      float q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = quotient(x[i][j], d);
      if (c0 + j < a.cols) *(uint2*)(a.codes_t + (c0 + j) * ldt + r0) = codes_of(q);
    }
}

hipError_t launch_quantize_blocks(const BlocksArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)((a.rows + 127) / 128), (uint32_t)((a.cols + 127) / 128));
  auto kernel = a.src_f32 ? (a.tile ? quantize_blocks_kernel<true, true> : quantize_blocks_kernel<true, false>)
                          : (a.tile ? quantize_blocks_kernel<false, true> : quantize_blocks_kernel<false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace kd
