// e4m3 in blocks of 128 that share a scale: the quantiser (kd_quantize_e4m3_blocks).  The product: kd_product.hip.
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_blocks.hpp"

namespace kd {

// ------------------------------------------------------------------------------------------------
// quantiser:  m = max(largest |x| of the block, 448 2^-126), scale = m / 448, code = e4m3(448 x / m)
//
// Bound by memory: two bytes (four) read, one written per element and order.  A workgroup holds 128 x 128 elements in registers, four rows x eight
// columns a thread: rows, columns and the tile each have their largest magnitude from there, so that both orders come from one reading.
// Codes of the other order are turned through LDS, so that a wave writes whole lines.  4096 x 4096 bf16 by rows, both orders: 20 us (22 between the products of a training step), of 14 at the rate of a
// copy; 4096 x 12288: 51 (eight rows a thread and columns' codes stored as threads have them: 25 and 74, too few waves to have loads on their
// way while others compute).  By tiles: 16 (18) and 38.  By rows each element is divided twice, by its row's largest and by its column's.
// ------------------------------------------------------------------------------------------------
constexpr int kTileRows = 4, kTileThreads = 16 * 128 / kTileRows;
template <bool F32, bool TILE>
__global__ __launch_bounds__(kTileThreads) void quantize_blocks_kernel(const BlocksArgs a) {
  constexpr int R = kTileRows, WAVES = kTileThreads / 64, PITCH = 128 + 4;
  __shared__ uint32_t tops[WAVES][128];
  __shared__ Divisor divisors[128];
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * PITCH];
  const int tid = threadIdx.x, tc = tid & 15, tr = tid >> 4, wave = tid >> 6;
  const int64_t n_cb = (a.cols + 127) / 128, n_rb = (a.rows + 127) / 128;
  const int64_t rb = blockIdx.x, cb = blockIdx.y;
  const int64_t r0 = rb * 128 + tr * R, c0 = cb * 128 + tc * 8;
  const int64_t ldc = (a.cols + 15) / 16 * 16, ldt = (a.rows + 15) / 16 * 16;
  float x[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (r0 + i < a.rows) load_row8<F32>(x[i], (const char*)a.src + (r0 + i) * a.ld * (F32 ? 4 : 2), c0, a.cols);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
  }
  uint32_t rm[R], cm[8];            // largest magnitude of the thread's rows' and columns' blocks
#pragma unroll
  for (int i = 0; i < R; ++i) rm[i] = kLeastBlock;
#pragma unroll
  for (int j = 0; j < 8; ++j) cm[j] = kLeastBlock;
#pragma unroll
  for (int i = 0; i < R; ++i)
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
    for (int i = 1; i < R; ++i) m = max(m, rm[i]);
    m = row_max(m);
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if ((tid & 63) == 0) tops[0][wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = max(m, tops[0][w]);
    one = divisor_of(m);
    if (tid == 0) {
      if (a.scales) a.scales[rb * n_cb + cb] = scale_of(m);
      if (a.scales_t) a.scales_t[cb * n_rb + rb] = scale_of(m);
    }
  } else {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) cm[j] = max(cm[j], (uint32_t)__shfl_xor((int)cm[j], o, 64));
    if ((tid & 63) < 16)
#pragma unroll
      for (int j = 0; j < 8; ++j) tops[wave][tc * 8 + j] = cm[j];
#pragma unroll
    for (int i = 0; i < R; ++i) rm[i] = row_max(rm[i]);
    if (a.scales && tc < R && r0 + tc < a.rows) {
      uint32_t m = rm[0];
#pragma unroll
      for (int i = 1; i < R; ++i) m = tc == i ? rm[i] : m;
      a.scales[(r0 + tc) * n_cb + cb] = scale_of(m);
    }
    __syncthreads();
    if (tid < 128) {
      uint32_t m = tops[0][tid];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) m = max(m, tops[w][tid]);
      divisors[tid] = divisor_of(m);
      if (cb * 128 + tid < a.cols) a.scales_t[(cb * 128 + tid) * n_rb + rb] = scale_of(m);
    }
  }
  if (a.codes && c0 < ldc)
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const Divisor d = TILE ? one : divisor_of(rm[i]);
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = quotient<F32>(x[i][j], d);
      if (r0 + i < a.rows) *(uint2*)(a.codes + (r0 + i) * ldc + c0) = codes_of(q);
    }
  if (!a.codes_t) return;
  if (!TILE) __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const Divisor d = TILE ? one : divisors[tc * 8 + j];
    float q[R];
#pragma unroll
    for (int i = 0; i < R; ++i) q[i] = quotient<F32>(x[i][j], d);
#pragma unroll
    for (int i = 0; i < R; i += 4) *(uint32_t*)(turned + (tc * 8 + j) * PITCH + tr * R + i) = codes_of4(q[i], q[i + 1], q[i + 2], q[i + 3]);
  }
  __syncthreads();
  // 128 bytes of a column's codes by eight threads
  for (int i = tid; i < 128 * 8; i += kTileThreads) {
    const int64_t c = cb * 128 + i / 8, r = rb * 128 + i % 8 * 16;
    const uint32_t* const from = (const uint32_t*)(turned + i / 8 * PITCH + i % 8 * 16);
    if (c < a.cols && r < ldt) *(u32x4_t*)(a.codes_t + c * ldt + r) = u32x4_t{from[0], from[1], from[2], from[3]};
  }
}

// Blocks of rows in the source's order alone: 16 lanes a block, eight elements a lane; W blocks of a row a workgroup (a power of two), 16 / W rows.
// 4096 x 4096 bf16: 11.2 us, 4.5 TB/s (two blocks a lane 11.7, four 13.7; 777 x 1008 fp32 2.9, 3.4, 4.7).
template <bool F32>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const BlocksArgs a, int w_shift) {
  const int group = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const int64_t n_cb = (a.cols + 127) / 128, ldc = (a.cols + 15) / 16 * 16;
  const int64_t cb = ((int64_t)blockIdx.y << w_shift) + (group & ((1 << w_shift) - 1)), c0 = cb * 128 + lane * 8;
  const int64_t r = (int64_t)blockIdx.x * (16 >> w_shift) + (group >> w_shift);
  if (cb >= n_cb || r >= a.rows) return;
  float x[8];
  load_row8<F32>(x, (const char*)a.src + r * a.ld * (F32 ? 4 : 2), c0, a.cols);
  uint32_t m = kLeastBlock;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, magnitude(x[i]));
  m = row_max(m);
  const Divisor d = divisor_of(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = quotient<F32>(x[i], d);
  if (c0 < ldc) *(uint2*)(a.codes + r * ldc + c0) = codes_of(x);
  if (lane == 0) a.scales[r * n_cb + cb] = scale_of(m);
}

hipError_t launch_quantize_blocks(const BlocksArgs& a, hipStream_t st) {
  if (!a.tile && !a.codes_t) {
    int w_shift = 0;
    while (w_shift < 3 && ((int64_t)128 << w_shift) < a.cols) ++w_shift;      // (two rows a workgroup at least: 2^24 rows are 2^31 threads)
    const int rows = 16 >> w_shift;
    const dim3 grid((uint32_t)((a.rows + rows - 1) / rows), (uint32_t)((a.cols + (128 << w_shift) - 1) / (128 << w_shift)));
    hipLaunchKernelGGL(a.src_f32 ? quantize_rows_kernel<true> : quantize_rows_kernel<false>, grid, dim3(256), 0, st, a, w_shift);
    return hipGetLastError();
  }
  const dim3 grid((uint32_t)((a.rows + 127) / 128), (uint32_t)((a.cols + 127) / 128));
  auto kernel = a.src_f32 ? (a.tile ? quantize_blocks_kernel<true, true> : quantize_blocks_kernel<true, false>)
                          : (a.tile ? quantize_blocks_kernel<false, true> : quantize_blocks_kernel<false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace kd
