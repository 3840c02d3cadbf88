// Device-side pieces that the kernels of several source files share.
#pragma once
#include "kd_launch.h"
#include "kd_mfma.hpp"
#include "kd_strip.hpp"

#include <atomic>

namespace kd {

// Number of this workgroup in a grid of flat_grid (kd_launch.h).
__device__ __forceinline__ int64_t flat_group() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Workgroups are dealt to the 8 XCDs round-robin by workgroup id.  Renumber so
// that consecutive logical ids sit on one XCD (and share its L2).
__device__ __forceinline__ int xcd_logical_id(int b, int G) {
  const int x = b % 8, q = G / 8, r = G % 8;       // XCD x holds q (+1 if x < r) of the G workgroups
  return x * q + (x < r ? x : r) + b / 8;
}

// Device-side plan, written by make_rowmap once the mask has been counted (the host never
// learns how many tokens are valid, so everything that depends on it is decided on the device).
// META_N_SPLIT: vocabulary ranges per token tile in the statistics passes; META_G_SPLIT, META_G_SPLIT_LAST: in the
// gradient kernel, for a full chunk and for the last one (strip loop).
enum { META_N_VALID = 0, META_N_TT = 1, META_N_SPLIT = 2, META_T_EFF = 3, META_G_SPLIT = 4, META_G_SPLIT_LAST = 5,
       META_WORDS = 6 };
__device__ __forceinline__ int meta_get(const int* meta, int i) { return uniform(meta[i]); }

// Index q over n_tt token tiles x n_split vocabulary splits: the token tiles in groups of at most four (of sizes
// that differ by one where four does not divide them), a group's splits one after the other.  32 consecutive
// indices, the workgroups of an XCD, then cover 4 x 8: the shape that streams the fewest rows into one L2.
__device__ __forceinline__ void group_decode(int q, int n_tt, int n_split, int& tt, int& split) {
  const int ng = (n_tt + 3) / 4, small = n_tt / ng, n_big = n_tt - small * ng;
  const int big_units = n_big * (small + 1) * n_split;
  int g = small, base = 0;
  if (q < big_units) g = small + 1;
  else { q -= big_units; base = n_big * (small + 1); }
  const int grp = q / (g * n_split), w = q - grp * g * n_split;
  tt = base + grp * g + w % g;
  split = w / g;
}

// dL/dz_s of a vocabulary chunk is kept in the order in which a lane of a finished logit tile holds it and in which the
// products read it: [64-token panel][32-column sub-step][16-token block][lane][8], lane 16 g + t with the columns
// 4 g .. + 3 and 16 + 4 g .. + 3 of token t of the block.  As the token operand of grad_h_s a lane's 16 bytes are its share of an
// MFMA (eight of the 32 columns contracted); as the column operand of grad_W_s they go through the transposing LDS reads.
// The panels are V_c columns apart.  Element offset of the 16 bytes of (panel, column sub-step, block, lane):
__device__ __forceinline__ int64_t dz_chunk(int ldz, int panel, int sub, int blk, int lane) {
  return (int64_t)panel * 64 * ldz + ((int64_t)(sub * 4 + blk) * 64 + lane) * 8;
}
// Column of row `row` (0 .. 15) of block i of an A_DZ tile (strip_loop).
__device__ __forceinline__ int dz_column(int i, int row) {
  return 32 * (i >> 1) + 16 * ((row >> 2) & 1) + 8 * (i & 1) + 4 * (row >> 3) + (row & 3);
}

// Merging the partial sums.  Every workgroup (one per token tile and vocabulary range) leaves its values as [range][value][T_pad], and
// with few tokens there are many ranges (256 at T <= 256; the eight-wave loop's four lanes of a token put theirs
// together first: a step of T = 200, H = 2048 / 512, V = 32000 148 -> 133 us, AKL at T = 150, H = 1024 / 512 347 -> 291).  A merge is bound by the latency of its loads:
// one thread walking all the parts of a token took 658 us at T = 256 and 47 us at T = 4096.  So a workgroup owns TX
// tokens and NT / TX threads share the parts of each: lanes run along the tokens (TX = 8: 32-byte runs, TX = 32:
// whole lines), the rest of the lanes and the waves along the parts; partial results meet by shuffles, then through
// LDS, in a fixed order.  Measured: combine_kernel 658 -> 23 us at T = 256, 47 -> 9 us at 128 parts, 6 us at 32 (T = 4096),
// one search merge of AKL 536 -> 15 us at T = 2048.
struct MergeSum {
  static __device__ __forceinline__ float op(float a, float b) { return a + b; }
};
struct MergeMax {
  static __device__ __forceinline__ float op(float a, float b) { return fmaxf(a, b); }
};
// v[i] of every thread -> the merged value of the thread's token, in every thread of that token
template <int TX, int NT, int NV, class Op>
__device__ __forceinline__ void merge_parts(float (&v)[NV], float* lds) {
  constexpr int NW = NT / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tx = lane % TX;
#pragma unroll
  for (int off = TX; off < 64; off <<= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = Op::op(v[i], __shfl_xor(v[i], off, 64));
  __syncthreads();                       // the values of an earlier merge have been read
  if (lane < TX)
#pragma unroll
    for (int i = 0; i < NV; ++i) lds[(wave * NV + i) * TX + tx] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float r = lds[i * TX + tx];
#pragma unroll
    for (int w = 1; w < NW; ++w) r = Op::op(r, lds[(w * NV + i) * TX + tx]);
    v[i] = r;
  }
}

// fp32 operands as bf16 parts laid side by side along K.  src_f32 == 1, the two-model losses: two parts, three products (see prepare);
// src_f32 == 2, the one-head losses: three parts, f = f0 + f1 + f2 to 24 bits, and the six products of them that are not below
// those bits, the head as [0 0 0 1 1 2], the hidden states as [0 1 2 0 1 0].
__device__ __forceinline__ int part_of_six(int place, bool head) { return (head ? 0x211000 : 0x010210) >> (4 * place) & 15; }
__device__ __forceinline__ bf16_t part_of(float f, int part) {
  const bf16_t hi = (bf16_t)f;
  if (part == 0) return hi;
  const float rest = f - (float)hi;
  const bf16_t mid = (bf16_t)rest;
  return part == 1 ? mid : (bf16_t)(rest - (float)mid);
}

#define KD_STRIP_KERNEL __global__ __launch_bounds__(StripCfg::NT, 1) __attribute__((amdgpu_waves_per_eu(1, 1)))

// Launch of a kernel that needs more dynamic LDS than the default limit.  The limit is a property of
// the kernel on a device: it is raised once per kernel and device (one flag word per instantiation,
// one bit per device), not on every launch: to `most_bytes` for a kernel whose launches take different amounts.
template <auto Kern>
static hipError_t launch_big(int grid, int threads, int smem_bytes, hipStream_t st, const void* args_ptr, int most_bytes = 0) {
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)Kern, hipFuncAttributeMaxDynamicSharedMemorySize, most_bytes ? most_bytes : smem_bytes);
    if (e != hipSuccess) return e;
    attr_done.fetch_or(bit, std::memory_order_release);
  }
  void* params[] = {const_cast<void*>(args_ptr)};
  return hipLaunchKernel((const void*)Kern, dim3(grid), dim3(threads), params, smem_bytes, st);
}

}  // namespace kd
