// Norm of many arrays taken together, and clipping (kd_grad_norm, kd_grad_clip).
//
// norm = sqrt(sum x^2) or max |x|;  out = x min(1, max_norm / norm).  Two readings and one writing of all elements, nothing else: bound by
// memory: 1.7 billion bf16 in 311 arrays, views of one at any offset, 591 to 613 us (5.6 to 5.8 TB/s), then 1545 (4.4), of 1420 for one reading and one writing at the
// rate of a copy; arrays of one size with an allocation each 565 to 572 and 1309 to 1316.  The arrays come as a table in the kernel's arguments (no copy to the device, so a call can be captured), cut into pieces
// of equal length that workgroups take in turn; squares are summed in 64 bits, where none overflows and the order of 10^9 terms does not matter
// much, in a fixed order all the same: a thread's, then a workgroup's, then all workgroups' by one more.
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_unaligned.hpp"

namespace kd {

// Array of a piece: the last whose first piece is not behind it (empty arrays have the next one's first piece).
template <class Table>
__device__ __forceinline__ int array_of(const Table& t, uint32_t piece) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

struct Piece {
  global_t in;
  int f32, array;
  int64_t begin;
  int n, head;      // elements; those in front of the first 16-byte boundary
};
__device__ __forceinline__ Piece piece_of(const GradTable& t, uint32_t piece) {
  Piece p;
  p.array = array_of(t, piece);
  const uint64_t a = t.in[p.array];
  p.f32 = (int)(a & 1);
  const int es = p.f32 ? 4 : 2;
  p.begin = (int64_t)(piece - t.first[p.array]) * kPieceElements;
  const int64_t left = (int64_t)t.count[p.array] - p.begin;
  p.n = (int)(left < (int64_t)kPieceElements ? left : (int64_t)kPieceElements);
  p.in = (global_t)(a & ~1ull) + p.begin * es;
  const int head = (int)((16 - ((uint64_t)p.in & 15)) & 15) / es;
  p.head = head < p.n ? head : p.n;
  return p;
}

__device__ __forceinline__ float element(global_t p, int f32, int64_t i) {
  return f32 ? ((KD_GLOBAL const float*)p)[i] : bf16_float(((KD_GLOBAL const uint16_t*)p)[i]);
}

constexpr int kNormThreads = 256;
constexpr int kNormUnroll = 8;          // 16-byte loads in flight per thread (four: the same within 2 %)

template <bool MAX>
__device__ __forceinline__ void put(double& s, float x) {
  if (MAX) {
    const double a = fabs((double)x);
    s = a > s || a != a ? a : s;        // (a NaN stays: nothing is larger)
  } else {
    s = fma((double)x, (double)x, s);
  }
}
template <bool MAX>
__device__ __forceinline__ double join(double a, double b) {
  return MAX ? (a != a || a >= b ? a : b) : a + b;
}

template <bool MAX, bool F32>
__device__ __forceinline__ void add_vector(double& s, const u32x4_t v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F32) put<MAX>(s, __uint_as_float(v[i]));
    else {
      put<MAX>(s, __uint_as_float(v[i] << 16));
      put<MAX>(s, __uint_as_float(v[i] & 0xffff0000u));
    }
  }
}
template <bool MAX, bool F32>
__device__ __forceinline__ void add_piece(double& s, const Piece& p) {
  constexpr int VE = F32 ? 4 : 8;
  if ((int)threadIdx.x < p.head) put<MAX>(s, element(p.in, F32, threadIdx.x));
  KD_GLOBAL const u32x4_t* const v = (KD_GLOBAL const u32x4_t*)(p.in + p.head * (F32 ? 4 : 2));
  const int nv = (p.n - p.head) / VE, rest = p.head + nv * VE;
  int i = threadIdx.x;
  for (; i + (kNormUnroll - 1) * kNormThreads < nv; i += kNormUnroll * kNormThreads) {
    u32x4_t x[kNormUnroll];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) x[j] = v[i + j * kNormThreads];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) add_vector<MAX, F32>(s, x[j]);
  }
  if (i < nv) {                         // (the last ones too are on their way together)
    u32x4_t x[kNormUnroll];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) x[j] = i + j * kNormThreads < nv ? v[i + j * kNormThreads] : u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) add_vector<MAX, F32>(s, x[j]);
  }
  if (rest + (int)threadIdx.x < p.n) put<MAX>(s, element(p.in, F32, rest + threadIdx.x));
}

template <bool MAX, int NT>
__device__ __forceinline__ double group_join(double s, double* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) s = join<MAX>(s, __shfl_xor(s, o, 64));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = lds[0];
  for (int w = 1; w < NT / 64; ++w) s = join<MAX>(s, lds[w]);
  return s;
}

template <bool MAX>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const GradTable t, double* partials) {
  __shared__ double lds[kNormThreads / 64];
  double s = 0;
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Piece p = piece_of(t, c);
    if (p.f32) add_piece<MAX, true>(s, p);
    else add_piece<MAX, false>(s, p);
  }
  s = group_join<MAX, kNormThreads>(s, lds);
  if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

template <bool MAX>
__global__ __launch_bounds__(1024) void grad_total_kernel(const double* partials, int64_t n, double* total) {
  __shared__ double lds[16];
  double s = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s = join<MAX>(s, partials[i]);
  s = group_join<MAX, 1024>(s, lds);
  if (threadIdx.x == 0) *total = s;
}

// Results pass the caches by: no part of this call reads them again, and what is still to be read stays (16 bytes at a time, in and out: 100 million elements
// of bf16 79 to 61 us, 3.2 million of fp32 8.7 to 7.6; no difference at 1.7 billion).
template <class V>
__device__ __forceinline__ void stream_out(global_t p, const V& v) {
  typedef V Any __attribute__((aligned(2)));
  __builtin_nontemporal_store(v, (KD_GLOBAL Any*)p);
}

// The factor as f 2^e, f from 1/2 to 1: below 2^-126 it would lose bits in 32 (gradients of 1e10 and a limit of 1e-30), and x f 2^e may be a normal number all the same.
struct Factor { float f; int e; };
__device__ __forceinline__ float scaled(float x, const Factor& f) { return ldexpf(x * f.f, f.e); }

template <bool IN32, bool OUT32>
__device__ __forceinline__ void scale_piece(const Piece& p, global_t out, const Factor& f) {
  constexpr int VE = IN32 ? 4 : 8;
  auto one = [&](int i) {
    const float y = scaled(element(p.in, IN32, i), f);
    if (OUT32) ((KD_GLOBAL float*)out)[i] = y;
    else ((KD_GLOBAL uint16_t*)out)[i] = bf16_bits(y);
  };
  if ((int)threadIdx.x < p.head) one(threadIdx.x);
  KD_GLOBAL const u32x4_t* const v = (KD_GLOBAL const u32x4_t*)(p.in + p.head * (IN32 ? 4 : 2));
  const global_t o = out + p.head * (OUT32 ? 4 : 2);
  const int nv = (p.n - p.head) / VE, rest = p.head + nv * VE;
  auto many = [&](int i, const u32x4_t x) {
    float y[VE];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (IN32) y[k] = scaled(__uint_as_float(x[k]), f);
      else {
        y[(2 * k) % VE] = scaled(__uint_as_float(x[k] << 16), f);
        y[(2 * k + 1) % VE] = scaled(__uint_as_float(x[k] & 0xffff0000u), f);
      }
    }
    if (OUT32) {
#pragma unroll
      for (int k = 0; k < VE; k += 4)
        stream_out(o + ((int64_t)i * VE + k) * 4, u32x4_t{__float_as_uint(y[k]), __float_as_uint(y[k + 1]), __float_as_uint(y[k + 2]), __float_as_uint(y[k + 3])});
    } else if (VE == 8) {
      stream_out(o + (int64_t)i * 16, u32x4_t{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4 % VE], y[5 % VE]), bf16_pair(y[6 % VE], y[7 % VE])});
    } else {
      stream_out(o + (int64_t)i * 8, u32x2_t{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])});
    }
  };
  int i = threadIdx.x;
  for (; i + (kNormUnroll - 1) * kNormThreads < nv; i += kNormUnroll * kNormThreads) {
    u32x4_t x[kNormUnroll];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) x[j] = v[i + j * kNormThreads];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) many(i + j * kNormThreads, x[j]);
  }
  if (i < nv) {
    u32x4_t x[kNormUnroll];
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j) x[j] = i + j * kNormThreads < nv ? v[i + j * kNormThreads] : u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kNormUnroll; ++j)
      if (i + j * kNormThreads < nv) many(i + j * kNormThreads, x[j]);
  }
  if (rest + (int)threadIdx.x < p.n) one(rest + threadIdx.x);
}

// The pieces are taken from the last to the first: the norm's pass has just read them, and what the last-level cache still holds of
// them (256 MB) does not come from memory again.
__global__ __launch_bounds__(kNormThreads) void grad_clip_kernel(const ClipTable c, int max_kind, const double* total, double max_norm,
                                                                 float* norm_out) {
  const double sum = *total, norm = max_kind ? sum : sqrt(sum);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool clips = norm > max_norm && norm < __builtin_inf();
  Factor f{1.f, 0};
  if (clips) f.f = (float)frexp(max_norm / norm, &f.e);
  for (uint32_t i = blockIdx.x; i < c.t.chunks; i += gridDim.x) {
    const Piece p = piece_of(c.t, c.t.chunks - 1 - i);
    const uint64_t o = c.out[p.array];
    if (!clips && o == c.t.in[p.array]) continue;
    const bool out32 = o & 1;
    const global_t out = (global_t)(o & ~1ull) + p.begin * (out32 ? 4 : 2);
    if (p.f32) out32 ? scale_piece<true, true>(p, out, f) : scale_piece<true, false>(p, out, f);
    else out32 ? scale_piece<false, true>(p, out, f) : scale_piece<false, false>(p, out, f);
  }
}

hipError_t launch_grad_norm(const GradTable& t, int max_kind, double* partials, int groups, hipStream_t st) {
  if (max_kind) hipLaunchKernelGGL(grad_norm_kernel<true>, dim3(groups), dim3(kNormThreads), 0, st, t, partials);
  else hipLaunchKernelGGL(grad_norm_kernel<false>, dim3(groups), dim3(kNormThreads), 0, st, t, partials);
  return hipGetLastError();
}

hipError_t launch_grad_total(const double* partials, int64_t n, int max_kind, double* total, hipStream_t st) {
  if (max_kind) hipLaunchKernelGGL(grad_total_kernel<true>, dim3(1), dim3(1024), 0, st, partials, n, total);
  else hipLaunchKernelGGL(grad_total_kernel<false>, dim3(1), dim3(1024), 0, st, partials, n, total);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const ClipTable& t, int max_kind, const double* total, double max_norm, float* norm, hipStream_t st) {
  const uint32_t groups = t.t.chunks < (uint32_t)kNormGroups ? (t.t.chunks ? t.t.chunks : 1) : kNormGroups;
  hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kNormThreads), 0, st, t, max_kind, total, max_norm, norm);
  return hipGetLastError();
}

}  // namespace kd
