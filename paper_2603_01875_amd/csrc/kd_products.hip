// The backward products' kernels for the two-model losses (kd_products.hpp), what finishes grad_h_s, and the launchers.
#include "kd_products.hpp"

namespace kd {

// ------------------------------------------------------------------------------------------
// before and behind them
// ------------------------------------------------------------------------------------------

// grad_h_s row t = sum over split-K parts of the fp32 partial sums of its compacted row (zero for a
// masked token), times *scale if there is one, converted to the output dtype.
__global__ void gradh_finish_kernel(const float* parts, int n_parts, int T, int H, const int* inv,
                                    const float* scale, int out_f32, void* out) {
  const int64_t i = (flat_group() * blockDim.x + threadIdx.x) * 4;
  const int64_t n = (int64_t)T * H;
  if (i >= n) return;
  const int t = (int)(i / H), h = (int)(i % H);
  const int j = inv[t];
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (j >= 0) {
    const float* src = parts + (int64_t)j * H + h;
    v = *(const f32x4*)src;
#pragma unroll 8
    for (int p = 1; p < n_parts; ++p) v += *(const f32x4*)(src + (int64_t)p * n);
    if (scale) v *= *scale;
  }
  if (out_f32) {
    *(f32x4*)((float*)out + i) = v;
  } else {
    *(bf16x4*)((bf16_t*)out + i) = to_bf16(v);
  }
}

// ------------------------------------------------------------------------------------------
// launchers
// ------------------------------------------------------------------------------------------
hipError_t launch_grad_W(const Problem& p, int v0, int width, hipStream_t st) {
  const int nb = grad_W_tile(p.H_s, width, p.n_cu) / 64;
  GradWArgs a = grad_w_args(p, v0, width, nb);
  if (p.n_tt == 1) {
    grad_w_few_args(p, width, a);
#define KD_GF(HV, F32, ADD) launch_big<grad_w_few_kernel<HV, F32, ADD>>(a.n_vt * a.n_ht, 256, GradWFew::SMEM_BYTES, st, &a)
    if (p.accumulate_grad_W)
      return p.w_hv ? (p.grad_f32 ? KD_GF(true, true, true) : KD_GF(true, false, true))
                    : (p.grad_f32 ? KD_GF(false, true, true) : KD_GF(false, false, true));
    return p.w_hv ? (p.grad_f32 ? KD_GF(true, true, false) : KD_GF(true, false, false))
                  : (p.grad_f32 ? KD_GF(false, true, false) : KD_GF(false, false, false));
#undef KD_GF
  }
  const int tiles = a.n_vt * a.n_ht, grid = tiles < p.n_cu ? tiles : p.n_cu;
#define KD_GW3(N, HV, F32) (p.accumulate_grad_W ? launch_big<grad_w_kernel<N, HV, F32, true>>(grid, 256, StripShape<16, N>::SMEM_BYTES, st, &a) \
                                               : launch_big<grad_w_kernel<N, HV, F32, false>>(grid, 256, StripShape<16, N>::SMEM_BYTES, st, &a))
#define KD_GW(N) (p.w_hv ? (p.grad_f32 ? KD_GW3(N, true, true) : KD_GW3(N, true, false)) \
                         : (p.grad_f32 ? KD_GW3(N, false, true) : KD_GW3(N, false, false)))
  switch (nb) {
    case 2: return KD_GW(2);
    case 3: return KD_GW(3);
    default: return KD_GW(4);
  }
#undef KD_GW3
#undef KD_GW
}

hipError_t launch_grad_h(const Problem& p, int v0, int width, bool first, hipStream_t st, const GradHPairs* pairs) {
  const int mb = p.gh_rows / 16;
  const GradHArgs a = grad_h_args(p, v0, width, first, pairs);
  const int tiles = a.n_ht * p.n_tt * a.n_split * a.n_pairs, grid = tiles < p.n_cu ? tiles : p.n_cu;   // worst case: no token masked
#define KD_GH(N) (p.w_hv_inplace ? launch_big<grad_h_kernel<N, true>>(grid, 256, StripShape<N, 4>::SMEM_BYTES, st, &a) \
                                 : launch_big<grad_h_kernel<N, false>>(grid, 256, StripShape<N, 4>::SMEM_BYTES, st, &a))
  switch (mb) {
    case 4: return KD_GH(4);
    case 8: return KD_GH(8);
    case 12: return KD_GH(12);
    default: return KD_GH(16);
  }
#undef KD_GH
}

hipError_t launch_gradh_finish(const Problem& p, hipStream_t st) {
  const int64_t n = (int64_t)p.T * p.H_s;
  const FlatGrid g = flat_grid(((n + 3) / 4 + 255) / 256);
  hipLaunchKernelGGL(gradh_finish_kernel, dim3(g.x, g.y), dim3(256), 0, st, p.gh32,
                     p.n_ksplit_h * (p.gh_pairs ? p.gh_pairs : 1), p.T, p.H_s, p.inv, p.out_scale, p.grad_f32, p.grad_h_s);
  return hipGetLastError();
}

}  // namespace kd
