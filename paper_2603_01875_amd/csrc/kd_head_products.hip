// grad_W of the one-head losses: the kernels of kd_products.hpp with a scaled product.  dL/dz is kept without its factor
// loss_scale / (n tau): that is one number for all tokens, and rounded into every entry it would shift all of them the same way (a label's
// entry is near -1 for every token), so it multiplies the fp32 sums.  fp32 gradients contract several copies of the token axis (dz_sets).
#include "kd_products.hpp"

namespace kd {

// Bound by the matrix pipe (T = 4096, 3584 computed, H = 1024, V = 151936: 862 us in five chunks, 1.34 PFLOP/s), of one token tile
// (head_gw_few_kernel) by the stores of grad_W (T = 100 66 us, 5.4 TB/s).  What the contraction adds in front of the rounding is one
// multiplication a result.
template <int NB, bool HV, bool F32, bool ADD>
KD_STRIP_KERNEL void head_gw_kernel(const GradWArgs a) { grad_w<NB, HV, F32, ADD, true>(a); }
template <bool HV, bool ADD>
__global__ __launch_bounds__(256, 2) void head_gw_few_kernel(const GradWArgs a) { grad_w_few<HV, false, ADD, true>(a); }

// grad_h with few tokens: bound by the head, which streams through once, so by how much of it is in flight.  The accumulator of 64 NB
// tokens leaves room for two workgroups a CU, 32 KiB each on their way (and the stores of one under the products of the other).  T = 128,
// H = 1024, V = 151936: 79 us, 4.4 TB/s (three workgroups a CU: slower).
template <int NB, bool HV>
__global__ __launch_bounds__(256, 2) void head_gh_few_kernel(const GradHArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  GradHWork<8, HV, NB> work(a);
  GradHEpi<8, NB> epi(a);
  strip_loop<1, false, StripShape<8, NB>, HV ? A_ROWS_DZ : A_KMAJOR_DZ>(work, epi, smem);
}

hipError_t launch_head_grad_h(const Problem& p, int v0, int width, bool first, hipStream_t st, const GradHPairs* pairs) {
  if (p.T > kFewHeadTokens) return launch_grad_h(p, v0, width, first, st, pairs);
  const GradHArgs a = grad_h_args(p, v0, width, first, pairs);
  const int tiles = a.n_ht * a.n_split * a.n_pairs, grid = tiles < kFewGradHGroups ? tiles : kFewGradHGroups;
#define KD_GHF(NB, HV) launch_big<head_gh_few_kernel<NB, HV>>(grid, 256, StripShape<8, NB>::SMEM_BYTES, st, &a)
  return p.T <= 64 ? (p.w_hv_inplace ? KD_GHF(1, true) : KD_GHF(1, false)) : (p.w_hv_inplace ? KD_GHF(2, true) : KD_GHF(2, false));
#undef KD_GHF
}

hipError_t launch_grad_W_scaled(const Problem& p, int v0, int width, hipStream_t st) {
  const int nb = grad_W_tile(p.H_s, width, p.n_cu) / 64;
  GradWArgs a = grad_w_args(p, v0, width, nb);
  const bool add = p.accumulate_grad_W != 0;
  if (p.n_tt == 1 && a.sets == 1) {
    grad_w_few_args(p, width, a);
#define KD_GF(HV, ADD) launch_big<head_gw_few_kernel<HV, ADD>>(a.n_vt * a.n_ht, 256, GradWFew::SMEM_BYTES, st, &a)
    return p.w_hv ? (add ? KD_GF(true, true) : KD_GF(true, false)) : (add ? KD_GF(false, true) : KD_GF(false, false));
#undef KD_GF
  }
  const int tiles = a.n_vt * a.n_ht, grid = tiles < p.n_cu ? tiles : p.n_cu;
#define KD_GW3(N, HV, F32) (add ? launch_big<head_gw_kernel<N, HV, F32, true>>(grid, 256, StripShape<16, N>::SMEM_BYTES, st, &a) \
                                : launch_big<head_gw_kernel<N, HV, F32, false>>(grid, 256, StripShape<16, N>::SMEM_BYTES, st, &a))
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

}  // namespace kd
