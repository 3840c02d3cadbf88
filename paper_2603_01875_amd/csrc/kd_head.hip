// The one-head losses: cross entropy with labels, and distillation from a teacher's top logits.  One call:
//   targets  : the caller's labels or top logits -> per token a sorted list of entries with their probabilities, and whether it counts
//   (row map and operand copies: operands_kernel, kd_kernels.hip)
//   stats    : logit tiles -> running max and sum beside the lists, the logits on them (kd_head.hpp)
//   combine  : log-sum-exp, the token's loss, the coefficients of its gradient, n, loss, the gradients' common factor; beside it h
//              transposed for grad_W
//   per chunk of the vocabulary:
//     grad   : logit tiles again -> dL/dz in the order of dz_chunk;  listed: its entries on the lists
//              (few enough logits are kept and read instead: dz)
//     the backward products (kd_products.hpp)
//   gradh_finish
// With few tokens (kd_head_few.hip) nothing is compacted: tokens that do not count are multiplied with the others, their results dropped.
#include "kd_head.hpp"

namespace kd {

// ------------------------------------------------------------------------------------------
// targets
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}
__device__ __forceinline__ double wave_max(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmax(x, __shfl_xor(x, off, 64));
  return x;
}

__global__ __launch_bounds__(256) void label_targets_kernel(const TargetArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t < a.T) (void)label_target(a, t);
}

// G threads per token, 64 or, of lists longer than that, 256 (4096 tokens with 64 entries 11 us).
// The entries that are there (a row that is not negative, a logit above minus infinity) go to the place that the
// count of smaller rows gives them: K compares each, out of LDS, four at a time (K = 217, 4546 tokens: 37.5 us).  Entries of the same row,
// which meet in one place, add up, in a second look that most calls do not need.  All sums in 64 bits: the mass beside the list is a
// difference from 1.
template <int G>
__global__ __launch_bounds__(256) void top_targets_kernel(const TargetArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ double sums[4][3];
  __shared__ int bad_of[4];
  constexpr int PER = 256 / G, WAVES = G / 64;         // tokens a workgroup, waves a token
  const int K = a.t.K, Kp = (K + 3) & ~3, mine = threadIdx.x / G, k0 = threadIdx.x % G, wave = threadIdx.x >> 6, w0 = mine * WAVES;
  const int t = blockIdx.x * PER + mine, lane = threadIdx.x & 63;
  double* const q = (double*)smem + mine * Kp;
  int* const row = (int*)(smem + PER * Kp * 8) + mine * 2 * Kp;
  int* const taken = row + Kp;                         // entries in a place; where some met: the rows, each once
  const bool there = t < a.T;
  const int64_t at = (int64_t)t * K;
  // sums over a token's waves of x, y, z, in one order
  auto all = [&](double x, double y, double z) {
    x = wave_sum(x); y = wave_sum(y); z = wave_sum(z);
    __syncthreads();
    if (lane == 0) { sums[wave][0] = x; sums[wave][1] = y; sums[wave][2] = z; }
    __syncthreads();
  };
  auto sum = [&](int i) {
    double r = sums[w0][i];
    for (int w = 1; w < WAVES; ++w) r += sums[w0 + w][i];
    return r;
  };
  bool bad = false;
  double top = -INFINITY;
  for (int k = k0; k < Kp; k += G) {
    row[k] = kNoEntry;
    taken[k] = 0;
    if (!there || k >= K) continue;
    const int64_t v = a.t.index64 ? ((const int64_t*)a.t.index)[at + k] : (int64_t)((const int*)a.t.index)[at + k];
    const float z = a.t.top_f32 ? ((const float*)a.t.top)[at + k] : (float)((const bf16_t*)a.t.top)[at + k];
    const bool in = v >= 0 && z != -INFINITY;
    bad = bad || (in && (v >= a.V || z != z));
    row[k] = in && v < a.V ? (int)v : kNoEntry;
    q[k] = (double)z * a.inv_tau;
    if (in) top = fmax(top, q[k]);
  }
  top = wave_max(top);
  if (lane == 0) sums[wave][0] = top;
  __syncthreads();
  top = sums[w0][0];
  for (int w = 1; w < WAVES; ++w) top = fmax(top, sums[w0 + w][0]);
  double norm = 0.0;
  if (a.t.tail == 0) {
    double mass = 0.0;
    for (int k = k0; k < K; k += G) mass += there && row[k] != kNoEntry ? exp(q[k] - top) : 0.0;
    all(mass, 0.0, 0.0);
    norm = top + log(sum(0));
  } else if (there) {
    norm = (double)a.t.lse[t];
  }
  for (int k = k0; k < K; k += G) q[k] = there && row[k] != kNoEntry ? exp(q[k] - norm) : 0.0;
  __syncthreads();
  int n = 0, met = 0;
  double held = 0.0, ent = 0.0;
  for (int k = k0; k < K; k += G) {
    const int v = row[k];
    if (v == kNoEntry) continue;
    int place = 0;
    for (int j = 0; j < Kp; j += 4) {
      const int4 r = *(const int4*)(row + j);
      place += (r.x < v) + (r.y < v) + (r.z < v) + (r.w < v);
    }
    ++n;
    met += atomicAdd(&taken[place], 1) != 0;
    a.t.list[at + place] = v;                          // (of entries that meet, either; done again below)
    a.t.q[at + place] = (float)q[k];
    held += q[k];
    ent += q[k] > 0.0 ? q[k] * log(q[k]) : 0.0;
  }
  const unsigned long long b_bad = __ballot(bad);
  all((double)n, (double)met, held);
  if (lane == 0) bad_of[wave] = b_bad != 0;
  __syncthreads();
  n = (int)sum(0);
  met = (int)sum(1);
  held = sum(2);
  bool any_bad = false;
  for (int w = 0; w < WAVES; ++w) any_bad = any_bad || bad_of[w0 + w];
  const int distinct = n - met;
  if (__syncthreads_or(met)) {                         // (in any token of the workgroup)
    for (int k = k0; k < K; k += G) {
      const int v = row[k];
      bool first = v != kNoEntry;
      for (int j = 0; j < k && first; ++j) first = row[j] != v;
      taken[k] = first ? v : kNoEntry;
    }
    __syncthreads();
    ent = 0.0;
    for (int k = k0; k < K; k += G) {
      const int v = taken[k];
      if (v == kNoEntry) continue;
      int place = 0;
      double total = 0.0;
      for (int j = 0; j < K; ++j) {
        place += taken[j] < v;
        total += row[j] == v ? q[j] : 0.0;
      }
      a.t.list[at + place] = v;
      a.t.q[at + place] = (float)total;
      ent += total > 0.0 ? total * log(total) : 0.0;
    }
  }
  all(ent, 0.0, 0.0);
  ent = sum(0);
  if (!there) return;
  for (int k = distinct + k0; k < K; k += G) a.t.list[at + k] = kNoEntry;
  if (k0) return;
  const double rest = a.t.tail == 1 ? fmax(1.0 - held, 0.0) : 0.0;
  double* const info = a.t.info + (int64_t)t * kTargetInfo;
  info[0] = any_bad || held != held ? __builtin_nan("") : held + rest;
  info[1] = rest;
  info[2] = ent + (rest > 0.0 ? rest * log(rest) : 0.0);
  info[3] = held;
  const bool counts_ = (n > 0 || any_bad) && (!a.t.mask || a.t.mask[t]);
  a.t.valid[t] = counts_;
  keep_places(a, t, counts_);
}

TargetArgs target_args(const HeadProblem& h) {
  return TargetArgs{h.t, h.p.T, h.p.V, 1.0 / (double)h.p.tau, h.few, h.p.meta, h.p.rowmap, h.p.inv};
}

hipError_t launch_targets(const HeadProblem& h, hipStream_t st) {
  const TargetArgs a = target_args(h);
  if (h.t.ce) hipLaunchKernelGGL(label_targets_kernel, dim3((h.p.T + 255) / 256), dim3(256), 0, st, a);
  else if (h.t.K <= 64) hipLaunchKernelGGL(top_targets_kernel<64>, dim3((h.p.T + 3) / 4), dim3(256), 64 * ((h.t.K + 3) & ~3), st, a);
  else hipLaunchKernelGGL(top_targets_kernel<256>, dim3(h.p.T), dim3(256), 16 * ((h.t.K + 3) & ~3), st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// fp32 heads
// ------------------------------------------------------------------------------------------
// The rows' bf16 parts side by side (part_of_six), zero from 6 H to K.  A thread reads eight values once and writes them to all six places;
// bound by its writes, 12 bytes a value.  (As one copy a place, prepare() of kd_kernels.hip read them six times: V = 32000, H = 1432
// 299 us; so 130 us, 5.7 TB/s.)
__global__ __launch_bounds__(256) void head_split_kernel(const float* src, int64_t V, int H, int K, bf16_t* dst) {
  const int wide = H / 8;
  const int64_t i = flat_group() * 256 + threadIdx.x, r = i / wide;
  const int c = (int)(i - r * wide) * 8;
  if (r >= V) return;
  const f32x4 x[2] = {*(const f32x4*)(src + r * H + c), *(const f32x4*)(src + r * H + c + 4)};
  bf16x8 part[3];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f = x[e >> 2][e & 3];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      part[p][e] = (bf16_t)f;
      f -= (float)part[p][e];
    }
  }
  bf16_t* const to = dst + r * K + c;
#pragma unroll
  for (int place = 0; place < 6; ++place) {
    const int p = part_of_six(place, true);
    *(bf16x8*)(to + place * H) = p == 0 ? part[0] : p == 1 ? part[1] : part[2];
  }
  bf16x8 zero;
#pragma unroll
  for (int e = 0; e < 8; ++e) zero[e] = (bf16_t)0.f;
  for (int k = 6 * H + c; k < K; k += H) *(bf16x8*)(dst + r * K + k) = zero;
}

hipError_t launch_head_split(const HeadProblem& h, hipStream_t st) {
  const Problem& p = h.p;
  const FlatGrid g = flat_grid(((int64_t)p.V * (p.H_s / 8) + 255) / 256);
  hipLaunchKernelGGL(head_split_kernel, dim3(g.x, g.y), dim3(256), 0, st, (const float*)p.user_W_s, (int64_t)p.V, p.H_s, p.K_s,
                     (bf16_t*)const_cast<void*>(p.W_s));
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// combine
// ------------------------------------------------------------------------------------------
struct PackHArgs {         // h transposed for grad_W: see pack_columns (kd_kernels.hip), `sets` copies of the token axis
  const void* src;
  bf16_t* dst;
  int src_f32, C, sets, T_pad;
  const int *meta, *rowmap, *inv;
};
struct LossSumArgs {
  const int *meta, *rowmap, *inv;
  const float* row_loss;
  float tau, weight;
  float *loss, *scale;
};
struct HeadCombineArgs {
  const float* partials;
  const int* meta;
  const int *rowmap, *inv;
  int T, T_pad, nv, K, n_parts;        // n_parts: 0 = the device's plan
  float c, z_loss;
  double uniform;                      // U
  const int* list;
  const float* q;
  const float* z;
  const float* kept;                   // the entries' logits among all of them, or null and in z
  int ldz;
  const double* info;
  f32x4* rowinfo;
  float* row_loss;
  float weight;
  float* per_token;
  int groups;              // workgroups that combine; those behind them pack h
  LossSumArgs sum;
  PackHArgs pack;
};

// Which bf16 part of h stands against copy s of dL/dz: dz 0 0 0 1 1 2 x h 0 1 2 0 1 0, or dz 0 1 2 x h itself.
__device__ __forceinline__ bf16_t h_part(float f, int s, int sets) {
  return part_of(f, sets == 6 ? part_of_six(s, false) : 0);
}

// Block b of 64 tokens x 64 hidden rows, by NT threads.
template <int NT>
__device__ __forceinline__ void pack_h(const PackHArgs& a, int b, float (*tile)[65]) {
  const int wide = a.T_pad / 64, by = b / wide, r0 = (b - by * wide) * 64, c0 = by * 64;
  const int eff = a.meta[META_T_EFF], n = a.meta[META_N_VALID];
  if (c0 >= a.C || r0 >= eff) return;
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6, c = c0 + tx, cc = min(c, a.C - 1);
  constexpr int ROWS = 4096 / NT;
  float v[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {         // (rowmap holds a token for every r < T_pad)
    const int r = r0 + ty + NT / 64 * i, token = a.rowmap[r];
    const int64_t at = (int64_t)token * a.C + cc;
    v[i] = a.src_f32 ? ((const float*)a.src)[at] : (float)((const bf16_t*)a.src)[at];
    if (r >= n || c >= a.C || a.inv[token] < 0) v[i] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) tile[ty + NT / 64 * i][tx] = v[i];
  __syncthreads();
  for (int p = ty; p < 8 * a.sets; p += NT / 64) {                     // a wave: 16 hidden rows x 32 tokens, 1 KiB
    const int s = p >> 3, sub = (p >> 2) & 1, blk = p & 3;
    if (c0 + 16 * blk >= a.C) continue;
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = h_part(tile[32 * sub + 8 * (tx >> 4) + e][16 * blk + (tx & 15)], s, a.sets);
    *(bf16x8*)(a.dst + ((int64_t)(c0 / 16 + blk) * (a.T_pad / 32 * a.sets) + (s * eff + r0) / 32 + sub) * 512 + tx * 8) = o;
  }
}

// The mean of the losses of the tokens that count, summed in a fixed order, and the gradients' common factor.
template <int NT>
__device__ __forceinline__ void sum_losses(const LossSumArgs& a, double* sums) {
  const int n_valid = a.meta[META_N_VALID];
  double acc = 0.0;
  int n = 0;
  for (int j = threadIdx.x; j < n_valid; j += NT) {
    acc += (double)a.row_loss[j];
    n += a.inv[a.rowmap[j]] >= 0;
  }
  double total = 0.0;
  for (int pass = 0; pass < 2; ++pass) {
    sums[threadIdx.x] = pass ? (double)n : acc;
    __syncthreads();
    for (int s = NT / 2; s > 0; s >>= 1) {
      if ((int)threadIdx.x < s) sums[threadIdx.x] += sums[threadIdx.x + s];
      __syncthreads();
    }
    if (pass == 0) {
      total = sums[0];
      __syncthreads();
    }
  }
  if (threadIdx.x == 0) {
    const double count = sums[0];
    *a.loss = count > 0.0 ? a.weight * (float)(total / count) : 0.f;
    *a.scale = count > 0.0 ? a.weight / ((float)count * a.tau) : 0.f;
  }
}

// Merges a token's partial sums and its listed logits: lse, and with it the loss and the coefficients of dL/dz (kd_head.hpp).  Bound by
// latency (T = 4096 22 us with packing h beside it, T = 100 with 256 partial sums a token 11 us).  Logarithms in base 2; what is a
// difference of large quantities in double (but for label smoothing's sum of all logits, which is an fp32 sum of V of them).
template <int TX, int NT>
__global__ __launch_bounds__(NT) void head_combine_kernel(const HeadCombineArgs a) {
  constexpr int BYTES = sizeof(float) * 64 * 65;
  __shared__ __attribute__((aligned(16))) char shared[BYTES];
  if (flat_group() >= a.groups) {
    if (a.pack.src) pack_h<NT>(a.pack, (int)(flat_group() - a.groups), (float(*)[65])shared);
    return;
  }
  float* const lds = (float*)shared;
  static_assert(NT / 64 * 4 * TX * 4 <= BYTES && NT * 8 <= BYTES, "the merges' and the sum's share");
  const int t = blockIdx.x * TX + threadIdx.x % TX, g = threadIdx.x / TX, G = NT / TX;
  const int n_valid = a.meta[META_N_VALID], n_parts = a.n_parts ? a.n_parts : a.meta[META_N_SPLIT];
  const int64_t token = a.rowmap[t];
  const bool counts = t < n_valid && a.inv[token] >= 0;
  const f32x4 nothing = {1.0e30f, 0.f, a.nv == 3 ? 0.f : 1.0e30f, 0.f};
  if (a.groups == 1)                     // (rows behind the workgroup's)
    for (int j = TX + threadIdx.x; j < a.T_pad; j += NT) a.rowinfo[j] = nothing;
  if (!counts && g == 0) {             // everything evaluates to 0
    a.rowinfo[t] = nothing;
    a.row_loss[t] = 0.f;
  }
  if (g == 0 && t < a.T && a.per_token && a.inv[t] < 0) a.per_token[t] = 0.f;
  if ((int)(blockIdx.x * TX) < n_valid) {
    const int64_t stride = (int64_t)a.nv * a.T_pad;
    const float* const q0 = a.partials + t;            // t < T_pad: allocated, whatever the row holds
    const int* const list = a.list + token * a.K;
    const float* const prob = a.q + token * a.K;
    auto z = [&](int k) {
      if (!a.kept) return a.z[(int64_t)t * a.K + k];
      const int v = list[k], c = v & 31;
      return a.kept[dz_chunk(a.ldz, t >> 6, v >> 5, (t >> 4) & 3, 16 * ((c & 15) >> 2) + (t & 15)) + 4 * (c >> 4) + (c & 3)];
    };
    float m[2] = {M_FLOOR, M_FLOOR};
#pragma unroll 4
    for (int p = g; p < n_parts; p += G) m[0] = fmaxf(m[0], q0[p * stride]);
    for (int k = g; k < a.K && list[k] != kNoEntry; k += G) m[1] = fmaxf(m[1], z(k) * a.c);
    merge_parts<TX, NT, 2, MergeMax>(m, lds);
    float v[4] = {0.f, 0.f, 0.f, 0.f};                 // sum beside the list, on it, sum of logits, sum q (z - max)
#pragma unroll 4
    for (int p = g; p < n_parts; p += G) {
      const float* const q = q0 + p * stride;
      v[0] = fmaf(q[a.T_pad], fexp2(q[0] - m[0]), v[0]);
      if (a.nv == 3) v[2] += q[2 * a.T_pad];
    }
    for (int k = g; k < a.K && list[k] != kNoEntry; k += G) {
      const float zk = z(k), d = fmaf(zk, a.c, -m[1]);
      v[1] += fexp2(d);
      if (a.nv == 3) v[2] += zk;
      if (prob[k] != 0.f) v[3] = fmaf(prob[k], d, v[3]);        // (0 log 0 = 0: a logit of minus infinity)
    }
    merge_parts<TX, NT, 4, MergeSum>(v, lds);
    if (g == 0 && counts) {
      const double ln2 = 0.6931471805599453;
      const double* const info = a.info + token * kTargetInfo;
      const double mass = info[0], rest = info[1], ent = info[2], held = info[3];
      const double lo = v[0] == 0.f ? -INFINITY : (double)m[0] + log2((double)v[0]);     // beside the list
      const double ll = v[1] == 0.f ? -INFINITY : (double)m[1] + log2((double)v[1]);
      const double big = fmax(lo, ll), lse = v[0] != v[0] || v[1] != v[1] ? __builtin_nan("") : big + log2(exp2(lo - big) + exp2(ll - big));
      const double nat = lse * ln2;
      // sum q z in base 2.  (The list's mass in double, as in `mass`: what the logits have in common is to cancel.  As an fp32 sum it left 1e-7 of
      // the largest logit over tau.)
      const double on = held != 0.0 ? (double)v[3] + (double)m[1] * held : 0.0;
      double loss = ent + mass * nat - ln2 * on - (a.nv == 3 ? a.uniform * (double)v[2] : 0.0) + (double)a.z_loss * nat * nat;
      const double in = mass + 2.0 * (double)a.z_loss * nat;
      double out = in, base = lse;
      if (rest > 0.0) {
        loss -= rest * lo * ln2;
        out = in * exp2(lo - lse) - rest;
        base = lo;
      }
      // (a logarithm as a float is up to 1e-6 off, the same way for all of a token's entries: that goes into the factors)
      const float high = (float)lse, high_out = (float)base;
      a.rowinfo[t] = f32x4{high, (float)(out * exp2((double)high_out - base)), a.nv == 3 ? (float)a.uniform : high_out,
                           (float)(in * exp2((double)high - lse))};
      a.row_loss[t] = (float)loss;
      if (a.per_token) a.per_token[token] = a.weight * (float)loss;
    }
  }
  if (a.groups == 1) {
    __syncthreads();                     // (one workgroup has written all the losses)
    sum_losses<NT>(a.sum, (double*)shared);
  }
}

// ... of more workgroups than one, in a launch of its own unless the gradients' first launch does it.  (The combining workgroup that is
// done last can not do it cheaply: what it needs is in eight L2 caches, and a fence that writes one back took 10 us and more.)
__global__ __launch_bounds__(1024) void head_sum_kernel(const LossSumArgs a) {
  __shared__ double sums[1024];
  sum_losses<1024>(a, sums);
}

static LossSumArgs loss_sum_args(const HeadProblem& h) {
  const Problem& p = h.p;
  return LossSumArgs{p.meta, p.rowmap, p.inv, p.row_loss, p.tau, p.out_weight, p.loss, h.t.scale};
}

hipError_t launch_head_combine(const HeadProblem& h, bool backward, bool pack_h, hipStream_t st) {
  const Problem& p = h.p;
  // 8 tokens x 128 threads where a token has many parts (see merge_parts) or a long list (128 entries 12.6 us, by 32 x 8 18.2, 64 entries of
  // 4096 tokens 37.8 and 23.5), 32 x 8 else; 32 x 32 where that is all the tokens and the sum can follow (one token 10.4 us; 8.7 and 4.6 in
  // two launches)
  const bool all = p.T <= 32, many = !all && ((h.few ? h.parts : p.n_split) >= 128 || h.t.K >= 128);
  HeadCombineArgs a{p.partials, p.meta, p.rowmap, p.inv, p.T, p.T_pad, h.t.smoothing > 0.f ? 3 : 2, h.t.K, h.few ? h.parts : 0,
                    1.4426950408889634f / p.tau, h.t.z_loss, (double)h.t.smoothing / p.V, h.t.list, h.t.q, h.t.z, h.kept, p.V_c, h.t.info,
                    (f32x4*)p.rowinfo, p.row_loss, p.out_weight, p.per_token_loss, all ? 1 : many ? p.T_pad / 8 : p.T_pad / 32,
                    loss_sum_args(h), {}};
  int64_t groups = a.groups;
  if (pack_h) {
    a.pack = PackHArgs{p.user_h_s, (bf16_t*)p.h_sT, p.in_f32, p.H_s, p.dz_sets, p.T_pad, p.meta, p.rowmap, p.inv};
    groups += (int64_t)(p.T_pad / 64) * ((p.H_s + 63) / 64);
  }
  const FlatGrid g = flat_grid(groups);
  if (all) hipLaunchKernelGGL((head_combine_kernel<32, 1024>), dim3(g.x, g.y), dim3(1024), 0, st, a);
  else if (many) hipLaunchKernelGGL((head_combine_kernel<8, 1024>), dim3(g.x, g.y), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((head_combine_kernel<32, 256>), dim3(g.x, g.y), dim3(256), 0, st, a);
  if (!all && !(h.kept && backward)) hipLaunchKernelGGL(head_sum_kernel, dim3(1), dim3(1024), 0, st, a.sum);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// logit tiles
// ------------------------------------------------------------------------------------------
HeadArgs head_args(const HeadProblem& h) {
  const Problem& p = h.p;
  HeadArgs a{};
  a.W = (const bf16_t*)p.W_s; a.h = (const bf16_t*)p.h_s;
  a.V = p.V; a.K = p.K_s;
  a.ld = p.w_hv_inplace ? p.V : p.prep_Ws ? p.K_s : p.H_s;
  a.meta = p.meta;
  a.T_pad = p.T_pad;
  a.c = 1.4426950408889634f / p.tau;
  a.partials = p.partials;
  a.rowmap = p.rowmap;
  a.list = h.t.list; a.n_list = h.t.K; a.z = h.t.z;
  a.rowinfo = (const f32x4*)p.rowinfo;
  a.kept = h.kept;
  a.dz = (bf16_t*)p.dz; a.ldz = p.V_c; a.sets = p.dz_sets;
  return a;
}

hipError_t launch_head_stats(const HeadProblem& h, hipStream_t st) {
  HeadArgs a = head_args(h);
  a.v_end = h.p.V;
  const int grid = h.p.n_tt * h.p.n_split;
  const bool hv = h.p.w_hv_inplace, smooth = h.t.smoothing > 0.f;
#define KD_HS(HV, S) (h.kept ? launch_big<head_stats_kernel<HV, S, true>>(grid, HeadCfg::NT, HeadCfg::STATE_SMEM_BYTES, st, &a) \
                             : launch_big<head_stats_kernel<HV, S, false>>(grid, HeadCfg::NT, HeadCfg::STATE_SMEM_BYTES, st, &a))
  return hv ? (smooth ? KD_HS(true, true) : KD_HS(true, false)) : (smooth ? KD_HS(false, true) : KD_HS(false, false));
#undef KD_HS
}

// dL/dz of a chunk on the lists: A_in p - q - U, where the tile kernel has written what it would be beside them.  One thread per entry;
// bound by latency (4096 tokens' lists of 64 5 us a chunk).
struct ListedArgs {
  const int *meta, *rowmap, *list;
  const float *q, *z;
  const f32x4* rowinfo;
  int K, v0, v_end, ldz, sets, smooth;
  float c;
  bf16_t* dz;
};
__global__ __launch_bounds__(256) void head_listed_kernel(const ListedArgs a) {
  const int64_t i = flat_group() * 256 + threadIdx.x;
  const int j = (int)(i / a.K), k = (int)(i - (int64_t)j * a.K);
  if (j >= a.meta[META_N_VALID]) return;
  const int64_t at = (int64_t)a.rowmap[j] * a.K + k;
  const int v = a.list[at];
  if (v < a.v0 || v >= a.v_end) return;
  const f32x4 ri = a.rowinfo[j];
  float x = listed_dz(ri, a.z[(int64_t)j * a.K + k], a.c, a.q[at], a.smooth ? ri[2] : 0.f);
  const int col = v - a.v0, c = col & 31, half = c >> 4, g = (c & 15) >> 2;
  const int64_t to = dz_chunk(a.ldz, j >> 6, col >> 5, (j >> 4) & 3, 16 * g + (j & 15)) + 4 * half + (c & 3);
  if (a.sets == 1) {
    a.dz[to] = (bf16_t)x;
    return;
  }
  const int64_t stride = (int64_t)a.meta[META_T_EFF] * a.ldz;
  for (int p = 0; p < 3; ++p) {
    const bf16_t o = (bf16_t)x;
    x -= (float)o;
    const int first = a.sets == 3 ? p : p == 0 ? 0 : p == 1 ? 3 : 5, n = a.sets == 3 ? 1 : 3 - p;
    for (int s = 0; s < n; ++s) a.dz[to + (first + s) * stride] = o;
  }
}

// All of it from kept logits (the whole vocabulary is one chunk).  A workgroup makes 256 columns of a panel of 64 tokens, 4 KiB of
// each 32; bound by memory, 6 bytes a logit (T = 200, three panels that count, V = 151936: 34 us, 5.1 TB/s).  Which of
// them are listed stands in LDS, a word per token and 32 columns.  With long lists by the latency of their marking and of loading
// their probabilities (T = 1909, V = 5424, K = 202: 29 us for 60 MB; one entry at a time 62 us).
struct KeptArgs {
  HeadArgs h;
  const int* inv;
  const float* q;
  int smooth;
  LossSumArgs sum;         // (if the merge has not done it: loss not null)
};
template <int PARTS>
__global__ __launch_bounds__(256, PARTS == 1 ? 5 : 4) void head_dz_kernel(const KeptArgs k) {
  __shared__ uint32_t listed[64][8];
  __shared__ int first[64], whose[64];
  const HeadArgs& a = k.h;
  __shared__ double sums[256];
  if (blockIdx.y == 0) {
    if (blockIdx.x == 0 && k.sum.loss) sum_losses<256>(k.sum, sums);
    return;
  }
  const int panel = blockIdx.y - 1, panels = a.meta[META_T_EFF] >> 6;
  if (panel >= panels) return;
  const int sub0 = blockIdx.x * 8, subs = min((a.V + 63) / 64 * 2 - sub0, 8);
  const int lane = threadIdx.x & 63, blk = threadIdx.x >> 6, g = lane >> 4, i = 16 * blk + (lane & 15);
  f32x4 z[8][2];                             // (all on their way before the lists are looked at; behind the last sub-step the last again)
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const float* const from = a.kept + dz_chunk(a.ldz, panel, sub0 + min(s, subs - 1), blk, lane);
    z[s][0] = *(const f32x4*)from;
    z[s][1] = *(const f32x4*)(from + 4);
  }
  const f32x4 ri = a.rowinfo[panel * 64 + i];
  const float base = k.smooth ? ri[0] : ri[2], u = k.smooth ? ri[2] : 0.f;
  {                                          // four threads a token, four entries each at a time
    const int i = threadIdx.x >> 2, r = threadIdx.x & 3, j = panel * 64 + i;
    const int token = j < a.meta[META_N_VALID] ? a.rowmap[j] : -1;
    const bool counts = token >= 0 && k.inv[token] >= 0;
    listed[i][2 * r] = listed[i][2 * r + 1] = 0u;            // (a token's four threads are one wave's: its LDS operations are made in order)
    __builtin_amdgcn_wave_barrier();
    if (r == 0) whose[i] = counts ? token : -1;
    if (counts) {
      const int* const list = a.list + (int64_t)token * a.n_list;
      const int from = first_entry(list, a.n_list, 32 * sub0);
      if (r == 0) first[i] = from;
      for (int at = from + r; at < a.n_list; at += 16) {
        int col[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) col[e] = list[min(at + 4 * e, a.n_list - 1)] - 32 * sub0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + 4 * e < a.n_list && col[e] < 256) atomicOr(&listed[i][col[e] >> 5], 1u << (col[e] & 31));
        if (col[3] >= 256) break;
      }
    }
  }
  __syncthreads();
  const int token = whose[i];                                              // (of tokens that do not count there may be no logits)
  const int64_t stride = (int64_t)panels * 64 * a.ldz;
  int rank = first[i];                                                     // entries of the list in front of the sub-step
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    if (s >= subs) break;
    const int64_t at = dz_chunk(a.ldz, panel, sub0 + s, blk, lane);
    const uint32_t word = listed[i][s], mine = (word >> (4 * g)) & 0x000f000fu;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool there = token >= 0 && (sub0 + s) * 32 + 4 * g + (e < 4 ? 0 : 16) < a.V;       // (V is a multiple of 8)
      const float d = unlisted_dz(ri[1], base, z[s][e >> 2][e & 3], a.c, u);
      x[e] = there ? d : 0.f;
    }
    if (mine) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {           // (four on their way together; with eight registers run out)
        float q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          q[e] = k.q[(int64_t)token * a.n_list + min(rank + (int)__popc(word & ((1u << (4 * g + 16 * half + e)) - 1)), a.n_list - 1)];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[4 * half + e] = mine >> (16 * half + e) & 1 ? listed_dz(ri, z[s][half][e], a.c, q[e], u) : x[4 * half + e];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    rank += __popc(word);
    store_dz<PARTS>(x, a.dz + at, stride, a.sets);
  }
}

hipError_t launch_head_grad(const HeadProblem& h, int v0, int width, hipStream_t st) {
  const Problem& p = h.p;
  HeadArgs a = head_args(h);
  a.v0 = v0; a.v_end = v0 + width;
  a.last_chunk = v0 + width >= p.V;
  const int grid = p.n_tt * p.g_split;
  const bool hv = p.w_hv_inplace, smooth = h.t.smoothing > 0.f, parts = p.dz_sets > 1;
#define KD_HG(HV, S) (parts ? launch_big<head_grad_kernel<HV, S, 3>>(grid, HeadCfg::NT, HeadCfg::STATE_SMEM_BYTES, st, &a) \
                            : launch_big<head_grad_kernel<HV, S, 1>>(grid, HeadCfg::NT, HeadCfg::STATE_SMEM_BYTES, st, &a))
  hipError_t e = hipSuccess;
  if (h.kept) {
    const dim3 blocks((p.V + 255) / 256, p.T_pad / 64 + 1);
    KeptArgs k{a, p.inv, h.t.q, smooth, loss_sum_args(h)};
    if (p.T <= 32) k.sum.loss = nullptr;
    if (parts) hipLaunchKernelGGL(head_dz_kernel<3>, blocks, dim3(256), 0, st, k);
    else hipLaunchKernelGGL(head_dz_kernel<1>, blocks, dim3(256), 0, st, k);
    return hipGetLastError();
  } else {
    e = hv ? (smooth ? KD_HG(true, true) : KD_HG(true, false)) : (smooth ? KD_HG(false, true) : KD_HG(false, false));
  }
#undef KD_HG
  if (e != hipSuccess) return e;
  const ListedArgs l{p.meta, p.rowmap, h.t.list, h.t.q, h.t.z, (const f32x4*)p.rowinfo, h.t.K, v0, v0 + width, p.V_c, p.dz_sets,
                     smooth, 1.4426950408889634f / p.tau, (bf16_t*)p.dz};
  const FlatGrid g = flat_grid(((int64_t)p.T * h.t.K + 255) / 256);
  hipLaunchKernelGGL(head_listed_kernel, dim3(g.x, g.y), dim3(256), 0, st, l);
  return hipGetLastError();
}

}  // namespace kd
