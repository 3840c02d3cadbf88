// C ABI of what stands beside the losses (e4m3 in blocks, top logits, sampling, gradient norm): argument checks, plans and launches.
// All checks are host-only and happen before the first HIP call.
#include <hip/hip_runtime.h>

#include "../../include/kdloss.h"
#include "kd_beside.h"
#include "kd_launch.h"
#include "kd_plan.hpp"

#include <cmath>

namespace {

using kd::aligned16;
using kd::round_up;

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool is_dtype(int32_t d) { return d == KD_BF16 || d == KD_F32; }
uintptr_t size_of(int32_t d) { return d == KD_F32 ? 4 : 2; }
uintptr_t index_size(int32_t d) { return d == KD_I64 ? 8 : 4; }

#define KD_TRY(expr)                                \
  do {                                              \
    if ((expr) != hipSuccess) return KD_ERR_LAUNCH; \
  } while (0)

constexpr int64_t kMostRows = 1 << 24, kMostColumns = 1 << 22;

// ---- e4m3 in blocks ----
kd_status check(const kd_blocks_params* p) {
  if (!p) return KD_ERR_NULL;
  if (p->rows < 1 || p->cols < 1 || p->rows > kMostRows || p->cols > kMostColumns || p->ld < p->cols) return KD_ERR_SHAPE;
  if (p->ld > ((int64_t)1 << 40)) return KD_ERR_SHAPE;
  if (!is_dtype(p->src_dtype) || (p->block != KD_BLOCK_ROW && p->block != KD_BLOCK_TILE)) return KD_ERR_PARAM;
  return p->reserved[0] == 0 && p->reserved[1] == 0 ? KD_OK : KD_ERR_PARAM;
}

kd_status check(const kd_linear_params* p) {
  if (!p) return KD_ERR_NULL;
  if (p->M < 1 || p->N < 1 || p->K < 1 || p->M > kMostRows || p->N > kMostRows || p->K > kMostColumns) return KD_ERR_SHAPE;
  if (!is_dtype(p->in_dtype) || !is_dtype(p->out_dtype)) return KD_ERR_PARAM;
  if ((p->b_block != KD_BLOCK_ROW && p->b_block != KD_BLOCK_TILE) || (p->accumulate != 0 && p->accumulate != 1)) return KD_ERR_PARAM;
  return p->reserved[0] == 0 && p->reserved[1] == 0 ? KD_OK : KD_ERR_PARAM;
}

struct LinearLayout { size_t codes, scales, sums, total; };
LinearLayout linear_layout(const kd_linear_params& p) {
  LinearLayout L{};
  size_t off = 0;
  auto take = [&](int64_t bytes) { size_t o = off; off = (size_t)round_up((int64_t)off + bytes, 256); return o; };
  L.codes = take(p.M * round_up(p.K, 16));
  L.scales = take(p.M * ((p.K + 127) / 128) * 4);
  const int parts = kd::product_parts(p.M, p.N, p.K, p.out_dtype == KD_F32);
  L.sums = take(parts > 1 ? parts * p.M * p.N * 4 : 0);
  L.total = off;
  return L;
}

kd::ProductArgs product_args(const kd_linear_params& p, const uint8_t* a, const float* a_scales, const uint8_t* b, const float* b_scales,
                             void* out, void* workspace) {
  float* const sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + linear_layout(p).sums);
  return kd::ProductArgs{a, b, a_scales, b_scales, out, p.M, p.N, p.K, p.out_dtype == KD_F32, p.b_block == KD_BLOCK_TILE, p.accumulate, sums, 1};
}

// ---- rows of logits ----
struct RowsLayout { size_t chunk, group, wide, mass, total; };

// Entries per thread of the first kernel: the most that leave 32 chunks in all and twelve groups for each entry of a list of `reach`;
// rows have at most 1024 chunks.  Many entries a thread: less is read twice over by the second kernel; few: more workgroups, and groups that hold less beside
// the list's entries.  us with 8, 16, 32 and 64 entries (T, V): top 20 of (512, 151936) 61, 46, 40, 39; top 256 of it 65, 50, 46, 54, of (64, 128256) 24, 20, 22, 27;
// a token of (1, 151936) 12, 12, 13, 14, of (7, 32003) 12, 13, 14, 17, of (512, 151936) 89, 78, 71, 73, among the first 700 of (64, 128256) 37, 36, 39, 47.
void plan_rows(kd::RowsArgs& r, RowsLayout& L, int64_t reach) {
  int e = 64;
  for (; e > 8; e >>= 1) {
    const int64_t chunks = (r.V + kd::kRowThreads * e - 1) / (kd::kRowThreads * e);
    if (r.T * chunks >= 32 && r.V / e >= 12 * reach) break;
    if ((r.V + kd::kRowThreads * e / 2 - 1) / (kd::kRowThreads * e / 2) > 1024) break;
  }
  r.per_thread = e;
  r.chunks = (int)((r.V + kd::kRowThreads * e - 1) / (kd::kRowThreads * e));
  size_t off = 0;
  auto take = [&](int64_t bytes) { size_t o = off; off = (size_t)round_up((int64_t)off + bytes, 256); return o; };
  L.chunk = take(r.T * r.chunks * (int64_t)sizeof(kd::RowChunk));
  L.group = take(r.T * r.chunks * kd::kRowThreads * 4);
  L.total = off;
}

kd_status check_rows(int64_t T, int64_t V, int64_t ld, int32_t in_dtype, int32_t index_dtype) {
  if (T < 1 || V < 1 || T > (1 << 22) || V > (1 << 24) || ld < V || ld > ((int64_t)1 << 40)) return KD_ERR_SHAPE;
  if (!is_dtype(in_dtype) || (index_dtype != KD_I32 && index_dtype != KD_I64)) return KD_ERR_PARAM;
  return KD_OK;
}

kd_status plan(const kd_top_logits_params* p, kd::RowsArgs& r, RowsLayout& L) {
  if (!p) return KD_ERR_NULL;
  const kd_status s = check_rows(p->T, p->V, p->ld, p->in_dtype, p->index_dtype);
  if (s != KD_OK) return s;
  if (p->K < 1 || p->K > KD_TOPK_MAX || p->K > p->V) return KD_ERR_SHAPE;
  if (!(p->tau >= 1e-6f && p->tau <= 1e6f) || p->reserved[0] || p->reserved[1]) return KD_ERR_PARAM;      // (also a tau of NaN)
  r.T = p->T; r.V = p->V; r.ld = p->ld; r.f32 = p->in_dtype == KD_F32; r.index64 = p->index_dtype == KD_I64;
  r.K = p->K; r.tau = p->tau;
  plan_rows(r, L, p->K);
  return KD_OK;
}

kd_status plan(const kd_sample_params* p, kd::RowsArgs& r, RowsLayout& L) {
  if (!p) return KD_ERR_NULL;
  const kd_status s = check_rows(p->T, p->V, p->ld, p->in_dtype, p->index_dtype);
  if (s != KD_OK) return s;
  if (!(p->temperature == 0.f || (p->temperature >= 1e-6f && p->temperature <= 1e6f)) || p->top_k < 0 ||
      !(p->top_p > 0.f && p->top_p <= 1.f) || !(p->min_p >= 0.f && p->min_p <= 1.f) || p->reserved[0] || p->reserved[1])
    return KD_ERR_PARAM;
  r.T = p->T; r.V = p->V; r.ld = p->ld; r.f32 = p->in_dtype == KD_F32; r.index64 = p->index_dtype == KD_I64;
  r.tau = p->temperature; r.top_k = p->top_k; r.top_p = p->top_p; r.min_p = p->min_p;
  plan_rows(r, L, p->top_k > 256 && p->top_k <= 1024 ? p->top_k : 256);
  if (r.V > kd::kWideList) {
    const int64_t rows = r.T < kd::kWideRows ? r.T : kd::kWideRows;
    const int64_t tiles = (r.V + kd::kWideTile - 1) / kd::kWideTile, parts = 4 * kd::kNumCU / rows;
    // (four workgroups a CU; one, four and eight: top-p 0.9 in 64 rows of 128256 fp32 74, 66 and 80 us, in 512 of 151936 bf16 282, 259 and 263)
    r.wide_parts = (int)(parts < 1 ? 1 : parts < tiles ? parts : tiles);
    L.wide = L.total;
    L.mass = (size_t)round_up((int64_t)L.wide + rows * (int64_t)sizeof(kd::RowWide), 256);
    L.total = (size_t)round_up((int64_t)L.mass + rows * tiles * 8, 256);
  }
  return KD_OK;
}

template <class Params>
kd_status rows_workspace(const Params* params, size_t* bytes) {
  if (!bytes) return KD_ERR_NULL;
  kd::RowsArgs r{};
  RowsLayout L{};
  const kd_status s = plan(params, r, L);
  if (s == KD_OK) *bytes = L.total;
  return s;
}

void carve(kd::RowsArgs& r, const RowsLayout& L, void* ws) {
  r.chunk = reinterpret_cast<kd::RowChunk*>(static_cast<char*>(ws) + L.chunk);
  r.group = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + L.group);
}

// ---- gradient norm ----
kd_status check_counts(int32_t n, const int64_t* counts) {
  if (n < 1 || n > KD_GRADS_MAX) return KD_ERR_SHAPE;
  if (!counts) return KD_ERR_NULL;
  int64_t all = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] < 0 || counts[i] > ((int64_t)1 << 40)) return KD_ERR_SHAPE;
    all += counts[i];
    if (all > ((int64_t)1 << 40)) return KD_ERR_SHAPE;
  }
  return KD_OK;
}

kd_status check_arrays(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes) {
  const kd_status s = check_counts(n, counts);
  if (s != KD_OK) return s;
  if (!grads || !dtypes) return KD_ERR_NULL;
  for (int32_t i = 0; i < n; ++i) {
    if (!is_dtype(dtypes[i])) return KD_ERR_PARAM;
    if (counts[i] && !grads[i]) return KD_ERR_NULL;
    if (counts[i] && !aligned(grads[i], size_of(dtypes[i]))) return KD_ERR_ALIGN;
  }
  return KD_OK;
}

// The arrays from `i` on that one launch takes; the next one's first.  Arrays without elements are left out.
int32_t fill(kd::GradTable& t, uint64_t* out, int32_t i, int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes,
             void* const* outs, const int32_t* out_dtypes) {
  t.n = 0;
  t.chunks = 0;
  for (; i < n && t.n < kd::kGradsPerLaunch; ++i) {
    if (!counts[i]) continue;
    const int64_t pieces = (counts[i] + kd::kPieceElements - 1) / kd::kPieceElements;
    t.in[t.n] = reinterpret_cast<uint64_t>(grads[i]) | (dtypes[i] == KD_F32);
    t.count[t.n] = (uint64_t)counts[i];
    t.first[t.n] = t.chunks;
    if (out) out[t.n] = outs ? reinterpret_cast<uint64_t>(outs[i]) | (out_dtypes[i] == KD_F32) : t.in[t.n];
    t.chunks += (uint32_t)pieces;
    ++t.n;
  }
  return i;
}

int groups_of(const kd::GradTable& t) { return t.chunks < (uint32_t)kd::kNormGroups ? (int)t.chunks : kd::kNormGroups; }

}  // namespace

extern "C" {

kd_status kd_quantize_e4m3_blocks(const kd_blocks_params* params, const void* src, uint8_t* codes, float* scales, uint8_t* codes_t,
                                  float* scales_t, void* hip_stream) {
  const kd_status s = check(params);
  if (s != KD_OK) return s;
  if (!src || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return KD_ERR_NULL;
  if (codes_t && params->rows > kMostColumns) return KD_ERR_SHAPE;
  if (!aligned(src, size_of(params->src_dtype)) || !aligned16(codes) || !aligned16(codes_t) || !aligned(scales, 4) || !aligned(scales_t, 4))
    return KD_ERR_ALIGN;
  const kd::BlocksArgs a{src, params->rows, params->cols, params->ld, params->src_dtype == KD_F32, params->block == KD_BLOCK_TILE,
                         codes, codes_t, scales, scales_t};
  KD_TRY(kd::launch_quantize_blocks(a, static_cast<hipStream_t>(hip_stream)));
  return KD_OK;
}

kd_status kd_linear_workspace_size(const kd_linear_params* params, size_t* bytes) {
  if (!bytes) return KD_ERR_NULL;
  const kd_status s = check(params);
  if (s == KD_OK) *bytes = linear_layout(*params).total;
  return s;
}

kd_status kd_matmul_e4m3(const kd_linear_params* params, const uint8_t* a, const float* a_scales, const uint8_t* b, const float* b_scales,
                         void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const kd_status s = check(params);
  if (s != KD_OK) return s;
  if (!a || !a_scales || !b || !b_scales || !out || !workspace) return KD_ERR_NULL;
  if (!aligned16(a) || !aligned16(b) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(out, size_of(params->out_dtype)) ||
      !aligned(workspace, 256))
    return KD_ERR_ALIGN;
  if (workspace_bytes < linear_layout(*params).total) return KD_ERR_WORKSPACE;
  KD_TRY(kd::launch_product(product_args(*params, a, a_scales, b, b_scales, out, workspace), static_cast<hipStream_t>(hip_stream)));
  return KD_OK;
}

kd_status kd_linear_e4m3(const kd_linear_params* params, const void* x, const uint8_t* w, const float* w_scales, void* out,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  const kd_status s = check(params);
  if (s != KD_OK) return s;
  if (params->b_block != KD_BLOCK_TILE) return KD_ERR_PARAM;
  if (!x || !w || !w_scales || !out || !workspace) return KD_ERR_NULL;
  if (!aligned(x, size_of(params->in_dtype)) || !aligned16(w) || !aligned(w_scales, 4) || !aligned(out, size_of(params->out_dtype)) ||
      !aligned(workspace, 256))
    return KD_ERR_ALIGN;
  const LinearLayout L = linear_layout(*params);
  if (workspace_bytes < L.total) return KD_ERR_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  uint8_t* const codes = static_cast<uint8_t*>(workspace) + L.codes;
  float* const scales = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.scales);
  if (kd::product_quantises(params->M, params->K)) {
    KD_TRY(kd::launch_linear_few(product_args(*params, nullptr, nullptr, w, w_scales, out, workspace), x, params->in_dtype == KD_F32, st));
    return KD_OK;
  }
  const kd::BlocksArgs q{x, params->M, params->K, params->K, params->in_dtype == KD_F32, 0, codes, nullptr, scales, nullptr};
  KD_TRY(kd::launch_quantize_blocks(q, st));
  KD_TRY(kd::launch_product(product_args(*params, codes, scales, w, w_scales, out, workspace), st));
  return KD_OK;
}

kd_status kd_top_logits_workspace_size(const kd_top_logits_params* params, size_t* bytes) { return rows_workspace(params, bytes); }
kd_status kd_sample_workspace_size(const kd_sample_params* params, size_t* bytes) { return rows_workspace(params, bytes); }

kd_status kd_top_logits(const kd_top_logits_params* params, const void* logits, void* top_logits, void* top_index, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  kd::RowsArgs r{};
  RowsLayout L{};
  const kd_status s = plan(params, r, L);
  if (s != KD_OK) return s;
  if (!logits || !top_logits || !top_index || !workspace) return KD_ERR_NULL;
  if (!aligned(logits, size_of(params->in_dtype)) || !aligned(top_logits, size_of(params->in_dtype)) ||
      !aligned(top_index, index_size(params->index_dtype)) || !aligned(lse, 4) || !aligned(workspace, 256))
    return KD_ERR_ALIGN;
  if (workspace_bytes < L.total) return KD_ERR_WORKSPACE;
  r.logits = logits; r.top = top_logits; r.index = top_index; r.lse = lse;
  carve(r, L, workspace);
  KD_TRY(kd::launch_top_logits(r, static_cast<hipStream_t>(hip_stream)));
  return KD_OK;
}

kd_status kd_sample(const kd_sample_params* params, const void* logits, const float* u, const float* temperature_rows,
                    const int32_t* top_k_rows, const float* top_p_rows, const float* min_p_rows, void* token, float* logp,
                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  kd::RowsArgs r{};
  RowsLayout L{};
  const kd_status s = plan(params, r, L);
  if (s != KD_OK) return s;
  if (!logits || !u || !token || !workspace) return KD_ERR_NULL;
  if (!aligned(logits, size_of(params->in_dtype)) || !aligned(u, 4) || !aligned(temperature_rows, 4) || !aligned(top_k_rows, 4) ||
      !aligned(top_p_rows, 4) || !aligned(min_p_rows, 4) || !aligned(token, index_size(params->index_dtype)) || !aligned(logp, 4) ||
      !aligned(workspace, 256))
    return KD_ERR_ALIGN;
  if (workspace_bytes < L.total) return KD_ERR_WORKSPACE;
  r.logits = logits; r.u = u; r.token = token; r.logp = logp;
  r.temperature_rows = temperature_rows; r.top_k_rows = top_k_rows; r.top_p_rows = top_p_rows; r.min_p_rows = min_p_rows;
  carve(r, L, workspace);
  // (who draws from all entries needs no groups)
  const bool same = !temperature_rows && !top_k_rows && !top_p_rows && !min_p_rows;
  if (same && r.tau > 0.f && (r.top_k == 0 || r.top_k >= r.V) && r.top_p == 1.f && r.min_p == 0.f) r.group = nullptr;
  const bool all_k = r.top_k_rows || r.top_k == 0 || r.top_k >= r.V, cuts = r.top_p_rows || r.min_p_rows || r.top_p < 1.f || r.min_p > 0.f;
  if (r.wide_parts && all_k && cuts) {
    r.wide = reinterpret_cast<kd::RowWide*>(static_cast<char*>(workspace) + L.wide);
    r.wide_mass = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + L.mass);
  }
  KD_TRY(kd::launch_sample(r, static_cast<hipStream_t>(hip_stream)));
  return KD_OK;
}

kd_status kd_grad_norm_workspace_size(int32_t n, const int64_t* counts, size_t* bytes) {
  if (!bytes) return KD_ERR_NULL;
  const kd_status s = check_counts(n, counts);
  if (s != KD_OK) return s;
  // (a partial sum per workgroup of every launch)
  *bytes = (size_t)((n + kd::kGradsPerLaunch - 1) / kd::kGradsPerLaunch) * kd::kNormGroups * sizeof(double);
  return KD_OK;
}

kd_status kd_grad_norm(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t norm_kind,
                       double* total, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const kd_status s = check_arrays(n, grads, counts, dtypes);
  if (s != KD_OK) return s;
  if (norm_kind != KD_NORM_L2 && norm_kind != KD_NORM_MAX) return KD_ERR_PARAM;
  if (!total || !workspace) return KD_ERR_NULL;
  if (!aligned(total, 8) || !aligned(workspace, 256)) return KD_ERR_ALIGN;
  size_t need = 0;
  kd_grad_norm_workspace_size(n, counts, &need);
  if (workspace_bytes < need) return KD_ERR_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double* const partials = static_cast<double*>(workspace);
  int64_t parts = 0;
  for (int32_t i = 0; i < n;) {
    kd::GradTable t{};
    i = fill(t, nullptr, i, n, grads, counts, dtypes, nullptr, nullptr);
    if (!t.n) break;
    KD_TRY(kd::launch_grad_norm(t, norm_kind == KD_NORM_MAX, partials + parts, groups_of(t), st));
    parts += groups_of(t);
  }
  KD_TRY(kd::launch_grad_total(partials, parts, norm_kind == KD_NORM_MAX, total, st));
  return KD_OK;
}

kd_status kd_grad_clip(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t norm_kind,
                       const double* total, double max_norm, void* const* out, const int32_t* out_dtypes, float* norm, void* hip_stream) {
  const kd_status s = check_arrays(n, grads, counts, dtypes);
  if (s != KD_OK) return s;
  if ((norm_kind != KD_NORM_L2 && norm_kind != KD_NORM_MAX) || !(max_norm >= 0 && std::isfinite(max_norm))) return KD_ERR_PARAM;
  if (!total || (out && !out_dtypes)) return KD_ERR_NULL;
  if (!aligned(total, 8) || !aligned(norm, 4)) return KD_ERR_ALIGN;
  if (out)
    for (int32_t i = 0; i < n; ++i) {
      if (!is_dtype(out_dtypes[i])) return KD_ERR_PARAM;
      if (!counts[i]) continue;
      if (!out[i]) return KD_ERR_NULL;
      if (!aligned(out[i], size_of(out_dtypes[i]))) return KD_ERR_ALIGN;
      if (out[i] == grads[i] && out_dtypes[i] != dtypes[i]) return KD_ERR_PARAM;
    }
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  int32_t i = 0;
  do {
    kd::ClipTable t{};
    i = fill(t.t, t.out, i, n, grads, counts, dtypes, out, out_dtypes);
    KD_TRY(kd::launch_grad_clip(t, norm_kind == KD_NORM_MAX, total, max_norm, norm, st));
    norm = nullptr;
  } while (i < n);
  return KD_OK;
}

}  // extern "C"
