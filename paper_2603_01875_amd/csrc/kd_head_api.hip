// C ABI of the one-head losses (kd_ce_*, kd_topk_*): argument checks, workspace planning and the launch sequence.
// All checks are host-only and happen before the first HIP call.
#include <hip/hip_runtime.h>

#include "../../include/kdloss.h"
#include "kd_launch.h"
#include "kd_plan.hpp"

#include <cmath>

namespace {

using kd::HeadProblem;
using kd::Problem;
using kd::Targets;
using kd::aligned16;
using kd::round_up;

// Most bytes of logits that a call with gradients keeps in its workspace, in fp32, instead of making them twice.  What they cost is a store
// and a load of 4 bytes, what they save is 2 H flop and the head's second reading.  All kept against none, us a call, bf16:
//   within the limit     T = 128, H = 1024, V = 151936 (78 MB) 285 / 380; T = 200, H = 2048, V = 151936 (156 MB) 570 / 734; T = 500,
//                        H = 1024, V = 50264 (103 MB) 266 / 276, H = 4096 677 / 825
//   beyond it            T = 256, V = 200000 (205 MB) H = 1024 509 / 540, H = 4096 1334 / 1719; T = 800, V = 100000 (410 MB, the most that one
//                        chunk has) H = 1024 686 / 724, H = 4096 1999 / 2481; T = 500, H = 1024, V = 151936, fp32 gradients (311 MB) 1151 / 1195
// so keeping them pays wherever the vocabulary is one chunk (3 to 8 % with H = 1024, 17 to 30 % with 4096, more with few tokens): the limit is
// there for the workspace alone, which would be 2 to 3 times as large (T = 256, H = 4096, V = 400000 686 MB for 276).
constexpr int64_t kKept = 160ll << 20;

// Most bytes of grad_h's partial sums for which the products of its parts get sums of their own, in one launch (one launch a product, each
// adding to the sums in front of it: T = 500, H = 1024, V = 32000 in fp32 286 us, so 208; T = 777, H = 1000, V = 50264, fp32 gradients
// of bf16 operands 306, so 263).
constexpr int64_t kPartialSums = 128ll << 20;

struct HeadLayout {
  size_t meta, rowmap, inv, row_loss, rowinfo, scale, valid, list, q, info, z;
  size_t prep_h, prep_W, partials, h_sT, dz, gh32, kept;
  size_t total;
};

// What both parameter blocks say.
struct Call {
  int64_t T, H, V;
  int K, in_dtype, grad_dtype, w_layout, index_dtype, top_dtype, tail, ce;
  float tau, smoothing, z_loss, weight;
  int accumulate, vocab_chunk;
};

kd_status check_call(const Call& c, float loss_scale) {
  if (c.T < 1 || c.H < 1 || c.V < 1 || c.T > (1 << 22) || c.V > (1 << 24) || c.H > 65536) return KD_ERR_SHAPE;
  if (c.K < 1 || c.K > KD_TOPK_MAX || c.K > c.V) return KD_ERR_SHAPE;
  if (c.H % 8 || c.V % 8) return KD_ERR_ALIGN;
  if (c.in_dtype != KD_BF16 && c.in_dtype != KD_F32) return KD_ERR_PARAM;
  if (c.grad_dtype != KD_BF16 && c.grad_dtype != KD_F32) return KD_ERR_PARAM;
  if (c.w_layout != KD_W_HV && c.w_layout != KD_W_VH) return KD_ERR_PARAM;
  if (c.index_dtype != KD_I32 && c.index_dtype != KD_I64) return KD_ERR_PARAM;
  if (c.accumulate != 0 && c.accumulate != 1) return KD_ERR_PARAM;
  if (c.vocab_chunk != 0 && (c.vocab_chunk < 256 || c.vocab_chunk > (1 << 20) || c.vocab_chunk % 256)) return KD_ERR_PARAM;
  if (!(std::isfinite(loss_scale) && loss_scale != 0.f)) return KD_ERR_PARAM;
  return KD_OK;
}

kd_status read_params(const kd_ce_params* p, Call& c) {
  if (!p) return KD_ERR_NULL;
  c = Call{p->T, p->H, p->V, 1, p->in_dtype, p->grad_dtype, p->w_layout, p->index_dtype, KD_F32, KD_TAIL_DROP, 1,
           1.f, p->label_smoothing, p->z_loss, p->loss_scale, p->accumulate_grad_W, p->vocab_chunk};
  const kd_status s = check_call(c, p->loss_scale);
  if (s != KD_OK) return s;
  if (!(p->label_smoothing >= 0.f && p->label_smoothing < 1.f)) return KD_ERR_PARAM;
  if (!(p->z_loss >= 0.f && p->z_loss < INFINITY)) return KD_ERR_PARAM;
  return p->reserved == 0 ? KD_OK : KD_ERR_PARAM;
}

kd_status read_params(const kd_topk_params* p, Call& c) {
  if (!p) return KD_ERR_NULL;
  c = Call{p->T, p->H, p->V, p->K, p->in_dtype, p->grad_dtype, p->w_layout, p->index_dtype, p->top_dtype, p->tail, 0,
           p->tau, 0.f, 0.f, p->loss_scale * ((p->flags & KD_FLAG_TAU2) ? p->tau * p->tau : 1.f), p->accumulate_grad_W, p->vocab_chunk};
  const kd_status s = check_call(c, p->loss_scale);
  if (s != KD_OK) return s;
  if (p->top_dtype != KD_BF16 && p->top_dtype != KD_F32) return KD_ERR_PARAM;
  if (p->tail < KD_TAIL_RENORM || p->tail > KD_TAIL_DROP) return KD_ERR_PARAM;
  if (p->tail == KD_TAIL_REST && p->K >= p->V) return KD_ERR_SHAPE;        // nothing would be left to be the rest
  if (!(p->tau >= 1e-6f && p->tau <= 1e6f)) return KD_ERR_PARAM;           // also rejects NaN
  if (p->flags & ~(int32_t)KD_FLAG_TAU2) return KD_ERR_PARAM;
  return p->reserved[0] == 0 && p->reserved[1] == 0 ? KD_OK : KD_ERR_PARAM;
}

// Tile counts, vocabulary chunk, split factors and the workspace.  Depends on the params and on `backward` only.
void plan(const Call& c, HeadProblem& h, HeadLayout& L, bool backward) {
  Problem& q = h.p;
  Targets& t = h.t;
  q.T = (int)c.T; q.V = (int)c.V; q.H_s = (int)c.H; q.H_t = 0;
  q.tau = c.tau;
  q.grad_f32 = c.grad_dtype == KD_F32;
  q.accumulate_grad_W = c.accumulate;
  q.out_weight = c.weight;
  q.n_cu = kd::kNumCU;
  q.in_f32 = c.in_dtype == KD_F32;
  q.f32_parts = 1;
  q.w_hv = c.w_layout == KD_W_HV;
  q.head_rows = kd::kHeadRows;
  // fp32 gradients are exact to fp32: dL/dz is held as three bf16 parts, h and W, if they are fp32, as well.  bf16 gradients of fp32 operands:
  // one product of first parts, each factor rounded to bf16 as the result is
  q.dz_sets = !q.grad_f32 ? 1 : q.in_f32 ? 6 : 3;
  q.K_s = (int)round_up(q.in_f32 ? 6 * c.H : c.H, 64);
  q.prep_hs = 1;                                       // (the strip loop reads packed tokens)
  // rows off the 64-element grid: as for the two-model losses (kd_api.hip)
  q.prep_Ws = q.in_f32 || (q.K_s != q.H_s && (q.w_hv || q.T > 1536 || 2ll * q.V * q.K_s <= (4ll << 20)));
  q.w_hv_inplace = q.w_hv && !q.prep_Ws && q.V % 64 == 0 && q.V < (1 << 23);
  if (q.w_hv && !q.w_hv_inplace) q.prep_Ws = 1;
  q.T_pad = (int)round_up(q.T, kd::kTileN);
  q.n_tt = q.T_pad / kd::kTileN;
  q.strip = 1;
  q.n_vt = (q.V + kd::kHeadRows - 1) / kd::kHeadRows;
  int ns = 2 * ((q.n_cu + q.n_tt - 1) / q.n_tt);       // vocabulary ranges: as for the two-model losses
  if (ns < 32) ns = 32;
  if (ns > q.n_cu) ns = q.n_cu;
  const int units = (q.V + 63) / 64;
  q.n_split = ns < units ? ns : units;
  q.g_split = q.n_split;

  const int64_t v_all = round_up(q.V, 256);
  int64_t vc = c.vocab_chunk;
  if (vc == 0) {
    // From 4096 tokens on 32768 columns, twice what the two-model losses take: a chunk's ends weigh more beside one model's products.
    // (T = 4096, H = 1024, V = 151936 3908 -> 3860 us, H = 2048, V = 128256 6503 -> 6432, T = 8192, H = 2048 13956 -> 13676.)
    vc = q.T_pad >= 4096 ? 32768 : kd::choose_chunk(q, v_all, q.K_s);
    while (vc > 1024 && (int64_t)q.T_pad * q.dz_sets * vc * 2 > (512ll << 20)) vc = round_up(vc / 2, 256);
  }
  q.V_c = (int)(vc < v_all ? vc : v_all);
  q.gh_pairs = q.dz_sets;
  if (q.T <= kd::kFewHeadTokens) {                     // parts that fill all places for workgroups, of at least eight k-steps
    const int steps = ((q.V < q.V_c ? q.V : q.V_c) + 63) / 64, tiles = (q.H_s + 127) / 128 * q.dz_sets;
    int parts = kd::kFewGradHGroups / tiles;
    if (parts > steps / 8) parts = steps / 8;
    if (parts < 1) parts = 1;
    q.gh_rows = 128;
    q.ksteps_h = (steps + parts - 1) / parts;
    q.n_ksplit_h = (steps + q.ksteps_h - 1) / q.ksteps_h;
  } else {
    kd::plan_grad_h(q, false, q.dz_sets);
    if (q.dz_sets > 1 && (int64_t)q.n_ksplit_h * q.dz_sets * q.T * q.H_s * 4 > kPartialSums) {
      q.gh_pairs = 1;
      kd::plan_grad_h(q, false);
    }
  }

  // (the loop for few tokens keeps whole panels of 64 tokens, the strip loop whole tiles)
  const bool few = q.T <= kd::kFewHeadTokens && !q.w_hv_inplace && (q.prep_Ws || q.K_s == q.H_s);
  const int64_t kept_bytes = (few ? round_up(q.T, 64) : q.T_pad) * v_all * 4;
  const bool keeps = backward && q.V_c == v_all && kept_bytes <= kKept;
  h.few = few && (keeps || !backward);
  if (h.few) {
    const int units32 = (q.V + 31) / 32;
    h.parts = units32 < q.n_cu ? units32 : q.n_cu;
    q.strip = 0;                                       // (tokens as rows, where they lie if they are whole k-steps of bf16)
    q.prep_hs = q.in_f32 || q.K_s != q.H_s;
  }

  t.ce = c.ce; t.K = c.K; t.index64 = c.index_dtype == KD_I64; t.top_f32 = c.top_dtype == KD_F32; t.tail = c.tail;
  t.smoothing = c.smoothing; t.z_loss = c.z_loss;

  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (size_t)round_up((int64_t)(off + bytes), 256); return o; };
  L.meta = take(64);
  L.rowmap = take((size_t)q.T_pad * 4);
  L.inv = take((size_t)q.T * 4);
  L.row_loss = take((size_t)q.T_pad * 4);
  L.rowinfo = take((size_t)q.T_pad * 16);
  L.scale = take(4);
  L.valid = take((size_t)q.T);
  L.list = take((size_t)q.T * t.K * 4);
  L.q = take((size_t)q.T * t.K * 4);
  L.info = take((size_t)q.T * kd::kTargetInfo * 8);
  L.z = take((size_t)q.T_pad * t.K * 4);
  L.prep_h = q.prep_hs ? take((size_t)q.T_pad * q.K_s * 2) : 0;
  L.prep_W = q.prep_Ws ? take((size_t)q.V * q.K_s * 2) : 0;
  const size_t partial_bytes = (size_t)(h.few ? h.parts : q.n_split) * (c.smoothing > 0.f ? 3 : 2) * q.T_pad * 4;
  L.h_sT = backward ? take((size_t)round_up(q.H_s, 16) * q.T_pad * q.dz_sets * 2) : 0;      // (packed beside the merge of the partials)
  L.partials = off;                                    // read for the last time before the backward pass writes what lies there
  if (backward) {
    L.dz = take((size_t)q.T_pad * q.dz_sets * q.V_c * 2);
    L.gh32 = take((size_t)q.n_ksplit_h * q.gh_pairs * q.T * q.H_s * 4);
  } else {
    L.dz = L.gh32 = off;
  }
  const size_t end = (size_t)round_up((int64_t)(L.partials + partial_bytes), 256);
  if (off < end) off = end;
  L.kept = off;
  if (keeps) take((size_t)kept_bytes);
  L.total = off;
  h.kept = keeps ? reinterpret_cast<float*>(1) : nullptr;      // (the address: carve)
}

void carve(HeadProblem& h, const HeadLayout& L, void* ws) {
  Problem& q = h.p;
  Targets& t = h.t;
  char* const b = static_cast<char*>(ws);
  q.meta = reinterpret_cast<int*>(b + L.meta);
  q.rowmap = reinterpret_cast<int*>(b + L.rowmap);
  q.inv = reinterpret_cast<int*>(b + L.inv);
  q.row_loss = reinterpret_cast<float*>(b + L.row_loss);
  q.rowinfo = reinterpret_cast<float*>(b + L.rowinfo);
  q.partials = reinterpret_cast<float*>(b + L.partials);
  q.h_sT = b + L.h_sT;
  q.dz = b + L.dz;
  q.gh32 = reinterpret_cast<float*>(b + L.gh32);
  t.scale = reinterpret_cast<float*>(b + L.scale);
  q.out_scale = t.scale;
  t.valid = reinterpret_cast<uint8_t*>(b + L.valid);
  t.list = reinterpret_cast<int*>(b + L.list);
  t.q = reinterpret_cast<float*>(b + L.q);
  t.info = reinterpret_cast<double*>(b + L.info);
  t.z = reinterpret_cast<float*>(b + L.z);
  if (h.kept) h.kept = reinterpret_cast<float*>(b + L.kept);
  q.mask = h.few ? nullptr : t.valid;                  // which tokens the row map keeps
  q.user_h_s = q.h_s; q.user_W_s = q.W_s;
  if (q.prep_hs) q.h_s = b + L.prep_h;
  if (q.prep_Ws) q.W_s = b + L.prep_W;
}

#define KD_TRY(expr)                                \
  do {                                              \
    if ((expr) != hipSuccess) return KD_ERR_LAUNCH; \
  } while (0)

// The products that make grad_h: a copy of dL/dz by a part of W's rows (places of the prepared head: part 0 first, part 1 fourth,
// part 2 sixth).
constexpr int kPairSet6[6] = {0, 0, 3, 0, 5, 3}, kPairPlace6[6] = {0, 3, 0, 5, 0, 3};

kd::GradHPairs grad_h_pairs(const Problem& q) {
  kd::GradHPairs pairs{q.dz_sets, {}, {}};
  for (int i = 0; i < pairs.n; ++i) {
    pairs.set[i] = pairs.n == 6 ? kPairSet6[i] : i;
    pairs.at[i] = pairs.n == 6 ? kPairPlace6[i] * q.H_s : 0;
  }
  return pairs;
}

kd_status run(const HeadProblem& h, bool backward, hipStream_t st) {
  const Problem& q = h.p;
  if (!(h.few && h.t.ce)) KD_TRY(kd::launch_targets(h, st));
  KD_TRY(kd::launch_operands(q, !h.few, true, false, st));
  if (q.in_f32 && !q.w_hv) KD_TRY(kd::launch_head_split(h, st));
  KD_TRY(h.few ? kd::launch_head_few(h, st) : kd::launch_head_stats(h, st));
  KD_TRY(kd::launch_head_combine(h, backward, backward && q.grad_W_s, st));
  if (!backward) return KD_OK;
  for (int64_t v0 = 0; v0 < q.V; v0 += q.V_c) {
    const int width = (int)((q.V - v0 < q.V_c) ? q.V - v0 : q.V_c);
    KD_TRY(kd::launch_head_grad(h, (int)v0, width, st));
    if (q.grad_W_s) KD_TRY(kd::launch_grad_W_scaled(q, (int)v0, width, st));
    if (q.grad_h_s) {
      // all products in one launch, or, where their partial sums would take too much memory, each adding to those of the one before
      const kd::GradHPairs all = grad_h_pairs(q);
      if (q.gh_pairs > 1) KD_TRY(kd::launch_head_grad_h(q, (int)v0, width, v0 == 0, st, &all));
      else
        for (int i = 0; i < all.n; ++i) {
          const kd::GradHPairs one{1, {all.set[i]}, {all.at[i]}};
          KD_TRY(kd::launch_head_grad_h(q, (int)v0, width, v0 == 0 && i == 0, st, &one));
        }
    }
  }
  if (q.grad_h_s) KD_TRY(kd::launch_gradh_finish(q, st));
  return KD_OK;
}

kd_status prepare(const Call& c, const void* h, const void* W, const void* index, const void* top, const float* lse, const uint8_t* mask,
                  float* loss, float* per_token_loss, void* grad_h, void* grad_W, bool backward, void* workspace, size_t workspace_bytes,
                  HeadProblem& hp) {
  if (!h || !W || !index || !loss || !workspace) return KD_ERR_NULL;
  if (!c.ce && (!top || (c.tail != KD_TAIL_RENORM && !lse))) return KD_ERR_NULL;
  if (backward && !grad_h && !grad_W) return KD_ERR_NULL;
  if (!aligned16(h) || !aligned16(W) || !aligned16(grad_h) || !aligned16(grad_W)) return KD_ERR_ALIGN;
  auto aligned = [](const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  if (!aligned(index, c.index_dtype == KD_I64 ? 8 : 4) || !aligned(top, c.top_dtype == KD_F32 ? 4 : 2) || !aligned(lse, 4) ||
      !aligned(loss, 4) || !aligned(per_token_loss, 4) || !aligned(workspace, 256))
    return KD_ERR_ALIGN;
  HeadLayout L{};
  plan(c, hp, L, backward);
  if (workspace_bytes < L.total) return KD_ERR_WORKSPACE;
  Problem& q = hp.p;
  q.h_s = h; q.W_s = W;
  q.loss = loss; q.per_token_loss = per_token_loss;
  q.grad_h_s = grad_h; q.grad_W_s = grad_W;
  hp.t.index = index; hp.t.top = top; hp.t.lse = lse; hp.t.mask = mask;
  carve(hp, L, workspace);
  return KD_OK;
}

template <class Params>
kd_status workspace_size(const Params* params, size_t* bytes) {
  if (!bytes) return KD_ERR_NULL;
  Call c{};
  const kd_status s = read_params(params, c);
  if (s != KD_OK) return s;
  HeadProblem h{};
  HeadLayout L{};
  plan(c, h, L, true);
  size_t most = L.total;
  HeadProblem f{};
  plan(c, f, L, false);
  *bytes = most > L.total ? most : L.total;
  return KD_OK;
}

}  // namespace

extern "C" {

kd_status kd_ce_workspace_size(const kd_ce_params* params, size_t* bytes) { return workspace_size(params, bytes); }
kd_status kd_topk_workspace_size(const kd_topk_params* params, size_t* bytes) { return workspace_size(params, bytes); }

kd_status kd_ce_fwd(const kd_ce_params* params, const void* h, const void* W, const void* labels, const uint8_t* mask, float* loss,
                    float* per_token_loss, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Call c{};
  kd_status s = read_params(params, c);
  if (s != KD_OK) return s;
  HeadProblem hp{};
  s = prepare(c, h, W, labels, nullptr, nullptr, mask, loss, per_token_loss, nullptr, nullptr, false, workspace, workspace_bytes, hp);
  return s == KD_OK ? run(hp, false, static_cast<hipStream_t>(hip_stream)) : s;
}

kd_status kd_ce_fwd_bwd(const kd_ce_params* params, const void* h, const void* W, const void* labels, const uint8_t* mask, float* loss,
                        float* per_token_loss, void* grad_h, void* grad_W, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Call c{};
  kd_status s = read_params(params, c);
  if (s != KD_OK) return s;
  HeadProblem hp{};
  s = prepare(c, h, W, labels, nullptr, nullptr, mask, loss, per_token_loss, grad_h, grad_W, true, workspace, workspace_bytes, hp);
  return s == KD_OK ? run(hp, true, static_cast<hipStream_t>(hip_stream)) : s;
}

kd_status kd_topk_fwd(const kd_topk_params* params, const void* top_logits, const void* top_index, const float* lse, const void* h_s,
                      const void* W_s, const uint8_t* mask, float* loss, float* per_token_loss, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
  Call c{};
  kd_status s = read_params(params, c);
  if (s != KD_OK) return s;
  HeadProblem hp{};
  s = prepare(c, h_s, W_s, top_index, top_logits, lse, mask, loss, per_token_loss, nullptr, nullptr, false, workspace, workspace_bytes, hp);
  return s == KD_OK ? run(hp, false, static_cast<hipStream_t>(hip_stream)) : s;
}

kd_status kd_topk_fwd_bwd(const kd_topk_params* params, const void* top_logits, const void* top_index, const float* lse, const void* h_s,
                          const void* W_s, const uint8_t* mask, float* loss, float* per_token_loss, void* grad_h_s, void* grad_W_s,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  Call c{};
  kd_status s = read_params(params, c);
  if (s != KD_OK) return s;
  HeadProblem hp{};
  s = prepare(c, h_s, W_s, top_index, top_logits, lse, mask, loss, per_token_loss, grad_h_s, grad_W_s, true, workspace, workspace_bytes, hp);
  return s == KD_OK ? run(hp, true, static_cast<hipStream_t>(hip_stream)) : s;
}

}  // extern "C"
