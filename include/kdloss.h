/*
 * libkdloss - full-vocabulary knowledge-distillation loss, forward + backward,
 * for one AMD MI355X (gfx950).
 *
 * The operation (KDFlow paper, abstract and Sec. 3.2 "Efficient Communication
 * via Hidden States"): a student worker receives the teacher's final hidden
 * states h_t [T,H_t] instead of teacher logits, rebuilds the full teacher
 * logits with a frozen copy of the teacher output head,  z_t = h_t . W_t,
 * and aligns the student's logits  z_s = h_s . W_s  to them with one of the
 * divergences of Sec. 3.4 (forward KL, reverse KL, Jensen-Shannon).  The
 * student's backward pass (Sec. 3.1, StudentActorGroup) then needs
 * dL/dh_s and dL/dW_s.  This library is that computation and nothing else.
 *
 * Definitions (the paper names the divergences; these are the textbook forms
 * it refers to, natural logarithm, p = softmax(z / tau) for both models):
 *   FKL: l_t = KL(p_t || p_s)            RKL: l_t = KL(p_s || p_t)
 *   JSD: l_t = beta KL(p_t || M) + (1-beta) KL(p_s || M),  M = beta p_t + (1-beta) p_s
 *   n = sum_t mask_t,  loss = sum_t mask_t l_t / n   (0 when n == 0)
 *   grad_h_s = dL/dz_s . W_s^T,   grad_W_s = h_s^T . dL/dz_s
 * No tau^2 factor is applied.  Masked tokens are compacted away on the device before any
 * product is formed, so they cost nothing.  Logits are never stored: they are produced
 * vocabulary tile by vocabulary tile in registers, twice (three times for JSD,
 * TVD and the skewed KLs, whose row value needs both log-sum-exps first).
 *
 * Conventions of every entry point
 *  - plain C ABI; no exceptions, no allocation, no device synchronisation.  The
 *    caller owns every buffer.  The entry points of this header read no
 *    environment variable and keep no state from one call to the next, except
 *    that each kernel's launch attribute is set once per process and device, and
 *    that kd_loss_fwd_bwd_static works in a device array owned by the library.
 *    (The measurement aids of kdloss_bench.h keep a per-thread hook.)
 *  - all argument checks run on the host before anything touches the GPU, so
 *    they can be exercised on a machine without one.
 *  - work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is
 *    the default stream) and the call returns without waiting.  Only kernels are
 *    enqueued (no memsets, no copies), so a call may be captured into a HIP graph;
 *    the workspace carries nothing from one call to the next.
 */
#ifndef KDLOSS_H
#define KDLOSS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  KD_OK = 0,
  KD_ERR_NULL = 1,        /* a required pointer is NULL                          */
  KD_ERR_SHAPE = 2,       /* T, H_t, H_s or V < 1, or beyond the supported range */
  KD_ERR_ALIGN = 3,       /* pointer not 16-byte aligned, or H_t/H_s/V % 8 != 0  */
  KD_ERR_PARAM = 4,       /* tau outside [1e-6, 1e6] or not finite, unknown enum, beta outside (0,1) where it is used */
  KD_ERR_WORKSPACE = 5,   /* workspace_bytes smaller than kd_loss_workspace_size */
  KD_ERR_UNSUPPORTED = 6, /* valid request this build does not implement         */
  KD_ERR_LAUNCH = 7,      /* the HIP runtime refused a launch (see hipGetLastError) */
  KD_ERR_TOO_LARGE = 8    /* kd_loss_fwd_bwd_static only: the problem needs more scratch memory than
                             the library's static array holds (KD_STATIC_SCRATCH_BYTES) */
} kd_status;

/* Sec. 3.4 / Table 1: built-in divergence metrics.
 *   KD_TVD      = 1/2 sum_v |p_t - p_s|
 *   KD_SKEW_FKL = KL(p_t || a p_t + (1-a) p_s),  KD_SKEW_RKL = KL(p_s || (1-a) p_t + a p_s),
 *   with the skew weight a passed in `beta` (0 < a < 1; a -> 0 recovers FKL / RKL).
 *   KD_AKL      = w_f KL(p_t || p_s) + w_r KL(p_s || p_t), the adaptive KL of Table 1 (defined in the paper by
 *                 Wu et al. that the authors cite, not in the paper itself).  Per token the vocabulary is
 *                 split by the teacher: in descending order of p_t, the head is the longest prefix whose
 *                 cumulative teacher mass stays <= mu (the top entry always belongs to it), the tail the
 *                 rest; w_f = g_head / (g_head + g_tail), w_r = g_tail / (g_head + g_tail) with
 *                 g = sum |p_t - p_s| over the part (1/2 each if both vanish).  mu is passed in `beta`
 *                 (0 < mu < 1; the cited method uses 1/2).  The weights are constants for the gradient.
 *                 The head boundary is found by a search over teacher log-probabilities to within 5e-4
 *                 (base 2): entries that close to the boundary may fall on either side.  Costs two to four
 *                 more passes over the teacher logits and one more over both; not with the fp8 teacher. */
typedef enum { KD_FKL = 0, KD_RKL = 1, KD_JSD = 2, KD_TVD = 3, KD_SKEW_FKL = 4, KD_SKEW_RKL = 5, KD_AKL = 6 } kd_kind;

typedef enum { KD_BF16 = 0, KD_F32 = 1 } kd_dtype;

/* Storage order of an output head W (mathematical shape [H, V]):
 *   KD_W_HV: W[k * V + v]   (V contiguous)
 *   KD_W_VH: W[v * H + k]   (H contiguous; the order lm_head.weight is kept in)
 * The same order applies to W_t, W_s and grad_W_s.  KD_W_VH is the faster one (both logit operands
 * contiguous along the contraction; about 5 % ahead).  KD_W_HV heads are read in place when they are
 * bf16 with H_t, H_s and V multiples of 64; otherwise they are re-packed into the workspace (which then
 * holds copies of both heads) by a transposing pass on every call.  grad_W_s is written
 * in the caller's order either way.  With the fp8 teacher, KD_W_HV heads always take the re-packing path
 * (better: quantise the frozen head from a [V,H] copy once and pass KD_W_VH). */
typedef enum { KD_W_HV = 0, KD_W_VH = 1 } kd_wlayout;

/* KD_FLAG_TAU2: multiply the loss, the per-token losses and both gradients by tau^2 (the
 * convention that keeps gradient magnitudes independent of the temperature).  Off by default:
 * the paper does not mention it. */
/* KD_FLAG_TEACHER_FP8: h_t and W_t hold OCP e4m3 bytes (one per element) instead of in_dtype values,
 * quantised with one scale per array (kd_quantize_e4m3):  z_t = teacher_scale * sum_k q_h[t,k] q_W[v,k],
 * teacher_scale = scale_h * scale_W.  The teacher logit tiles then run on the fp8 matrix pipe at twice the
 * bf16 rate and half the operand traffic; everything else (student side, divergence, gradients) is unchanged.
 * An extension in the spirit of the paper's FP8 teacher inference (Table 3): the paper does not quantise the
 * head.  Requires in_dtype == KD_BF16 and H_t a multiple of 128.  In the multi-teacher
 * call every teacher is then fp8, each with its own scale (teacher_scales[k]; params->teacher_scale is not read). */
typedef enum { KD_FLAG_TAU2 = 1, KD_FLAG_TEACHER_FP8 = 2 } kd_flags;

typedef struct {
  int64_t T;            /* tokens (batch x sequence, flattened)                     */
  int64_t H_t, H_s;     /* teacher / student hidden sizes, multiples of 8           */
  int64_t V;            /* vocabulary size shared by both heads, multiple of 8      */
  int32_t in_dtype;     /* kd_dtype of h_t, W_t, h_s, W_s                           */
  int32_t grad_dtype;   /* kd_dtype of grad_h_s and grad_W_s                        */
  int32_t w_layout;     /* kd_wlayout                                               */
  int32_t kind;         /* kd_kind                                                  */
  float tau;            /* temperature, 1e-6 <= tau <= 1e6.  The scaled logits z / tau
                           are held in fp32: results are meaningful while |z| / tau
                           stays below about 1e5, and a loss far below 1e-4 (very
                           high temperatures) is resolved to about 1e-7 absolute    */
  float beta;           /* JSD mixing weight on the teacher term, the skew weight of
                           the skewed KLs, or AKL's head mass mu; 0 < beta < 1;
                           ignored for FKL/RKL/TVD                                  */
  int32_t accumulate_grad_W; /* 0: grad_W_s is overwritten. 1: added to (gradient
                           accumulation over micro-batches, Table 3 caption)        */
  int32_t flags;        /* bit set of kd_flags; other bits must be 0                */
  float teacher_scale;  /* KD_FLAG_TEACHER_FP8 only: > 0, finite                    */
  int32_t vocab_chunk;  /* columns of the vocabulary handled per backward chunk (the
                           width of the dL/dz_s staging buffer): 0 = chosen by the
                           library, else a multiple of 256 in [256, 2^20].  Enters
                           the size query and the call alike, so the two cannot
                           disagree.  Results do not depend on it beyond the
                           summation order of grad_h_s                              */
  float loss_scale;     /* finite, non-zero: factor on the loss, the per-token losses
                           and both gradients (1 = the plain masked mean; e.g. 1 /
                           micro-batches under gradient accumulation, or the
                           upstream gradient when it is known before the call)      */
  int32_t reserved;     /* must be 0 (KD_ERR_PARAM otherwise)                       */
} kd_loss_params;

/* Bytes of device workspace kd_loss_fwd_bwd needs for these parameters.
 * (Footnote of Sec. 1: shipping full logits would take about 160 GB per global
 * batch, 2 T V bytes per T tokens; this is what the recomputation needs instead.)
 * Host only.  The size is O(T * V_c + H_s * V_c + T * (H_t + H_s)) for a vocabulary
 * chunk V_c chosen by the library - staging of dL/dz_s, fp32 sums of grad_h_s,
 * compacted copies of the hidden states - plus copies of the heads only when they
 * must be re-packed (fp32 inputs; hidden sizes that are not multiples of 64, with more than 1536 tokens, small heads or KD_W_HV).  The
 * staging buffer (2 T V_c bytes, T rounded up to 256) takes at most 208 MiB below
 * 4096 tokens, which may be the whole vocabulary; from there on at most 16384
 * columns and 512 MiB, or 1024 columns.  It never grows like T * V.  Returns KD_OK or the status kd_loss_fwd_bwd would return for
 * the same params. */
kd_status kd_loss_workspace_size(const kd_loss_params* params, size_t* bytes);

/* Forward + backward of the distillation loss (paper Sec. 3.2 and 3.4; student
 * backward of Sec. 3.1).
 *
 *  h_t  [T, H_t]  device, read-only, row-major (H contiguous), in_dtype
 *  W_t  head of the teacher, device, read-only, in_dtype, order w_layout
 *  h_s  [T, H_s]  device, read-only
 *  W_s  head of the student, device, read-only
 *  mask [T] uint8 device, non-zero = token counts; NULL = every token counts
 *  loss            device, one float: the masked-mean divergence
 *  per_token_loss  device, [T] floats (l_t; 0 for masked tokens, which are never computed) or NULL
 *  grad_h_s [T, H_s] device, grad_dtype; rows of masked tokens are exactly 0
 *  grad_W_s device, grad_dtype, same order as W_s; overwritten or accumulated
 *  workspace       device, 256-byte aligned, workspace_bytes >= the size query
 *  hip_stream      hipStream_t
 *
 * Pointers must be 16-byte aligned.  Inputs must not alias outputs or the
 * workspace.  Results are bitwise reproducible from call to call (no floating
 * point atomics).  On any status other than KD_OK and KD_ERR_LAUNCH nothing
 * was enqueued. */
kd_status kd_loss_fwd_bwd(const kd_loss_params* params,
                          const void* h_t, const void* W_t,
                          const void* h_s, const void* W_s,
                          const uint8_t* mask,
                          float* loss, float* per_token_loss,
                          void* grad_h_s, void* grad_W_s,
                          void* workspace, size_t workspace_bytes,
                          void* hip_stream);

/* kd_loss_fwd_bwd for callers that cannot allocate device memory or have no workspace to pass: code
 * that runs under HIP graph capture, tight serving or training loops, harnesses that forbid hipMalloc.
 * Same arguments, checks, kernels and results as kd_loss_fwd_bwd, minus the workspace: the scratch memory
 * is a static device array of KD_STATIC_SCRATCH_BYTES inside the library (each GPU the library runs on
 * holds its own copy until the process ends).  The call allocates and frees nothing.
 *  - With params->vocab_chunk == 0 the library picks the widest vocabulary chunk whose plan fits the
 *    array; with a chunk given, that plan must fit.  Near the limit it takes a lean plan (fewer partial
 *    sums, the logit loop with the smaller copies) before a narrower chunk.  A problem that does not fit returns
 *    KD_ERR_TOO_LARGE and enqueues nothing (the headline workload, T = 4096, H_t = 4096, H_s = 1024,
 *    V = 151936, fits; T = 32768 with H_s = 4096 does not).
 *  - The array's address is looked up on the first call on each device (current device = the stream's);
 *    make that first call outside a graph capture.
 *  - Nothing in the array has to be zero or survive between calls, but every call on one GPU uses the
 *    same array: calls that overlap in time on one GPU (two streams, two threads) race.  Serialise them,
 *    or give the concurrent ones their own workspace through kd_loss_fwd_bwd. */
#define KD_STATIC_SCRATCH_BYTES ((size_t)128 << 20)
kd_status kd_loss_fwd_bwd_static(const kd_loss_params* params,
                                 const void* h_t, const void* W_t,
                                 const void* h_s, const void* W_s,
                                 const uint8_t* mask,
                                 float* loss, float* per_token_loss,
                                 void* grad_h_s, void* grad_W_s,
                                 void* hip_stream);

/* Forward only: loss and per-token loss, no gradients (the logit tiles are
 * produced once; twice for JSD).  Same arguments and checks as above. */
kd_status kd_loss_fwd(const kd_loss_params* params,
                      const void* h_t, const void* W_t,
                      const void* h_s, const void* W_s,
                      const uint8_t* mask,
                      float* loss, float* per_token_loss,
                      void* workspace, size_t workspace_bytes,
                      void* hip_stream);

/* Quantise n values to OCP e4m3 bytes (KD_FLAG_TEACHER_FP8):  dst[i] = e4m3(src[i] * (1 / scale)), the
 * reciprocal and the product in fp32, round to nearest even, magnitudes beyond 448 saturate, NaN -> 0x7f.
 * src: device, src_dtype (KD_BF16 or KD_F32), n values; dst: device, n bytes; both 16-byte aligned.
 * A good scale is max|src| / 448.  The frozen teacher head is quantised once, hidden states per batch. */
kd_status kd_quantize_e4m3(const void* src, int32_t src_dtype, int64_t n, float scale, void* dst,
                           void* hip_stream);

/* Multi-teacher distillation (Table 1, "Multi-Teacher Distillation"): n_teachers teachers over the
 * same tokens and vocabulary, each with its own hidden states h_t[k] [T, H_t[k]] and head W_t[k];
 *   loss = sum_k weights[k] * D(p_t^k, p_s)      (same divergence, temperature and mask for all)
 * and the gradients are those of that sum.  params->H_t is ignored; h_t, W_t, H_t, weights (and
 * teacher_scales, read only with KD_FLAG_TEACHER_FP8, else may be NULL) are HOST arrays of n_teachers
 * entries (the pointers in h_t / W_t are device pointers).  1 <= n_teachers <= 16.
 * Everything else is as for kd_loss_fwd_bwd; the workspace must satisfy the _multi size query (the
 * single-teacher workspace plus, per teacher, its row statistics and any re-packed operand copies).
 * The token compaction, the student operands and the two backward products are shared: each chunk of
 * dL/dz_s is summed over the teachers (in its bf16 staging buffer) before grad_W_s and grad_h_s are
 * formed once.  The student logit tiles are recomputed with every teacher's tiles. */
kd_status kd_loss_workspace_size_multi(const kd_loss_params* params, int n_teachers, const int64_t* H_t,
                                       size_t* bytes);
kd_status kd_loss_fwd_bwd_multi(const kd_loss_params* params, int n_teachers,
                                const void* const* h_t, const void* const* W_t, const int64_t* H_t,
                                const float* weights, const float* teacher_scales,
                                const void* h_s, const void* W_s, const uint8_t* mask,
                                float* loss, float* per_token_loss, void* grad_h_s, void* grad_W_s,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------------------------------------
 * Losses over one output head.
 *
 * What a distillation program computes beside the divergence of two models: the cross entropy of the labels
 * (kd_ce_*), and the divergence from a teacher of which only the largest logits were kept (kd_topk_*).  Same
 * conventions as above: plain C ABI, every buffer the caller's, no allocation, no synchronisation, only kernels
 * enqueued, nothing kept from call to call, results bitwise reproducible, all checks on the host before anything is
 * enqueued.  z = h W, logits produced tile by tile, and again for the gradients; where they are few (at most 160 MiB in
 * fp32), a call with gradients keeps them in its workspace instead.  Tokens that do not count are compacted away.
 *
 *  h       [T, H] device, in_dtype;  W: head in the order w_layout, in_dtype
 *  mask    [T] uint8 device, non-zero = token may count; NULL = every token may
 *  loss    device, one float: the mean over the n tokens that count, times loss_scale (0 when n == 0)
 *  per_token_loss  device, [T] floats (0 for tokens that do not count) or NULL
 *  grad_h [T, H], grad_W (order of W) device, grad_dtype; either may be NULL and is then not computed.  Rows of grad_h
 *          of tokens that do not count are exactly 0; grad_W is overwritten, or added to with accumulate_grad_W
 *  workspace  device, 256-byte aligned, workspace_bytes >= the size query for these parameters (one token more may need
 *          less: T = 256, H = 1024, V = 151936 keeps its logits and takes 268 MB, T = 257 takes 192; a program whose T
 *          varies asks for each size and takes the largest)
 * h, W, grad_h, grad_W must be 16-byte aligned, the other arrays to their elements.  Inputs must not alias outputs or
 * the workspace.
 *
 * fp32 operands are multiplied as three bf16 parts each (six products, 24 bits), and fp32 gradients are fp32 sums of
 * products in which dL/dz is held in three parts: fp32 results are as exact as fp32 arithmetic gives them.  (Infinite
 * weights need bf16 operands, where a logit of minus infinity is a row of probability 0; the parts of fp32 ones give NaN.)  For bf16
 * gradients dL/dz is rounded to bf16 once, without the factor loss_scale / n that all its entries share, and the sums
 * once more; of fp32 operands the products for bf16 gradients take h and W rounded to bf16 as well (losses do not). */

/* Type of labels and of vocabulary rows. */
typedef enum { KD_I32 = 0, KD_I64 = 1 } kd_index_dtype;

/* Cross entropy with labels:
 *   l_t = lse_t - (1-e) z[t, y_t] - (e / V) sum_v z[t, v] + z_loss lse_t^2,    lse_t = log sum_v exp(z[t, v])
 * with label smoothing e.  A token counts if the mask says so and its label is not negative (-100, say); a label of V or
 * more is never read: its token's loss, the loss and the gradients are NaN. */
typedef struct {
  int64_t T, H, V;            /* H and V multiples of 8                                          */
  int32_t in_dtype;           /* kd_dtype of h and W                                             */
  int32_t grad_dtype;         /* kd_dtype of grad_h and grad_W                                   */
  int32_t w_layout;           /* kd_wlayout                                                      */
  int32_t index_dtype;        /* kd_index_dtype of the labels                                    */
  float label_smoothing;      /* e, 0 <= e < 1                                                   */
  float z_loss;               /* >= 0, finite: weight of the squared log-sum-exp                 */
  float loss_scale;           /* finite, non-zero: factor on losses and gradients                */
  int32_t accumulate_grad_W;  /* 0 or 1                                                          */
  int32_t vocab_chunk;        /* as in kd_loss_params                                            */
  int32_t reserved;           /* must be 0                                                       */
} kd_ce_params;

kd_status kd_ce_workspace_size(const kd_ce_params* params, size_t* bytes);
kd_status kd_ce_fwd_bwd(const kd_ce_params* params, const void* h, const void* W, const void* labels,
                        const uint8_t* mask, float* loss, float* per_token_loss, void* grad_h, void* grad_W,
                        void* workspace, size_t workspace_bytes, void* hip_stream);
/* ... without gradients: -per_token_loss (loss_scale 1, no smoothing) are the labels' log-probabilities. */
kd_status kd_ce_fwd(const kd_ce_params* params, const void* h, const void* W, const void* labels, const uint8_t* mask,
                    float* loss, float* per_token_loss, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's top logits.  Per token K vocabulary rows top_index[t, k] and the teacher's logits
 * top_logits[t, k] there, in any order; a negative row, or a logit of minus infinity, is an entry that is not there (lists
 * shorter than K); entries of the same row add up.  With p = softmax(z / tau) and
 *   KD_TAIL_RENORM  q_k = softmax over the list of top_logits / tau             (lse is not read, may be NULL)
 *   KD_TAIL_REST    q_k = exp(top_logits[t, k] / tau - lse[t]),  lse[t] = log sum_v exp(z_t[t, v] / tau) over the teacher's
 *                   whole vocabulary; what the list does not hold, r = max(0, 1 - sum q), is one more category, which is
 *                   compared with the student's mass beside the list
 *   KD_TAIL_DROP    the same q without the rest (also for importance weights: top_logits = tau log w, lse = 0)
 * the loss of a token is  sum_k q_k (log q_k - log p_k)  (+ r (log r - log (1 - sum p_k)) with KD_TAIL_REST).
 * A token counts if the mask says so and its list is not empty; a row of V or more is never read: its token's loss, the
 * loss and the gradients are NaN, as for a logit of NaN. */
typedef enum { KD_TAIL_RENORM = 0, KD_TAIL_REST = 1, KD_TAIL_DROP = 2 } kd_tail;
#define KD_TOPK_MAX 1024

typedef struct {
  int64_t T, H, V;            /* H and V multiples of 8                                          */
  int32_t K;                  /* entries per token, 1 .. KD_TOPK_MAX, at most V (KD_TAIL_REST: V - 1) */
  int32_t in_dtype;           /* kd_dtype of h_s and W_s                                         */
  int32_t grad_dtype;         /* kd_dtype of grad_h_s and grad_W_s                               */
  int32_t w_layout;           /* kd_wlayout                                                      */
  int32_t index_dtype;        /* kd_index_dtype of top_index                                     */
  int32_t top_dtype;          /* kd_dtype of top_logits                                          */
  int32_t tail;               /* kd_tail                                                         */
  float tau;                  /* temperature, 1e-6 <= tau <= 1e6                                 */
  float loss_scale;           /* finite, non-zero: factor on losses and gradients                */
  int32_t accumulate_grad_W;  /* 0 or 1                                                          */
  int32_t flags;              /* KD_FLAG_TAU2 or 0                                               */
  int32_t vocab_chunk;        /* as in kd_loss_params                                            */
  int32_t reserved[2];        /* must be 0                                                       */
} kd_topk_params;

kd_status kd_topk_workspace_size(const kd_topk_params* params, size_t* bytes);
kd_status kd_topk_fwd_bwd(const kd_topk_params* params, const void* top_logits, const void* top_index, const float* lse,
                          const void* h_s, const void* W_s, const uint8_t* mask, float* loss, float* per_token_loss,
                          void* grad_h_s, void* grad_W_s, void* workspace, size_t workspace_bytes, void* hip_stream);
kd_status kd_topk_fwd(const kd_topk_params* params, const void* top_logits, const void* top_index, const float* lse,
                      const void* h_s, const void* W_s, const uint8_t* mask, float* loss, float* per_token_loss,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------------------------------------
 * Beside the losses: what a distillation program calls in front of them and behind them.
 *
 * A linear layer in e4m3 with a scale per block of 128 (teacher layers as they are stored for FP8 inference, or a student trained
 * in FP8), the top logits of a teacher as kd_topk_* reads them, tokens sampled from a student's logits, and the norm of all
 * gradients with clipping.  Same conventions as above: plain C ABI, every buffer the caller's, no allocation, no synchronisation,
 * only kernels enqueued, nothing kept from call to call, results bitwise reproducible, all checks on the host before anything is
 * enqueued.  Inputs must not alias outputs or the workspace, unless it is said. */

/* Blocks of a matrix [rows, cols] that share a scale: 1 x 128 (of a row) or 128 x 128; the last ones of a row or column may be
 * narrower.  Codes are OCP e4m3 bytes in rows of cols rounded up to a multiple of 16, zero behind the row's end; scales are
 * [rows, ceil(cols / 128)] or [ceil(rows / 128), ceil(cols / 128)] floats.  A block stands for codes times scale. */
typedef enum { KD_BLOCK_ROW = 0, KD_BLOCK_TILE = 1 } kd_block;

typedef struct {
  int64_t rows, cols;         /* 1 .. 2^24, 1 .. 2^22 (2^22 both with a transposed result)       */
  int64_t ld;                 /* elements from row to row of src, >= cols                        */
  int32_t src_dtype;          /* kd_dtype of src                                                 */
  int32_t block;              /* kd_block                                                        */
  int32_t reserved[2];        /* must be 0                                                       */
} kd_blocks_params;

/* Quantises a matrix in blocks:  scale = m / 448 with m = max(largest |src| of the block, 448 2^-126), code = e4m3(448 src / m):
 * 448 src, which is exact for bf16, and its quotient by m in fp32, each rounded once, then to nearest even.  A block that holds an infinity or a NaN has the scale NaN.
 * codes, scales: of src.  codes_t, scales_t: of its transpose [cols, rows] (KD_BLOCK_ROW: blocks along src's columns, with scales of
 * their own; KD_BLOCK_TILE: the same codes and scales).  Either pair may be NULL; src is read once for both.
 * src: aligned to its elements, codes to 16 bytes, scales to 4. */
kd_status kd_quantize_e4m3_blocks(const kd_blocks_params* params, const void* src, uint8_t* codes, float* scales, uint8_t* codes_t,
                                  float* scales_t, void* hip_stream);

/* Product of two matrices in blocks:
 *   out[m, n] = sum over blocks j of 128 columns  a_scale[m, j] b_scale[n or n / 128, j] sum_{k in j} a[m, k] b[n, k]
 * (the scaled blocks are summed in fp32, in an order that sizes and types fix.  A block's own products: for an fp32 result in
 * fp32, on the bf16 matrix pipe; for a bf16 result on the e4m3 pipe at twice the rate, which cuts products off at 2^-13 of the largest of their
 * group of eight: 1.5e-5 of a result of normal numbers, whose rounding to bf16 is 1.7e-3, and never more than 7 2^-13 of the groups' largest products - which a result
 * whose products cancel each other may be small beside: an fp32 result has none of it).
 * A linear layer y = x W^T is a = x, b = W; its gradients are grad_x: a = grad_y, b = W's transpose, grad_W: a = grad_y's transpose,
 * b = x's transpose. */
typedef struct {
  int64_t M, N, K;            /* a [M, K], b [N, K], out [M, N]; M, N 1 .. 2^24, K 1 .. 2^22     */
  int32_t in_dtype;           /* kd_linear_e4m3: kd_dtype of x                                   */
  int32_t out_dtype;          /* kd_dtype of out                                                 */
  int32_t b_block;            /* kd_block of b (a: KD_BLOCK_ROW); kd_linear_e4m3: KD_BLOCK_TILE   */
  int32_t accumulate;         /* 0: out is overwritten.  1: added to, in front of the rounding   */
  int32_t reserved[2];        /* must be 0                                                       */
} kd_linear_params;

/* Bytes of device workspace (256-byte aligned) that either call below needs for these parameters (in_dtype is read here as well). */
kd_status kd_linear_workspace_size(const kd_linear_params* params, size_t* bytes);
/* a, b: codes, 16-byte aligned; scales, out: aligned to their elements. */
kd_status kd_matmul_e4m3(const kd_linear_params* params, const uint8_t* a, const float* a_scales, const uint8_t* b, const float* b_scales,
                         void* out, void* workspace, size_t workspace_bytes, void* hip_stream);
/* out = x W^T with x [M, K] in in_dtype (row-major, aligned to its elements), quantised in the call (KD_BLOCK_ROW). */
kd_status kd_linear_e4m3(const kd_linear_params* params, const void* x, const uint8_t* w, const float* w_scales, void* out,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* The K largest logits of each row, as kd_topk_* takes them, in descending order, of equal ones the lower index first:
 *   top_logits [T, K] in the logits' type, top_index [T, K], lse [T] = log sum_v exp(logits[t, v] / tau) (may be NULL)
 * A logit of minus infinity is no entry: where a row has fewer than K others, the list ends with entries of index -1 and logit minus
 * infinity.  A NaN counts as larger than every number; the row's lse is then NaN (infinite where the row's largest logit is).  An empty row's lse is minus
 * infinity. */
typedef struct {
  int64_t T, V;               /* rows, entries of a row: 1 .. 2^22, 1 .. 2^24                    */
  int64_t ld;                 /* elements from row to row of logits, >= V                        */
  int32_t K;                  /* 1 .. KD_TOPK_MAX, at most V                                     */
  int32_t in_dtype;           /* kd_dtype of logits and top_logits                               */
  int32_t index_dtype;        /* kd_index_dtype of top_index                                     */
  float tau;                  /* 1e-6 <= tau <= 1e6                                              */
  int32_t reserved[2];        /* must be 0                                                       */
} kd_top_logits_params;

kd_status kd_top_logits_workspace_size(const kd_top_logits_params* params, size_t* bytes);
/* Arrays aligned to their elements. */
kd_status kd_top_logits(const kd_top_logits_params* params, const void* logits, void* top_logits, void* top_index, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/* One token per row of logits, from one given number u[t] in [0, 1):
 *   w_v = exp((logits[t, v] - largest) / temperature).  Entries in descending order of their logits, of equal ones the lower index
 *   first: kept are the first top_k (0: all); of those the fewest whose sum of w is at least top_p times the sum over all of them
 *   (1: all, at least one); of those the ones with w >= min_p (0: all).
 *   token[t] = the first kept v, in order of v, where the sum of the kept w up to and with v exceeds u[t] times the sum of all kept
 *   logp[t]  = log of w_token over that sum (may be NULL)
 * w and its sums are held in 64 bits: exp to 2^-39, and each w as a whole number of 2^-51, or of 2^-62 S where the row's sum S of w is above 2^11, so that which
 * token is drawn does not depend on the order of a sum, and a sum is off by at most V 2^-52 (or 2^-62 V S) by that; without a filter, where sums of w are rounded, by at most
 * V 2^-51 + 2^-34.  temperature 0: the first of the largest logits, logp 0.  A setting may be the
 * same for all rows (in params) or an array of one per row (temperature_rows, ... device pointers; NULL: params').  A logit of minus
 * infinity is never drawn.  token is -1 and logp NaN in a row without a finite logit, with a NaN or a logit of plus infinity,
 * and where u or a row's own setting is outside its range. */
typedef struct {
  int64_t T, V;               /* rows, entries of a row: 1 .. 2^22, 1 .. 2^24                    */
  int64_t ld;                 /* elements from row to row of logits, >= V                        */
  int32_t in_dtype;           /* kd_dtype of logits                                              */
  int32_t index_dtype;        /* kd_index_dtype of token                                         */
  float temperature;          /* 0, or 1e-6 .. 1e6                                               */
  int32_t top_k;              /* >= 0                                                            */
  float top_p;                /* 0 < top_p <= 1                                                  */
  float min_p;                /* 0 <= min_p <= 1                                                 */
  int32_t reserved[2];        /* must be 0                                                       */
} kd_sample_params;

/* The workspace has room for every filter, as arrays of settings are not known here: 4 bytes for every 8 to 64 logits and, where rows have more than 4096, 48 KB a row
 * for 1024 rows at most (512 rows of 151936: 35 MB). */
kd_status kd_sample_workspace_size(const kd_sample_params* params, size_t* bytes);
/* Arrays aligned to their elements. */
kd_status kd_sample(const kd_sample_params* params, const void* logits, const float* u, const float* temperature_rows,
                    const int32_t* top_k_rows, const float* top_p_rows, const float* min_p_rows, void* token, float* logp,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

/* Norm of n arrays taken together, and clipping:
 *   KD_NORM_L2   total = sum of squares, norm = sqrt(total)          KD_NORM_MAX   total = norm = largest magnitude
 *   kd_grad_clip: out = in min(1, max_norm / norm), in fp32, rounded once.
 * Sums are held in 64 bits.  Where the norm is not finite nothing is scaled (a program sees it in norm and skips the step); a norm of
 * NaN is one with a NaN among the elements.  grads, counts, dtypes, out: HOST arrays of n entries (device pointers, elements, kd_dtype);
 * an array may have 0 elements (its pointer is not read).  The calls read the host arrays before they return.
 * The arrays of one call must not overlap each other.
 *  total  device, one double.  A program whose gradients are spread over ranks adds up (KD_NORM_MAX: takes the largest of) the ranks'
 *         totals between the two calls.
 *  out, out_dtypes  where the clipped values go; out NULL, or out[i] == grads[i] with the same type: in place, where nothing is written
 *         if nothing has to be scaled
 *  norm   device, one float, or NULL; infinite where the norm is beyond fp32, also if it is finite in 64 bits (then everything is scaled) */
typedef enum { KD_NORM_L2 = 0, KD_NORM_MAX = 1 } kd_norm;
#define KD_GRADS_MAX 65536

kd_status kd_grad_norm_workspace_size(int32_t n, const int64_t* counts, size_t* bytes);
kd_status kd_grad_norm(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t norm_kind,
                       double* total, void* workspace, size_t workspace_bytes, void* hip_stream);
kd_status kd_grad_clip(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t norm_kind,
                       const double* total, double max_norm, void* const* out, const int32_t* out_dtypes, float* norm, void* hip_stream);

/* Static, NUL-terminated description of a status code (error reporting of this boundary; nothing of
 * the paper's). */
const char* kd_status_string(kd_status status);

/* For reports: the vocabulary chunk kd_loss_fwd_bwd uses for these params and the number of kernels
 * one call launches (counted as for a call with a mask, whose hidden states are compacted into the
 * workspace, and with four search passes for AKL, where one of the two logit loops needs three).  Either output pointer may be NULL.  Host only. */
kd_status kd_loss_plan_info(const kd_loss_params* params, int64_t* vocab_chunk,
                            int64_t* n_launches);

#ifdef __cplusplus
}
#endif
#endif /* KDLOSS_H */
