/*
 * kdtopk.h - C ABI of the fused, chunked top-K KL distillation loss for
 * AMD MI355X (gfx950).
 *
 * The operation is the "full chunked KL computation" of §3.2.3 and
 * Algorithm 1 of "Efficient Knowledge Distillation for LLMs: Offline Top-K
 * Logits and a Fused Chunked KL Loss": the student output projection
 * z = h W^T is fused into a forward KL against a cached top-K teacher, the
 * rows are processed in chunks of C_s tokens, and the [N, V] logit tensor is
 * never stored. Per token t (Eq. 1 and its decomposition Eq. 2 in §3.2):
 *
 *     l_t = sum_{k} p_tk log p_tk  -  sum_{k} p_tk y_t[idx_tk]  +  M_t log Z_t
 *
 * with y_t = z_t / tau, log Z_t = logsumexp_v y_tv, p_t = softmax over the K
 * cached entries of teacher_logit_t / tau and M_t = sum_k p_tk. The loss is the
 * mean of l_t over non-ignored tokens (§3, after Eq. 1). Gradients use the
 * closed form of Eq. (3) (§3.2.3): dL/dz_tv = g_t / tau (M_t q_tv - p_tv) with
 * q_t = softmax(y_t) and g_t = 1/N_valid for non-ignored tokens, 0 otherwise;
 * grad_hidden = G W and grad_W (+)= G^T h, as in Algorithm 1's backward.
 *
 * Conventions for every entry point:
 *   - All tensor pointers are DEVICE pointers, row-major, densely packed.
 *   - The caller allocates and owns every buffer, including the workspace.
 *     The library never allocates, frees, or keeps a pointer after return.
 *   - Work is enqueued asynchronously on `hip_stream` (a hipStream_t passed as
 *     void*, NULL = the default stream). kd_topk_kl_fwd_bwd never
 *     synchronises: read `loss` after synchronising the stream.
 *   - Every argument is checked on the host before anything is enqueued. On
 *     any error nothing is launched, no output is touched, and the function
 *     returns the error code.
 *   - Results are deterministic: identical inputs and chunk size give
 *     bitwise identical outputs (no floating-point atomics).
 *   - Calls are reentrant; concurrent calls need distinct workspaces.
 */
#ifndef KDTOPK_H
#define KDTOPK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KDTOPK_ABI_VERSION 5

typedef enum kd_status {
  KD_OK = 0,
  KD_ERR_NULL_PTR = 1,           /* a required pointer is NULL */
  KD_ERR_BAD_SHAPE = 2,          /* N < 0, D/V/K <= 0, K > V, K > 4096, or a size limit */
  KD_ERR_BAD_ARG = 3,            /* chunk <= 0, tau not finite or <= 0, flags */
  KD_ERR_UNSUPPORTED = 4,        /* dtype, D % 64 != 0, misaligned pointer */
  KD_ERR_WORKSPACE_TOO_SMALL = 5,
  KD_ERR_BAD_INDEX = 6,          /* a teacher index outside [0, V) or repeated */
  KD_ERR_DEVICE = 7              /* a HIP launch or runtime error */
} kd_status;

typedef enum kd_dtype {
  KD_F32 = 0,                    /* fp32 inputs; contractions at fp32 accuracy (each
                                    operand as the exact sum of three bf16 terms,
                                    bf16 MFMA, fp32 accumulate) and fp32 elsewhere.
                                    Operands below 1e-33 keep fewer than 24 bits */
  KD_BF16 = 1,                   /* bf16 inputs, bf16 MFMA, fp32 accumulate */
  KD_MX4 = 2                     /* hidden rows of kd_mx4_logits only: kd_mx4_write's
                                    codes and scales */
} kd_dtype;

/* Problem description (Algorithm 1's inputs: h, W, the support and C_s). */
typedef struct kd_problem {
  int64_t N;           /* tokens = rows of hidden; 0 <= N < 2^31            */
  int64_t D;           /* hidden size d; 64 <= D <= 65536, D % 64 == 0       */
  int64_t V;           /* vocabulary size; 1 <= V <= 1048576                 */
  int64_t chunk;       /* rows per chunk C_s; >= 1 (min(chunk, N) is used)   */
  int32_t K;           /* cached teacher entries per token; 1 <= K <= V, K <= 4096 */
  int32_t dtype;       /* kd_dtype of hidden, W and grad_hidden              */
  float temperature;   /* tau; finite and > 0                                */
  int32_t flags;       /* 0 or KD_FLAG_TEACHER_LOGPROBS | KD_FLAG_GRAD_HIDDEN_F32 */
} kd_problem;

/*
 * Teacher representation (§3.2). Default (flags = 0): teacher_logit holds
 * logits of the K cached entries; the teacher distribution is their softmax
 * over the K entries at temperature tau (retained mass M = 1).
 * KD_FLAG_TEACHER_LOGPROBS: teacher_logit holds the teacher's log-probabilities
 * over the full vocabulary at the K cached entries (the partial-mass cache of
 * §3.2): p = exp(value) as given, M = sum_k p <= 1, no renormalisation and no
 * temperature (tau still divides the student's logits). Values must be <= 0
 * and sum_k exp(value) <= 1; this is not checked.
 */
#define KD_FLAG_TEACHER_LOGPROBS 1

/*
 * KD_FLAG_GRAD_HIDDEN_F32: grad_hidden is written as fp32 whatever the
 * problem's dtype (kd_topk_kl_fwd_bwd and kd_topk_kl_bwd), so that a caller
 * who scales it later (kd_scale_grads) rounds to the hidden dtype only once.
 * The pointer's buffer is then [N, D] fp32.
 */
#define KD_FLAG_GRAD_HIDDEN_F32 2

/*
 * Bytes of device workspace kd_topk_kl_fwd_bwd, kd_topk_kl_fwd and
 * kd_topk_kl_bwd need for problem *p. Pure host
 * function: touches no device. The size is O(N/4 + G C_s (V + K + 1) + D G C_s),
 * with G C_s <= 16384 the tokens whose dZ rows one grad_W contraction
 * gathers (at most 4 GiB of them), plus at most 128 MiB for the partial tiles
 * of grad_hidden's and grad_W's contractions when their tiles leave the last
 * round of the compute units partly filled: it grows with N only through an
 * array of loss partials (one per 4 tokens), never as N*V.
 * Errors: KD_ERR_NULL_PTR if p or bytes is NULL; the shape/argument errors of
 * kd_topk_kl_fwd_bwd otherwise.
 */
kd_status kd_topk_kl_workspace_size(const kd_problem* p, size_t* bytes);

/*
 * Fused chunked top-K KL forward + backward (§3.2.3, Algorithm 1, Eqs. 1-3).
 *
 *   hidden        [N, D] dtype        student hidden states h (row t = token t)
 *   W             [V, D] dtype        output projection
 *   teacher_idx   [N, K] int32        support S_t: K indices in [0, V) per
 *                                     row (not range-checked here unless
 *                                     KD_DEBUG_CHECK=1; see
 *                                     kd_topk_kl_check_indices). An index
 *                                     outside [0, V) is skipped; an index
 *                                     repeated in a row counts once with the
 *                                     sum of the repeated entries'
 *                                     probabilities (the dense teacher row
 *                                     of §3.2.1)
 *   teacher_logit [N, K] fp32         teacher logits of the support; the
 *                                     teacher distribution is their softmax
 *                                     over the K entries at temperature tau
 *                                     (log-probabilities with
 *                                     KD_FLAG_TEACHER_LOGPROBS)
 *   ignore        [N] uint8 or NULL   nonzero = token excluded from the loss
 *                                     and from the mean's count; NULL = none
 *   loss          [1] fp32            out: mean of l_t over non-ignored
 *                                     tokens (0 if there are none)
 *   loss_per_token [N] fp32 or NULL   out: l_t (0 on ignored tokens)
 *   grad_hidden   [N, D] dtype or NULL  out: dL/dh (fp32 with
 *                                     KD_FLAG_GRAD_HIDDEN_F32); NULL skips
 *                                     its GEMMs
 *   grad_W        [V, D] fp32 or NULL   out: dL/dW; NULL skips its GEMMs
 *   accumulate_grad_W  0: grad_W = dL/dW;  1: grad_W += dL/dW (micro-batch
 *                                     accumulation)
 *   workspace, workspace_bytes        device scratch of at least
 *                                     kd_topk_kl_workspace_size bytes,
 *                                     16-byte aligned
 *   hip_stream                        hipStream_t or NULL
 *
 * Schedule: with grad_hidden or grad_W requested, each chunk is projected
 * once. A chunk's log Z is complete once its own projection has run, and the
 * upstream gradient of the mean is known up front, so the projection that
 * yields the normaliser also yields the gradient, stored up to a factor per
 * token that the dH and dW contractions apply once log Z is merged, in place
 * of Algorithm 1's logit recompute (which the split entry points below
 * keep). The transient [chunk, V] buffer is the same one; nothing of size
 * N x V exists. The stream's device must be the current device.
 *
 * With an ignore mask, the ignored tokens take no part in the contractions
 * (with or without gradients requested, and likewise in kd_topk_kl_fwd and
 * kd_topk_kl_bwd): their loss terms and gradient rows
 * are 0 (Eq. 3 weights every row of G by its mask), so each group of up to
 * 16384 tokens is first compacted to its tokens that are not ignored, the
 * projection, dH and dW run over those only (the count stays on the device:
 * no host synchronisation), and the ignored tokens' loss_per_token entries
 * and grad_hidden rows are written as 0. The results are those of the
 * uncompacted computation up to the order of fp32 sums.
 *
 * Pointers hidden, W, grad_hidden, grad_W and workspace must be 16-byte
 * aligned (KD_ERR_UNSUPPORTED otherwise). hidden, W, teacher_idx,
 * teacher_logit and loss are required (KD_ERR_NULL_PTR); with N == 0 only
 * loss (and grad_W when given) are written. Launch failures return
 * KD_ERR_DEVICE; work enqueued before the failure may have run.
 */
kd_status kd_topk_kl_fwd_bwd(const kd_problem* p,
                             const void* hidden,
                             const void* W,
                             const int32_t* teacher_idx,
                             const float* teacher_logit,
                             const uint8_t* ignore,
                             float* loss,
                             float* loss_per_token,
                             void* grad_hidden,
                             float* grad_W,
                             int accumulate_grad_W,
                             void* workspace,
                             size_t workspace_bytes,
                             void* hip_stream);

/*
 * Forward only: the loss of Algorithm 1's two forward passes (normaliser, then
 * the loss; §3.2.3), without any gradient work, plus the per-token
 * log-normaliser the backward needs.
 *
 *   hidden, W, teacher_idx, teacher_logit, ignore   as for kd_topk_kl_fwd_bwd
 *   loss          [1] fp32            out: mean of l_t over non-ignored tokens
 *   loss_per_token [N] fp32 or NULL   out: l_t (0 on ignored tokens)
 *   saved_logz    [N] fp32            out: log Z_t = logsumexp_v z_tv / tau
 *                                     (0 on ignored tokens, which are left
 *                                     out as in kd_topk_kl_fwd_bwd)
 *   workspace, workspace_bytes, hip_stream   as for kd_topk_kl_fwd_bwd
 *
 * One projection per chunk (the normaliser and the student logits at the
 * teacher entries come from the same tile). Values are bitwise identical to
 * the corresponding outputs of kd_topk_kl_fwd_bwd called without gradients.
 * Errors as for kd_topk_kl_fwd_bwd; saved_logz is required.
 */
kd_status kd_topk_kl_fwd(const kd_problem* p,
                         const void* hidden,
                         const void* W,
                         const int32_t* teacher_idx,
                         const float* teacher_logit,
                         const uint8_t* ignore,
                         float* loss,
                         float* loss_per_token,
                         float* saved_logz,
                         void* workspace,
                         size_t workspace_bytes,
                         void* hip_stream);

/*
 * Backward only (Algorithm 1's backward: per chunk the logits are recomputed,
 * q_t = exp(z_t / tau - log Z_t) with log Z_t from the forward, Eq. 3, then
 * grad_hidden = G W and grad_W (+)= G^T h).
 *
 *   hidden, W, teacher_idx, teacher_logit, ignore   as for the forward call
 *   saved_logz    [N] fp32            log Z_t written by kd_topk_kl_fwd (read
 *                                     for the tokens not ignored)
 *   grad_loss     [1] fp32 or NULL    upstream gradient of the mean loss
 *                                     (device scalar); NULL = 1
 *   grad_loss_per_token [N] fp32 or NULL   upstream gradients u_t of the
 *                                     per-token losses; when given, G uses
 *                                     g_t = u_t (ignored tokens 0) instead of
 *                                     grad_loss / N_valid
 *   grad_hidden   [N, D] dtype (fp32 with KD_FLAG_GRAD_HIDDEN_F32) or NULL,
 *   grad_W        [V, D] fp32 or NULL,
 *   accumulate_grad_W                 as for kd_topk_kl_fwd_bwd
 *
 * With grad_loss = NULL and no per-token gradients the results equal
 * kd_topk_kl_fwd_bwd's gradients up to the rounding of log Z through fp32.
 * Errors as for kd_topk_kl_fwd_bwd; saved_logz is required.
 */
kd_status kd_topk_kl_bwd(const kd_problem* p,
                         const void* hidden,
                         const void* W,
                         const int32_t* teacher_idx,
                         const float* teacher_logit,
                         const uint8_t* ignore,
                         const float* saved_logz,
                         const float* grad_loss,
                         const float* grad_loss_per_token,
                         void* grad_hidden,
                         float* grad_W,
                         int accumulate_grad_W,
                         void* workspace,
                         size_t workspace_bytes,
                         void* hip_stream);

/*
 * Checks that every teacher index lies in [0, V) and that no row repeats an
 * index (the support S_t of §3.2 is a set; the loss accepts repeats and sums
 * them, but a top-K cache never repeats an index, so a repeat points at a
 * broken cache). Synchronises `hip_stream`.
 * Returns KD_OK, KD_ERR_BAD_INDEX, or an argument/device error. Uses the
 * first 256 bytes of `workspace` (KD_ERR_WORKSPACE_TOO_SMALL if it has fewer),
 * whatever the problem's D, chunk and dtype.
 *
 * Debug mode: with the environment variable KD_DEBUG_CHECK set to 1 when a
 * call is made, kd_topk_kl_fwd_bwd, kd_topk_kl_fwd and kd_topk_kl_bwd run
 * this check first (synchronising their stream, so the call is no longer
 * asynchronous) and return KD_ERR_BAD_INDEX with nothing else enqueued and no
 * output touched when it fails. Without it, indices are not checked.
 */
kd_status kd_topk_kl_check_indices(const kd_problem* p,
                                   const int32_t* teacher_idx,
                                   void* workspace,
                                   size_t workspace_bytes,
                                   void* hip_stream);

/*
 * kd_topk_kl_fwd_bwd for callers that cannot allocate device memory (code
 * being captured into a HIP graph, tight serving loops, harnesses that forbid
 * allocation): the same arguments without the workspace. The workspace is a
 * static per-device array inside the library, KD_SCRATCH_BYTES and 8 MiB for
 * partial sums that do not count against it, which each device the library runs
 * on holds from the first use of the library on that
 * device until the process ends; the call itself allocates nothing (no
 * hipMalloc, no events, no allocating library routine) and only enqueues
 * kernels on hip_stream. The caller still provides every output.
 *
 * The plan is kd_topk_kl_fwd_bwd's when its workspace fits the array: results
 * are then bitwise identical to kd_topk_kl_fwd_bwd's. Otherwise fewer chunks'
 * dZ rows are gathered per grad_W contraction, and the contractions may be split
 * into fewer ranges (every output may then differ in the order of its fp32
 * sums); if one chunk's workspace does not fit (about
 * chunk * V * (element size) bytes plus small terms), the call returns
 * KD_ERR_WORKSPACE_TOO_SMALL before touching the device: use a smaller chunk.
 *
 * Every call on a device shares that device's array, and calls keep no state
 * in it (nothing in it has to start at zero; each call writes what it reads).
 * Calls that overlap in time on one device (two streams, two threads) race on
 * the array and give wrong results: order them on one stream. With
 * KD_DEBUG_CHECK=1 the index check synchronises the stream, as for the other
 * entry points. Errors as for kd_topk_kl_fwd_bwd, plus KD_ERR_WORKSPACE_TOO_SMALL
 * as above and KD_ERR_DEVICE if the array's address cannot be obtained.
 */
#define KD_SCRATCH_BYTES (256u << 20)

kd_status kd_topk_kl_fwd_bwd_noalloc(const kd_problem* p,
                                     const void* hidden,
                                     const void* W,
                                     const int32_t* teacher_idx,
                                     const float* teacher_logit,
                                     const uint8_t* ignore,
                                     float* loss,
                                     float* loss_per_token,
                                     void* grad_hidden,
                                     float* grad_W,
                                     int accumulate_grad_W,
                                     void* hip_stream);

/*
 * Scales the gradients of the mean loss by the upstream gradient g of that
 * mean, a device fp32 scalar: Algorithm 1's backward forms G = (M g) q - p g
 * (§3.2.3); the loss is linear in g, so the gradients kd_topk_kl_fwd_bwd
 * computed with g = 1 become those for any g by one multiplication. For a
 * caller (an autograd function) that runs the fused call in its forward,
 * before g is known: with KD_FLAG_GRAD_HIDDEN_F32 both gradients come out of
 * the fused call in fp32, and each is rounded once, here, to its dtype.
 *
 *   grad_loss        [1] fp32                g (device)
 *   grad_hidden_f32  [n_hidden] fp32 or NULL  input: dL/dh of the mean
 *   grad_hidden_out  [n_hidden] hidden_dtype or NULL   out: g * input
 *   grad_W_f32       [n_W] fp32 or NULL       input: dL/dW of the mean
 *   grad_W_out       [n_W] w_dtype or NULL    out: g * input
 *   hip_stream                                hipStream_t or NULL
 *
 * Each output is rounded once to its dtype (KD_F32 or KD_BF16). An fp32
 * output may be its input itself (in place); otherwise output and input must
 * not overlap. A NULL pair (or a zero count) skips that gradient. grad_hidden
 * comes first where one pair's buffers overlap what the other writes.
 * Asynchronous on hip_stream. Errors, all detected before any launch:
 * KD_ERR_NULL_PTR (grad_loss NULL, or one of a pair NULL), KD_ERR_BAD_SHAPE
 * (a negative count), KD_ERR_UNSUPPORTED (an output dtype other than KD_F32
 * or KD_BF16, or a pointer not 16-byte aligned), KD_ERR_BAD_ARG (an output
 * overlapping its input other than in place); KD_ERR_DEVICE (launch).
 */
kd_status kd_scale_grads(const float* grad_loss,
                         const float* grad_hidden_f32,
                         int32_t hidden_dtype,
                         void* grad_hidden_out,
                         int64_t n_hidden,
                         const float* grad_W_f32,
                         int32_t w_dtype,
                         void* grad_W_out,
                         int64_t n_W,
                         void* hip_stream);

/*
 * Cross entropy against labels, the other half of a distillation run's objective:
 * the same projection, chunks and gradients for a target of one entry a token.
 *
 *     l_t = ln Z_t - z_t[label_t] + z_loss (ln Z_t)^2
 *
 * (the last term, the "z-loss", keeps the normaliser near 1; z_loss = 0 leaves it
 * out), the loss their mean over the tokens whose label is in [0, V); tokens with
 * another label (-100, say) are ignored as the loss above ignores them. Gradients:
 * dL/dz_tv = g_t ((1 + 2 z_loss ln Z_t) q_tv - [v = label_t]), grad_hidden = G W,
 * grad_W (+)= G^T h. (The weight 1 + 2 z_loss ln Z_t is held 2^-24 away from 0.)
 */
typedef struct kd_label_problem {
  int64_t N, D, V, chunk;  /* as in kd_problem                                 */
  int32_t dtype;           /* kd_dtype of hidden, W and grad_hidden             */
  float z_loss;            /* finite and >= 0                                   */
  int32_t flags;           /* 0 or KD_FLAG_GRAD_HIDDEN_F32 (with a part for
                              grad_W too: see kd_cross_entropy_fwd_bwd)         */
} kd_label_problem;

/* Workspace of the three calls below: kd_topk_kl_workspace_size's for K = 1, and 9
 * bytes a token. */
kd_status kd_cross_entropy_workspace_size(const kd_label_problem* p, size_t* bytes);

/*
 * kd_topk_kl_fwd_bwd, kd_topk_kl_fwd and kd_topk_kl_bwd for labels: loss and
 * gradients with one projection a chunk; the loss with the log-normaliser; the
 * gradients from it. labels [N] int64 (8-byte aligned) take the place of the
 * teacher's arrays and the mask; the other arguments, their results on ignored tokens,
 * and the errors are those calls' (KD_ERR_BAD_ARG also for z_loss). KD_DEBUG_CHECK
 * has nothing to check here.
 *
 * In bf16 the entries of dL/dz are held in bf16 on their way into the gradients, and with
 * one projection the hidden rows are rounded to bf16 once more for grad_W. With
 * KD_FLAG_GRAD_HIDDEN_F32, kd_cross_entropy_fwd_bwd keeps this off each token's label:
 * its part of both gradients (of grad_W alone too, with grad_hidden NULL) is formed in
 * fp32. Without the flag results are bitwise kd_topk_kl_fwd_bwd's for a teacher of one
 * entry.
 */
kd_status kd_cross_entropy_fwd_bwd(const kd_label_problem* p, const void* hidden, const void* W,
                                   const int64_t* labels, float* loss, float* loss_per_token,
                                   void* grad_hidden, float* grad_W, int accumulate_grad_W,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);
kd_status kd_cross_entropy_fwd(const kd_label_problem* p, const void* hidden, const void* W,
                               const int64_t* labels, float* loss, float* loss_per_token,
                               float* saved_logz, void* workspace, size_t workspace_bytes,
                               void* hip_stream);
kd_status kd_cross_entropy_bwd(const kd_label_problem* p, const void* hidden, const void* W,
                               const int64_t* labels, const float* saved_logz,
                               const float* grad_loss, const float* grad_loss_per_token,
                               void* grad_hidden, float* grad_W, int accumulate_grad_W,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Operators around the loss ------------------------------------------
 * The conventions above hold for them too (device pointers, the caller's
 * buffers, checks before anything is enqueued, one stream, the same bits from
 * the same inputs). They allocate nothing and never synchronise, so they may be
 * captured into a HIP graph; calls that overlap in time need workspaces of their
 * own. An output or the workspace overlaps no other buffer of the call.
 * kd_profile_enable times the loss's kernels only.
 *
 * Logits rows are [N, ld] with V <= ld columns used (the rest is never read),
 * and may start at any element boundary. A logit that is not a number counts
 * as -inf everywhere below; +inf is the largest value.
 */

/* Rows of logits of which the K largest are wanted. */
typedef struct kd_rows {
  int64_t N;           /* rows; 0 <= N < 2^31                                */
  int64_t V;           /* vocabulary size; 1 <= V <= 1048576                 */
  int64_t ld;          /* elements between rows; V <= ld <= 2^31             */
  int32_t K;           /* 1 <= K <= V, K <= 4096                             */
  int32_t dtype;       /* kd_dtype of the logits                             */
  int32_t flags;       /* 0 or KD_FLAG_TEACHER_LOGPROBS                      */
} kd_rows;

/*
 * Bytes of device workspace kd_topk_entries and kd_teacher_cache_write need: at
 * most 64 MiB (or one row's, up to 72 KiB) and small terms. Pure host function.
 */
kd_status kd_topk_entries_workspace_size(const kd_rows* p, size_t* bytes);

/*
 * The K largest logits of each row, as the loss takes them: the target of a
 * teacher that runs beside the student, or the proposal of a drafting student.
 *
 *   logits   [N, ld] dtype
 *   idx      [N, K] int32  out: vocabulary indices, largest logit first, of
 *                          equal ones the lowest index first
 *   value    [N, K] fp32   out: the logits; with KD_FLAG_TEACHER_LOGPROBS the
 *                          log-probabilities over the whole vocabulary
 *                          (z - log sum exp z; -inf in a row of -inf only)
 *   workspace, workspace_bytes   at least kd_topk_entries_workspace_size bytes,
 *                          16-byte aligned
 *
 * A row with fewer than K logits above -inf has its list filled with -inf at
 * the lowest indices of such columns. The loss is not a number for a row whose
 * entries are all -inf (value[n, 0] = -inf: it has no target and has to be ignored
 * there, as kd_teacher_cache_read marks it) or hold +inf. Errors: KD_ERR_NULL_PTR, KD_ERR_BAD_SHAPE,
 * KD_ERR_BAD_ARG (flags), KD_ERR_UNSUPPORTED (dtype, a pointer that is not
 * aligned to its elements, workspace not to 16 bytes),
 * KD_ERR_WORKSPACE_TOO_SMALL, KD_ERR_DEVICE.
 */
kd_status kd_topk_entries(const kd_rows* p, const void* logits, int32_t* idx, float* value,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The same selection written to a teacher cache at half the bytes: an entry is
 * index << 12 | code, and a row has a scale (top, step):
 *   value of an entry = top - code * step, code 0..4094; code 4095 = no entry.
 * step = (largest - least kept logit) / 4094 in fp32, so a kept value is off by
 * at most step / 2 before it is rounded to fp32 (where the kept logits lie within
 * 2^-125, whose step fp32 cannot hold, by at most that range). Entries that are -inf or more than 1024 below the row's
 * largest (whose probability is 0 at every temperature up to 9) are not
 * kept: their code is 4095. top is the largest logit, or its log-probability
 * with KD_FLAG_TEACHER_LOGPROBS; -inf marks a row that keeps nothing. Infinite
 * logits are stored as the largest finite number.
 *
 *   entries  [N, K] uint32   out
 *   scale    [N, 2] fp32     out
 *
 * Arguments and errors as for kd_topk_entries. A part of a larger cache is
 * written through pointers to its first row.
 */
kd_status kd_teacher_cache_write(const kd_rows* p, const void* logits, uint32_t* entries,
                                 float* scale, void* workspace, size_t workspace_bytes,
                                 void* hip_stream);

/*
 * Rows of a teacher cache as the loss takes them.
 *
 *   entries [N, K] uint32, scale [N, 2] fp32   the cache (N K may pass 2^32)
 *   rows          [M] int64 or NULL   the cache row of each token; NULL: row m
 *                                     (then M <= N). A row may be named twice
 *   teacher_idx   [M, K] int32        out: indices
 *   teacher_logit [M, K] fp32         out: top - code * step, rounded once;
 *                                     -inf for an entry that was not kept
 *   ignore        [M] uint8 or NULL   out: 1 for a token without a target (a
 *                                     cache row that keeps nothing, or a row
 *                                     number outside [0, N)), else 0. Such a
 *                                     token's indices are -1 and its logits 0
 *
 * The three outputs are the loss's arguments of these names (a token without a
 * target has to be ignored there). Errors: KD_ERR_NULL_PTR, KD_ERR_BAD_SHAPE
 * (N or M < 0, M >= 2^31, K outside 1..4096, M > N without rows),
 * KD_ERR_UNSUPPORTED (alignment to the elements), KD_ERR_DEVICE.
 */
kd_status kd_teacher_cache_read(int64_t N, int32_t K, const uint32_t* entries, const float* scale,
                                const int64_t* rows, int64_t M, int32_t* teacher_idx,
                                float* teacher_logit, uint8_t* ignore, void* hip_stream);

/*
 * Hidden states in 8 bits, held from a forward to its backward: 1.03 bytes an
 * element instead of 2 or 4. Each block of 32 consecutive columns has one byte s
 * as scale 2^(s - 127) and its elements as e4m3 codes, rounded to nearest even:
 * 4 significant bits, off by at most 2^-4 of the element, or by 2^-10 of the
 * scale where the element is below 2^-6 of it. The scale is the least power of
 * two, at least 2^-127, that leaves the block's largest magnitude at 448 or
 * below. (The last 1/32 of the types' range, which would round to 2^128, is held
 * as 1.875 2^127.) A block with an element that is infinite or not a number has s = 255
 * and reads back as not a number.
 *
 *   hidden   [N, D] dtype; D a multiple of 32, 32 <= D <= 65536
 *   codes    [N, D] uint8, scales [N, D / 32] uint8
 *
 * kd_checkpoint_read gives the values back in either dtype (exact in both above
 * 2^-133). hidden and codes 16-byte aligned. Errors: KD_ERR_NULL_PTR,
 * KD_ERR_BAD_SHAPE, KD_ERR_UNSUPPORTED (dtype, D % 32, alignment),
 * KD_ERR_DEVICE.
 */
kd_status kd_checkpoint_write(int64_t N, int64_t D, int32_t dtype, const void* hidden,
                              uint8_t* codes, uint8_t* scales, void* hip_stream);
kd_status kd_checkpoint_read(int64_t N, int64_t D, int32_t dtype, const uint8_t* codes,
                             const uint8_t* scales, void* hidden, void* hip_stream);

/*
 * The loss's backward from such a checkpoint: kd_topk_kl_bwd with the hidden rows
 * h^ that the codes stand for. The gradient is the loss's own at h^: log Z is
 * formed again from h^ (a log Z of the exact rows would leave the
 * probabilities of a confident token summing to something other than 1, and a
 * gradient where there is none), in the same projection as the gradient, so the
 * three contractions of kd_topk_kl_fwd_bwd run and no saved log Z is needed. With
 * grad_loss = NULL and no per-token gradients the results are bitwise those of
 * kd_topk_kl_fwd_bwd on the rows of kd_checkpoint_read.
 *
 *   codes, scales     [N, D], [N, D / 32] uint8   kd_checkpoint_write's; the
 *                                     problem's dtype is that of W, grad_hidden and
 *                                     the decoded rows. codes 16-byte aligned
 *   the other arguments, the workspace and the errors as for kd_topk_kl_bwd
 */
kd_status kd_topk_kl_bwd_checkpoint(const kd_problem* p,
                                    const uint8_t* codes,
                                    const uint8_t* scales,
                                    const void* W,
                                    const int32_t* teacher_idx,
                                    const float* teacher_logit,
                                    const uint8_t* ignore,
                                    const float* grad_loss,
                                    const float* grad_loss_per_token,
                                    void* grad_hidden,
                                    float* grad_W,
                                    int accumulate_grad_W,
                                    void* workspace,
                                    size_t workspace_bytes,
                                    void* hip_stream);

/* Sequences with drafted tokens. */
typedef struct kd_draft {
  int64_t B;           /* sequences; 0 <= B <= 2^20                          */
  int64_t T;           /* drafted tokens of a sequence at most; 0..1024      */
  int64_t V;           /* vocabulary size; 1 <= V <= 1048576                 */
  int64_t ld_target;   /* elements between the target's rows; >= V           */
  int64_t ld_draft;    /* between the draft's rows (dense draft only); >= V  */
  int32_t K;           /* entries of the draft's distribution, 1..4096 and
                          <= V; 0 = the draft's logits are dense             */
  int32_t dtype;       /* kd_dtype of the target's and a dense draft's logits */
  double temperature;  /* tau of both distributions; finite and > 0 (64 bits,
                          as what it divides is)                             */
  int32_t flags;       /* 0                                                  */
} kd_draft;

kd_status kd_verify_draft_workspace_size(const kd_draft* p, size_t* bytes);

/*
 * Verification of drafted tokens (speculative sampling) with a distilled
 * student as draft: the tokens that come out are distributed as the target's
 * own. Per sequence, with p_t = softmax(target logits / tau) and q_t the
 * draft's distribution at place t, the drafted tokens d_0, d_1, ... are kept
 * while u_t q_t(d_t) < p_t(d_t); the next token behind the r kept ones is the
 * first v at which the running sum of x passes u_T sum(x), where x = max(p_r -
 * q_r, 0) if d_r was rejected and p_r if all were kept (x = p_r too where
 * p_r - q_r is nowhere above 0; a difference within 2^-46 of p_r, the rounding of
 * the two, is none). All of it is held and compared in 64 bits; each 2^(z / tau) is
 * off by at most 2^-42 of itself.
 *
 *   target_logits [B, T + 1, ld_target] dtype   row t: behind t drafted tokens
 *   draft_tokens  [B, T] int32     a token outside [0, V) is rejected
 *   draft_idx     [B, T, K] int32, draft_logit [B, T, K] fp32   K > 0: the
 *                                  draft's distribution is the softmax of the
 *                                  K logits at tau, 0 elsewhere (kd_topk_entries
 *                                  of the draft's logits). An index outside
 *                                  [0, V) belongs to no token; one that repeats
 *                                  counts with the sum
 *   draft_logits  [B, T, ld_draft] dtype        K = 0: dense
 *   uniform       [B, T + 1] fp32  random numbers in [0, 1): T for the
 *                                  comparisons, the last for the next token
 *   lengths       [B] int32 or NULL   drafted tokens of each sequence (values
 *                                  outside 0..T count as the nearer end); NULL =
 *                                  T. Rows behind a sequence's end are not read
 *   tokens        [B, T + 1] int32 out: kept tokens, the next token, then -1.
 *                                  The next token is -1 where the target's row
 *                                  is -inf throughout
 *   accepted      [B] int32        out: r
 *   accept_prob   [B, T] fp32 or NULL   out: min(1, p_t(d_t) / q_t(d_t)) of each
 *                                  drafted token (1 where only q is 0, 0 where
 *                                  both are), 0 behind the sequence's end
 *
 * The draft's arrays are not used with T = 0 (a draw from the target alone). A
 * small tau gives the greedy check. B (2 T + 1) times the 2048-column segments
 * of a row may be at most 2^25. Errors: KD_ERR_NULL_PTR, KD_ERR_BAD_SHAPE,
 * KD_ERR_BAD_ARG (temperature, flags), KD_ERR_UNSUPPORTED (dtype, alignment),
 * KD_ERR_WORKSPACE_TOO_SMALL, KD_ERR_DEVICE.
 */
kd_status kd_verify_draft(const kd_draft* p, const void* target_logits,
                          const int32_t* draft_tokens, const int32_t* draft_idx,
                          const float* draft_logit, const void* draft_logits,
                          const float* uniform, const int32_t* lengths, int32_t* tokens,
                          int32_t* accepted, float* accept_prob, void* workspace,
                          size_t workspace_bytes, void* hip_stream);

/*
 * Matrices in 4 bits (microscaled floating point): a student's head after training,
 * or hidden states, at 17/32 of a byte an element. Each block of 32 consecutive
 * columns has one byte s as scale 2^(s - 127) and its elements as e2m1 codes,
 * rounded to nearest even: the codes 0 to 7 stand for 0, 0.5, 1, 1.5, 2, 3, 4 and
 * 6 scales, 8 to 15 for their negatives. The scale is the least power of two, at
 * least 2^-127, that leaves the block's largest magnitude at 6 or below: an element
 * is off by at most a fifth of itself, or by a quarter of the scale where it is below
 * the scale. (At the scale 2^126 an element of 3.5 of it and more, which would round to
 * 2^128, is held as 3.)
 * A block with an element that is infinite or not a number has s = 255 and reads
 * back as not a number.
 *
 *   x        [N, D] dtype; D a multiple of 32, 32 <= D <= 65536
 *   codes    [N, D / 2] uint8; the even column in the low half of its byte
 *   scales   [N, D / 32] uint8
 *
 * kd_mx4_read gives the values back in either dtype (exact in both). x and codes
 * 16-byte aligned. Errors: KD_ERR_NULL_PTR, KD_ERR_BAD_SHAPE, KD_ERR_UNSUPPORTED
 * (dtype, D % 32, alignment), KD_ERR_DEVICE.
 */
kd_status kd_mx4_write(int64_t N, int64_t D, int32_t dtype, const void* x, uint8_t* codes,
                       uint8_t* scales, void* hip_stream);
kd_status kd_mx4_read(int64_t N, int64_t D, int32_t dtype, const uint8_t* codes,
                      const uint8_t* scales, void* x, void* hip_stream);

/* Logits of hidden rows with a head held in 4 bits. */
typedef struct kd_mx4_head {
  int64_t N;           /* hidden rows; 0 <= N < 2^31                         */
  int64_t D;           /* hidden size; 32 <= D <= 65536, D % 32 == 0         */
  int64_t V;           /* rows of the head; 1 <= V <= 1048576                */
  int64_t ld_hidden;   /* elements between hidden rows (bf16 and fp32); D <=
                          ld_hidden <= 2^31, a multiple of 16 bytes          */
  int64_t ld_out;      /* elements between output rows; V <= ld_out <= 2^31  */
  int32_t dtype;       /* of the hidden rows: KD_BF16, KD_F32 or KD_MX4      */
  int32_t out_dtype;   /* of the logits: KD_BF16 or KD_F32                   */
  int32_t flags;       /* 0                                                  */
} kd_mx4_head;

/*
 * Bytes of device workspace with which kd_mx4_logits takes N hidden rows and any fewer
 * (the other sizes as they are): 256 for most products of up to 64 hidden rows; for
 * larger ones 1/32 of a byte an element of the head and of 4-bit hidden rows, or 6 an
 * element of fp32 ones (at most 256 MiB at a time); and up to 64 MiB of sums where the
 * columns are split into ranges, which fewer rows may need and more not. Pure host
 * function.
 */
kd_status kd_mx4_logits_workspace_size(const kd_mx4_head* p, size_t* bytes);

/*
 * out = hidden W^T with the values W that the head's codes and scales stand for:
 * what a drafting student runs before kd_topk_entries and kd_verify_draft, or a
 * teacher before kd_teacher_cache_write. bf16 and fp32 hidden rows are used as they
 * are (products exact in fp32: fp32 elements as the exact sum of three bf16 terms,
 * of which those below 2^-126 may count as 0), 4-bit ones as the values they stand
 * for; sums are fp32, rounded once to out's dtype.
 *
 *   hidden         [N, ld_hidden] dtype, or [N, D / 2] uint8 codes (KD_MX4)
 *   hidden_scales  [N, D / 32] uint8 (KD_MX4), else not used
 *   codes, scales  [V, D / 2], [V, D / 32] uint8   kd_mx4_write's of the head
 *   out            [N, ld_out] out_dtype   out: columns V and on are left as they are
 *   workspace, workspace_bytes   kd_mx4_logits_workspace_size bytes or more (of this N or a
 *                  larger one), 16-byte aligned
 *
 * hidden, codes and workspace 16-byte aligned. A head's row with a block that is not
 * a number gives logits that are not a number. Errors: KD_ERR_NULL_PTR,
 * KD_ERR_BAD_SHAPE, KD_ERR_BAD_ARG (flags), KD_ERR_UNSUPPORTED (dtypes, D % 32,
 * alignment), KD_ERR_WORKSPACE_TOO_SMALL, KD_ERR_DEVICE.
 */
kd_status kd_mx4_logits(const kd_mx4_head* p, const void* hidden, const uint8_t* hidden_scales,
                        const uint8_t* codes, const uint8_t* scales, void* out, void* workspace,
                        size_t workspace_bytes, void* hip_stream);

/*
 * Instrumentation, not part of the method: per-kernel timing with HIP events.
 * kd_profile_enable(mode), process-wide: 0 off; 1 the entry points record a
 * HIP event pair on their stream around each kernel launch; 2 only around the
 * contraction kernels (the projection, dH and dW launches, whose `flops` is
 * nonzero), which keeps the events' own cost out of the rest of the step.
 * Another mode gives KD_ERR_BAD_ARG. kd_profile_read waits for the recorded
 * events, writes up to `max` entries (one per kernel kind that ran), clears the
 * records and returns the number of entries written (negative on a HIP error).
 * `flops` is the algorithmic floating-point work of the recorded launches (the
 * 2*rows*D*V contractions of each chunk; 0 for the other kernels).
 * Creating events is an allocation: leave profiling off where that matters.
 */
typedef struct kd_kernel_time {
  char name[32];       /* kernel kind, e.g. "logits_lse", "dz", "dh", "dw" */
  int64_t launches;
  double total_ms;     /* sum of event-measured durations */
  double flops;        /* sum of algorithmic FLOP over the launches */
} kd_kernel_time;

kd_status kd_profile_enable(int mode);
int kd_profile_read(kd_kernel_time* out, int max);

/* Static, NUL-terminated description of a status code (never NULL). */
const char* kd_status_string(int status);

/* KDTOPK_ABI_VERSION of the loaded library. */
int kd_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* KDTOPK_H */
