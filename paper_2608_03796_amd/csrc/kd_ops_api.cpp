// C ABI of the operators around the loss (top-K entries, the teacher cache,
// 8-bit checkpoints, draft verification): argument checks and workspace plans.
// Plain C++: every device operation goes through the launchers of kd_ops.hip.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/kdtopk.h"
#include "kd_ops.h"

namespace {

constexpr int64_t kMaxN = (int64_t)1 << 31;
constexpr int64_t kMaxV = (int64_t)1 << 20;   // an entry holds its index in 20 bits
constexpr int64_t kMaxLd = (int64_t)1 << 31;
constexpr int64_t kMaxK = 4096;
constexpr int64_t kMaxD = 65536;
constexpr int64_t kMaxB = (int64_t)1 << 20;
constexpr int64_t kMaxT = 1024;
constexpr int64_t kMaxWaves = (int64_t)1 << 25;  // segments of one launch

inline bool aligned(const void* q, uintptr_t n) { return ((uintptr_t)q & (n - 1)) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int elem_bytes(int32_t dtype) { return dtype == KD_BF16 ? 2 : 4; }

kd_status check_rows(const kd_rows* p) {
  if (p == nullptr) return KD_ERR_NULL_PTR;
  if ((p->flags & ~KD_FLAG_TEACHER_LOGPROBS) != 0) return KD_ERR_BAD_ARG;
  if (p->dtype != KD_F32 && p->dtype != KD_BF16) return KD_ERR_UNSUPPORTED;
  if (p->N < 0 || p->N >= kMaxN) return KD_ERR_BAD_SHAPE;
  if (p->V < 1 || p->V > kMaxV || p->ld < p->V || p->ld > kMaxLd) return KD_ERR_BAD_SHAPE;
  if (p->K < 1 || (int64_t)p->K > p->V || p->K > kMaxK) return KD_ERR_BAD_SHAPE;
  return KD_OK;
}

// Rows whose group maxima and sums are held at a time: at most 64 MiB of them
// (about 7600 rows of 2^17 columns, whose select pass fills the chip many times).
struct TopkPlan {
  int64_t rows, nseg;
  size_t off_pm, off_ps, total;
};
TopkPlan topk_plan(const kd_rows* p) {
  TopkPlan t;
  t.nseg = kd_row_segs(p->V, elem_bytes(p->dtype));
  const int64_t per = t.nseg * (kSegGroups + 2) * 4;
  t.rows = std::max<int64_t>(1, std::min<int64_t>(p->N, ((int64_t)64 << 20) / per));
  t.off_pm = align256((size_t)(t.rows * t.nseg) * kSegGroups * 4);
  t.off_ps = align256(t.off_pm + (size_t)(t.rows * t.nseg) * 4);
  t.total = align256(t.off_ps + (size_t)(t.rows * t.nseg) * 4);
  return t;
}

kd_status topk(const kd_rows* p, const void* logits, int32_t* idx, float* value, uint32_t* entries,
               float* scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (workspace == nullptr) return KD_ERR_NULL_PTR;
  if (p->N > 0 && (logits == nullptr || ((idx == nullptr || value == nullptr) &&
                                         (entries == nullptr || scale == nullptr))))
    return KD_ERR_NULL_PTR;
  const int eb = elem_bytes(p->dtype);
  if (!aligned(logits, eb) || !aligned(idx, 4) || !aligned(value, 4) || !aligned(entries, 4) ||
      !aligned(scale, 4) || !aligned(workspace, 16))
    return KD_ERR_UNSUPPORTED;
  const TopkPlan t = topk_plan(p);
  if (workspace_bytes < t.total) return KD_ERR_WORKSPACE_TOO_SMALL;
  char* ws = static_cast<char*>(workspace);
  KdTopkArgs a{};
  a.ld = p->ld;
  a.dtype = p->dtype;
  a.V = (int)p->V;
  a.K = p->K;
  a.nseg = (int)kd_row_segs(p->V, eb, aligned(logits, 16) && p->ld * eb % 16 == 0);
  a.logprobs = (p->flags & KD_FLAG_TEACHER_LOGPROBS) ? 1 : 0;
  a.gmax = reinterpret_cast<float*>(ws);
  a.pm = reinterpret_cast<float*>(ws + t.off_pm);
  a.ps = reinterpret_cast<float*>(ws + t.off_ps);
  for (int64_t r = 0; r < p->N; r += t.rows) {
    a.logits = static_cast<const char*>(logits) + r * p->ld * eb;
    a.rows = std::min<int64_t>(t.rows, p->N - r);
    a.idx = idx != nullptr ? idx + r * p->K : nullptr;
    a.value = value != nullptr ? value + r * p->K : nullptr;
    a.entries = entries != nullptr ? entries + r * p->K : nullptr;
    a.scale = scale != nullptr ? scale + r * 2 : nullptr;
    if (kd_launch_topk(&a, stream) != 0) return KD_ERR_DEVICE;
  }
  return KD_OK;
}

kd_status check_checkpoint(int64_t N, int64_t D, int32_t dtype, const void* hidden,
                           const void* codes, const void* scales) {
  if (dtype != KD_F32 && dtype != KD_BF16) return KD_ERR_UNSUPPORTED;
  if (N < 0 || N >= kMaxN || D < 32 || D > kMaxD) return KD_ERR_BAD_SHAPE;
  if (D % 32 != 0) return KD_ERR_UNSUPPORTED;
  if (N > 0 && (hidden == nullptr || codes == nullptr || scales == nullptr))
    return KD_ERR_NULL_PTR;
  if (!aligned(hidden, 16) || !aligned(codes, 16)) return KD_ERR_UNSUPPORTED;
  return KD_OK;
}

kd_status check_draft(const kd_draft* p) {
  if (p == nullptr) return KD_ERR_NULL_PTR;
  if (p->flags != 0) return KD_ERR_BAD_ARG;
  if (p->dtype != KD_F32 && p->dtype != KD_BF16) return KD_ERR_UNSUPPORTED;
  if (p->B < 0 || p->B > kMaxB || p->T < 0 || p->T > kMaxT) return KD_ERR_BAD_SHAPE;
  if (p->V < 1 || p->V > kMaxV || p->ld_target < p->V || p->ld_target > kMaxLd)
    return KD_ERR_BAD_SHAPE;
  if (p->K < 0 || p->K > kMaxK || (int64_t)p->K > p->V) return KD_ERR_BAD_SHAPE;
  if (p->K == 0 && p->T > 0 && (p->ld_draft < p->V || p->ld_draft > kMaxLd))
    return KD_ERR_BAD_SHAPE;
  if (!(isfinite(p->temperature) && p->temperature > 0.0)) return KD_ERR_BAD_ARG;
  const int64_t rows = p->B * (2 * p->T + 1);
  if (rows * kd_row_segs(p->V, elem_bytes(p->dtype)) > kMaxWaves) return KD_ERR_BAD_SHAPE;
  return KD_OK;
}

struct DraftPlan {
  int64_t nseg;
  size_t off_segm, off_segr, off_norm, total;
};
DraftPlan draft_plan(const kd_draft* p) {
  DraftPlan t;
  t.nseg = kd_row_segs(p->V, elem_bytes(p->dtype));
  const bool dense = p->K == 0 && p->T > 0;
  const size_t rows = (size_t)(p->B * (p->T + 1 + (dense ? p->T : 0)));
  t.off_segm = align256(rows * t.nseg * 8);
  t.off_segr = align256(t.off_segm + rows * t.nseg * 4);
  t.off_norm = align256(t.off_segr + (dense ? (size_t)(p->B * t.nseg) * 8 : 0));
  t.total = align256(t.off_norm + (dense ? (size_t)p->B * 32 : 0) + 1);
  return t;
}

}  // namespace

extern "C" {

kd_status kd_topk_entries_workspace_size(const kd_rows* p, size_t* bytes) {
  if (p == nullptr || bytes == nullptr) return KD_ERR_NULL_PTR;
  const kd_status st = check_rows(p);
  if (st != KD_OK) return st;
  *bytes = topk_plan(p).total;
  return KD_OK;
}

kd_status kd_topk_entries(const kd_rows* p, const void* logits, int32_t* idx, float* value,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  const kd_status st = check_rows(p);
  if (st != KD_OK) return st;
  return topk(p, logits, idx, value, nullptr, nullptr, workspace, workspace_bytes, hip_stream);
}

kd_status kd_teacher_cache_write(const kd_rows* p, const void* logits, uint32_t* entries,
                                 float* scale, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  const kd_status st = check_rows(p);
  if (st != KD_OK) return st;
  return topk(p, logits, nullptr, nullptr, entries, scale, workspace, workspace_bytes, hip_stream);
}

kd_status kd_teacher_cache_read(int64_t N, int32_t K, const uint32_t* entries, const float* scale,
                                const int64_t* rows, int64_t M, int32_t* teacher_idx,
                                float* teacher_logit, uint8_t* ignore, void* hip_stream) {
  if (N < 0 || M < 0 || M >= kMaxN || K < 1 || K > kMaxK) return KD_ERR_BAD_SHAPE;
  if (rows == nullptr && M > N) return KD_ERR_BAD_SHAPE;
  if (M == 0) return KD_OK;
  if (teacher_idx == nullptr || teacher_logit == nullptr) return KD_ERR_NULL_PTR;
  if (N > 0 && (entries == nullptr || scale == nullptr)) return KD_ERR_NULL_PTR;
  if (!aligned(entries, 4) || !aligned(scale, 4) || !aligned(rows, 8) ||
      !aligned(teacher_idx, 4) || !aligned(teacher_logit, 4))
    return KD_ERR_UNSUPPORTED;
  const KdCacheReadArgs a{entries, scale, rows, N, M, K, teacher_idx, teacher_logit, ignore};
  return kd_launch_cache_read(&a, hip_stream) == 0 ? KD_OK : KD_ERR_DEVICE;
}

kd_status kd_checkpoint_write(int64_t N, int64_t D, int32_t dtype, const void* hidden,
                              uint8_t* codes, uint8_t* scales, void* hip_stream) {
  const kd_status st = check_checkpoint(N, D, dtype, hidden, codes, scales);
  if (st != KD_OK) return st;
  if (N == 0) return KD_OK;
  return kd_launch_ckpt_write(hidden, dtype, N * D, codes, scales, hip_stream) == 0
             ? KD_OK : KD_ERR_DEVICE;
}

kd_status kd_checkpoint_read(int64_t N, int64_t D, int32_t dtype, const uint8_t* codes,
                             const uint8_t* scales, void* hidden, void* hip_stream) {
  const kd_status st = check_checkpoint(N, D, dtype, hidden, codes, scales);
  if (st != KD_OK) return st;
  if (N == 0) return KD_OK;
  return kd_launch_ckpt_read(codes, scales, dtype, N * D, hidden, hip_stream) == 0
             ? KD_OK : KD_ERR_DEVICE;
}

kd_status kd_verify_draft_workspace_size(const kd_draft* p, size_t* bytes) {
  if (p == nullptr || bytes == nullptr) return KD_ERR_NULL_PTR;
  const kd_status st = check_draft(p);
  if (st != KD_OK) return st;
  *bytes = draft_plan(p).total;
  return KD_OK;
}

kd_status kd_verify_draft(const kd_draft* p, const void* target_logits,
                          const int32_t* draft_tokens, const int32_t* draft_idx,
                          const float* draft_logit, const void* draft_logits,
                          const float* uniform, const int32_t* lengths, int32_t* tokens,
                          int32_t* accepted, float* accept_prob, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  const kd_status st = check_draft(p);
  if (st != KD_OK) return st;
  if (workspace == nullptr) return KD_ERR_NULL_PTR;
  const bool dense = p->K == 0 && p->T > 0;
  if (p->B > 0) {
    if (target_logits == nullptr || uniform == nullptr || tokens == nullptr || accepted == nullptr)
      return KD_ERR_NULL_PTR;
    if (p->T > 0 && draft_tokens == nullptr) return KD_ERR_NULL_PTR;
    if (p->T > 0 && (dense ? draft_logits == nullptr
                           : draft_idx == nullptr || draft_logit == nullptr))
      return KD_ERR_NULL_PTR;
  }
  const int eb = elem_bytes(p->dtype);
  if (!aligned(target_logits, eb) || !aligned(draft_logits, eb) || !aligned(draft_tokens, 4) ||
      !aligned(draft_idx, 4) || !aligned(draft_logit, 4) || !aligned(uniform, 4) ||
      !aligned(lengths, 4) || !aligned(tokens, 4) || !aligned(accepted, 4) ||
      !aligned(accept_prob, 4) || !aligned(workspace, 16))
    return KD_ERR_UNSUPPORTED;
  const DraftPlan t = draft_plan(p);
  if (workspace_bytes < t.total) return KD_ERR_WORKSPACE_TOO_SMALL;
  if (p->B == 0) return KD_OK;
  char* ws = static_cast<char*>(workspace);
  KdVerifyArgs a{};
  a.target = target_logits;
  a.draft = dense ? draft_logits : nullptr;
  a.ld_t = p->ld_target;
  a.ld_d = p->ld_draft;
  a.dtype = p->dtype;
  a.B = (int)p->B;
  a.T = (int)p->T;
  a.V = (int)p->V;
  a.K = p->K;
  // (places count from the target's boundaries in the draft's rows too)
  a.nseg = (int)kd_row_segs(p->V, eb, aligned(target_logits, 16) && p->ld_target * eb % 16 == 0 &&
                                          (!dense || (aligned(draft_logits, 16) &&
                                                      p->ld_draft * eb % 16 == 0)));
  a.tokens = draft_tokens;
  a.didx = draft_idx;
  a.dlogit = draft_logit;
  a.uniform = uniform;
  a.lengths = lengths;
  a.c = 1.4426950408889634074 / p->temperature;
  a.out_tokens = tokens;
  a.accepted = accepted;
  a.prob = p->T > 0 ? accept_prob : nullptr;
  a.segs = reinterpret_cast<double*>(ws);
  a.segm = reinterpret_cast<float*>(ws + t.off_segm);
  a.segr = reinterpret_cast<double*>(ws + t.off_segr);
  a.norm = reinterpret_cast<double*>(ws + t.off_norm);
  return kd_launch_verify(&a, hip_stream) == 0 ? KD_OK : KD_ERR_DEVICE;
}

}  // extern "C"
