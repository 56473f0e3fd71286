// C ABI of the operators around the loss (top-K entries, the teacher cache,
// 8-bit checkpoints, draft verification, 4-bit matrices and their products): argument
// checks and workspace plans. Plain C++: every device operation goes through the
// launchers of kd_ops.hip and kd_mx4.hip.
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

kd_status check_mx4(int64_t N, int64_t D, int32_t dtype, const void* x, const void* codes,
                    const void* scales) {
  if (dtype != KD_F32 && dtype != KD_BF16) return KD_ERR_UNSUPPORTED;
  if (N < 0 || N >= kMaxN || D < 32 || D > kMaxD) return KD_ERR_BAD_SHAPE;
  if (D % 32 != 0) return KD_ERR_UNSUPPORTED;
  if (N > 0 && (x == nullptr || codes == nullptr || scales == nullptr)) return KD_ERR_NULL_PTR;
  if (!aligned(x, 16) || !aligned(codes, 16)) return KD_ERR_UNSUPPORTED;
  return KD_OK;
}

kd_status check_head(const kd_mx4_head* p) {
  if (p == nullptr) return KD_ERR_NULL_PTR;
  if (p->flags != 0) return KD_ERR_BAD_ARG;
  if (p->dtype != KD_F32 && p->dtype != KD_BF16 && p->dtype != KD_MX4) return KD_ERR_UNSUPPORTED;
  if (p->out_dtype != KD_F32 && p->out_dtype != KD_BF16) return KD_ERR_UNSUPPORTED;
  if (p->N < 0 || p->N >= kMaxN || p->D < 32 || p->D > kMaxD) return KD_ERR_BAD_SHAPE;
  if (p->V < 1 || p->V > kMaxV || p->ld_out < p->V || p->ld_out > kMaxLd) return KD_ERR_BAD_SHAPE;
  if (p->D % 32 != 0) return KD_ERR_UNSUPPORTED;
  if (p->dtype != KD_MX4) {
    if (p->ld_hidden < p->D || p->ld_hidden > kMaxLd) return KD_ERR_BAD_SHAPE;
    if (p->ld_hidden * elem_bytes(p->dtype) % 16 != 0) return KD_ERR_UNSUPPORTED;
  }
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

// The bounds below are fits to products timed with every kernel; over 180 of them (N 24 to
// 256, D 512 to 4096, V 3001 to 100001) the choice takes on average 1.03 of the best one's
// time (fp32 hidden rows 1.06, 4-bit ones 1.05; at most 1.54). bf16, us, wide and tiles: 96 x 2048 x 30001 21.9 and 33.7; 256 x
// 2048 x 55001 69.5 and 53.9; 96 x 4096 x 55001 60.3 and 64.2; 256 x 4096 x 55001 116 and
// 90.2. Rows of the head a wave (1, 2, 4): 64 x 4096 x 55001 48.2, 39.7, 57.8; 64 x 4096 x
// 100001 89.6, 73.1, 58.5.
KdMx4Plan kd_mx4_plan(int64_t N, int64_t D, int64_t V, int dtype, int64_t ld_hidden) {
  KdMx4Plan p{};
  p.splits = 1;
  p.rows = N;
  const bool f32 = dtype == KD_F32, mx4 = dtype == KD_MX4;
  const int64_t pieces = (D + 255) / 256;
  const int64_t hld = mx4 ? D / 2 : ld_hidden * elem_bytes(dtype);
  auto cdiv = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  // pieces of the workgroups of 64 hidden rows by 128 of the head
  const int64_t work = cdiv(V, 128) * cdiv(N, 64) * pieces;
  size_t t = 0;
  // (tiles reach their hidden rows by 32-bit offsets)
  if (N > 64 && work > (f32 ? 1500 : mx4 ? 4000 : 3000) && 256 * hld < ((int64_t)1 << 31)) {
    p.kind = KD_MX4_TILES;
    // 256 MiB of terms, and grids that the launch takes
    const int64_t Dp = cdiv(D, 64) * 64;
    p.rows = (int64_t)1 << 18;
    if (f32) p.rows = std::max<int64_t>(256, (((int64_t)256 << 20) / (Dp * 6)) & ~255);
    p.rows = std::min(p.rows, N);
    // tiles of 128 hidden rows take 0.6 of the time of one of 256
    const int64_t tv = cdiv(V, 256);
    p.tok = p.rows > 128 && cdiv(tv * cdiv(p.rows, 256), 256) * 10 <=
                                cdiv(tv * cdiv(p.rows, 128), 256) * 6
                ? 256
                : 128;
    const int64_t tiles = tv * cdiv(p.rows, p.tok);
    // a range is a multiple of 256 columns (of every term), the scales' loads
    const int64_t unit = f32 ? 12 : mx4 ? 1 : 4, most = mx4 ? 128 : 256;
    const int64_t splits = tiles * 2 <= most ? std::min<int64_t>(most / tiles, pieces) : 1;
    const int64_t per = cdiv(pieces, splits);
    p.per = (int)(per * unit);
    p.splits = (int)cdiv(pieces, per);
    const int64_t T = pieces * 2;
    p.off_wst = 0;
    p.off_hidden = align256((size_t)(tv * 4 * T * 256));
    t = p.off_hidden;
    if (f32) t += (size_t)(p.rows * Dp * 6);
    if (mx4) t += (size_t)(cdiv(p.rows, 256) * 4 * T) * 256;
  } else if (N <= 16 && V <= (f32 || N > 4 ? 24576 : 49152)) {
    p.kind = KD_MX4_ROWS;
    p.r = V <= 6144 ? 1 : 2;
    p.ks = 1;
    while (p.ks < (V <= 16384 ? 8 : 4) && p.ks < pieces) p.ks *= 2;
  } else {
    p.kind = KD_MX4_WIDE;
    p.nb = N <= 16 ? 1 : N <= 32 || (N <= 64 && !mx4 && work < 2000) ? 2 : 4;
    p.rows = std::min<int64_t>(N, (int64_t)65535 * 16 * p.nb);
    // rows of the head a wave: as many as leave most compute units a workgroup
    const int64_t toks = cdiv(p.rows, 16 * p.nb), least = f32 && pieces >= 8 ? 64 : 180;
    p.r = 1;
    if (cdiv(V, 256) * toks >= least && !(p.nb == 4 && mx4)) p.r = 2;
    // (two rows of 16 run a workgroup a compute unit: four where those take a second round)
    if (p.nb == 4 && (mx4 ? cdiv(V, 512) * toks >= 180 : cdiv(V, 256) * toks > 256)) p.r = 4;
    const int64_t groups = cdiv(V, 128 * p.r) * toks;
    int64_t splits = 1;
    if (groups <= (pieces >= 8 ? 128 : f32 && pieces >= 4 ? 64 : 0))
      splits = std::max<int64_t>(1, std::min<int64_t>(256 / groups, pieces / 2));
    const int64_t per = cdiv(pieces, splits);
    p.per = (int)per;
    p.splits = (int)cdiv(pieces, per);
  }
  p.off_part = align256(t);
  p.total = std::max<size_t>(256, p.off_part);
  if (p.splits > 1) p.total += align256((size_t)(p.splits * p.rows * cdiv(V, 4) * 4) * 4);
  return p;
}

// Workspace of up to N hidden rows. Only the ranges' sums make fewer rows need more than
// N; ranges take at most 128 workgroups (V <= 65536) of at most 128 hidden rows each. The
// plan is the same for all rows up to a multiple of 16, and from 64 on of 64 (of one tile of
// a kernel), but for its space, which grows with them. At most 259 plans, 10 us.
static size_t mx4_workspace(const kd_mx4_head* p) {
  auto bytes = [&](int64_t n) { return kd_mx4_plan(n, p->D, p->V, p->dtype, p->ld_hidden).total; };
  size_t most = bytes(p->N);
  if (p->V > 65536) return most;
  for (int64_t n = 16; n < p->N && n <= 128 * 128; n += n < 64 ? 16 : 64)
    most = std::max(most, bytes(n));
  return most;
}

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

kd_status kd_mx4_write(int64_t N, int64_t D, int32_t dtype, const void* x, uint8_t* codes,
                       uint8_t* scales, void* hip_stream) {
  const kd_status st = check_mx4(N, D, dtype, x, codes, scales);
  if (st != KD_OK || N == 0) return st;
  return kd_launch_mx4_write(x, dtype, N * D, codes, scales, hip_stream) == 0 ? KD_OK
                                                                              : KD_ERR_DEVICE;
}

kd_status kd_mx4_read(int64_t N, int64_t D, int32_t dtype, const uint8_t* codes,
                      const uint8_t* scales, void* x, void* hip_stream) {
  const kd_status st = check_mx4(N, D, dtype, x, codes, scales);
  if (st != KD_OK || N == 0) return st;
  return kd_launch_mx4_read(codes, scales, dtype, N * D, x, hip_stream) == 0 ? KD_OK
                                                                             : KD_ERR_DEVICE;
}

kd_status kd_mx4_logits_workspace_size(const kd_mx4_head* p, size_t* bytes) {
  if (p == nullptr || bytes == nullptr) return KD_ERR_NULL_PTR;
  const kd_status st = check_head(p);
  if (st != KD_OK) return st;
  *bytes = mx4_workspace(p);
  return KD_OK;
}

kd_status kd_mx4_logits(const kd_mx4_head* p, const void* hidden, const uint8_t* hidden_scales,
                        const uint8_t* codes, const uint8_t* scales, void* out, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  const kd_status st = check_head(p);
  if (st != KD_OK) return st;
  const bool mx4 = p->dtype == KD_MX4;
  if (workspace == nullptr) return KD_ERR_NULL_PTR;
  if (p->N > 0 && (hidden == nullptr || (mx4 && hidden_scales == nullptr) || codes == nullptr ||
                   scales == nullptr || out == nullptr))
    return KD_ERR_NULL_PTR;
  if (!aligned(hidden, 16) || !aligned(codes, 16) || !aligned(workspace, 16) ||
      !aligned(out, elem_bytes(p->out_dtype)))
    return KD_ERR_UNSUPPORTED;
  if (workspace_bytes < kd_mx4_plan(p->N, p->D, p->V, p->dtype, p->ld_hidden).total)
    return KD_ERR_WORKSPACE_TOO_SMALL;
  if (p->N == 0) return KD_OK;
  KdMx4Args a{};
  a.hidden = hidden;
  a.hscales = mx4 ? hidden_scales : nullptr;
  a.codes = codes;
  a.scales = scales;
  a.out = out;
  a.ws = static_cast<char*>(workspace);
  a.N = p->N;
  a.D = p->D;
  a.V = p->V;
  a.ld_hidden = p->ld_hidden;
  a.ld_out = p->ld_out;
  a.dtype = p->dtype;
  a.out_dtype = p->out_dtype;
  return kd_launch_mx4_logits(&a, hip_stream) == 0 ? KD_OK : KD_ERR_DEVICE;
}

}  // extern "C"
