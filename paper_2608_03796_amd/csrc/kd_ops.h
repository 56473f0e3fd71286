// Internal interface between the checks of the vocabulary and cache operators
// (kd_ops_api.cpp, plain C++) and their HIP launchers (kd_ops.hip). No HIP types:
// streams travel as void*.
#pragma once

#include <stddef.h>
#include <stdint.h>

// A wave streams a segment of a logits row: 2048 columns, counted from the
// 16-byte boundary at or before the row's first element; its 32 groups of 64
// columns (one or two 128-byte lines) are what the selection works on.
constexpr int kSegCols = 2048;
constexpr int kGroupCols = 64;
constexpr int kSegGroups = kSegCols / kGroupCols;
// segments of a row of V elements of eb bytes, wherever it starts, or of rows that
// all start on a 16-byte boundary
constexpr int64_t kd_row_segs(int64_t V, int eb, bool aligned = false) {
  return (V + (aligned ? 0 : 16 / eb - 1) + kSegCols - 1) / kSegCols;
}

// Cache entry: index << 12 | code. Codes 0..4094 count steps below the row's
// largest value; 4095 = no entry (-inf, or further than kCacheReach below it).
constexpr int kCacheCodeBits = 12;
constexpr int kCacheCodeMax = 4094;
constexpr int kCacheNone = 4095;
constexpr double kCacheReach = 1024.0;

struct KdTopkArgs {
  const void* logits;       // [rows, ld]
  int64_t rows, ld;
  int dtype, V, K, nseg, logprobs;
  float* gmax;              // [rows, nseg * kSegGroups] largest value of each group
  float *pm, *ps;           // [rows, nseg] (max, sum of exp) of each segment (logprobs)
  int32_t* idx;             // [rows, K] or null
  float* value;             // [rows, K] or null
  uint32_t* entries;        // [rows, K] or null
  float* scale;             // [rows, 2] or null
};

struct KdCacheReadArgs {
  const uint32_t* entries;  // [N, K]
  const float* scale;       // [N, 2]
  const int64_t* rows;      // [M], or null: row m
  int64_t N, M;
  int K;
  int32_t* idx;             // [M, K]
  float* value;             // [M, K]
  uint8_t* ignore;          // [M] or null
};

struct KdVerifyArgs {
  const void* target;       // [B, T + 1, ld_t]
  const void* draft;        // [B, T, ld_d] or null
  int64_t ld_t, ld_d;
  int dtype, B, T, V, K, nseg;
  const int32_t* tokens;    // [B, T]
  const int32_t* didx;      // [B, T, K] or null
  const float* dlogit;      // [B, T, K] or null
  const float* uniform;     // [B, T + 1]
  const int32_t* lengths;   // [B] or null
  double c;                 // log2(e) / tau
  int32_t* out_tokens;      // [B, T + 1]
  int32_t* accepted;        // [B]
  float* prob;              // [B, T] or null
  // workspace
  float* segm;              // [rows, nseg] a reference of each segment; rows = the
  double* segs;             // target's, then the draft's. segs: sums of 2^(c (z - segm))
  double* segr;             // [B, nseg] dense draft: sums of the remaining mass
  double* norm;             // [B, 4] dense draft: M, S of the target's and the draft's row
};

// How a product of N hidden rows with a head of V rows runs:
//  ROWS   up to 16 hidden rows: a workgroup per 16 r rows of the head, its ks waves
//         sharing the columns
//  WIDE   16 nb hidden rows by 128 r of the head a workgroup, in `splits` ranges of `per`
//         256-column pieces
//  TILES  `tok` hidden rows by 256 of the head, in `splits` ranges of `per` steps (64
//         columns, of each of three terms with fp32 hidden rows; 256 with 4-bit ones)
// `rows` hidden rows at a time. Workspace: with several ranges their fp32 sums, joined
// afterwards; for tiles the head's scales, and the hidden rows' terms or scales, as they
// take them.
enum { KD_MX4_ROWS = 0, KD_MX4_WIDE = 1, KD_MX4_TILES = 2 };
struct KdMx4Plan {
  int kind, nb, r, ks, tok, per, splits;
  int64_t rows;
  size_t off_wst, off_hidden, off_part, total;
};
KdMx4Plan kd_mx4_plan(int64_t N, int64_t D, int64_t V, int dtype, int64_t ld_hidden);

struct KdMx4Args {
  const void* hidden;       // [N, ld_hidden], or [N, D / 2] codes
  const uint8_t* hscales;   // [N, D / 32] (4-bit hidden rows) or null
  const uint8_t* codes;     // [V, D / 2]
  const uint8_t* scales;    // [V, D / 32]
  void* out;                // [N, ld_out]
  char* ws;                 // kd_mx4_plan's bytes
  int64_t N, D, V, ld_hidden, ld_out;
  int dtype, out_dtype;     // of the hidden rows (2 = 4 bits) and the output
};

extern "C" {
int kd_launch_mx4_write(const void* x, int dtype, int64_t n, uint8_t* codes, uint8_t* scales,
                        void* stream);
int kd_launch_mx4_read(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t n, void* x,
                       void* stream);
int kd_launch_mx4_logits(const KdMx4Args* a, void* stream);
int kd_launch_topk(const KdTopkArgs* a, void* stream);
int kd_launch_cache_read(const KdCacheReadArgs* a, void* stream);
int kd_launch_ckpt_write(const void* hidden, int dtype, int64_t n, uint8_t* codes, uint8_t* scales,
                         void* stream);
int kd_launch_ckpt_read(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t n,
                        void* hidden, void* stream);
int kd_launch_verify(const KdVerifyArgs* a, void* stream);
}
