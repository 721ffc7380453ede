// Operators on caller-owned tensors without a context: products over rows
// grouped by cluster, dropout, label scores.  Arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "rng.h"

// Workgroups of 256 threads that one launch may have.  A launch has fewer than
// 2^32 threads: the runtime takes their number modulo that, without an error.
constexpr int64_t kMaxBlocks = ((int64_t)1 << 32) / 256 - 1;

// ---------------------------------------------------------------- dropout
// Threshold and factor of a dropout probability: an element is kept when its
// 16-bit draw is at least `thr`, which has probability 1 - thr / 65536.
struct Drop {
  uint64_t key;
  uint32_t thr;  // 0: everything is kept
  float scale;   // 65536 / (65536 - thr)
};

// Word of four draws for columns 4 c4 .. 4 c4 + 3 of row `row` of a tensor
// with `words` = ceil(cols / 4) words a row: SplitMix64's output number
// row * words + c4 from state `key`.
__device__ __forceinline__ uint64_t drop_word(uint64_t key, int64_t row, int64_t words, int c4) {
  return gc_mix64(key + (uint64_t)(row * words + c4 + 1) * GCPSL_GOLDEN);
}
__device__ __forceinline__ bool drop_keeps(uint64_t word, int j, uint32_t thr) {
  return ((uint32_t)(word >> (16 * j)) & 0xffffu) >= thr;
}

hipError_t launch_dropout(int dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *y, int64_t ldy,
                          const Drop &d, hipStream_t s);

// --------------------------------------------------------- grouped products
// out[m][c] = sum_q A(m, q) B(c, q) for the rows of every group g (rows
// [offsets[g], offsets[g+1])):
//   forward      A = x rows,  q = input feature,  B(c, q) = w_g[c][q]
//   input grad   A = dy rows, q = output feature, B(c, q) = w_g[q][c]
//   weight grad  A(m, q) = dy[q][m], B(c, q) = x[q][c], q = row of the group
enum GroupMode { GROUP_FWD = 0, GROUP_DX = 1, GROUP_DW = 2 };
struct GroupArgs {
  const int32_t *off;  // device [G + 1]
  int G, M, N, Q;      // M: rows of the tensors (weight grad: output features), N columns of out; Q: length of
                       // the sums (weight grad: rows of the tensors)
  const void *a, *b;
  int64_t lda, ldb, b_gs;   // row strides; b's stride from group to group (weights)
  void *out;
  int64_t ldo, out_gs;      // out's row stride; weight grad: stride from group to group
  const float *bias;        // forward: [G] rows of N, or null
  int64_t bias_gs;
  float *db;                // weight grad: [G] rows of M, or null
  int64_t db_gs;
  int relu;                 // forward
  const void *gate;         // input grad: rows of N, or null
  int64_t ldg;
  Drop drop;                // forward: applied to the result; input grad: its scale multiplies where the gate is > 0
  // weight grad: a group of c rows is summed in max(1, round(c / piece)) pieces; those of groups of more than one
  // go to partials, [slots][M][N] and [slots][M]
  int piece, slots;
  float *part, *part_db;
};
// Rows of a piece of a weight gradient's sums and the partials that this can make (host).
struct GroupPieces {
  int piece, slots;
};
GroupPieces group_pieces(int dtype, int G, int64_t rows, int n, int k);
hipError_t launch_group(int dtype, int mode, const GroupArgs &a, hipStream_t s);

// ------------------------------------------------------------ label scores
constexpr int kMaxTop = 32;
struct ScoreArgs {
  const void *z;
  int64_t ldz, rows;
  int L, top;
  const int32_t *labels;  // or null
  float *logp, *entropy, *lse, *top_logp;
  int32_t *top_class;
  void *work;
};
size_t score_work_bytes(int dtype, int64_t rows, int L, int top);
hipError_t launch_score(int dtype, const ScoreArgs &a, hipStream_t s);
struct ScoreGradArgs {
  const void *z;
  int64_t ldz, rows;
  int L;
  const int32_t *labels;
  const float *lse, *entropy, *g_logp, *g_entropy;
  void *dz;
  int64_t lddz;
};
hipError_t launch_score_grad(int dtype, const ScoreGradArgs &a, hipStream_t s);
