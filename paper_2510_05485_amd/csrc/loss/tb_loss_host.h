// The kernels' launchers, as the entry points call them.
#pragma once

#include "tb_loss.h"

namespace tb {

hipError_t grant_dynamic_lds(const void* kernel, size_t bytes);  // (../tb_kernels.h)

namespace loss {

struct Call {
  Rows rows;
  RowOut out;
  Policy policy;
  Mean mean;
  Teacher teacher;
  Given given;
  int type;      // tb_type_t of the logits
  bool entropy;  // the operator needs it
  hipStream_t stream;
  int groups;  // (set by rows_of) workgroups that have left their terms in out.partial
};

// A launch has less than 2^32 threads: from so many rows on, workgroups take several.
constexpr int64_t kMostGroups = 1 << 22;
// Workgroups that the card holds at a time take all rows of up to kLaneChunks chunks: 8 of 4 wavefronts on each of
// 256 units.
constexpr int kLaneGroups = 2048, kLaneChunks = 512;

// About how many workgroups the launch of rows_of has.
inline int64_t workgroups_of(Op op, const Call& c) {
  const int64_t rows = int64_t(c.rows.B) * c.rows.T;
  const int chunks = c.rows.V / (c.type == TB_FLOAT32 ? 4 : 8);
  if (chunks < (op == kDistill ? 2 : 1) || chunks > kLaneChunks) return rows < kMostGroups ? rows : kMostGroups;
  // a workgroup's rows at a time: of two to four chunks a lane; of 16 lanes or a wavefront
  const int at_a_time = op != kDistill ? (chunks < 256 ? 1024 / chunks : 4) : chunks <= 128 && c.teacher.K <= 64 ? 16 : 4;
  const int64_t groups = (rows + at_a_time - 1) / at_a_time;
  return groups < kLaneGroups ? groups : kLaneGroups;
}

// A pass over all rows: statistics, the operator's values, and the gradient where rows.g is set.
template <typename X>
hipError_t rows_of(Op op, Call& c);
// The gradient alone, of rows whose statistics and cotangents are given.
template <typename X>
hipError_t gradient_of(Op op, const Call& c);

// How many positions of each sequence count (n [B]), or of parts of all positions (n [kCountParts]).
constexpr int kCountParts = 256;
hipError_t run_counts(const Rows& r, int32_t* n, hipStream_t stream);
hipError_t run_part_counts(const Rows& r, int32_t* n, hipStream_t stream);
// weight[b] of the positions of every sequence, from their numbers.
hipError_t run_weights(int B, int average, const int32_t* n, float* weight, hipStream_t stream);

// terms[i] = sum over workgroups of partial[workgroup][i], i < n; more: scratch of kMoreSums * 4 doubles.
constexpr int kMoreSums = 256;
hipError_t run_terms(int64_t groups, const double* partial, double* more, float* terms, int n, hipStream_t stream);

struct Pairs {
  const float* ref_lp;  // [B, T]
  const double* lp;     // [B, T]
  float *terms, *sequence_lp, *margins, *d_sequence;
  double* partial;  // [B / 2, 3]
  int kind;
  float beta, smooth;
};
hipError_t run_pairs(const Rows& r, const Pairs& p, hipStream_t stream);

}  // namespace loss
}  // namespace tb
