// The kernels' launchers, as the entry points call them.
#pragma once

#include "tb_loss.h"

namespace tb {
namespace loss {

struct Call {
  Rows rows;
  RowOut out;
  Policy policy;
  Teacher teacher;
  Given given;
  int type;      // tb_type_t of the logits
  bool entropy;  // the operator needs it
  hipStream_t stream;
};

// A pass over all rows: statistics, the operator's values, and the gradient where rows.g is set.
hipError_t run_rows(Op op, const Call& c);
// The gradient alone, of rows whose statistics and cotangents are given.
hipError_t run_gradient(Op op, const Call& c);

// weight[b] of every sequence's positions; counts [B] is scratch.
hipError_t run_weights(const Rows& r, int average, int32_t* counts, float* weight, hipStream_t stream);

// terms[i] = sum over positions of weight[b] row_terms[b, t][i], i < n; partial: scratch of
// kPartials * 4 doubles.
constexpr int kPartials = 512;
hipError_t run_terms(const Rows& r, const float4* row_terms, const float* weight, double* partial, float* terms,
                     int n, hipStream_t stream);

struct Pairs {
  const float* ref_lp;
  const float4* state;
  float *terms, *sequence_lp, *margins, *d_sequence;
  double* partial;  // [B / 2, 3]
  int kind;
  float beta, smooth;
};
hipError_t run_pairs(const Rows& r, const Pairs& p, hipStream_t stream);

}  // namespace loss
}  // namespace tb
