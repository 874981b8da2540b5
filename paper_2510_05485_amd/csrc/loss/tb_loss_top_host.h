// The launchers of top log-probabilities, as the entry points call them.
#pragma once

#include <algorithm>

#include "tb_loss_host.h"

namespace tb {
namespace loss {

struct Top {
  void* ids;
  float* logprobs;
  int K, long_ids;
};
struct Split {  // of long rows; parts 1: none
  uint64_t* keys;  // [row][part][K], in descending order, 0 for none
  float4* stats;   // [row][part]: reference logit, sums of 2^((x - m) k) and of these times their logarithms, token's logit
  int parts;
  int tiles;      // of a part, that a workgroup takes one after the other
  int64_t first;  // part of the launch
  int by_values;  // a wavefront's bound goes by its values, not by what lanes have the largest
};
struct TopGiven {
  const float4* state;
  const float *d_top, *d_lp, *d_entropy;  // (the last two may be null)
};
struct TopCall {
  Rows rows;
  RowOut out;
  Top top;
  Split split;
  TopGiven given;
  int type;
  bool entropy;
  hipStream_t stream;
};

constexpr size_t kPlainLds = 65536;  // dynamic LDS that needs no grant

template <typename X>
hipError_t top_of(const TopCall& c);
template <typename X>
hipError_t top_gradient_of(const TopCall& c);

}  // namespace loss
}  // namespace tb
