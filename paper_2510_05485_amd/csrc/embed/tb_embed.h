// Embeddings of token ids: what the kernels and the entry points share.
#pragma once

#include <type_traits>

#include "../loss/tb_loss.h"
#include "tensorembed.h"

namespace tb {
namespace embed {

using loss::At;
using loss::BF16;
using loss::F16;
using loss::F32;
using loss::kWave;
using loss::Rows;
using loss::u32x4;
using loss::u32x4_any;

// Of a lookup, r.x and r.x_pos are the table and its row stride, r.g the embeddings; of a gradient r.x are the
// rows and r.g, r.g_pos the table's gradient and its row stride.
struct Lookup {
  Rows r;
  int D, type;
  float scale;
  hipStream_t stream;
};

// Tokens are sorted by a digit, some of their lower bits (so that the likeliest tokens, whose ids are neighbours in most
// vocabularies, fall to different workgroups; but neighbouring rows of narrow tables, whole lines of memory, to one),
// then by their other bits.
struct Buckets {
  int low, bits;  // the digit is (token >> low) & (2^bits - 1)
  int rows;       // of a bucket
  int held;       // of these by a workgroup of the sort, whose counters of them are in LDS
};
constexpr int kPartBlock = 2048;

struct Entry {
  uint32_t token, position;
};

struct Gradient {
  Rows r;
  int D, type, out_type, accumulate;
  float scale;
  Buckets by;
  int32_t* tokens;     // [positions], -1 for none; null: few positions, whose tokens are read where they are needed
  Entry* sorted;       // [positions]
  Entry* parted;       // [positions], of many positions: by digit alone
  int32_t* counts;     // [digit][block] of these, then where each begins
  int32_t* totals;     // [digit]
  int32_t* valid;      // how many positions there are in `sorted`
  int32_t* joins;      // how many tokens go over the end of a slice
  int32_t* join_from;  // the slices in which these begin
  float* partial;      // [slice][2][D]: sums of tokens that go on from the slice before, or into the next one
  int blocks;          // of kPartBlock positions; 0: not parted
  int slice;           // entries of `sorted` that are added up together
  int64_t slices;
  hipStream_t stream;
};

// Accesses of a wavefront's lanes to shared memory keep their order; this keeps the compiler from moving them.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

hipError_t run_lookup(const Lookup& c);
hipError_t run_gradient(const Gradient& c);

}  // namespace embed
}  // namespace tb
