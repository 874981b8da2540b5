// Passes over rows of logits: log-probabilities and entropies, the policy loss, the distillation loss,
// and their gradients.  Each type of logits is instantiated in a file of its own.
//
// Long rows are bound by HBM: a row is read once and its gradient written once, with two exponentials (which
// issue at a quarter of the rate) and about seven other instructions a value in between.  Kernels by the
// length of a row:
//   lanes_kernel     up to 512 chunks of 16 bytes: 2 to 64 lanes of a wavefront hold a row
//   held_kernel      a workgroup holds a row in its registers, and in LDS
//   distill_kernel   the same with a teacher's entries: 16 lanes, a wavefront or a workgroup
//   sweep_kernel     a workgroup reads the row from memory in each of two sweeps (any length)
//   gradient_kernel  the second sweep alone, with statistics given
// Calls on one MI355X, with their gradients: the policy loss of 32 x 1024 rows of 50257 values in bfloat16, 62 % of
// which count, 1014 us (5.3 TB/s; rows copied alone 5.2 to 5.7), of 16384 rows of 8191 110 us (4.9), of 1048576
// rows of 64 71 us (3.8); distillation of 4096 rows of 32000 106 us (5.0).  Statistics alone: 6.2 to 6.9 TB/s.
// Cards differ by 2 to 5 %; single launches under the profiler take 3 to 5 % longer.
#pragma once

#include <type_traits>

#include "tb_loss_host.h"

namespace tb {
namespace loss {
namespace {

constexpr uint32_t kNan = 0x7FC00000u;

// ---- what all kernels do for a row ------------------------------------------------------------

// M = m k of the weights 2^(x k - M): rounded, and the same wherever it is formed (the compiler must
// not take the product into a fused multiply-add, whose M would be another one).
__device__ __forceinline__ float scaled(float m, float k) {
#pragma clang fp contract(off)
  return m * k;
}
// M is off by half a unit in its last place: by 8 at most below 2^28, from where on weights are formed as
// 2^((x - m) k) only.
__device__ __forceinline__ bool scales(float m, float k) { return fabsf(scaled(m, k)) < 0x1p28f; }
// Kernels that form weights as 2^((x - m) k) have sums that differ from those of 2^(x k - M) by a factor
// that rounds M; the state of a row that is kept for the backward pass is of the latter, where M is used.
__device__ __forceinline__ float to_scaled(float m, float k) {
  return scales(m, k) ? exp2_fast(fmaf(m, k, -scaled(m, k))) : 1.f;
}
__device__ __forceinline__ float from_scaled(float m, float k) {
  return scales(m, k) ? exp2_fast(-fmaf(m, k, -scaled(m, k))) : 1.f;
}
// 1 / x, to 1 unit in the last place
__device__ __forceinline__ float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }

// What the gradient of a row is made of: values 2^a (by_weight + by_log a), a = (x - m) k, and `token`
// more at the row's token.
struct Slope {
  float by_weight, by_log, token;
};

// from the cotangents of lp and H
__device__ __forceinline__ Slope slope_of(float s, float H, float d_lp, float d_H, float scale) {
  const float f = scale * reciprocal(s);
  return {f * (-d_lp - d_H * (H - logf(s))), -f * d_H * kLn2, scale * d_lp};
}
template <bool kEntropy>
__device__ __forceinline__ float gradient_at(float a, Slope f) {
  return exp2_fast(a) * (kEntropy ? f.by_weight + f.by_log * finite(a) : f.by_weight);
}

// Loss and cotangents of a position (every thread of the workgroup computes them).
struct Position {
  float4 terms;  // loss, kl, clipped, entropy
  float d_lp, d_H;
};
__device__ __forceinline__ Position policy_position(const Policy& p, float old_lp, float ref_lp, float A, float lp,
                                                    float H, float w) {
  const float ratio = expf(lp - old_lp);
  const bool clipped = (A > 0 && ratio > 1 + p.high) || (A < 0 && ratio < 1 - p.low);
  const float held = A > 0 ? 1 + p.high : 1 - p.low;
  Position o;
  float loss = -(clipped ? held : ratio) * A, kl = 0.f;
  o.d_lp = clipped ? 0.f : -ratio * A;
  if (p.kl_coef != 0.f) {
    const float d = ref_lp - lp, e = expf(d);
    // near 0 the difference of e^d and 1 + d is its series' next terms: d^2 (1/2 + d/6 + ...)
    kl = fabsf(d) < 0.02f ? d * d * (0.5f + d * (1.f / 6 + d * (1.f / 24 + d * (1.f / 120)))) : e - d - 1.f;
    loss += p.kl_coef * kl;
    o.d_lp += p.kl_coef * (fabsf(d) < 0.02f ? -d * (1.f + d * (0.5f + d * (1.f / 6 + d * (1.f / 24)))) : 1.f - e);
  }
  if (p.entropy_coef != 0.f) loss -= p.entropy_coef * H;
  o.terms = {loss, kl, clipped ? 1.f : 0.f, p.entropy_coef != 0.f ? H : 0.f};
  o.d_lp *= w;
  o.d_H = -p.entropy_coef * w;
  return o;
}
__device__ __forceinline__ Position policy_position(const Policy& p, int b, int64_t at, float lp, float H, float w) {
  return policy_position(p, p.old_lp[at], p.kl_coef != 0.f ? p.ref_lp[at] : 0.f, p.advantages[p.each ? at : b], lp, H, w);
}

__device__ __forceinline__ float teacher_value(const Teacher& q, int64_t i) {
  if (q.type == TB_FLOAT32) return static_cast<const float*>(q.logits)[i];
  return q.type == TB_BFLOAT16 ? BF16::load(static_cast<const uint16_t*>(q.logits) + i)
                               : F16::load(static_cast<const _Float16*>(q.logits) + i);
}

// The row's token, or -1 (reported by the thread that has `tell`) for one outside the vocabulary.
__device__ __forceinline__ int take_token(const Rows& r, int b, int t, bool tell) {
  const int64_t token = load_id(r.tokens, r.long_tokens, b * r.token_seq + t);
  if (token >= 0 && token < r.V) return int(token);
  if (tell && r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
  return -1;
}

// A log-probability for sums over whole sequences: a_tok = log2 of the token's weight, s the sum of all.  In
// 32 bits the logarithm alone is off by up to 5e-7, as much as a pair's mean margin of 0.02 bears.
__device__ __forceinline__ double exact_lp(double a_tok, float s) { return a_tok * 0.693147180559945309417 - log(double(s)); }

// What the position that does not count leaves, but for its gradient.
__device__ __forceinline__ void leave_nothing(const RowOut& o, int64_t at) {
  if (o.logprobs) o.logprobs[at] = 0.f;
  if (o.entropy) o.entropy[at] = 0.f;
  if (o.state) o.state[at] = {};
  if (o.d_logprobs) o.d_logprobs[at] = 0.f;
  if (o.d_entropy) o.d_entropy[at] = 0.f;
}

// The thread's share of the total, and the weight of a sequence's positions.
__device__ __forceinline__ int share_of_total(const Rows& r, const Mean& mean) {
  constexpr int kAhead = 8;  // loads under way
  const int32_t* from = mean.n ? mean.n : r.lengths;
  int n = 0;
  if (mean.weight || mean.average == TB_SUM) return n;
  if (r.mask && !mean.n) {  // (few positions)
    for (int i = threadIdx.x; i < r.B * r.T; i += blockDim.x) {
      const At pos = position(r, i);
      n += counts(r, pos.b, pos.t);
    }
    return n;
  }
  if (!from) return n;
  const int most = mean.n ? INT32_MAX : r.T, threads = blockDim.x;
  for (int i = threadIdx.x; i < mean.parts; i += kAhead * threads) {
    int m[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) m[j] = i + j * threads < mean.parts ? from[i + j * threads] : 0;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int c = clamped(m[j], most);
      n += mean.average == TB_MEAN_TOKENS ? c : c > 0;
    }
  }
  return n;
}
__device__ __forceinline__ float weight_of(const Rows& r, const Mean& mean, int b, int length, int total) {
  if (mean.weight) return mean.weight[b];
  if (mean.average == TB_SUM) return 1.f;
  if (!mean.n && !r.lengths && !r.mask) total = mean.average == TB_MEAN_TOKENS ? r.B * r.T : r.B;
  if (mean.average == TB_MEAN_TOKENS) return 1.f / float(total);
  return reciprocal(float(total) * float(mean.n ? mean.n[b] : length));
}
__device__ __forceinline__ float weight_of(const Rows& r, const Mean& mean, int b, int total) {
  return weight_of(r, mean, b, r.lengths ? clamped(r.lengths[b], r.T) : r.T, total);
}

// Which row a workgroup takes: neighbouring workgroups go to different XCDs, neighbouring rows to one.
// Which XCD begins changes from block to block, so that the ends of sequences, whose rows do not count, fall
// to all of them alike (512 sequences of 32 positions, half of which count: 212 us without).
__device__ __forceinline__ int64_t row_of_group(int64_t group, int64_t rows) {
  constexpr int kXcds = 8, kRun = 4;
  const int64_t block = group / (kXcds * kRun), in = group % (kXcds * kRun);
  if ((block + 1) * kXcds * kRun > rows) return group;
  return block * kXcds * kRun + (in + block) % kXcds * kRun + in / kXcds;
}

// Sum over the lanes that share a row (kLanes of a wavefront), in all of them.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xf, 0xf, true));
}
// The value of a lane whose group of kStep lanes is the neighbour of the own one; all lanes of a group
// hold the same value.
template <int kStep>
__device__ __forceinline__ float neighbour(float v) {
  if constexpr (kStep == 1) return dpp<0xB1>(v);        // quad_perm [1, 0, 3, 2]
  else if constexpr (kStep == 2) return dpp<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  else if constexpr (kStep == 4) return dpp<0x141>(v);  // row_half_mirror
  else if constexpr (kStep == 8) return dpp<0x140>(v);  // row_mirror
  else return __shfl_xor(v, kStep);
}
template <bool kEntropy, int kLanes, int kStep = 1, typename Join>
__device__ __forceinline__ Stats joined_lanes(const Stats& mine, Join join) {
  if constexpr (kStep == kLanes) return mine;
  else {
    const Stats other = {neighbour<kStep>(mine.m), neighbour<kStep>(mine.s), kEntropy ? neighbour<kStep>(mine.t) : 0.f};
    return joined_lanes<kEntropy, kLanes, kStep * 2>(join(mine, other), join);
  }
}

// A barrier of the threads that share a row: in a wavefront, whose accesses keep their order, it only
// keeps the compiler from moving them.
template <int kThreads>
__device__ __forceinline__ void meet() {
  if constexpr (kThreads <= kWave) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    __syncthreads();
  }
}

// ---- rows in the registers of some lanes ------------------------------------------------------

// The part of a row that a lane of kLanes holds: chunks lane + k kLanes of 16 bytes from the row's first
// value on, at any address.  The last chunk ends with the row: where a row is not a whole number of chunks it
// has values of the chunk before once more, which count once and get the same gradient twice.
template <typename X, int kLanes, int kChunks>
struct Part {
  u32x4 c[kChunks];
  // the first value of chunk k, or -1
  static __device__ __forceinline__ int at(int V, int lane, int k) {
    const int i = (lane + k * kLanes) * X::kPer;
    return i < V ? min(i, V - X::kPer) : -1;
  }
  __device__ __forceinline__ void load(const typename X::type* row, int V, int lane, bool live) {
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      c[k] = u32x4{X::kNone, X::kNone, X::kNone, X::kNone};
      const int i = at(V, lane, k);
      if (live && i >= 0) c[k] = *reinterpret_cast<const u32x4_any*>(row + i);
    }
  }
  // values of chunk k, those that count elsewhere as -inf
  __device__ __forceinline__ void once(int V, int lane, int k, float* v) const {
    X::unpack(c[k], v);
    if (V % X::kPer == 0 || k != (V - 1) / X::kPer / kLanes) return;  // (the same for all rows)
    const int again = (lane + k * kLanes) * X::kPer - (V - X::kPer);
#pragma unroll
    for (int i = 0; i < X::kPer - 1; ++i)
      if (i < again) v[i] = -INFINITY;
  }
  __device__ __forceinline__ void keep_packed() {  // (as in Held)
#pragma unroll
    for (int k = 0; k < kChunks; ++k) asm volatile("" : "+v"(c[k]));
  }
};

template <bool kEntropy, int kLanes, typename X, int kChunks>
__device__ __forceinline__ Stats part_stats(Part<X, kLanes, kChunks>& p, int V, int lane, float k) {
  Stats mine = {kLowest, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[X::kPer];
    X::unpack(p.c[j], v);
#pragma unroll
    for (int i = 0; i < X::kPer; i += 2) mine.m = max3(mine.m, v[i], v[i + 1]);
  }
  p.keep_packed();
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[X::kPer];
    p.once(V, lane, j, v);
#pragma unroll
    for (int i = 0; i < X::kPer; ++i) {
      const float a = (v[i] - mine.m) * k, w = exp2_fast(a);
      mine.s += w;
      if (kEntropy) mine.t += w * finite(a);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  p.keep_packed();
  return joined_lanes<kEntropy, kLanes>(mine, [k](const Stats& a, const Stats& b) { return joined<kEntropy>(a, b, k); });
}

// Writes the gradients of a wavefront's rows, the first of which is row `from`; zeros where `live` is false.
// Lanes that hold pieces of 16 or 32 bytes of a row would store as many pieces of lines; so the chunks go
// through LDS, from where neighbouring lanes take neighbouring chunks (4096 x 512 rows of 64 values, the
// gradient alone: 180 us without, 117 so).  `stage`: room for the wavefront's chunks.
template <bool kEntropy, int kLanes, typename X, int kChunks>
__device__ __forceinline__ void write_part(const Part<X, kLanes, kChunks>& p, const Rows& r, int64_t from, int V,
                                           bool live, int token, float x, float m, float k, Slope f, u32x4_at16* stage) {
  using T = typename X::type;
  constexpr int kSlots = kLanes * kChunks, kSpread = kSlots % 8 == 0 ? 8 : kSlots % 4 == 0 ? 4 : 2;
  const int lane = threadIdx.x % kLanes, thread = threadIdx.x % kWave, row = thread / kLanes;
  auto slot_of = [](int row, int slot) { return row * kSlots + (slot ^ (row % kSpread)); };  // (other banks for other rows)
  const bool any = __any(live);
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    u32x4 c = {};
    if (any) {
      float v[X::kPer];
      X::unpack(p.c[j], v);
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) v[i] = gradient_at<kEntropy>((v[i] - m) * k, f);
      if (live) c = X::pack(v);
    }
    stage[slot_of(row, lane + j * kLanes)] = c;
    __builtin_amdgcn_sched_barrier(0);  // (one chunk's values in registers at a time)
  }
  meet<kWave>();
  if (live && token >= 0 && lane == 0) {
    const float v = f.token + gradient_at<kEntropy>((x - m) * k, f);
    const int chunk = token / X::kPer, last = (V - 1) / X::kPer, tail = token - (V - X::kPer);
    if (chunk < V / X::kPer) X::store(reinterpret_cast<T*>(stage + slot_of(row, chunk)) + token % X::kPer, v);
    if (tail >= 0) X::store(reinterpret_cast<T*>(stage + slot_of(row, last)) + tail, v);
  }
  meet<kWave>();
  const int64_t rows = int64_t(r.B) * r.T;
#pragma unroll 1
  for (int j = 0; j < kChunks; ++j) {
    const int q = j * kWave + thread, other = q / kSlots, slot = q % kSlots;
    const int i = Part<X, kLanes, kChunks>::at(V, slot, 0);
    if (i < 0 || from + other >= rows) continue;
    const At pos = position(r, from + other);
    *reinterpret_cast<u32x4_any*>(gradient_of<X>(r, pos.b, pos.t) + i) = stage[slot_of(other, slot)];
  }
  meet<kWave>();  // (before the next rows' chunks)
}

constexpr int kLaneThreads = 256;

// What a position brings besides its row, on its way while the position before is worked on: with one
// round trip after the other in front of every row (length, token, the token's logit, the sampling policy's
// value ...) 4096 x 512 rows of 64 values took a sixth longer.
template <int kOp, bool kEntropy>
struct Ahead {
  int64_t token;
  float old_lp, ref_lp, advantage;  // kPolicy
  float4 state;                     // kGiven
  float d_lp, d_H;
  int length, mask, b, t;

  __device__ __forceinline__ void fetch(const Rows& r, const Policy& p, const Given& v, int64_t at) {
    const At pos = position(r, at);
    b = pos.b;
    t = pos.t;
    length = r.lengths ? r.lengths[b] : r.T;
    mask = r.mask ? r.mask[at] : 1;
    token = load_id(r.tokens, r.long_tokens, b * r.token_seq + t);
    if constexpr (kOp == kPolicy) {
      old_lp = p.old_lp[at];
      ref_lp = p.kl_coef != 0.f ? p.ref_lp[at] : 0.f;
      advantage = p.advantages[p.each ? at : b];
    }
    if constexpr (kOp == kGiven) {
      state = v.state[at];
      d_lp = v.d_lp[b * v.d_seq + t * v.d_pos];
      d_H = kEntropy ? v.d_entropy[b * v.d_seq + t * v.d_pos] : 0.f;
    }
  }
};

// kLanes lanes of a wavefront a row, kLaneThreads / kLanes rows a workgroup at a time.  Nothing of it
// needs a barrier, and a row's statistics meet in one to six steps between lanes.  Few lanes with four
// chunks each share what is done once a row, a third of all instructions at 64 values.
template <typename X, int kOp, bool kEntropy, int kLanes, int kChunks>
__global__ __launch_bounds__(kLaneThreads) void lanes_kernel(Rows r, RowOut o, Policy p, Mean mean, Given v) {
  constexpr int kTeams = kLaneThreads / kLanes, kWaves = kLaneThreads / kWave;
  __shared__ double sums[kWaves][4];
  __shared__ int totals[kWaves];
  __shared__ u32x4_at16 stage[kOp == kScore ? 1 : kWaves * kWave * kChunks];
  const int lane = threadIdx.x % kLanes;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  constexpr int kRows = kWave / kLanes;  // of a wavefront
  const int wave = threadIdx.x / kWave, row_in_wave = threadIdx.x % kWave / kLanes;
  // Round by round the workgroups take the next rows, each one's place in a round being its neighbour's in
  // the round before: in the same place it would meet the same positions of every sequence, the ends of
  // which do not count (161 us for the rows above, 121 so).
  auto first_of = [&](uint32_t round) {
    uint32_t place = blockIdx.x + round;
    if (place >= gridDim.x) place %= gridDim.x;
    return (int64_t(round) * gridDim.x + place) * kTeams + wave * kRows;
  };
  int64_t from = first_of(0);
  auto within = [&](int64_t i) { return i < rows ? i : rows - 1; };
  Ahead<kOp, kEntropy> next;
  next.fetch(r, p, v, within(from + row_in_wave));
  int total = 0;
  if (kOp == kPolicy) {
    const int part = full_wave_sum(share_of_total(r, mean));
    if (threadIdx.x % kWave == 0) totals[threadIdx.x / kWave] = part;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) total += totals[w];
  }
  const float up = kOp == kGiven && v.upstream ? *v.upstream : 1.f;
  double sum[4] = {};
  const int64_t a_round = int64_t(gridDim.x) * kTeams;
  for (uint32_t round = 0; round * a_round < rows; ++round) {
    const int64_t at = from + row_in_wave, follows = first_of(round + 1);
    // (keeps the compiler from working out the lanes' masks once for all rows, for which there are no registers)
    int V = r.V;
    asm volatile("" : "+s"(V));
    const Ahead<kOp, kEntropy> now = next;
    next.fetch(r, p, v, within(follows + row_in_wave));
    const bool inside = at < rows, live = inside && now.t < now.length && now.mask != 0;
    const typename X::type* row = row_of<X>(r, now.b, now.t);
    Part<X, kLanes, kChunks> part;
    part.load(row, V, lane, live);
    const int token = live && now.token >= 0 && now.token < V ? int(now.token) : -1;
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(row + token);
    if (kOp != kGiven && lane == 0 && inside && r.status) {
      if (now.t == 0 && (now.length < 0 || now.length > r.T)) atomicOr(r.status, TB_DEV_LENGTH_RANGE);
      if (live && token < 0) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
    }
    Slope f = {};
    float m = 0.f;
    if (live) {
      if constexpr (kOp == kGiven) {
        m = now.state.x;
        f = slope_of(now.state.y * from_scaled(m, k), now.state.z, token < 0 ? x : now.d_lp * up, now.d_H * up,
                     r.g_scale * r.inv_temp);
      } else {
        const Stats s = part_stats<kEntropy, kLanes>(part, V, lane, k);
        const float log_s = logf(s.s), lp = (x - s.m) * r.inv_temp - log_s;
        const float H = kEntropy ? log_s - kLn2 * s.t / s.s : 0.f;
        m = s.m;
        Position q = {};
        if constexpr (kOp == kPolicy) {
          const float w = weight_of(r, mean, now.b, clamped(now.length, r.T), total);
          q = policy_position(p, now.old_lp, now.ref_lp, now.advantage, lp, H, w);
          if (lane == 0) {
            const double by = w;
            sum[0] = fma(by, double(q.terms.x), sum[0]);
            if (p.kl_coef != 0.f) sum[1] = fma(by, double(q.terms.y), sum[1]);
            sum[2] = fma(by, double(q.terms.z), sum[2]);
            if (kEntropy) sum[3] = fma(by, double(q.terms.w), sum[3]);
          }
          f = slope_of(s.s, H, q.d_lp, q.d_H, r.g_scale * r.inv_temp);
        }
        if (lane == 0) {
          if (o.logprobs) o.logprobs[at] = lp;
          if (kOp == kScore && o.entropy) o.entropy[at] = H;
          if (kOp == kScore && o.exact) o.exact[at] = exact_lp(double(x - s.m) * k, s.s);
          if (o.state) o.state[at] = {s.m, s.s * to_scaled(s.m, k), H, lp};
          if (kOp == kPolicy && o.d_logprobs) o.d_logprobs[at] = q.d_lp;
          if (kOp == kPolicy && o.d_entropy) o.d_entropy[at] = q.d_H;
        }
      }
    } else if (kOp != kGiven && lane == 0 && inside) {
      leave_nothing(o, at);
    }
    if (kOp == kGiven || (kOp == kPolicy && r.g))
      write_part<kEntropy>(part, r, from, V, live, token, x, m, k, f, stage + wave * (kWave * kChunks));
    from = follows;
  }
  if constexpr (kOp == kPolicy) {
    for (int j = 0; j < 4; ++j) {
      sum[j] = wave_sum(sum[j]);
      if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave][j] = sum[j];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
      double all = 0;
      for (int w = 0; w < kWaves; ++w) all += sums[w][threadIdx.x];
      o.partial[int64_t(blockIdx.x) * 4 + threadIdx.x] = all;
    }
  }
}

// ---- sweeps over a row in memory --------------------------------------------------------------

// Statistics of a row, in every thread.  Reads the row once.
// (kThreads: threads of the workgroup, or of the wavefront that has the row to itself; 0: blockDim.x)
template <typename X, bool kEntropy, int kThreads = 0, typename Row>
__device__ __forceinline__ Stats row_stats(const Row& row, float k, int thread, Stats* parts) {
  const int threads = kThreads ? kThreads : blockDim.x;
  Stats mine = {kLowest, 0.f, 0.f};
  auto take = [&](const float* v, auto count) {
    constexpr int n = decltype(count)::value;
    float top = mine.m;
#pragma unroll
    for (int i = 0; i + 1 < n; i += 2) top = max3(top, v[i], v[i + 1]);
    if (n % 2) top = fmaxf(top, v[n - 1]);
    const float d = (mine.m - top) * k, e = exp2_fast(d);
    mine.t = kEntropy ? e * (mine.t + finite(d) * mine.s) : 0.f;
    mine.s *= e;
    mine.m = top;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float a = (v[i] - top) * k, w = exp2_fast(a);
      mine.s += w;
      if (kEntropy) mine.t += w * finite(a);
    }
  };
  constexpr int kAhead = 4;  // chunks under way
  int c = thread;
  for (; c + (kAhead - 1) * threads < row.chunks; c += kAhead * threads) {
    u32x4 u[kAhead];
    float v[kAhead * X::kPer];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) u[j] = row.chunk(c + j * threads);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) X::unpack(u[j], v + j * X::kPer);
    take(v, std::integral_constant<int, kAhead * X::kPer>());
  }
  for (; c < row.chunks; c += threads) {
    float v[X::kPer];
    X::unpack(row.chunk(c), v);
    take(v, std::integral_constant<int, X::kPer>());
  }
  for (int j = thread; j < row.kEdge; j += threads) {
    const int e = row.edge(j);
    if (e < 0) break;
    const float v[1] = {X::load(row.x + e)};
    take(v, std::integral_constant<int, 1>());
  }
  constexpr int kLanes = kThreads && kThreads < kWave ? kThreads : kWave;
  mine = joined_lanes<kEntropy, kLanes>(mine, [k](const Stats& a, const Stats& b) { return joined<kEntropy>(a, b, k); });
  if constexpr (kThreads && kThreads <= kWave) return mine;
  if (thread % kWave == 0) parts[thread / kWave] = mine;
  __syncthreads();
  Stats all = parts[0];
  for (int w = 1; w < threads / kWave; ++w) all = joined<kEntropy>(all, parts[w], k);
  return all;
}

// The gradient of a row, but for the additions at the token.
template <typename X, bool kEntropy, int kThreads = 0, typename Row>
__device__ __forceinline__ void write_gradient(const Row& row, typename X::type* g, int thread, float m, float k,
                                               Slope f) {
  const int threads = kThreads ? kThreads : blockDim.x;
  for (int c = thread; c < row.chunks; c += threads) {
    float v[X::kPer];
    X::unpack(row.chunk(c), v);
#pragma unroll
    for (int i = 0; i < X::kPer; ++i) v[i] = gradient_at<kEntropy>((v[i] - m) * k, f);
    *reinterpret_cast<u32x4_any*>(g + row.at(c)) = X::pack(v);
  }
  for (int j = thread; j < row.kEdge; j += threads) {
    const int e = row.edge(j);
    if (e >= 0) X::store(g + e, gradient_at<kEntropy>((X::load(row.x + e) - m) * k, f));
  }
}

// Zeros for a gradient's row.
template <typename X>
__device__ __forceinline__ void write_zeros(const Rows& r, int b, int t, int thread, int threads) {
  typename X::type* g = gradient_of<X>(r, b, t);
  const Line<X> row(g, r.V);
  for (int c = thread; c < row.chunks; c += threads) *reinterpret_cast<u32x4_at16*>(g + row.at(c)) = u32x4{};
  for (int j = thread; j < row.kEdge; j += threads) {
    const int e = row.edge(j);
    if (e >= 0) X::store(g + e, 0.f);
  }
}

// The token's value, added where its owner has just stored the rest (stores of one thread to one
// address keep their order).
template <typename X, bool kEntropy>
__device__ __forceinline__ void add_token(const Line<X>& row, typename X::type* g, int token, float x, float m,
                                          float k, Slope f) {
  if (row.owner(token, blockDim.x) == int(threadIdx.x))
    X::store(g + token, f.token + gradient_at<kEntropy>((x - m) * k, f));
}

// The teacher's entries of a row, in LDS: ids (-1: none, or one outside the vocabulary, which makes
// the row NaN), their probabilities, and their sum by id.
struct Entries {
  int id[TB_TEACHER_MOST];
  float q[TB_TEACHER_MOST], log_q[TB_TEACHER_MOST], x[TB_TEACHER_MOST];  // x: the row's logits there
  float part[16];
};

template <typename V>
__device__ __forceinline__ V block_sum(V v, V* part) {  // part: one a wavefront
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < int(blockDim.x / kWave); ++w) v += part[w];
  return v;
}
__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < int(blockDim.x / kWave); ++w) v = fmaxf(v, part[w]);
  return v;
}

// Fills `e`; the sum of exponentials: 0 for a row without entries, NaN for one with a wrong id.
template <typename X>
__device__ __forceinline__ float take_entries(const Rows& r, const Line<X>& row, const Teacher& q, int64_t at, float k,
                                              Entries& e) {
  float top = kLowest;
  for (int j = threadIdx.x; j < q.K; j += blockDim.x) {
    const float v = teacher_value(q, at * q.K + j);
    int id = -1;
    if (v != -INFINITY) {
      const int64_t wide = load_id(q.ids, q.long_ids, at * q.K + j);
      if (wide >= 0 && wide < r.V) id = int(wide);
      else if (r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
    }
    e.id[j] = id;
    e.x[j] = id < 0 ? 0.f : X::load(row.x + id);
    e.log_q[j] = v != -INFINITY && id < 0 ? __uint_as_float(kNan) : v;
    top = fmaxf(top, v);
  }
  top = block_max(top, e.part);
  float sum = 0.f;
  for (int j = threadIdx.x; j < q.K; j += blockDim.x) {
    const float a = (e.log_q[j] - top) * k;
    e.log_q[j] = a * kLn2;
    e.q[j] = exp2_fast(a);
    sum += e.q[j];
  }
  sum = block_sum(sum, e.part);
  const float log_sum = logf(sum), by = sum == 0.f ? 0.f : 1.f / sum;
  for (int j = threadIdx.x; j < q.K; j += blockDim.x) {
    e.log_q[j] -= log_sum;
    e.q[j] *= by;
  }
  __syncthreads();
  return sum;
}

// The gradient at the teacher's entries, behind a barrier after everything else is stored.
template <typename X>
__device__ __forceinline__ void add_entries(const Line<X>& row, typename X::type* g, const Teacher& q,
                                            const Entries& e, float m, float k, Slope f) {
  for (int j = threadIdx.x; j < q.K; j += blockDim.x) {
    const int id = e.id[j];
    if (id < 0) continue;
    float sum = 0.f;
    for (int i = 0; i < q.K; ++i) sum += e.id[i] == id ? e.q[i] : 0.f;
    X::store(g + id, exp2_fast((e.x[j] - m) * k) * f.by_weight - f.token * sum);
  }
}

// The gradient of a row's divergence; m, s: the row's statistics, sum: of take_entries, w: cotangent.
template <typename X>
__device__ __forceinline__ void write_distilled(const Rows& r, const Line<X>& row, const Teacher& q, const Entries& e,
                                                int b, int t, float m, float s, float sum, float w, float k) {
  if (sum == 0.f) {
    write_zeros<X>(r, b, t, threadIdx.x, blockDim.x);
    return;
  }
  typename X::type* g = gradient_of<X>(r, b, t);
  Slope f = {0.f, 0.f, q.tau * w * r.g_scale};
  f.by_weight = sum == sum ? f.token / s : sum;
  write_gradient<X, false>(row, g, threadIdx.x, m, k, f);
  __syncthreads();  // (what it has stored comes before what follows)
  add_entries<X>(row, g, q, e, m, k, f);
}

template <int kOp>
struct Shared {
  Stats parts[8];
  int totals[8];
};
template <>
struct Shared<kDistill> {
  Stats parts[8];
  int totals[8];
  Entries entries;
};

template <typename X, int kOp, bool kEntropy>
__device__ __forceinline__ float4 sweep_row(const Rows& r, const RowOut& o, const Policy& p, const Teacher& q, float w,
                                            int b, int t, int64_t at, Shared<kOp>& shared) {
  const bool first = threadIdx.x == 0;
  const Line<X> row(row_of<X>(r, b, t), r.V);
  const float k = r.inv_temp * kLog2e;
  if constexpr (kOp != kDistill) {
    const int token = take_token(r, b, t, first);
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(row.x + token);
    const Stats s = row_stats<X, kEntropy>(row, k, threadIdx.x, shared.parts);
    const float log_s = logf(s.s), lp = (x - s.m) * r.inv_temp - log_s;
    const float H = kEntropy ? log_s - kLn2 * s.t / s.s : 0.f;
    Position v = {};
    if (kOp == kPolicy) v = policy_position(p, b, at, lp, H, w);
    if (first) {
      if (o.logprobs) o.logprobs[at] = lp;
      if (o.entropy) o.entropy[at] = H;
      if (kOp == kScore && o.exact) o.exact[at] = exact_lp(double(x - s.m) * k, s.s);
      if (o.state) o.state[at] = {s.m, s.s * to_scaled(s.m, k), H, lp};
      if (o.d_logprobs) o.d_logprobs[at] = v.d_lp;
      if (o.d_entropy) o.d_entropy[at] = v.d_H;
    }
    if (kOp == kPolicy && r.g) {
      const Slope f = slope_of(s.s, H, v.d_lp, v.d_H, r.g_scale * r.inv_temp);
      typename X::type* g = gradient_of<X>(r, b, t);
      write_gradient<X, kEntropy>(row, g, threadIdx.x, s.m, k, f);
      if (token >= 0) add_token<X, kEntropy>(row, g, token, x, s.m, k, f);
    }
    return v.terms;
  } else {
    Entries& e = shared.entries;
    const float sum = take_entries<X>(r, row, q, at, k, e);
    const Stats s = row_stats<X, false>(row, k, threadIdx.x, shared.parts);
    const float log_s = logf(s.s);
    float d = 0.f;
    for (int j = threadIdx.x; j < q.K; j += blockDim.x)
      if (!(e.q[j] <= 0.f)) d += e.q[j] * (e.log_q[j] - ((e.x[j] - s.m) * r.inv_temp - log_s));
    d = block_sum(d, e.part) * q.tau * q.tau;
    if (sum == 0.f) w = 0.f;
    if (first) {
      if (o.state) o.state[at] = {s.m, s.s * to_scaled(s.m, k), 0.f, d};
      if (o.d_logprobs) o.d_logprobs[at] = w;
      if (o.logprobs) o.logprobs[at] = d;
    }
    if (r.g) write_distilled<X>(r, row, q, e, b, t, s.m, s.s, sum, w, k);
    return {d, 0.f, 0.f, 0.f};
  }
}

// One workgroup a row; the row is read from memory in every sweep over it.
template <typename X, int kOp, bool kEntropy>
__global__ __launch_bounds__(512) void sweep_kernel(Rows r, RowOut o, Policy p, Mean mean, Teacher q) {
  __shared__ Shared<kOp> shared;
  const int64_t rows = int64_t(r.B) * r.T;
  int total = 0;
  if (kOp != kScore) {
    const int part = full_wave_sum(share_of_total(r, mean));
    if (threadIdx.x % kWave == 0) shared.totals[threadIdx.x / kWave] = part;
    __syncthreads();
    for (int w = 0; w < int(blockDim.x / kWave); ++w) total += shared.totals[w];
  }
  double sum[4] = {};
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    const int64_t at = row_of_group(i, rows);
    const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
    if (threadIdx.x == 0 && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    if (counts(r, b, t)) {
      const float w = kOp == kScore ? 0.f : weight_of(r, mean, b, total);
      const float4 v = sweep_row<X, kOp, kEntropy>(r, o, p, q, w, b, t, at, shared);
      sum[0] += double(w) * v.x;
      sum[1] += double(w) * v.y;
      sum[2] += double(w) * v.z;
      sum[3] += double(w) * v.w;
    } else {
      if (threadIdx.x == 0) leave_nothing(o, at);
      if (r.g) write_zeros<X>(r, b, t, threadIdx.x, blockDim.x);
    }
    __syncthreads();  // (before the next row takes the shared memory)
  }
  if (kOp != kScore && threadIdx.x == 0)
    for (int j = 0; j < 4; ++j) o.partial[int64_t(blockIdx.x) * 4 + j] = sum[j];
}

// The gradient of a row whose statistics are given.
template <typename X, int kOp, bool kEntropy>
__device__ __forceinline__ void given_row(const Rows& r, const Given& v, const Teacher& q, int b, int t, int64_t at,
                                          Shared<kOp>& shared) {
  const Line<X> row(row_of<X>(r, b, t), r.V);
  const float k = r.inv_temp * kLog2e, up = v.upstream ? *v.upstream : 1.f;
  const float4 state = v.state[at];
  const float d = v.d_lp[b * v.d_seq + t * v.d_pos] * up;
  if constexpr (kOp != kDistill) {
    const float d_H = kEntropy ? v.d_entropy[b * v.d_seq + t * v.d_pos] * up : 0.f;
    const int token = take_token(r, b, t, false);
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(row.x + token);
    __syncthreads();  // (the row may be the gradient's own memory)
    const Slope f = slope_of(state.y * from_scaled(state.x, k), state.z, token < 0 ? x : d, d_H, r.g_scale * r.inv_temp);
    typename X::type* g = gradient_of<X>(r, b, t);
    write_gradient<X, kEntropy>(row, g, threadIdx.x, state.x, k, f);
    if (token >= 0) add_token<X, kEntropy>(row, g, token, x, state.x, k, f);
  } else {
    const float sum = take_entries<X>(r, row, q, at, k, shared.entries);
    write_distilled<X>(r, row, q, shared.entries, b, t, state.x, state.y * from_scaled(state.x, k), sum, d, k);
  }
}

template <typename X, int kOp, bool kEntropy>
__global__ __launch_bounds__(512) void gradient_kernel(Rows r, Given v, Teacher q) {
  __shared__ Shared<kOp> shared;
  const int64_t rows = int64_t(r.B) * r.T;
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    const int64_t at = row_of_group(i, rows);
    const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
    if (counts(r, b, t)) given_row<X, kOp, kEntropy>(r, v, q, b, t, at, shared);
    else write_zeros<X>(r, b, t, threadIdx.x, blockDim.x);
    __syncthreads();
  }
}

// ---- rows in the registers of a workgroup -----------------------------------------------------

constexpr int kHeldThreads = 512;

// A row's chunks in registers of kThreads threads, kChunks each: chunk k * kThreads + thread.  With
// kChunks = V / kPer / kThreads rounded up, all but the last two are there in every thread (the row's head
// takes up to eight chunks from the last but one); what lies beyond the row is -inf.
// With kMore, chunks from kChunks on are in LDS, where they come without passing through registers: the
// registers and the LDS of a compute unit hold 512 KB of a row together.
extern __shared__ u32x4 more_chunks[];
template <typename X, int kThreads, int kChunks, bool kMore = false>
struct Held {
  // (a wavefront's lanes would have two values of head and rest each if it read whole lines)
  using Row = Span<X, kThreads <= kWave ? 16 : kLine>;
  static_assert(Row::kEdge <= kThreads);
  static constexpr int kSure = kChunks - (kMore ? 1 : 2);
  u32x4 c[kChunks];
  float edge;
  int edge_at;
  int more;  // chunks in LDS
  __device__ __forceinline__ void load(const Row& row, int thread) {
    const char* from = reinterpret_cast<const char*>(row.x + row.head);
    const uint32_t lane = thread * 16u;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      if (k >= kSure) c[k] = u32x4{X::kNone, X::kNone, X::kNone, X::kNone};
      if (k < kSure || there(row, thread, k)) c[k] = *reinterpret_cast<const u32x4_at16*>(from + k * (kThreads * 16) + lane);
    }
    more = 0;
    if constexpr (kMore) {
      more = (row.chunks + kThreads - 1) / kThreads - kChunks;
      for (int j = 0; j < more; ++j)
        if (there(row, thread, kChunks + j))
          __builtin_amdgcn_global_load_lds(
              (const __attribute__((address_space(1))) void*)(from + int64_t(kChunks + j) * (kThreads * 16) + lane),
              (__attribute__((address_space(3))) void*)(more_chunks + j * kThreads + thread / kWave * kWave), 16, 0, 0);
    }
    edge_at = row.edge(thread);
    edge = edge_at >= 0 ? X::load(row.x + edge_at) : -INFINITY;
  }
  // LDS chunk j of the thread, when all that has been loaded is there
  __device__ __forceinline__ u32x4 chunk_in_lds(const Row& row, int thread, int j) const {
    const u32x4 none = {X::kNone, X::kNone, X::kNone, X::kNone};
    return there(row, thread, kChunks + j) ? more_chunks[j * kThreads + thread] : none;
  }
  static __device__ __forceinline__ bool there(const Row& row, int thread, int k) {
    return thread + k * kThreads < row.chunks;
  }
  // Keeps the compiler from holding the values that it has unpacked until they are used again, which
  // would take twice the registers of the row itself.
  __device__ __forceinline__ void keep_packed() {
#pragma unroll
    for (int k = 0; k < kChunks; ++k) asm volatile("" : "+v"(c[k]));
  }
};

// Over the lanes of a wavefront that share a row, all of them or 16.
template <int kThreads>
__device__ __forceinline__ float lanes_max(float v) {
  static_assert(kThreads == 16 || kThreads >= kWave);
  if constexpr (kThreads >= kWave) return full_wave_max(v);
  v = fmaxf(v, neighbour<1>(v));
  v = fmaxf(v, neighbour<2>(v));
  v = fmaxf(v, neighbour<4>(v));
  return fmaxf(v, neighbour<8>(v));
}
template <int kThreads>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (kThreads >= kWave) return full_wave_sum(v);
  v += neighbour<1>(v);
  v += neighbour<2>(v);
  v += neighbour<4>(v);
  return v + neighbour<8>(v);
}

// Statistics of a wavefront's part of a row, the same in all lanes, of weights 2^(x k - M), M = scaled(m, k).
// m need not be the largest value: any that keeps the weights in range does.  It is the largest of the
// lanes' own, found on the packed values as signed integers: right where a lane has a value above 0, else
// the lane's smallest (half an instruction a value instead of two and a half).  Where that takes the sum
// out of range, `fine` is false and the row has to be swept.  So it is where a wavefront's part of a row has
// a sum beyond 2^88: another part's reference may be so much larger that this one's factor, 2^-126 and
// below, is 0, and what is lost no longer negligible (otherwise it is below 2^-30 of the row's sum).
template <bool kEntropy, typename X, int kThreads, int kChunks, bool kMore>
__device__ __forceinline__ Stats wave_stats(const typename Held<X, kThreads, kChunks, kMore>::Row& row,
                                            Held<X, kThreads, kChunks, kMore>& h, int thread, float k) {
  Stats mine = {fmaxf(h.edge, -kExtreme), 0.f, 0.f};
  if constexpr (kChunks > 2) mine.m = fmaxf(mine.m, X::template upper<kChunks - 2>(h.c));
#pragma unroll
  for (int j = kChunks > 2 ? kChunks - 2 : 0; j < kChunks; ++j) {  // (with what lies beyond the row)
    float v[X::kPer];
    X::unpack(h.c[j], v);
#pragma unroll
    for (int i = 0; i < X::kPer; i += 2) mine.m = max3(mine.m, v[i], v[i + 1]);
  }
  mine.m = lanes_max<kThreads>(mine.m);
  const float M = scaled(mine.m, k);
  auto take = [&](float x) {
    const float a = fmaf(x, k, -M), w = exp2_fast(a);
    mine.s += w;
    if (kEntropy) mine.t += w * finite(a);
  };
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[X::kPer];
    X::unpack(h.c[j], v);
#pragma unroll
    for (int i = 0; i < X::kPer; ++i) take(v[i]);
  }
  take(h.edge);
  h.keep_packed();
  if constexpr (kMore) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what a wavefront has asked for is in LDS then)
    for (int j = 0; j < h.more; ++j) {
      float v[X::kPer];
      X::unpack(h.chunk_in_lds(row, thread, j), v);
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) take(v[i]);
    }
  }
  mine.s = lanes_sum<kThreads>(mine.s);
  if (kEntropy) mine.t = lanes_sum<kThreads>(mine.t);
  if (kThreads > kWave && mine.s > 0x1p88f) mine.s = __uint_as_float(kNan);
  return mine;
}
__device__ __forceinline__ bool fine(const Stats& s, float k) {
  return scales(s.m, k) && s.s > 0x1p-40f && s.s < 0x1p40f;
}

template <bool kEntropy, typename X, int kThreads, int kChunks, bool kMore>
__device__ __forceinline__ void write_held(const typename Held<X, kThreads, kChunks, kMore>::Row& row,
                                           const Held<X, kThreads, kChunks, kMore>& h, typename X::type* g, int thread,
                                           float m, float k, Slope f) {
  const float M = scaled(m, k);
  char* to = reinterpret_cast<char*>(g + row.head);
  const uint32_t lane = thread * 16u;
  auto value = [&](float x) { return gradient_at<kEntropy>(fmaf(x, k, -M), f); };
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    float v[X::kPer];
    X::unpack(h.c[j], v);
#pragma unroll
    for (int i = 0; i < X::kPer; ++i) v[i] = value(v[i]);
    if (j < h.kSure || h.there(row, thread, j))
      *reinterpret_cast<u32x4_any*>(to + j * (kThreads * 16) + lane) = X::pack(v);
  }
  if constexpr (kMore)
    for (int j = 0; j < h.more; ++j) {
      float v[X::kPer];
      X::unpack(h.chunk_in_lds(row, thread, j), v);
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) v[i] = value(v[i]);
      if (h.there(row, thread, kChunks + j))
        *reinterpret_cast<u32x4_any*>(to + int64_t(kChunks + j) * (kThreads * 16) + lane) = X::pack(v);
    }
  if (h.edge_at >= 0) X::store(g + h.edge_at, value(h.edge));
}

// Statistics of the row, in every thread, of the parts that four or eight wavefronts leave: one a lane,
// joined in two or three steps.
template <bool kEntropy, int kWaves>
__device__ __forceinline__ Stats block_stats(const Stats* parts, float k) {
  static_assert(kWaves == 8 || kWaves == 4);
  Stats s = parts[threadIdx.x % kWaves];
  float m = s.m;
  m = fmaxf(m, neighbour<1>(m));
  m = fmaxf(m, neighbour<2>(m));
  if (kWaves == 8) m = fmaxf(m, neighbour<4>(m));
  const float d = scaled(s.m, k) - scaled(m, k), e = exp2_fast(d);
  if (kEntropy) s.t = e * (s.t + finite(d) * s.s);
  s.s *= e;
  s.s += neighbour<1>(s.s);
  s.s += neighbour<2>(s.s);
  if (kWaves == 8) s.s += neighbour<4>(s.s);
  if (kEntropy) {
    s.t += neighbour<1>(s.t);
    s.t += neighbour<2>(s.t);
    if (kWaves == 8) s.t += neighbour<4>(s.t);
  }
  auto uniform = [](float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); };
  return {uniform(m), uniform(s.s), kEntropy ? uniform(s.t) : 0.f};
}

// One workgroup a row; the score, and the policy loss.
template <typename X, int kOp, bool kEntropy, int kThreads, int kChunks, bool kMore = false>
__global__ __launch_bounds__(kThreads) void held_kernel(Rows r, RowOut o, Policy p, Mean mean) {
  constexpr int kWaves = kThreads / kWave;
  __shared__ Stats parts[kWaves];
  __shared__ int totals[kWaves];
  const int64_t at = row_of_group(blockIdx.x, int64_t(r.B) * r.T);
  const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
  const bool first = threadIdx.x == 0;
  if (first && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
  if (!counts(r, b, t)) {
    if (first) leave_nothing(o, at);
    if (kOp == kPolicy && threadIdx.x < 4) o.partial[int64_t(blockIdx.x) * 4 + threadIdx.x] = 0.0;
    if (r.g) write_zeros<X>(r, b, t, threadIdx.x, blockDim.x);
    return;
  }
  const Line<X> row(row_of<X>(r, b, t), r.V);
  // (what comes first is waited for first: not behind the whole row)
  const int token = take_token(r, b, t, first), share = kOp == kPolicy ? share_of_total(r, mean) : 0;
  Held<X, kThreads, kChunks, kMore> h;
  h.load(row, threadIdx.x);
  const float x = token < 0 ? __uint_as_float(kNan) : X::load(row.x + token);
  const float k = r.inv_temp * kLog2e;
  if (kOp == kPolicy) {
    const int part = full_wave_sum(share);
    if (threadIdx.x % kWave == 0) totals[threadIdx.x / kWave] = part;
  }
  const Stats part = wave_stats<kEntropy>(row, h, threadIdx.x, k);
  if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = part;
  __syncthreads();
  Stats s = block_stats<kEntropy, kWaves>(parts, k);
  const bool extreme = !fine(s, k);
  if (extreme) {
    __syncthreads();
    s = row_stats<X, kEntropy>(row, k, threadIdx.x, parts);
  }
  const float log_s = logf(s.s);
  const float lp = (extreme ? (x - s.m) * r.inv_temp : fmaf(x, k, -scaled(s.m, k)) * kLn2) - log_s;
  const float H = kEntropy ? log_s - kLn2 * s.t / s.s : 0.f;
  Position v = {};
  if constexpr (kOp == kPolicy) {
    int total = 0;
    for (int w = 0; w < kWaves; ++w) total += totals[w];
    const float w = weight_of(r, mean, b, total);
    v = policy_position(p, b, at, lp, H, w);
    if (first) {
      double* to = o.partial + int64_t(blockIdx.x) * 4;
      to[0] = double(w) * v.terms.x;
      to[1] = double(w) * v.terms.y;
      to[2] = double(w) * v.terms.z;
      to[3] = double(w) * v.terms.w;
    }
  }
  if (first) {
    if (o.logprobs) o.logprobs[at] = lp;
    if (o.entropy) o.entropy[at] = H;
    if (kOp == kScore && o.exact)
      o.exact[at] = exact_lp(extreme ? double(x - s.m) * k : double(x) * k - double(scaled(s.m, k)), s.s);
    if (o.state) o.state[at] = {s.m, extreme ? s.s * to_scaled(s.m, k) : s.s, H, lp};
    if (o.d_logprobs) o.d_logprobs[at] = v.d_lp;
    if (o.d_entropy) o.d_entropy[at] = v.d_H;
  }
  if (kOp == kScore || !r.g) return;
  const Slope f = slope_of(s.s, H, v.d_lp, v.d_H, r.g_scale * r.inv_temp);
  typename X::type* g = gradient_of<X>(r, b, t);
  if (extreme) {
    write_gradient<X, kEntropy>(row, g, threadIdx.x, s.m, k, f);
    if (token >= 0) add_token<X, kEntropy>(row, g, token, x, s.m, k, f);
    return;
  }
  write_held<kEntropy>(row, h, g, threadIdx.x, s.m, k, f);
  if (token >= 0 && row.owner(token, kThreads) == int(threadIdx.x))
    X::store(g + token, f.token + gradient_at<kEntropy>(fmaf(x, k, -scaled(s.m, k)), f));
}

// ---- distillation on rows in registers --------------------------------------------------------

// kThreads threads a row, kEntries entries of the teacher each: a workgroup, or a wavefront or 16 lanes of
// one that then take several rows.  While the row is on its way to the registers, its threads look for ids
// that come up twice; entry j's thread writes the gradient at id j behind the others' stores, with the
// sum of the probabilities of this id if it does.
template <typename X, int kThreads, int kChunks, int kEntries, bool kMore = false>
__global__ __launch_bounds__(kThreads <= kWave ? kLaneThreads : kThreads) void distill_kernel(Rows r, RowOut o, Mean mean,
                                                                                           Teacher q) {
  constexpr bool kAlone = kThreads > kWave;  // (the workgroup has one row)
  constexpr int kTeams = kAlone ? 1 : kLaneThreads / kThreads, kWaves = kAlone ? kThreads / kWave : 1;
  constexpr int kLanes = kAlone ? kWave : kThreads, kRoom = kThreads * kEntries;
  __shared__ __attribute__((aligned(16))) int ids[kTeams][kRoom];
  __shared__ __attribute__((aligned(16))) float shares[kTeams][kRoom];
  __shared__ Stats parts[kTeams][kWaves], teachers[kTeams][kWaves];
  __shared__ float losses[kTeams][kWaves];
  __shared__ int totals[kAlone ? kWaves : kLaneThreads / kWave];
  const int team = threadIdx.x / kThreads, thread = threadIdx.x % kThreads, wave = thread / kWave;
  const bool first = thread == 0;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  int total = 0;
  if constexpr (!kAlone) {
    const int part = full_wave_sum(share_of_total(r, mean));
    if (threadIdx.x % kWave == 0) totals[threadIdx.x / kWave] = part;
    __syncthreads();
    for (int w = 0; w < kLaneThreads / kWave; ++w) total += totals[w];
  }
  double sum = 0;
  auto take_row = [&](int64_t i) {
    const int64_t at = kAlone ? row_of_group(i, rows) : i;
    const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
    if (first && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    typename X::type* g = r.g ? gradient_of<X>(r, b, t) : nullptr;
    auto zeros = [&] {
      if (g) write_zeros<X>(r, b, t, thread, kThreads);
    };
    if (!counts(r, b, t)) {
      if (first) leave_nothing(o, at);
      zeros();
      return;
    }
    const typename Held<X, kThreads, kChunks, kMore>::Row row(row_of<X>(r, b, t), r.V);
    // (what comes first is waited for first: not behind the whole row)
    float v[kEntries], x[kEntries];
    int64_t wide[kEntries];
    int id[kEntries];
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      const int j = thread + e * kThreads;
      v[e] = -INFINITY;
      wide[e] = -1;
      if (j < q.K) {
        v[e] = teacher_value(q, at * q.K + j);
        wide[e] = load_id(q.ids, q.long_ids, at * q.K + j);
      }
    }
    const int share = kAlone ? share_of_total(r, mean) : 0;
    Held<X, kThreads, kChunks, kMore> h;
    h.load(row, thread);
    Stats teacher = {kLowest, 0.f, 0.f};
    bool wrong = false;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      const bool entry = v[e] != -INFINITY, fits = wide[e] >= 0 && wide[e] < r.V;
      if (entry && !fits) {
        wrong = true;
        v[e] = __uint_as_float(kNan);
      }
      id[e] = entry && fits ? int(wide[e]) : -1;
      x[e] = id[e] >= 0 ? X::load(row.x + id[e]) : 0.f;
      const int j = thread + e * kThreads;
      ids[team][j] = id[e] >= 0 ? id[e] : ~j;
      teacher.m = fmaxf(teacher.m, v[e]);
    }
    if (wrong && r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
#pragma unroll
    for (int e = 0; e < kEntries; ++e) teacher.s += exp2_fast((v[e] - teacher.m) * k);
    teacher = joined_lanes<false, kLanes>(teacher, [k](const Stats& a, const Stats& c) { return joined<false>(a, c, k); });
    if constexpr (kAlone) {
      const int part = full_wave_sum(share);
      if (thread % kWave == 0) {
        totals[wave] = part;
        teachers[team][wave] = teacher;
      }
    }
    meet<kThreads>();
    uint32_t twice = 0;  // (bit e: entry e's id has others)
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      const int j = thread + e * kThreads;
      if (j >= q.K) continue;
      int found = 0;
      for (int c = 0; c < q.K; c += 4) {
        const int4 u = *reinterpret_cast<const int4*>(&ids[team][c]);
        found += (u.x == id[e]) + (u.y == id[e]) + (u.z == id[e]) + (u.w == id[e]);
      }
      if (found > 1) twice |= 1u << e;
    }
    const Stats mine = wave_stats<false>(row, h, thread, k);
    Stats s = mine;
    if constexpr (kAlone) {
      if (thread % kWave == 0) parts[team][wave] = mine;
      __syncthreads();
      s = block_stats<false, kWaves>(parts[team], k);
      teacher = teachers[team][0];
      for (int w = 1; w < kWaves; ++w) teacher = joined<false>(teacher, teachers[team][w], k);
      total = 0;
      for (int w = 0; w < kWaves; ++w) total += totals[w];
    }
    const bool extreme = !fine(s, k);
    if (extreme) {
      meet<kThreads>();
      s = row_stats<X, false, kThreads>(row, k, thread, parts[team]);
    }
    const float log_s = logf(s.s), log_t = logf(teacher.s), by = teacher.s == 0.f ? 0.f : 1.f / teacher.s;
    const float M = scaled(s.m, k);
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      const float a = (v[e] - teacher.m) * k, share_e = exp2_fast(a) * by;
      const float z = extreme ? (x[e] - s.m) * k : fmaf(x[e], k, -M);
      if (!(share_e <= 0.f)) d += share_e * ((a - z) * kLn2 - (log_t - log_s));
      v[e] = share_e;
      x[e] = z;
      shares[team][thread + e * kThreads] = share_e;
    }
    d = lanes_sum<kThreads>(d);
    if (thread % kWave == 0) losses[team][wave] = d;
    const float w = teacher.s == 0.f ? 0.f : weight_of(r, mean, b, total);
    Slope f = {0.f, 0.f, q.tau * w * r.g_scale};
    f.by_weight = teacher.s == teacher.s ? f.token / s.s : teacher.s;
    if (teacher.s == 0.f) zeros();
    else if (g && extreme) write_gradient<X, false, kThreads>(row, g, thread, s.m, k, f);
    else if (g) write_held<false>(row, h, g, thread, s.m, k, f);
    meet<kThreads>();  // (what it has stored comes before what follows)
    if (g && teacher.s != 0.f) {
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        if (id[e] < 0) continue;
        float sum_e = v[e];
        if (twice >> e & 1) {
          sum_e = 0.f;
          for (int c = 0; c < q.K; ++c) sum_e += ids[team][c] == id[e] ? shares[team][c] : 0.f;
        }
        X::store(g + id[e], exp2_fast(x[e]) * f.by_weight - f.token * sum_e);
      }
    }
    d = 0.f;
    for (int c = 0; c < kWaves; ++c) d += losses[team][c];
    d *= q.tau * q.tau;
    if (first) {
      if (o.state) o.state[at] = {s.m, extreme ? s.s * to_scaled(s.m, k) : s.s, 0.f, d};
      if (o.d_logprobs) o.d_logprobs[at] = w;
      if (o.logprobs) o.logprobs[at] = d;
    }
    sum += double(w) * d;
  };
  // (a workgroup takes one row: what lives from row to row would cost it registers)
  if constexpr (!kAlone) {
    for (int64_t i = int64_t(blockIdx.x) * kTeams + team; i < rows; i += int64_t(gridDim.x) * kTeams) {
      take_row(i);
      meet<kThreads>();  // (before the next row takes the shared memory)
    }
  } else {
    take_row(blockIdx.x);
  }
  __shared__ double sums[kTeams];
  if (first) sums[team] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kTeams; ++w) sum += sums[w];
    double* to = o.partial + int64_t(blockIdx.x) * 4;
    to[0] = sum;
    to[1] = to[2] = to[3] = 0.0;
  }
}

// ---- launches ---------------------------------------------------------------------------------

int grid_of(const Rows& r) {
  const int64_t rows = int64_t(r.B) * r.T;
  return int(rows < kMostGroups ? rows : kMostGroups);
}
// Of a workgroup that sweeps over a row: two chunks a thread at least (the gradient alone of 32760 rows of
// 4097 values in bfloat16: 172 us with 512 threads, 97 with 128).
int threads_of(const Rows& r, int per) {
  const int chunks = r.V / per;
  return chunks >= 1280 ? 512 : chunks >= 768 ? 256 : chunks >= 256 ? 128 : kWave;
}

template <typename X, int kOp, bool kEntropy>
bool launch_lanes(Call& c) {
  const Rows& r = c.rows;
  const int64_t rows = int64_t(r.B) * r.T;
  auto go = [&](auto kernel, int lanes) {
    const int64_t teams = kLaneThreads / lanes, groups = (rows + teams - 1) / teams;
    c.groups = int(groups < kLaneGroups ? groups : kLaneGroups);
    kernel<<<c.groups, kLaneThreads, 0, c.stream>>>(r, c.out, c.policy, c.mean, c.given);
    return true;
  };
  const int chunks = (r.V + X::kPer - 1) / X::kPer;
  if (r.V < X::kPer) return false;
#define LANES(lanes, n) \
  if (chunks <= lanes * n) return go(lanes_kernel<X, kOp, kEntropy, lanes, n>, lanes);
  LANES(2, 3) LANES(2, 4) LANES(4, 3) LANES(4, 4) LANES(8, 3) LANES(8, 4) LANES(16, 3) LANES(16, 4) LANES(16, 5) LANES(16, 6) LANES(32, 4)
  LANES(64, 3) LANES(64, 4) LANES(64, 5) LANES(64, 6) LANES(64, 7) LANES(64, 8)
#undef LANES
  return false;
}

// Longer rows than 32 chunks a thread: 32 or 46 of them in registers and up to 18 in LDS, one workgroup a unit.
// 46 are as many as a thread has registers for beside its work, with which rows of 64 fit; they have to be there in
// every thread, so that rows of up to 46 hold 32.  Where both would do, 47 to 50, 46 take 1 to 4 % less (2048 rows of 200003
// values in bfloat16, of which three quarters count: policy loss 325 and 331 us, distilled 342 and 356).
// 2047 rows of 262144 values in bfloat16, distilled: 655 us with sweeps and 443 so, on one card; 449 to 482 on others
// (4.2 to 4.6 TB/s).
constexpr int kMoreFrom = 32, kFewer = 32, kMostHeld = 46, kMostMore = 18;
template <typename Kernel>
bool more_in_lds(Kernel kernel, int chunks, size_t* bytes) {
  *bytes = size_t(chunks) * kHeldThreads * sizeof(u32x4);
  return grant_dynamic_lds(reinterpret_cast<const void*>(kernel), *bytes) == hipSuccess;
}

template <typename X, int kOp, bool kEntropy>
bool launch_held(Call& c) {
  const Rows& r = c.rows;
  const int64_t rows = int64_t(r.B) * r.T;
  if (rows > kMostGroups || r.V < 2 * X::kPer) return false;
  c.groups = int(rows);
  const int need = (r.V / X::kPer + kHeldThreads - 1) / kHeldThreads;
  if (kOp == kPolicy && need > kMoreFrom) {
    auto go = [&](auto kernel, int held) {
      size_t bytes;
      if (need - held > kMostMore || !more_in_lds(kernel, need - held, &bytes)) return false;
      kernel<<<int(rows), kHeldThreads, bytes, c.stream>>>(r, c.out, c.policy, c.mean);
      return true;
    };
    return need <= kMostHeld ? go(held_kernel<X, kPolicy, kEntropy, kHeldThreads, kFewer, true>, kFewer)
                                      : go(held_kernel<X, kPolicy, kEntropy, kHeldThreads, kMostHeld, true>, kMostHeld);
  }
#define HELD(n) \
  case n: held_kernel<X, kOp, kEntropy, kHeldThreads, n><<<int(rows), kHeldThreads, 0, c.stream>>>(r, c.out, c.policy, c.mean); return true;
#define HALF(n) \
  case n: held_kernel<X, kOp, kEntropy, kHeldThreads / 2, n><<<int(rows), kHeldThreads / 2, 0, c.stream>>>(r, c.out, c.policy, c.mean); return true;
  // rows of up to 2048 chunks by half as many threads, which more of them keep busy (policy
  // loss on 26840 rows of 5000 values in bfloat16: 170 us with all, 107 so); rows of up to 512 chunks have gone to lanes
  switch ((r.V / X::kPer + kHeldThreads / 2 - 1) / (kHeldThreads / 2)) { HALF(2) HALF(3) HALF(4) HALF(5) HALF(6) HALF(7) HALF(8) }
  switch (need) {
    HELD(5) HELD(6) HELD(7) HELD(8) HELD(9) HELD(10) HELD(11) HELD(12) HELD(13) HELD(14)
    HELD(15) HELD(16) HELD(17) HELD(18) HELD(19) HELD(20) HELD(21) HELD(22) HELD(23) HELD(24) HELD(25) HELD(26) HELD(27)
    HELD(28) HELD(29) HELD(30) HELD(31) HELD(32)
  }
#undef HALF
#undef HELD
  return false;
}

// 16 lanes of a wavefront a row of up to 128 chunks, a wavefront one of up to 512, a workgroup one of more.
// kFrom: chunks a lane that shorter rows leave to fewer lanes.
template <typename X, int kThreads, int kEntries, int kFrom = 1>
bool launch_distill_lanes(Call& c) {
  const Rows& r = c.rows;
  constexpr int kTeams = kLaneThreads / kThreads;
  const int64_t groups = (int64_t(r.B) * r.T + kTeams - 1) / kTeams;
  c.groups = int(groups < kLaneGroups ? groups : kLaneGroups);
#define HELD(n) \
  case n: if constexpr (n >= kFrom) { distill_kernel<X, kThreads, n, kEntries><<<c.groups, kLaneThreads, 0, c.stream>>>(r, c.out, c.mean, c.teacher); return true; } else break;
  switch ((r.V / X::kPer + kThreads - 1) / kThreads) { HELD(1) HELD(2) HELD(3) HELD(4) HELD(5) HELD(6) HELD(7) HELD(8) }
#undef HELD
  return false;
}
template <typename X, int kEntries>
bool launch_distill_block(Call& c) {
  const Rows& r = c.rows;
  if (int64_t(r.B) * r.T > kMostGroups) return false;
  c.groups = grid_of(r);
#define HELD(n) \
  case n: distill_kernel<X, kHeldThreads, n, kEntries><<<c.groups, kHeldThreads, 0, c.stream>>>(r, c.out, c.mean, c.teacher); return true;
  const int need = (r.V / X::kPer + kHeldThreads - 1) / kHeldThreads;
  if (need > kMoreFrom) {
    auto go = [&](auto kernel, int held) {
      size_t bytes;
      if (need - held > kMostMore || !more_in_lds(kernel, need - held, &bytes)) return false;
      kernel<<<c.groups, kHeldThreads, bytes, c.stream>>>(r, c.out, c.mean, c.teacher);
      return true;
    };
    return need <= kMostHeld ? go(distill_kernel<X, kHeldThreads, kFewer, kEntries, true>, kFewer)
                                      : go(distill_kernel<X, kHeldThreads, kMostHeld, kEntries, true>, kMostHeld);
  }
#define HALF(n) \
  case n: distill_kernel<X, kHeldThreads / 2, n, 2 * kEntries><<<c.groups, kHeldThreads / 2, 0, c.stream>>>(r, c.out, c.mean, c.teacher); return true;
  // (rows of up to 512 whole chunks have gone to wavefronts)
  switch ((r.V / X::kPer + kHeldThreads / 2 - 1) / (kHeldThreads / 2)) { HALF(3) HALF(4) HALF(5) HALF(6) HALF(7) HALF(8) }
#undef HALF
  switch (need) {
    HELD(5) HELD(6) HELD(7) HELD(8) HELD(9) HELD(10) HELD(11) HELD(12) HELD(13) HELD(14)
    HELD(15) HELD(16) HELD(17) HELD(18) HELD(19) HELD(20) HELD(21) HELD(22) HELD(23) HELD(24) HELD(25) HELD(26) HELD(27)
    HELD(28) HELD(29) HELD(30) HELD(31) HELD(32)
  }
#undef HELD
  return false;
}
template <typename X>
bool launch_distill(Call& c) {
  if (c.rows.V < 2 * X::kPer) return false;
  const int K = c.teacher.K;
  if (K <= 16 && launch_distill_lanes<X, 16, 1>(c)) return true;
  if (K <= 64) return launch_distill_lanes<X, 16, 4>(c) || launch_distill_lanes<X, kWave, 1, 3>(c) || launch_distill_block<X, 1>(c);
  if (K <= 256) return launch_distill_lanes<X, kWave, 4>(c) || launch_distill_block<X, 1>(c);
  return launch_distill_lanes<X, kWave, 16>(c) || (K <= 512 ? launch_distill_block<X, 1>(c) : launch_distill_block<X, 2>(c));
}

template <typename X, int kOp, bool kEntropy>
void launch_sweep(Call& c) {
  c.groups = grid_of(c.rows);
  sweep_kernel<X, kOp, kEntropy>
      <<<c.groups, threads_of(c.rows, X::kPer), 0, c.stream>>>(c.rows, c.out, c.policy, c.mean, c.teacher);
}

template <typename X, bool kEntropy>
hipError_t launch_rows(Op op, Call& c) {
  if (op == kDistill) launch_distill<X>(c) || (launch_sweep<X, kDistill, false>(c), true);
  else if (op == kPolicy)
    launch_lanes<X, kPolicy, kEntropy>(c) || launch_held<X, kPolicy, kEntropy>(c) || (launch_sweep<X, kPolicy, kEntropy>(c), true);
  else
    launch_lanes<X, kScore, kEntropy>(c) || launch_held<X, kScore, kEntropy>(c) || (launch_sweep<X, kScore, kEntropy>(c), true);
  return hipGetLastError();
}
template <typename X, bool kEntropy>
hipError_t launch_gradient(Op op, Call c) {
  const Rows& r = c.rows;
  const int grid = grid_of(r), threads = threads_of(r, X::kPer);
  if (op == kDistill) gradient_kernel<X, kDistill, false><<<grid, threads, 0, c.stream>>>(r, c.given, c.teacher);
  else if (!launch_lanes<X, kGiven, kEntropy>(c))
    gradient_kernel<X, kGiven, kEntropy><<<grid, threads, 0, c.stream>>>(r, c.given, c.teacher);
  return hipGetLastError();
}

}  // namespace

template <typename X>
hipError_t rows_of(Op op, Call& c) {
  return c.entropy ? launch_rows<X, true>(op, c) : launch_rows<X, false>(op, c);
}
template <typename X>
hipError_t gradient_of(Op op, const Call& c) {
  return c.entropy ? launch_gradient<X, true>(op, c) : launch_gradient<X, false>(op, c);
}

}  // namespace loss
}  // namespace tb
