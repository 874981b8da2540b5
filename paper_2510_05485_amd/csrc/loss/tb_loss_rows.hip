// Passes over rows of logits: log-probabilities and entropies, the policy loss, the distillation loss,
// and their gradients.
#include "tb_loss_host.h"

namespace tb {
namespace loss {
namespace {

constexpr uint32_t kNan = 0x7FC00000u;

// What the gradient of a row is made of: values 2^a (by_weight + by_log a), a = (x - m) k, and `token`
// more at the row's token.
struct Slope {
  float by_weight, by_log, token;
};

// from the cotangents of lp and H
__device__ __forceinline__ Slope slope_of(float s, float H, float d_lp, float d_H, float scale) {
  const float f = scale / s;
  return {f * (-d_lp - d_H * (H - logf(s))), -f * d_H * kLn2, scale * d_lp};
}

// Statistics of a row, in every thread.  Reads the row once.
template <typename X, bool kEntropy>
__device__ __forceinline__ Stats row_stats(const Span<X>& row, float k, Stats* parts) {
  Stats mine = {kLowest, 0.f, 0.f};
  auto take = [&](const float* v, int n) {
    float top = mine.m;
#pragma unroll
    for (int i = 0; i < X::kPer; ++i)
      if (i < n) top = fmaxf(top, v[i]);
    const float d = (mine.m - top) * k, e = exp2_fast(d);
    mine.t = kEntropy ? e * (mine.t + finite(d) * mine.s) : 0.f;
    mine.s *= e;
    mine.m = top;
#pragma unroll
    for (int i = 0; i < X::kPer; ++i)
      if (i < n) {
        const float a = (v[i] - top) * k, w = exp2_fast(a);
        mine.s += w;
        if (kEntropy) mine.t += w * finite(a);
      }
  };
  for (int c = threadIdx.x; c < row.chunks; c += blockDim.x) {
    float v[X::kPer];
    X::unpack(row.chunk(c), v);
    take(v, X::kPer);
  }
  const int e = row.edge(threadIdx.x);
  if (e >= 0) {
    const float v[X::kPer] = {X::load(row.x + e)};
    take(v, 1);
  }
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const Stats other = {__shfl_xor(mine.m, d), __shfl_xor(mine.s, d), __shfl_xor(mine.t, d)};
    mine = joined<kEntropy>(mine, other, k);
  }
  if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = mine;
  __syncthreads();
  Stats all = parts[0];
  for (int w = 1; w < int(blockDim.x / kWave); ++w) all = joined<kEntropy>(all, parts[w], k);
  return all;
}

// The gradient of a row, but for the additions at the token.
template <typename X, bool kEntropy>
__device__ __forceinline__ void write_gradient(const Span<X>& row, typename X::type* g, float m, float k, Slope f) {
  auto value = [&](float x) {
    const float a = (x - m) * k, w = exp2_fast(a);
    return w * (kEntropy ? f.by_weight + f.by_log * finite(a) : f.by_weight);
  };
  for (int c = threadIdx.x; c < row.chunks; c += blockDim.x) {
    float v[X::kPer];
    X::unpack(row.chunk(c), v);
#pragma unroll
    for (int i = 0; i < X::kPer; ++i) v[i] = value(v[i]);
    *reinterpret_cast<u32x4_any*>(g + row.at(c)) = X::pack(v);
  }
  const int e = row.edge(threadIdx.x);
  if (e >= 0) X::store(g + e, value(X::load(row.x + e)));
}

template <typename X>
__device__ __forceinline__ void write_zeros(const Rows& r, int b, int t) {
  const Span<X> row(gradient_of<X>(r, b, t), r.V);
  typename X::type* g = gradient_of<X>(r, b, t);
  for (int c = threadIdx.x; c < row.chunks; c += blockDim.x) *reinterpret_cast<u32x4*>(g + row.at(c)) = u32x4{};
  const int e = row.edge(threadIdx.x);
  if (e >= 0) X::store(g + e, 0.f);
}

// The token's value, added where its owner has just stored the rest (stores of one thread to one
// address keep their order).
template <typename X, bool kEntropy>
__device__ __forceinline__ void add_token(const Span<X>& row, typename X::type* g, int token, float x, float m,
                                          float k, Slope f) {
  if (row.owner(token, blockDim.x) != int(threadIdx.x)) return;
  const float a = (x - m) * k, w = exp2_fast(a);
  X::store(g + token, f.token + w * (kEntropy ? f.by_weight + f.by_log * finite(a) : f.by_weight));
}

// Loss and cotangents of a position (every thread of the workgroup computes them).
struct Position {
  float4 terms;  // loss, kl, clipped, entropy
  float d_lp, d_H;
};
__device__ __forceinline__ Position policy_position(const Policy& p, int b, int64_t r, float lp, float H, float w) {
  const float ratio = expf(lp - p.old_lp[r]), A = p.each ? p.advantages[r] : p.advantages[b];
  const bool clipped = (A > 0 && ratio > 1 + p.high) || (A < 0 && ratio < 1 - p.low);
  const float held = A > 0 ? 1 + p.high : 1 - p.low;
  Position o;
  float loss = -(clipped ? held : ratio) * A, kl = 0.f;
  o.d_lp = clipped ? 0.f : -ratio * A;
  if (p.kl_coef != 0.f) {
    const float d = p.ref_lp[r] - lp, e = expf(d);
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

__device__ __forceinline__ float teacher_value(const Teacher& q, int64_t i) {
  if (q.type == TB_FLOAT32) return static_cast<const float*>(q.logits)[i];
  return q.type == TB_BFLOAT16 ? BF16::load(static_cast<const uint16_t*>(q.logits) + i)
                               : F16::load(static_cast<const _Float16*>(q.logits) + i);
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
__device__ __forceinline__ float take_entries(const Rows& r, const Span<X>& row, const Teacher& q, int64_t at, float k,
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
__device__ __forceinline__ void add_entries(const Span<X>& row, typename X::type* g, const Teacher& q,
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
__device__ __forceinline__ void write_distilled(const Rows& r, const Span<X>& row, const Teacher& q, const Entries& e,
                                                int b, int t, float m, float s, float sum, float w, float k) {
  if (sum == 0.f) {
    write_zeros<X>(r, b, t);
    return;
  }
  typename X::type* g = gradient_of<X>(r, b, t);
  Slope f = {0.f, 0.f, q.tau * w * r.g_scale};
  f.by_weight = sum == sum ? f.token / s : sum;
  write_gradient<X, false>(row, g, m, k, f);
  __syncthreads();  // (what it has stored comes before what follows)
  add_entries<X>(row, g, q, e, m, k, f);
}

// A position that does not count.
template <typename X>
__device__ __forceinline__ void nothing(const Rows& r, const RowOut& o, int b, int t, int64_t at) {
  if (threadIdx.x == 0) {
    if (o.logprobs) o.logprobs[at] = 0.f;
    if (o.entropy) o.entropy[at] = 0.f;
    if (o.state) o.state[at] = {};
    if (o.d_logprobs) o.d_logprobs[at] = 0.f;
    if (o.d_entropy) o.d_entropy[at] = 0.f;
    if (o.terms) o.terms[at] = {};
  }
  if (r.g) write_zeros<X>(r, b, t);
}

// The row's token, or -1 (reported) for one outside the vocabulary.
__device__ __forceinline__ int take_token(const Rows& r, int b, int t) {
  const int64_t token = load_id(r.tokens, r.long_tokens, b * r.token_seq + t);
  if (token >= 0 && token < r.V) return int(token);
  if (threadIdx.x == 0 && r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
  return -1;
}

template <int kOp>
struct Shared {
  Stats parts[8];
  Entries entries;
};
template <>
struct Shared<kScore> {
  Stats parts[8];
};
template <>
struct Shared<kPolicy> : Shared<kScore> {};

template <typename X, int kOp, bool kEntropy>
__device__ __forceinline__ void sweep_row(const Rows& r, const RowOut& o, const Policy& p, const Teacher& q, int b,
                                          int t, int64_t at, Shared<kOp>& shared) {
  const bool first = threadIdx.x == 0;
  const Span<X> row(row_of<X>(r, b, t), r.V);
  const float k = r.inv_temp * kLog2e;
  Slope f;
  if constexpr (kOp != kDistill) {
    const int token = take_token(r, b, t);
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(row.x + token);
    const Stats s = row_stats<X, kEntropy>(row, k, shared.parts);
    const float log_s = logf(s.s), lp = (x - s.m) * r.inv_temp - log_s;
    const float H = kEntropy ? log_s - kLn2 * s.t / s.s : 0.f;
    Position v = {};
    if (kOp == kPolicy) v = policy_position(p, b, at, lp, H, p.weight[b]);
    if (first) {
      if (o.logprobs) o.logprobs[at] = lp;
      if (o.entropy) o.entropy[at] = H;
      if (o.state) o.state[at] = {s.m, s.s, H, lp};
      if (kOp == kPolicy) {
        if (o.d_logprobs) o.d_logprobs[at] = v.d_lp;
        if (o.d_entropy) o.d_entropy[at] = v.d_H;
        o.terms[at] = v.terms;
      }
    }
    if (kOp == kScore || !r.g) return;
    f = slope_of(s.s, H, v.d_lp, v.d_H, r.g_scale * r.inv_temp);
    typename X::type* g = gradient_of<X>(r, b, t);
    write_gradient<X, kEntropy>(row, g, s.m, k, f);
    if (token >= 0) add_token<X, kEntropy>(row, g, token, x, s.m, k, f);
  } else {
    Entries& e = shared.entries;
    const float sum = take_entries<X>(r, row, q, at, k, e);
    const Stats s = row_stats<X, false>(row, k, shared.parts);
    const float log_s = logf(s.s);
    float d = 0.f;
    for (int j = threadIdx.x; j < q.K; j += blockDim.x)
      if (!(e.q[j] <= 0.f)) d += e.q[j] * (e.log_q[j] - ((e.x[j] - s.m) * r.inv_temp - log_s));
    d = block_sum(d, e.part) * q.tau * q.tau;
    const float w = sum == 0.f ? 0.f : q.weight[b];
    if (first) {
      if (o.state) o.state[at] = {s.m, s.s, 0.f, d};
      if (o.d_logprobs) o.d_logprobs[at] = w;
      if (o.logprobs) o.logprobs[at] = d;
      o.terms[at] = {d, 0.f, 0.f, 0.f};
    }
    if (r.g) write_distilled<X>(r, row, q, e, b, t, s.m, s.s, sum, w, k);
  }
}

// One workgroup a row; the row is read from memory in every sweep over it.
template <typename X, int kOp, bool kEntropy>
__global__ __launch_bounds__(512) void sweep_kernel(Rows r, RowOut o, Policy p, Teacher q) {
  __shared__ Shared<kOp> shared;
  const int64_t rows = int64_t(r.B) * r.T;
  for (int64_t at = blockIdx.x; at < rows; at += gridDim.x) {
    const int b = int(uint32_t(at) / uint32_t(r.T)), t = int(uint32_t(at) % uint32_t(r.T));
    if (threadIdx.x == 0 && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    if (counts(r, b, t)) sweep_row<X, kOp, kEntropy>(r, o, p, q, b, t, at, shared);
    else nothing<X>(r, o, b, t, at);
    __syncthreads();  // (before the next row takes the shared memory)
  }
}

// The gradient of a row whose statistics are given.
template <typename X, int kOp, bool kEntropy>
__device__ __forceinline__ void given_row(const Rows& r, const Given& v, const Teacher& q, int b, int t, int64_t at,
                                          Shared<kOp>& shared) {
  const Span<X> row(row_of<X>(r, b, t), r.V);
  const float k = r.inv_temp * kLog2e, up = v.upstream ? *v.upstream : 1.f;
  const float4 state = v.state[at];
  const float d = v.d_lp[b * v.d_seq + t * v.d_pos] * up;
  if constexpr (kOp != kDistill) {
    const float d_H = kEntropy ? v.d_entropy[b * v.d_seq + t * v.d_pos] * up : 0.f;
    const int token = take_token(r, b, t);
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(row.x + token);
    __syncthreads();  // (the row may be the gradient's own memory)
    const Slope f = slope_of(state.y, state.z, token < 0 ? x : d, d_H, r.g_scale * r.inv_temp);
    typename X::type* g = gradient_of<X>(r, b, t);
    write_gradient<X, kEntropy>(row, g, state.x, k, f);
    if (token >= 0) add_token<X, kEntropy>(row, g, token, x, state.x, k, f);
  } else {
    const float sum = take_entries<X>(r, row, q, at, k, shared.entries);
    write_distilled<X>(r, row, q, shared.entries, b, t, state.x, state.y, sum, d, k);
  }
}

template <typename X, int kOp, bool kEntropy>
__global__ __launch_bounds__(512) void gradient_kernel(Rows r, Given v, Teacher q) {
  __shared__ Shared<kOp> shared;
  const int64_t rows = int64_t(r.B) * r.T;
  for (int64_t at = blockIdx.x; at < rows; at += gridDim.x) {
    const int b = int(uint32_t(at) / uint32_t(r.T)), t = int(uint32_t(at) % uint32_t(r.T));
    if (counts(r, b, t)) given_row<X, kOp, kEntropy>(r, v, q, b, t, at, shared);
    else write_zeros<X>(r, b, t);
    __syncthreads();
  }
}

// A launch has less than 2^32 threads: from so many rows on, workgroups take several.
constexpr int64_t kMostGroups = 1 << 22;
int grid_of(const Rows& r) {
  const int64_t rows = int64_t(r.B) * r.T;
  return int(rows < kMostGroups ? rows : kMostGroups);
}

int threads_of(const Rows& r, int per) {
  const int chunks = (r.V + per - 1) / per;
  const int t = (chunks + kWave - 1) / kWave * kWave;
  return t > 512 ? 512 : t;
}

template <typename X, bool kEntropy>
hipError_t rows_of(Op op, const Call& c) {
  const Rows& r = c.rows;
  const int grid = grid_of(r), threads = threads_of(r, X::kPer);
  switch (op) {
    case kScore: sweep_kernel<X, kScore, kEntropy><<<grid, threads, 0, c.stream>>>(r, c.out, c.policy, c.teacher); break;
    case kPolicy: sweep_kernel<X, kPolicy, kEntropy><<<grid, threads, 0, c.stream>>>(r, c.out, c.policy, c.teacher); break;
    case kDistill: sweep_kernel<X, kDistill, false><<<grid, threads, 0, c.stream>>>(r, c.out, c.policy, c.teacher); break;
  }
  return hipGetLastError();
}
template <typename X, bool kEntropy>
hipError_t gradient_of(Op op, const Call& c) {
  const Rows& r = c.rows;
  const int grid = grid_of(r), threads = threads_of(r, X::kPer);
  if (op == kDistill) gradient_kernel<X, kDistill, false><<<grid, threads, 0, c.stream>>>(r, c.given, c.teacher);
  else gradient_kernel<X, kScore, kEntropy><<<grid, threads, 0, c.stream>>>(r, c.given, c.teacher);
  return hipGetLastError();
}

}  // namespace

hipError_t run_rows(Op op, const Call& c) {
  if (c.type == TB_FLOAT32) return c.entropy ? rows_of<F32, true>(op, c) : rows_of<F32, false>(op, c);
  if (c.type == TB_BFLOAT16) return c.entropy ? rows_of<BF16, true>(op, c) : rows_of<BF16, false>(op, c);
  return c.entropy ? rows_of<F16, true>(op, c) : rows_of<F16, false>(op, c);
}
hipError_t run_gradient(Op op, const Call& c) {
  if (c.type == TB_FLOAT32) return c.entropy ? gradient_of<F32, true>(op, c) : gradient_of<F32, false>(op, c);
  if (c.type == TB_BFLOAT16) return c.entropy ? gradient_of<BF16, true>(op, c) : gradient_of<BF16, false>(op, c);
  return c.entropy ? gradient_of<F16, true>(op, c) : gradient_of<F16, false>(op, c);
}

}  // namespace loss
}  // namespace tb
