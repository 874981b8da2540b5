// Sums over positions: how many count, the weights that make a mean, the terms of a loss, and the
// margins of pairs of sequences.
#include "tb_loss_host.h"

namespace tb {
namespace loss {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// kTeam threads a sequence (a workgroup or a wavefront): how many of its positions count.
template <int kTeam>
__global__ __launch_bounds__(kThreads) void count_kernel(Rows r, int32_t* n) {
  constexpr int kTeams = kThreads / kTeam;
  __shared__ int part[kWaves];
  const int thread = threadIdx.x % kTeam;
  for (int64_t b = int64_t(blockIdx.x) * kTeams + threadIdx.x / kTeam; b < r.B; b += int64_t(gridDim.x) * kTeams) {
    const int length = r.lengths ? clamped(r.lengths[b], r.T) : r.T;
    int c = 0;
    if (!r.mask) c = thread == 0 ? length : 0;
    else
      for (int t = thread; t < length; t += kTeam) c += r.mask[b * r.T + t] != 0;
    c = wave_sum(c);
    if (kTeam > kWave) {
      if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = c;
      __syncthreads();
      c = 0;
      for (int w = 0; w < kWaves; ++w) c += part[w];
      __syncthreads();
    }
    if (thread == 0) n[b] = c;
  }
}

// Parts of all positions of a mask, kCountParts workgroups.
__global__ __launch_bounds__(kThreads) void part_count_kernel(Rows r, int32_t* n) {
  __shared__ int part[kWaves];
  const int64_t rows = int64_t(r.B) * r.T;
  int c = 0;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < rows; i += int64_t(kCountParts) * kThreads)
    c += counts(r, position(r, i).b, position(r, i).t);
  c = wave_sum(c);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = c;
  __syncthreads();
  if (threadIdx.x == 0) n[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// One workgroup: weights of means (over tokens or sequences) from the counts.
__global__ __launch_bounds__(1024) void weight_kernel(int B, int average, const int32_t* n, float* weight) {
  __shared__ long long part[16];
  long long sum = 0;
  for (int b = threadIdx.x; b < B; b += 1024) sum += average == TB_MEAN_TOKENS ? n[b] : n[b] > 0;
  sum = wave_sum(sum);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < 16; ++w) sum += part[w];
  for (int b = threadIdx.x; b < B; b += 1024) {
    weight[b] = n[b] > 0 ? float(1.0 / (average == TB_MEAN_TOKENS ? double(sum) : double(sum) * n[b])) : 0.f;
  }
}

// Sums of n columns of `parts` rows, in an order that only their number fixes.  Several workgroups leave a
// row each in `to`, a single one the columns' sums times `by` in `terms`.
__global__ __launch_bounds__(1024) void sum_kernel(int64_t parts, const double* partial, int n, int step, double by,
                                                   double* to, float* terms) {
  __shared__ double part[16][4];
  double sum[4] = {};
  for (int64_t i = int64_t(blockIdx.x) * 1024 + threadIdx.x; i < parts; i += int64_t(gridDim.x) * 1024)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) sum[j] += partial[i * step + j];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sum[j] = wave_sum(sum[j]);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave][j] = sum[j];
  }
  __syncthreads();
  if (int(threadIdx.x) < n) {
    double all = 0;
    for (int w = 0; w < 16; ++w) all += part[w][threadIdx.x];
    if (terms) terms[threadIdx.x] = float(all * by);
    else to[blockIdx.x * 4 + threadIdx.x] = all;
  }
}

// Of a sequence: sums of lp and of lp - ref, and how many positions count; of the thread's share.
struct Sequence {
  double lp, d;
  int n;
};
__device__ __forceinline__ Sequence sequence_part(const Rows& r, const Pairs& p, int64_t b, int thread, int threads) {
  const int length = r.lengths ? clamped(r.lengths[b], r.T) : r.T;
  Sequence s = {};
  for (int t = thread; t < length; t += threads) {
    const int64_t at = b * r.T + t;
    if (r.mask && !r.mask[at]) continue;
    const double lp = p.lp[at];
    s.lp += lp;
    s.d += lp - p.ref_lp[at];
    s.n += 1;
  }
  return {wave_sum(s.lp), wave_sum(s.d), wave_sum(s.n)};
}

// Loss and margin of pair i from its sequences' sums; leaves the pair's values.
struct Pair {
  double loss, margin;
};
__device__ __forceinline__ Pair pair_values(const Pairs& p, int pairs, int i, Sequence s, Sequence u) {
  const double of_s = p.kind == TB_PAIR_IPO ? 1.0 / (s.n > 0 ? s.n : 1) : 1.0;
  const double of_u = p.kind == TB_PAIR_IPO ? 1.0 / (u.n > 0 ? u.n : 1) : 1.0;
  const double margin = s.d * of_s - u.d * of_u, beta = p.beta, h = beta * margin;
  double loss, slope;
  if (p.kind == TB_PAIR_IPO) {
    const double off = margin - 0.5 / beta;
    loss = off * off;
    slope = 2 * off;
  } else if (p.kind == TB_PAIR_HINGE) {
    loss = h < 1 ? 1 - h : (h == h ? 0.0 : h);
    slope = h < 1 ? -beta : (h == h ? 0.0 : h);
  } else {
    const double low = log1p(exp(-fabs(h))), e = p.smooth;  // softplus(-h) and softplus(h) without overflow
    loss = low + (1 - e) * fmax(-h, 0.0) + (e > 0 ? e * fmax(h, 0.0) : 0.0);  // (h may be infinite)
    slope = beta * (e / (1 + exp(-h)) - (1 - e) / (1 + exp(h)));
  }
  slope /= pairs;
  p.sequence_lp[i] = float(s.lp);
  p.sequence_lp[i + pairs] = float(u.lp);
  p.margins[i] = float(margin);
  p.d_sequence[i] = float(slope * of_s);
  p.d_sequence[i + pairs] = float(-slope * of_u);
  return {loss, margin};
}

// One workgroup a pair; several pairs where there are more than a launch may have workgroups.
__global__ __launch_bounds__(kThreads) void pair_kernel(Rows r, Pairs p) {
  __shared__ Sequence part[2][kWaves];
  const int pairs = r.B / 2;
  for (int i = blockIdx.x; i < pairs; i += gridDim.x) {
    for (int side = 0; side < 2; ++side) {
      const Sequence s = sequence_part(r, p, i + int64_t(side) * pairs, threadIdx.x, kThreads);
      if (threadIdx.x % kWave == 0) part[side][threadIdx.x / kWave] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      Sequence s[2] = {};
      for (int side = 0; side < 2; ++side)
        for (int w = 0; w < kWaves; ++w) {
          s[side].lp += part[side][w].lp;
          s[side].d += part[side][w].d;
          s[side].n += part[side][w].n;
        }
      const Pair v = pair_values(p, pairs, i, s[0], s[1]);
      p.partial[3 * int64_t(i)] = v.loss;
      p.partial[3 * int64_t(i) + 1] = v.margin > 0;
      p.partial[3 * int64_t(i) + 2] = v.margin;
    }
    __syncthreads();  // (before the next pair's parts)
  }
}

// All pairs in one workgroup, a wavefront a sequence, and the means over them.
constexpr int kFewSequences = 256;
__global__ __launch_bounds__(1024) void few_pairs_kernel(Rows r, Pairs p) {
  __shared__ Sequence all[kFewSequences];
  __shared__ double part[16][3];
  const int pairs = r.B / 2, lane = threadIdx.x % kWave;
  for (int b = threadIdx.x / kWave; b < r.B; b += 16) {
    const Sequence s = sequence_part(r, p, b, lane, kWave);
    if (lane == 0) all[b] = s;
  }
  __syncthreads();
  double sum[3] = {};
  const int i = threadIdx.x;
  if (i < pairs) {
    const Pair v = pair_values(p, pairs, i, all[i], all[i + pairs]);
    sum[0] = v.loss;
    sum[1] = v.margin > 0;
    sum[2] = v.margin;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    sum[j] = wave_sum(sum[j]);
    if (lane == 0) part[threadIdx.x / kWave][j] = sum[j];
  }
  __syncthreads();
  if (i < 3) {
    double total = 0;
    for (int w = 0; w < 16; ++w) total += part[w][i];
    p.terms[i] = float(total / pairs);
  }
}

}  // namespace

hipError_t run_counts(const Rows& r, int32_t* n, hipStream_t stream) {
  if (r.T > 512) {
    count_kernel<kThreads><<<r.B < 4096 ? r.B : 4096, kThreads, 0, stream>>>(r, n);
  } else {
    const int64_t groups = (int64_t(r.B) + kWaves - 1) / kWaves;
    count_kernel<kWave><<<int(groups < 4096 ? groups : 4096), kThreads, 0, stream>>>(r, n);
  }
  return hipGetLastError();
}
hipError_t run_part_counts(const Rows& r, int32_t* n, hipStream_t stream) {
  part_count_kernel<<<kCountParts, kThreads, 0, stream>>>(r, n);
  return hipGetLastError();
}
hipError_t run_weights(int B, int average, const int32_t* n, float* weight, hipStream_t stream) {
  weight_kernel<<<1, 1024, 0, stream>>>(B, average, n, weight);
  return hipGetLastError();
}

hipError_t run_terms(int64_t groups, const double* partial, double* more, float* terms, int n, hipStream_t stream) {
  if (groups > 16 * 1024) {  // (one workgroup reads 512 KB in 6 us, several and then one take 9 for any number)
    sum_kernel<<<kMoreSums, 1024, 0, stream>>>(groups, partial, n, 4, 1.0, more, nullptr);
    partial = more;
    groups = kMoreSums;
  }
  sum_kernel<<<1, 1024, 0, stream>>>(groups, partial, n, 4, 1.0, nullptr, terms);
  return hipGetLastError();
}

hipError_t run_pairs(const Rows& r, const Pairs& p, hipStream_t stream) {
  const int pairs = r.B / 2;
  // one workgroup takes 4.4 us for 64 positions a wavefront, 11 to 13 for 1024; two launches take 10
  if (pairs && r.B <= kFewSequences && int64_t(r.B + 15) / 16 * r.T <= 512) {
    few_pairs_kernel<<<1, 1024, 0, stream>>>(r, p);
    return hipGetLastError();
  }
  if (pairs) pair_kernel<<<int(pairs < kMostGroups ? pairs : kMostGroups), kThreads, 0, stream>>>(r, p);
  sum_kernel<<<1, 1024, 0, stream>>>(pairs, p.partial, 3, 3, pairs ? 1.0 / pairs : 0.0, nullptr, p.terms);
  return hipGetLastError();
}

}  // namespace loss
}  // namespace tb
