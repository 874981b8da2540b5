// Sums over positions: how many count, the weights that make a mean, the terms of a loss, and the
// margins of pairs of sequences.
#include "tb_loss_host.h"

namespace tb {
namespace loss {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// One wavefront a sequence: how many of its positions count.
__global__ __launch_bounds__(kThreads) void count_kernel(Rows r, int32_t* n) {
  const int lane = threadIdx.x % kWave;
  for (int64_t b = int64_t(blockIdx.x) * kWaves + threadIdx.x / kWave; b < r.B; b += int64_t(gridDim.x) * kWaves) {
    const int length = r.lengths ? held_length(r.lengths[b], r.T, nullptr) : r.T;
    int c = 0;
    if (!r.mask) c = lane == 0 ? length : 0;
    else
      for (int t = lane; t < length; t += kWave) c += r.mask[b * r.T + t] != 0;
    c = wave_sum(c);
    if (lane == 0) n[b] = c;
  }
}

// One workgroup: weights from the counts.
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
    float w = 0.f;
    if (n[b] > 0)
      w = average == TB_SUM ? 1.f : float(1.0 / (average == TB_MEAN_TOKENS ? double(sum) : double(sum) * n[b]));
    weight[b] = w;
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

// One workgroup a pair.
__global__ __launch_bounds__(kThreads) void pair_kernel(Rows r, Pairs p) {
  __shared__ double part[kWaves][2][3];
  const int pairs = r.B / 2, i = blockIdx.x;
  for (int side = 0; side < 2; ++side) {
    const int64_t b = i + int64_t(side) * pairs;
    const int length = r.lengths ? held_length(r.lengths[b], r.T, nullptr) : r.T;
    double lp_sum = 0, d_sum = 0, n = 0;
    for (int t = threadIdx.x; t < length; t += kThreads) {
      const int64_t at = b * r.T + t;
      if (r.mask && !r.mask[at]) continue;
      const float lp = p.state[at].w;
      lp_sum += lp;
      d_sum += double(lp) - p.ref_lp[at];
      n += 1;
    }
    lp_sum = wave_sum(lp_sum);
    d_sum = wave_sum(d_sum);
    n = wave_sum(n);
    if (threadIdx.x % kWave == 0) {
      double* to = part[threadIdx.x / kWave][side];
      to[0] = lp_sum;
      to[1] = d_sum;
      to[2] = n;
    }
  }
  __syncthreads();
  if (threadIdx.x) return;
  double lp[2] = {}, d[2] = {}, share[2];
  for (int side = 0; side < 2; ++side) {
    double n = 0;
    for (int w = 0; w < kWaves; ++w) {
      lp[side] += part[w][side][0];
      d[side] += part[w][side][1];
      n += part[w][side][2];
    }
    share[side] = p.kind == TB_PAIR_IPO ? 1.0 / (n > 0 ? n : 1.0) : 1.0;
    d[side] *= share[side];
    p.sequence_lp[i + side * pairs] = float(lp[side]);
  }
  const double margin = d[0] - d[1], h = p.beta * margin, beta = p.beta;
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
    loss = low + (1 - e) * fmax(-h, 0.0) + e * fmax(h, 0.0);
    slope = beta * (e / (1 + exp(-h)) - (1 - e) / (1 + exp(h)));
  }
  p.margins[i] = float(margin);
  p.partial[3 * i] = loss;
  p.partial[3 * i + 1] = margin > 0;
  p.partial[3 * i + 2] = margin;
  slope /= pairs;
  p.d_sequence[i] = float(slope * share[0]);
  p.d_sequence[i + pairs] = float(-slope * share[1]);
}

}  // namespace

hipError_t run_weights(const Rows& r, int average, int32_t* counts, float* weight, hipStream_t stream) {
  const int64_t groups = (int64_t(r.B) + kWaves - 1) / kWaves;
  count_kernel<<<int(groups < 4096 ? groups : 4096), kThreads, 0, stream>>>(r, counts);
  weight_kernel<<<1, 1024, 0, stream>>>(r.B, average, counts, weight);
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
  if (pairs) pair_kernel<<<pairs, kThreads, 0, stream>>>(r, p);
  sum_kernel<<<1, 1024, 0, stream>>>(pairs, p.partial, 3, 3, pairs ? 1.0 / pairs : 0.0, nullptr, p.terms);
  return hipGetLastError();
}

}  // namespace loss
}  // namespace tb
