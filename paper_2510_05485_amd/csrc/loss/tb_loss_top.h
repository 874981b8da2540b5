// The K likeliest tokens of every position, with their log-probabilities, beside those of given tokens and
// entropies; and the gradient of all of these in the logits.
//
// z = x / temperature, lp = z - log sum exp z.  The order of the alternatives is that of x, equal ones by their
// ids.  A row is read once, with its softmax's statistics formed on the way as for the losses; nothing of it is
// sorted.  The K-th largest of the maxima that lanes have of their parts of the row is a bound that K values reach at
// least, and about K (1 + K / 2 maxima) do; these are collected in LDS, and each one's place is the number of those
// before it.  Kernels by the length of a row:
//   best_kernel   up to 128 chunks of 16 bytes and eight alternatives: 2 to 32 lanes of a wavefront hold a row and keep
//                 the best of their chunks
//   short_kernel  up to 64 chunks: 2 to 64 lanes, a chunk each, and the best of the lanes' best is taken K times
//   top_kernel    a wavefront, or a workgroup, holds a row (or a part of a long one) in its registers, or tile by tile
//   join_kernel   joins the parts of long rows, where there are few
//
// Long rows are bound by HBM and, with entropies, by the vector units alike: 10 to 11 vector instructions a value, one of
// them an exponential at a quarter of the rate, under way for 76 % of a unit's busy cycles.  On one MI355X, among other
// calls: 16 x 256 rows (three in four of which count) of 32000 values in bfloat16, K = 64, 47 us (4.2 TB/s); 10240 of
// 50257, K = 20, with entropies 204 us (5.1); 1842 of 262144 in float16, K = 256, 248 us (3.9); 3884 of 50257 in float32,
// K = 20, with entropies 190 us (4.1); 1113000 of 64, K = 5, 79 us (3.4; issue and stores); one row of 50257 8.3 us, on
// one unit; four of 262144 in float32 12 us, two launches.  Far from that: many alternatives of short rows (66582 of 635,
// K = 134, 338 us), and more than 512 alternatives, of rows taken tile by tile (1024 of 262144 in float32: K = 512 292 us,
// 1024 6230, in 18 sweeps) and of others (4096 of 32000 in bfloat16, K = 1024, 1142 us: the order of the candidates).
#pragma once

#include "tb_loss_rows.h"
#include "tb_loss_top_host.h"

namespace tb {
namespace loss {
namespace {

// ---- the order of logits as one of whole numbers ----------------------------------------------

typedef int int_alias __attribute__((may_alias));  // (values inside chunks)
typedef short short_alias __attribute__((may_alias));

// Order: value x -> int32 that grows with x, -0 and 0 alike: sign and magnitude as two's complement.
template <typename X>
struct Order;
template <>
struct Order<F32> {
  static constexpr int kNone = -0x7F800000;  // of -inf
  static constexpr int kShift = 16;          // of a bound in 16 bits
  static __device__ __forceinline__ uint32_t of_packed(uint32_t u) {
    const int mask = int(u) >> 31;
    return uint32_t((int(u & 0x7FFFFFFFu) ^ mask) - mask);
  }
  static __device__ __forceinline__ float value(int t) {
    return __uint_as_float(t < 0 ? 0x80000000u | uint32_t(-t) : uint32_t(t));
  }
  static constexpr int kMost = 0x7F7FFFFF;  // of the largest value
  static __device__ __forceinline__ int raw(float v) { return __float_as_int(v); }
  static __device__ __forceinline__ int of(float v) { return int(of_packed(__float_as_uint(v))); }
  template <typename Take>
  static __device__ __forceinline__ void each(u32x4 c, Take take) {
#pragma unroll
    for (int i = 0; i < 4; ++i) take(i, int(c[i]));
  }
  static __device__ __forceinline__ int in_chunk(const u32x4* c, int i) { return reinterpret_cast<const int_alias*>(c)[i]; }
  static __device__ __forceinline__ int largest(u32x4 c) { return max(max(int(c[0]), int(c[1])), max(int(c[2]), int(c[3]))); }
};
struct Order16 {
  static constexpr int kShift = 0;
  static __device__ __forceinline__ uint32_t of_packed(uint32_t u) {
    i16x2 v;
    __builtin_memcpy(&v, &u, 4);
    const i16x2 mask = v >> 15, t = ((v & i16x2{0x7FFF, 0x7FFF}) ^ mask) - mask;
    __builtin_memcpy(&u, &t, 4);
    return u;
  }
  template <typename Take>
  static __device__ __forceinline__ void each(u32x4 c, Take take) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      take(2 * i, int(short(c[i] & 0xFFFFu)));
      take(2 * i + 1, int(c[i]) >> 16);
    }
  }
  static __device__ __forceinline__ int in_chunk(const u32x4* c, int i) { return reinterpret_cast<const short_alias*>(c)[i]; }
  static __device__ __forceinline__ int largest(u32x4 c) {
    const i16x2 top = upper_pair<1>(&c);
    return max(int(top[0]), int(top[1]));
  }
};
template <>
struct Order<BF16> : Order16 {
  static constexpr int kNone = -0x7F80, kMost = 0x7F7F;
  static __device__ __forceinline__ float value(int t) { return Order<F32>::value(t * 65536); }
  static __device__ __forceinline__ int raw(float v) { return __float_as_int(v) >> 16; }
  static __device__ __forceinline__ int of(float v) { return short(of_packed(uint32_t(raw(v)))); }
};
template <>
struct Order<F16> : Order16 {
  static constexpr int kNone = -0x7C00, kMost = 0x7BFF;
  static __device__ __forceinline__ float value(int t) {
    const uint16_t u = uint16_t(t < 0 ? 0x8000 | -t : t);
    _Float16 h;
    __builtin_memcpy(&h, &u, 2);
    return float(h);
  }
  static __device__ __forceinline__ int raw(float v) {
    const _Float16 h = _Float16(v);
    short s;
    __builtin_memcpy(&s, &h, 2);
    return s;
  }
  static __device__ __forceinline__ int of(float v) { return short(of_packed(uint32_t(raw(v)))); }
};
// Logits before others have larger keys; no key of a logit is 0.
__device__ __forceinline__ uint64_t key_of(int t, int at) {
  return uint64_t(uint32_t(t) ^ 0x80000000u) << 32 | uint32_t(~at);
}
__device__ __forceinline__ int order_in(uint64_t key) { return int(uint32_t(key >> 32) ^ 0x80000000u); }
__device__ __forceinline__ int place_in(uint64_t key) { return int(~uint32_t(key)); }

// ---- what a row leaves ------------------------------------------------------------------------

__device__ __forceinline__ void put_id(const Top& q, int64_t i, int id) {
  if (q.long_ids) static_cast<int64_t*>(q.ids)[i] = id;
  else static_cast<int32_t*>(q.ids)[i] = id;
}
// Entries from `from` on that are not there.
__device__ __forceinline__ void put_none(const Top& q, int64_t at, int from, float lp, int thread, int threads) {
  for (int j = from + thread; j < q.K; j += threads) {
    put_id(q, at * q.K + j, -1);
    q.logprobs[at * q.K + j] = lp;
  }
}

// Statistics of a row and how its log-probabilities follow: of weights 2^(x k - M), or 2^((x - m) k).
struct Found {
  float m, s, t;
  bool apart;  // the second
};
__device__ __forceinline__ float scaled_logit(const Found& f, float x, float k) {
  return f.apart ? (x - f.m) * k : fmaf(x, k, -scaled(f.m, k));
}
__device__ __forceinline__ float logprob(const Found& f, float x, float k, float inv_temp, float log_s) {
  const float z = (x - f.m) * inv_temp, scaled_z = f.apart ? z : scaled_logit(f, x, k) * kLn2;
  // (x k overflows where x / temperature does not: a mask of the type's lowest value)
  return (scaled_z == -INFINITY ? z : scaled_z) - log_s;
}
// A row without a finite logit, or with +inf or NaN
__device__ __forceinline__ bool lost(const Found& f) { return !(f.s > 0.f); }

template <bool kEntropy>
__device__ __forceinline__ void put_values(const Rows& r, const RowOut& o, const Found& f, float x, float k, float log_s,
                                           int64_t at) {
  const float lp = logprob(f, x, k, r.inv_temp, log_s), H = kEntropy ? log_s - kLn2 * f.t / f.s : 0.f;
  if (o.logprobs) o.logprobs[at] = lp;
  if (o.entropy) o.entropy[at] = H;
  if (o.state) o.state[at] = {f.m, f.apart ? f.s * to_scaled(f.m, k) : f.s, H, lp};
}

// Which rows a workgroup of several takes: those of eight neighbours (one to an XCD) come in another order from block
// to block, for the same reason as in row_of_group.
__device__ __forceinline__ int64_t turned(int64_t group, int64_t groups) {
  const int64_t block = group / 8;
  return (block + 1) * 8 > groups ? group : block * 8 + (group + block) % 8;
}

// ---- rows in registers ------------------------------------------------------------------------

__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// Chunks k kThreads + thread of a row, k < kChunks, of which all but the last kStep + 2 are there in every thread
// (kStep: how many lengths one kernel serves; one for the row's head, one for parts that differ in length).
template <typename X, int kThreads, int kChunks, int kStep>
struct Taken {
  using Row = Span<X, kThreads <= kWave ? 16 : kLine>;
  using O = Order<X>;
  static_assert(Row::kEdge <= kThreads);
  static constexpr int kSure = kChunks - kStep - 2 > 0 ? kChunks - kStep - 2 : 0;
  u32x4 c[kChunks];
  float edge;
  int edge_at;

  static __device__ __forceinline__ bool there(const Row& row, int thread, int k) { return thread + k * kThreads < row.chunks; }
  __device__ __forceinline__ void load(const Row& row, int thread) {
    const char* from = reinterpret_cast<const char*>(row.x + row.head);
    const uint32_t lane = thread * 16u;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      if (k >= kSure) c[k] = u32x4{X::kNone, X::kNone, X::kNone, X::kNone};
      if (k < kSure || there(row, thread, k)) c[k] = *reinterpret_cast<const u32x4_at16*>(from + k * (kThreads * 16) + lane);
    }
    edge_at = row.edge(thread);
    edge = edge_at >= 0 ? X::load(row.x + edge_at) : -INFINITY;
  }
  __device__ __forceinline__ void keep_packed() {  // (as in Held)
#pragma unroll
    for (int k = 0; k < kChunks; ++k) asm volatile("" : "+v"(c[k]));
  }
  // The chunks as whole numbers in the order of their values.
  __device__ __forceinline__ void to_order() {
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[k][i] = O::of_packed(c[k][i]);
    keep_packed();
  }
  // The largest of the thread's values, in kParts groups.
  static constexpr int kParts = 4;
  __device__ __forceinline__ void largest(int* most, int edge_order) const {
    most[0] = edge_order;
#pragma unroll
    for (int j = 1; j < kParts; ++j) most[j] = INT32_MIN;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) most[k % kParts] = max(most[k % kParts], O::largest(c[k]));
  }
  // A number that `need` of a wavefront's values reach, 16 bits of it, when the chunks are whole numbers in the values'
  // order: the largest such, by halving; three instructions a value and step, two of them scalar.
  __device__ __forceinline__ int value_bound(int edge_order, int need) {
    constexpr int kBias = 32768;
    int b = 0;
#pragma unroll 1
    for (int bit = 1 << 15; bit; bit >>= 1) {
      keep_packed();
      const int least = ((b | bit) - kBias) * (1 << O::kShift);
      int n = __popcll(__ballot(edge_order >= least));
#pragma unroll
      for (int k = 0; k < kChunks; ++k) O::each(c[k], [&](int, int t) { n += __popcll(__ballot(t >= least)); });
      if (n >= need) b |= bit;
    }
    return (b - kBias) * (1 << O::kShift);
  }
  // Chunks with a value from `least` on, with the places of their first values, into a list of the wavefront: how many
  // there are (of which `room` are kept).
  __device__ __forceinline__ int hits(const Row& row, int thread, int least, u32x4* chunks, int* places, int room) {
    int n = 0, at = row.at(thread);
    keep_packed();
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const bool is = O::largest(c[k]) >= least;
      const uint64_t mask = __ballot(is);
      if (mask) {
        const int slot = n + lanes_before(mask);
        if (is && slot < room) {
          chunks[slot] = c[k];
          places[slot] = at;
        }
        n += __popcll(mask);
      }
      at += kThreads * X::kPer;
      asm volatile("" : "+v"(at));  // (the compiler would hold all places)
    }
    return n;
  }
};

// Statistics of a wavefront's part of a row, as in wave_stats; most: what its lanes' largest values are, as raw bits.
template <bool kEntropy, typename X, int kThreads, int kChunks, int kStep>
__device__ __forceinline__ Stats taken_stats(Taken<X, kThreads, kChunks, kStep>& h, float k) {
  Stats mine = {fmaxf(h.edge, -kExtreme), 0.f, 0.f};
  constexpr int kSure = Taken<X, kThreads, kChunks, kStep>::kSure;
  if constexpr (kSure > 0) mine.m = fmaxf(mine.m, X::template upper<kSure>(h.c));
#pragma unroll
  for (int j = kSure; j < kChunks; ++j) {  // (with what lies beyond the row)
    float v[X::kPer];
    X::unpack(h.c[j], v);
#pragma unroll
    for (int i = 0; i < X::kPer; i += 2) mine.m = max3(mine.m, v[i], v[i + 1]);
  }
  mine.m = full_wave_max(mine.m);
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
  mine.s = full_wave_sum(mine.s);
  if (kEntropy) mine.t = full_wave_sum(mine.t);
  if (kThreads > kWave && mine.s > 0x1p88f) mine.s = __uint_as_float(kNan);
  return mine;
}

// A number that `need` of a wavefront's lanes' largest values reach (in all lanes), 16 bits of it: these, or those of
// the four groups that each lane has where more are needed.  The least number if there are not so many.
template <typename X>
__device__ __forceinline__ int wave_bound(const int* most, int need) {
  constexpr int kBias = 32768, kParts = 4;
  int u[kParts];
#pragma unroll
  for (int j = 0; j < kParts; ++j) u[j] = (most[j] >> Order<X>::kShift) + kBias;
  int b = 0;
  if (need <= kWave / 2) {
    const int v = max(max(u[0], u[1]), max(u[2], u[3]));
    for (int bit = 1 << 15; bit; bit >>= 1)
      if (__popcll(__ballot(v >= (b | bit))) >= need) b |= bit;
  } else {
    for (int bit = 1 << 15; bit; bit >>= 1) {
      int n = 0;
#pragma unroll
      for (int j = 0; j < kParts; ++j) n += __popcll(__ballot(u[j] >= (b | bit)));
      if (n >= need) b |= bit;
    }
  }
  return (b - kBias) * (1 << Order<X>::kShift);
}

// Sum over groups of kLanes neighbouring lanes, in all of them.
template <int kLanes, int kStep = 1>
__device__ __forceinline__ int lanes_total(int v) {
  if constexpr (kStep == kLanes) return v;
  else return lanes_total<kLanes, kStep * 2>(v + __float_as_int(neighbour<kStep>(__int_as_float(v))));
}

template <int kLanes, int kStep = 1>
__device__ __forceinline__ float lanes_added(float v) {
  if constexpr (kStep == kLanes) return v;
  else return lanes_added<kLanes, kStep * 2>(v + neighbour<kStep>(v));
}

// What the threads that share a row leave for one another; counted: two, taken in turn.
template <int kWaves>
struct TopShared {
  Stats parts[kWaves];
  int bounds[4][kWaves], counts[kWaves], counted[2][kWaves];
};

// The same of the keys that a wavefront has found, or no number (of -inf) if there are not so many.
constexpr int kMostKeys = 514;
template <typename X>
__device__ __forceinline__ int list_bound(const uint64_t* own, int found, int need) {
  constexpr int kBias = 32768, kBlocks = (kMostKeys + kWave - 1) / kWave;
  if (found < need) return Order<X>::kNone;
  const int lane = threadIdx.x % kWave;
  int u[kBlocks];
#pragma unroll
  for (int j = 0; j < kBlocks; ++j) {
    const int i = j * kWave + lane;
    u[j] = i < found ? (order_in(own[i]) >> Order<X>::kShift) + kBias : -1;
  }
  int b = 0;
  for (int bit = 1 << 15; bit; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
      if (j * kWave < found) n += __popcll(__ballot(u[j] >= (b | bit)));
    if (n >= need) b |= bit;
  }
  return (b - kBias) * (1 << Order<X>::kShift);
}

// Sums of weights 2^(x k - M) of two parts of a row, M the scaled reference of each.
template <bool kEntropy>
__device__ __forceinline__ Stats joined_scaled(const Stats& p, const Stats& q, float k) {
  Stats r;
  r.m = fmaxf(p.m, q.m);
  const float M = scaled(r.m, k), dp = scaled(p.m, k) - M, dq = scaled(q.m, k) - M;
  const float ep = exp2_fast(dp), eq = exp2_fast(dq);
  r.s = ep * p.s + eq * q.s;
  r.t = kEntropy ? ep * (p.t + finite(dp) * p.s) + eq * (q.t + finite(dq) * q.s) : 0.f;
  return r;
}

// A wavefront's keys in descending order, `found` of them in room for the next power of two (Batcher's exchanges).
__device__ __forceinline__ void sort_list(uint64_t* own, int found) {
  const int lane = threadIdx.x % kWave;
  int n = 2;
  while (n < found) n *= 2;
  for (int i = found + lane; i < n; i += kWave) own[i] = 0;
  meet<kWave>();
  for (int size = 2; size <= n; size *= 2)
    for (int d = size / 2; d; d /= 2) {
      for (int i = lane; i < n / 2; i += kWave) {
        const int lo = 2 * i - (i & (d - 1)), hi = lo + d;
        const uint64_t a = own[lo], b = own[hi];
        if ((a < b) == !(lo & size)) {
          own[lo] = b;
          own[hi] = a;
        }
      }
      meet<kWave>();
    }
}

// take(order, place) for each of a thread's values of a row, read from memory.
template <typename X, int kThreads, typename Row, typename Take>
__device__ __forceinline__ void sweep_orders(const Row& row, int thread, Take take) {
  using O = Order<X>;
#pragma unroll 1
  for (int c = thread; c < row.chunks; c += kThreads) {
    u32x4 u = row.chunk(c);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = O::of_packed(u[i]);
    const int at = row.at(c);
    O::each(u, [&](int i, int t) { take(t, at + i); });
  }
#pragma unroll 1
  for (int j = thread; j < row.kEdge; j += kThreads) {
    const int e = row.edge(j);
    if (e >= 0) take(O::of(X::load(row.x + e)), e);
  }
}

// Statistics of a row from one sweep over it, as row_stats, with few registers: rows whose reference is out of range, as
// where a mask of -inf leaves some of a wavefront's part, all below 0.
template <typename X, bool kEntropy, int kThreads, typename Row>
__device__ __forceinline__ Stats swept_stats(const Row& row, float k, int thread, Stats* parts) {
  Stats mine = {kLowest, 0.f, 0.f};
  auto take = [&](const float* v, auto count) {
    constexpr int n = decltype(count)::value;
    float top = mine.m;
#pragma unroll
    for (int i = 0; i < n; ++i) top = fmaxf(top, v[i]);
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
#pragma unroll 1
  for (int c = thread; c < row.chunks; c += kThreads) {
    float v[X::kPer];
    X::unpack(row.chunk(c), v);
    take(v, std::integral_constant<int, X::kPer>());
  }
#pragma unroll 1
  for (int j = thread; j < row.kEdge; j += kThreads) {
    const int e = row.edge(j);
    if (e < 0) continue;
    const float v[1] = {X::load(row.x + e)};
    take(v, std::integral_constant<int, 1>());
  }
  mine = joined_lanes<kEntropy, kWave>(mine, [k](const Stats& a, const Stats& b) { return joined<kEntropy>(a, b, k); });
  if constexpr (kThreads <= kWave) return mine;
  if (thread % kWave == 0) parts[thread / kWave] = mine;
  __syncthreads();
  Stats all = parts[0];
  for (int w = 1; w < kThreads / kWave; ++w) all = joined<kEntropy>(all, parts[w], k);
  return all;
}

// Where the values that a bound lets through are too many: keys of the K before all others, in any order, from keys[0] on;
// returns how many there are.  Ties and masks of the lowest value, where the smallest of these values has less than K
// above it, take two sweeps over the row, which comes from the caches; others (large values all in one place) as many more
// as it takes to find the K-th value by quarters, 8 or 16.
template <typename X, int kThreads, typename Row, typename Shared>
__device__ __forceinline__ int exact_keys(const Row& row, int thread, int K, int from, int bound, Shared& shared, uint64_t* keys) {
  using O = Order<X>;
  constexpr int kWaves = kThreads > kWave ? kThreads / kWave : 1;
  const int wave = thread / kWave, lane = thread % kWave;
  int turn = 0;
  // over all threads
  auto over_all = [&](int v, auto join) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v = join(v, __shfl_xor(v, d));
    if constexpr (kThreads > kWave) {
      turn ^= 1;
      if (lane == 0) shared.counted[turn][wave] = v;
      __syncthreads();
      v = shared.counted[turn][0];
      for (int w = 1; w < kWaves; ++w) v = join(v, shared.counted[turn][w]);
    }
    return v;
  };
  auto sum = [](int a, int b) { return a + b; };
  int least = INT32_MAX, at_least = 0, count = 0;
  sweep_orders<X, kThreads>(row, thread, [&](int t, int) {
    if (t < bound) return;
    ++count;
    at_least = t < least ? 1 : at_least + (t == least);
    least = min(least, t);
  });
  const int mine = least;
  least = over_all(least, [](int a, int b) { return min(a, b); });
  count = over_all(count, sum);
  int above = count - over_all(mine == least ? at_least : 0, sum);
  if (above >= K) {  // the K-th value: `least` is reached by K, `high` by `above` less than K
    int64_t low = least, high = int64_t(O::kMost) + 1;
    above = 0;
    while (high - low > 1) {
      const int64_t step = max((high - low) / 4, int64_t(1));
      const int m0 = int(low + step), m1 = int(min(low + 2 * step, high - 1)), m2 = int(min(low + 3 * step, high - 1));
      int n0 = 0, n1 = 0, n2 = 0;
      sweep_orders<X, kThreads>(row, thread, [&](int t, int) {
        n0 += t >= m0;
        n1 += t >= m1;
        n2 += t >= m2;
      });
      n0 = over_all(n0, sum);
      n1 = over_all(n1, sum);
      n2 = over_all(n2, sum);
      if (n2 >= K) {
        low = m2;
      } else if (n1 >= K) {
        low = m1;
        high = m2;
        above = n2;
      } else if (n0 >= K) {
        low = m0;
        high = m1;
        above = n1;
      } else {
        high = m0;
        above = n0;
      }
    }
    least = int(low);
  }
  // those above it, and of its equals the first ones: their numbers among all threads' values in the order of places
  int equals = K - above, slots = 0;
  auto take = [&](const int* t, int n, int at) {
    int larger = 0, same = 0;
    for (int i = 0; i < n; ++i) {
      larger += t[i] > least;
      same += t[i] == least;
    }
    int before = same << 16 | larger;  // (both at once: 4096 values at most)
    const int own = before;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int v = __shfl_up(before, d);
      if (lane >= d) before += v;
    }
    int all = __shfl(before, kWave - 1);
    before -= own;
    if constexpr (kThreads > kWave) {
      turn ^= 1;
      if (lane == 0) shared.counted[turn][wave] = all;
      __syncthreads();
      all = 0;
      for (int w = 0; w < kWaves; ++w) {
        const int v = shared.counted[turn][w];
        if (w < wave) before += v;
        all += v;
      }
    }
    // (the larger ones first, then as many of the equals as are wanted still)
    const int taken = min(all >> 16, equals);
    int to = slots + (before & 0xFFFF), rank = before >> 16;
    const int equal_slots = slots + (all & 0xFFFF);
    for (int i = 0; i < n; ++i) {
      if (t[i] > least) keys[to++] = key_of(t[i], from + at + i);
      if (t[i] == least) {
        if (rank < taken) keys[equal_slots + rank] = key_of(t[i], from + at + i);
        ++rank;
      }
    }
    equals -= taken;
    slots = equal_slots + taken;
  };
  // (a thread's values of the row's head, then of its chunks, then of what is behind these)
  const int none = INT32_MIN;
  {
    const int t[1] = {thread < row.head ? O::of(X::load(row.x + thread)) : none};
    take(t, 1, thread);
  }
#pragma unroll 1
  for (int c = 0; c < row.chunks; c += kThreads) {
    int t[X::kPer];
    const bool there = c + thread < row.chunks;
    u32x4 u = {};
    if (there) u = row.chunk(c + thread);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = O::of_packed(u[i]);
    O::each(u, [&](int i, int order) { t[i] = there ? order : none; });
    take(t, X::kPer, row.at(c + thread));
  }
  {
    const int e = row.head + row.chunks * X::kPer + thread;
    const int t[1] = {e < row.V ? O::of(X::load(row.x + e)) : none};
    take(t, 1, e);
  }
  if (thread == 0) keys[slots] = 0;  // (read in pairs)
  return slots;
}

// Joined parts of a row, of weights 2^((x - m) k) (apart), for parts that a kernel after this one joins.
__device__ __forceinline__ Found moved_apart(const Found& f, float k) {
  if (f.apart || !scales(f.m, k)) return {f.m, f.s, f.t, true};
  const float d = -fmaf(f.m, k, -scaled(f.m, k)), e = exp2_fast(d);
  return {f.m, e * f.s, e * (f.t + d * f.s), true};
}

constexpr int64_t kManyRows = 512;
constexpr int kCounted = 128;
// What a wavefront may find: chunks with candidates (of a tile), and candidates.
struct Room {
  int hits, keys;  // (keys: an even number, more than K by all that share a row, at most kMostKeys)
};
constexpr int kHitBytes = sizeof(u32x4) + sizeof(int);
constexpr int kTopThreads = 256;  // of a workgroup whose wavefronts have rows of their own

// The first value of a part of a long row: multiples of 64, so that parts are alike in length up to 64 values.
__device__ __forceinline__ int part_from(int V, int part, int parts) {
  return part == parts ? V : int(int64_t(V) * part / parts) & ~63;
}

// kThreads threads a row, or a part of one: a wavefront of four in a workgroup, or a workgroup.  With kTiled a row (or
// part) is longer than the registers hold, and is taken tile by tile: what has been found in those before is a
// bound for the next ones.
template <typename X, bool kEntropy, int kThreads, int kChunks, int kStep, bool kTiled = false>
__global__ __launch_bounds__(kThreads <= kWave ? kTopThreads : kThreads) void top_kernel(Rows r, RowOut o, Top q, Split split,
                                                                                      Room room) {
  constexpr bool kAlone = kThreads > kWave;
  constexpr int kTeams = kAlone ? 1 : kTopThreads / kThreads, kWaves = kAlone ? kThreads / kWave : 1;
  using H = Taken<X, kThreads, kChunks, kStep>;
  using O = Order<X>;
  // of each wavefront: chunks with candidates, their places, the candidates' keys
  extern __shared__ __attribute__((aligned(16))) uint64_t candidates[];
  __shared__ TopShared<kWaves> all[kTeams];
  const int team = threadIdx.x / kThreads, thread = threadIdx.x % kThreads, wave = thread / kWave, lane = threadIdx.x % kWave;
  const bool first = thread == 0;
  TopShared<kWaves>& shared = all[team];
  constexpr int kAllWaves = kTeams * kWaves;
  u32x4* chunks = reinterpret_cast<u32x4*>(candidates) + threadIdx.x / kWave * room.hits;
  int* places = reinterpret_cast<int*>(reinterpret_cast<u32x4*>(candidates) + kAllWaves * room.hits) + threadIdx.x / kWave * room.hits;
  uint64_t* keys = candidates + kAllWaves * (room.hits * kHitBytes / 8) + team * kWaves * room.keys;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  auto take_unit = [&](int64_t unit, int thread, int lane) {
    const int64_t which = split.parts == 1 ? unit : unit / split.parts;
    const int part = int(unit - which * split.parts);
    const int64_t at = kAlone && split.parts == 1 ? row_of_group(which, rows) : which;
    const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
    if (first && part == 0 && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    if (!counts(r, b, t)) {
      if (part == 0) {
        if (first) leave_nothing(o, at);
        put_none(q, at, 0, -INFINITY, thread, kThreads);
      }
      return;
    }
    const int from = kAlone ? part_from(r.V, part, split.parts) : 0;
    int V = kAlone ? part_from(r.V, part + 1, split.parts) - from : r.V;
    if constexpr (!kAlone) asm volatile("" : "+s"(V));
    const typename X::type* values = row_of<X>(r, b, t) + from;
    // (what comes first is waited for first: not behind the whole row)
    const int token = r.tokens && part == 0 ? take_token(r, b, t, first) : -1;
    float x = __uint_as_float(kNan);
    const int need = (q.K + kWaves - 1) / kWaves, tiles = kTiled ? split.tiles : 1;
    int found = 0, bound = O::kNone + 1, turn = 0;
    bool much = false;
    Stats s = {};
    uint64_t* own = keys + wave * room.keys;
    auto start_of = [&](int tile) { return kTiled ? part_from(V, tile, tiles) : 0; };
    auto tile_of = [&](int tile) {
      return typename H::Row(values + start_of(tile), kTiled ? start_of(tile + 1) - start_of(tile) : V);
    };
    H h;
    h.load(tile_of(0), thread);
    if (token >= 0) x = X::load(values - from + token);
    for (int tile = 0; tile < tiles; ++tile) {
      const int start = start_of(tile);
      const typename H::Row row = tile_of(tile);
      const Stats mine = taken_stats<kEntropy>(h, k);
      s = tile ? joined_scaled<kEntropy>(s, mine, k) : mine;
      // the workgroup's bound: what all wavefronts have `need` values from
      int least;
      auto shared_bound = [&](int turn) {
        if constexpr (kAlone) {
          if (lane == 0) shared.bounds[turn][wave] = least;
          __syncthreads();
          for (int w = 0; w < kWaves; ++w) least = min(least, shared.bounds[turn][w]);
        }
        bound = max(bound, least);
      };
      // Raw bits as signed integers are in the values' order from 0 on, with all others below: they do as long as
      // the bound is above 0.
      int most[H::kParts], edge_order = O::raw(h.edge);
      bool by_values = false;
      if constexpr (!kAlone) by_values = split.by_values;
      if (tile == 0) {
        if (!by_values) {
          h.largest(most, edge_order);
          least = wave_bound<X>(most, need);
          if (least < 1) least = O::kNone;
          shared_bound(0);
        }
      } else {
        // a new bound from what has been found: all tiles together find about K log(tiles) candidates
        least = list_bound<X>(own, found, need);
        shared_bound(2 + turn);
        turn ^= 1;
        int kept = 0;
        for (int i = 0; i < found; i += kWave) {
          const uint64_t key = i + lane < found ? own[i + lane] : 0;
          const bool is = i + lane < found && order_in(key) >= bound;
          const uint64_t mask = __ballot(is);
          meet<kWave>();
          if (is) own[kept + lanes_before(mask)] = key;
          kept += __popcll(mask);
        }
        found = kept;
        meet<kWave>();
      }
      if (bound < 1) {
        h.to_order();
        edge_order = O::of(h.edge);
        if (tile == 0) {
          if (by_values) {
            least = h.value_bound(edge_order, need);
          } else {
            h.largest(most, edge_order);
            least = wave_bound<X>(most, need);
          }
          shared_bound(1);
        }
      }
      // The values from the bound on, as keys in LDS, a part for each wavefront: first the chunks that have some,
      // with one lane storing all of its chunk, then each value of these.
      int from_here = bound;
      int hits = h.hits(row, thread, from_here, chunks, places, room.hits);
      if (kTiled && tile > 0 && hits > room.hits / 2) {
        // more than the tiles before let expect (rising values): no wavefront needs more than its own K largest
        h.largest(most, edge_order);
        const int local = wave_bound<X>(most, q.K);
        if (local > from_here) {
          from_here = local;
          meet<kWave>();
          hits = h.hits(row, thread, from_here, chunks, places, room.hits);
        }
      }
      const int edge_at = h.edge_at;
      if (kTiled && tile + 1 < tiles) h.load(tile_of(tile + 1), thread);
      meet<kWave>();
      auto take = [&](bool is, int order, int place) {
        const uint64_t mask = __ballot(is);
        const int slot = found + lanes_before(mask);
        if (is && slot < room.keys) own[slot] = key_of(order, from + start + place);
        found += __popcll(mask);
      };
      much = much || hits > room.hits;
      hits = min(hits, room.hits);
      for (int e = 0; e < hits; e += kWave / X::kPer) {
        const int hit = e + lane / X::kPer, i = lane % X::kPer;
        const bool there = hit < hits;
        const int order = there ? O::in_chunk(chunks + hit, i) : O::kNone, place = there ? places[hit] + i : 0;
        take(there && order >= from_here, order, place);
      }
      if (__any(edge_order >= from_here)) take(edge_order >= from_here, edge_order, edge_at);
      much = much || found > room.keys;
      found = min(found, room.keys);
      meet<kWave>();
    }
    if (lane == 0) {
      if (found < room.keys) own[found] = 0;  // (keys are read in pairs)
      if (kAlone) {
        shared.parts[wave] = s;
        shared.counts[wave] = much ? -1 : found;
      }
    }
    meet<kThreads>();
    int total = found;
    if constexpr (kAlone) {
      s = block_stats<kEntropy, kWaves>(shared.parts, k);
      total = 0;
      for (int w = 0; w < kWaves; ++w) {
        const int n = shared.counts[w];
        total += n;
        much = much || n < 0;
      }
    }
    const typename H::Row row(values, V);
    const bool extreme = !fine(s, k);
    if (extreme) {
      meet<kThreads>();
      s = swept_stats<X, kEntropy, kThreads>(row, k, thread, shared.parts);
    }
    const Found f = {s.m, s.s, s.t, extreme};
    const bool none = f.s != f.s || (split.parts == 1 && lost(f));
    if (none) total = found = 0;
    else if (much) {
      meet<kThreads>();
      total = exact_keys<X, kThreads>(row, thread, q.K, from, bound, shared, keys);  // (in the first wavefronts' parts)
      found = kAlone ? max(min(total - wave * room.keys, room.keys), 0) : total;
      if (kAlone && lane == 0) shared.counts[wave] = found;
      meet<kThreads>();
    }
    const float log_s = logf(f.s);
    auto put_key = [&](int rank, uint64_t key) {
      if (split.parts > 1) {
        split.keys[unit * q.K + rank] = key;
      } else {
        put_id(q, at * q.K + rank, place_in(key));
        q.logprobs[at * q.K + rank] = logprob(f, O::value(order_in(key)), k, r.inv_temp, log_s);
      }
    };
    // Each one's place is the number of larger keys: kWaves lanes count those of a wavefront's part each.  Many of a
    // wavefront are sorted: counting takes found^2 / 64 comparisons.
    const bool sorted = !kAlone && found > kCounted && found <= (room.keys & ~3);  // (the next power of two fits)
    if (sorted) {
      sort_list(own, found);
      for (int i = lane; i < min(found, q.K); i += kWave) put_key(i, own[i]);
      found = 0;
    }
    const int share = lane % kWaves;
    const uint64_t* others = keys + share * room.keys;
    const int theirs = kAlone ? shared.counts[share] : found;
    for (int i = lane / kWaves; i < found; i += kWave / kWaves) {
      const uint64_t key = own[i];
      int rank = 0, j = 0;
      for (; j + 4 < theirs; j += 4) {
        const ulonglong2 one = *reinterpret_cast<const ulonglong2*>(others + j), two = *reinterpret_cast<const ulonglong2*>(others + j + 2);
        rank += (one.x > key) + (one.y > key) + (two.x > key) + (two.y > key);
      }
      for (; j < theirs; j += 2) {
        const ulonglong2 one = *reinterpret_cast<const ulonglong2*>(others + j);
        rank += (one.x > key) + (one.y > key);
      }
      rank = lanes_total<kWaves>(rank);
      if (rank < q.K && !share) put_key(rank, key);
    }
    if (split.parts > 1) {
      for (int j = min(total, q.K) + thread; j < q.K; j += kThreads) split.keys[unit * q.K + j] = 0;
      const Found g = moved_apart(f, k);
      if (first) split.stats[unit] = {g.m, g.s, g.t, x};
    } else {
      put_none(q, at, min(total, q.K), none ? __uint_as_float(kNan) : -INFINITY, thread, kThreads);
      if (first) put_values<kEntropy>(r, o, f, x, k, log_s, at);
    }
  };
  // (a workgroup takes one row: what lives from row to row would cost it registers)
  if constexpr (kAlone) {
    take_unit(split.first + blockIdx.x, thread, lane);
  } else {
    for (int64_t group = blockIdx.x; group * kTeams < rows; group += gridDim.x) {
      const int64_t unit = turned(group, (rows + kTeams - 1) / kTeams) * kTeams + team;
      int now = thread;  // (keeps the compiler from working out places and masks once for all rows, 50 registers)
      asm volatile("" : "+v"(now));
      if (unit < rows) take_unit(unit, now, now);
      meet<kThreads>();  // (before the next row takes the shared memory)
    }
  }
}

// ---- the parts of long rows -------------------------------------------------------------------

// `last`: over the workgroup's threads, the largest or smallest key.
template <bool kLargest>
__device__ __forceinline__ uint64_t block_key(uint64_t v, uint64_t* part) {
#pragma unroll
  for (int d = kWave / 2; d; d >>= 1) {
    const uint64_t u = __shfl_xor(static_cast<unsigned long long>(v), d);
    v = (u > v) == kLargest ? u : v;
  }
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < kTopThreads / kWave; ++w) v = (part[w] > v) == kLargest ? part[w] : v;
  return v;
}

// One workgroup a row.  Every part's keys are in descending order: the largest of the parts' K-th keys is reached by K
// keys, and so is the smallest of their (K / parts)-th ones.
constexpr int kJoinRoom = 2048;
template <typename X, bool kEntropy>
__global__ __launch_bounds__(kTopThreads) void join_kernel(Rows r, RowOut o, Top q, Split split) {
  __shared__ __attribute__((aligned(16))) uint64_t keys[kJoinRoom + 2];
  __shared__ uint64_t tops[kTopThreads / kWave], lows[kTopThreads / kWave];
  __shared__ int counted[2][kTopThreads / kWave], slots;
  __shared__ Stats joints[kTopThreads / kWave];
  const int thread = threadIdx.x;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  for (int64_t at = blockIdx.x; at < rows; at += gridDim.x) {
    const At pos = position(r, at);
    if (!counts(r, pos.b, pos.t)) continue;  // (the kernel before has written what is left of it)
    const uint64_t* from = split.keys + at * split.parts * q.K;
    const float4* stats = split.stats + at * split.parts;
    const int K = q.K, share = (K + split.parts - 1) / split.parts;
    const int64_t n = int64_t(split.parts) * K;
    if (thread == 0) slots = 0;
    // (what is read first is under way together)
    const uint64_t own = thread < n ? from[thread] : 0;
    uint64_t top = 0, low = ~uint64_t(0);
    Stats s = {kLowest, 0.f, 0.f};
    for (int p = thread; p < split.parts; p += kTopThreads) {
      top = max(top, from[int64_t(p) * K + K - 1]);
      low = min(low, from[int64_t(p) * K + share - 1]);
      const float4 v = stats[p];
      s = joined<kEntropy>(s, Stats{v.x, v.y, v.z}, k);
    }
    const float x = stats[0].w;
    s = joined_lanes<kEntropy, kWave>(s, [k](const Stats& a, const Stats& b) { return joined<kEntropy>(a, b, k); });
    if (thread % kWave == 0) joints[thread / kWave] = s;
    top = block_key<true>(top, tops);
    low = block_key<false>(low, lows);
    uint64_t bound = max(max(top, low), uint64_t(1));
    s = joints[0];
    for (int w = 1; w < kTopThreads / kWave; ++w) s = joined<kEntropy>(s, joints[w], k);
    const Found f = {s.m, s.s, s.t, true};
    const float log_s = logf(f.s);
    const bool none = lost(f);
    int total = 0;
    while (!none) {
      for (int64_t i = thread; i < n; i += kTopThreads) {
        const uint64_t key = i == thread ? own : from[i];
        if (key < bound) continue;
        const int slot = atomicAdd(&slots, 1);
        if (slot < kJoinRoom) keys[slot] = key;
      }
      __syncthreads();
      total = slots;
      if (total <= kJoinRoom) break;
      // the K-th key itself, by halving: keys differ from one another
      uint64_t high = ~uint64_t(0);
      int turn = 0;
      while (high - bound > 1) {
        const uint64_t mid = bound + (high - bound) / 2;
        int c = 0;
        for (int64_t i = thread; i < n; i += kTopThreads) c += from[i] >= mid;
        c = full_wave_sum(c);
        turn ^= 1;
        if (thread % kWave == 0) counted[turn][thread / kWave] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < kTopThreads / kWave; ++w) c += counted[turn][w];
        if (c >= K) bound = mid;
        else high = mid;
      }
      if (thread == 0) slots = 0;
      __syncthreads();
    }
    if (thread == 0) keys[total] = 0;  // (read in pairs)
    __syncthreads();
    for (int i = thread; i < total; i += kTopThreads) {
      const uint64_t key = keys[i];
      int rank = 0;
      for (int j = 0; j < total; j += 2) {
        const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(keys + j);
        rank += (two.x > key) + (two.y > key);
      }
      if (rank >= K) continue;
      put_id(q, at * K + rank, place_in(key));
      q.logprobs[at * K + rank] = logprob(f, Order<X>::value(order_in(key)), k, r.inv_temp, log_s);
    }
    put_none(q, at, min(total, K), none ? __uint_as_float(kNan) : -INFINITY, thread, kTopThreads);
    if (thread == 0) put_values<kEntropy>(r, o, f, x, k, log_s, at);
    __syncthreads();  // (before the next row takes the shared memory)
  }
}

// ---- short rows -------------------------------------------------------------------------------

// The largest key of the lanes that share a row, in all of them.
template <int kLanes, int kStep = 1>
__device__ __forceinline__ uint32_t lanes_most(uint32_t v) {
  if constexpr (kStep == kLanes) return v;
  else return lanes_most<kLanes, kStep * 2>(max(v, __float_as_uint(neighbour<kStep>(__uint_as_float(v)))));
}
template <int kLanes, int kStep = 1>
__device__ __forceinline__ uint64_t lanes_most(uint64_t v) {
  if constexpr (kStep == kLanes) return v;
  else {
    const uint32_t high = __float_as_uint(neighbour<kStep>(__uint_as_float(uint32_t(v >> 32))));
    const uint32_t low = __float_as_uint(neighbour<kStep>(__uint_as_float(uint32_t(v))));
    return lanes_most<kLanes, kStep * 2>(max(v, uint64_t(high) << 32 | low));
  }
}

// Keys in descending order: Batcher's exchanges (1968) for four and eight.
template <typename Key>
__device__ __forceinline__ void exchange(Key* v, int i, int j) {
  const Key a = v[i], b = v[j];
  v[i] = max(a, b);
  v[j] = min(a, b);
}
template <typename Key, int kN>
__device__ __forceinline__ void sort_keys(Key* v) {
  static_assert(kN == 4 || kN == 8);
#pragma unroll
  for (int h = 0; h < kN; h += 4) {
    exchange(v, h, h + 1);
    exchange(v, h + 2, h + 3);
    exchange(v, h, h + 2);
    exchange(v, h + 1, h + 3);
    exchange(v, h + 1, h + 2);
  }
  if constexpr (kN == 8) {
    exchange(v, 0, 4);
    exchange(v, 1, 5);
    exchange(v, 2, 6);
    exchange(v, 3, 7);
    exchange(v, 2, 4);
    exchange(v, 3, 5);
    exchange(v, 1, 2);
    exchange(v, 3, 4);
    exchange(v, 5, 6);
  }
}

// The eight largest keys of two descending lists: no key of the one is behind its counterpart of the other in reverse,
// and what that leaves rises and then falls (Batcher).
template <typename Key>
__device__ __forceinline__ void merge_keys(Key* v, const Key* u) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = max(v[i], u[7 - i]);
#pragma unroll
  for (int d = 4; d; d >>= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & d)) exchange(v, i, i + d);
}
template <int kStep>
__device__ __forceinline__ uint32_t neighbour_key(uint32_t v) {
  return __float_as_uint(neighbour<kStep>(__uint_as_float(v)));
}
template <int kStep>
__device__ __forceinline__ uint64_t neighbour_key(uint64_t v) {
  return uint64_t(neighbour_key<kStep>(uint32_t(v >> 32))) << 32 | neighbour_key<kStep>(uint32_t(v));
}
// Of the lanes that share a row, in all of them.
template <int kLanes, int kStep = 1, typename Key>
__device__ __forceinline__ void merge_lanes(Key* v) {
  if constexpr (kStep < kLanes) {
    Key u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = neighbour_key<kStep>(v[i]);
    merge_keys(v, u);
    merge_lanes<kLanes, kStep * 2>(v);
  }
}

// A key into the descending list `v`, of which kFilled are there, when kBefore of these are known to be larger: an
// instruction a place.
template <int kKeep, int kFilled, int kBefore = 0>
__device__ __forceinline__ void insert_key(uint32_t* v, uint32_t key) {
  uint32_t old[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) old[i] = v[i];
#pragma unroll
  for (int i = kBefore; i < kKeep; ++i) {
    if (i > kFilled) break;
    if (i == kFilled) v[i] = i == kBefore ? key : min(old[i - 1], key);
    else if (i == kBefore) v[i] = max(old[i], key);
    else v[i] = max(min(key, old[i]), min(max(key, old[i]), old[i - 1]));  // (the median of three)
  }
}
template <int kKeep, int kI = 0>
__device__ __forceinline__ void insert_keys(uint32_t* v, const uint32_t* keys, bool first) {
  if constexpr (kI < 8) {
    if (first) insert_key<kKeep, kI < kKeep ? kI : kKeep>(v, keys[kI]);
    else insert_key<kKeep, kKeep>(v, keys[kI]);
    insert_keys<kKeep, kI + 1>(v, keys, first);
  }
}
// Two lists: the second one's places are known to be none before their own.
template <int kKeep, int kI = 0>
__device__ __forceinline__ void insert_list(uint32_t* v, const uint32_t* u) {
  if constexpr (kI < kKeep) {
    insert_key<kKeep, kKeep, kI>(v, u[kI]);
    insert_list<kKeep, kI + 1>(v, u);
  }
}
template <int kKeep, int kLanes, int kStep = 1>
__device__ __forceinline__ void insert_lanes(uint32_t* v) {
  if constexpr (kStep < kLanes) {
    uint32_t u[kKeep];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) u[i] = neighbour_key<kStep>(v[i]);
    insert_list<kKeep>(v, u);
    insert_lanes<kKeep, kLanes, kStep * 2>(v);
  }
}

// Keys of short rows: in 32 bits with the place in the lower half where values have 16.
template <typename X>
struct ShortKey {
  using type = uint32_t;
  static __device__ __forceinline__ int order(type key) { return int(key >> 16) - 32768; }
  static __device__ __forceinline__ int place(type key) { return 0xFFFF - int(key & 0xFFFFu); }
  static __device__ __forceinline__ type of(int t, int place) { return uint32_t(t + 32768) << 16 | uint32_t(0xFFFF - place); }
  // of a chunk's values, the first of which is at `place`
  static __device__ __forceinline__ void of_chunk(u32x4 c, int place, type* keys) {
    const uint32_t low = uint32_t(0xFFFF - place);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = Order<X>::of_packed(c[i]) ^ 0x80008000u;
      keys[2 * i] = t << 16 | (low - 2 * i);
      keys[2 * i + 1] = (t & 0xFFFF0000u) | (low - 2 * i - 1);
    }
  }
};
template <>
struct ShortKey<F32> {
  using type = uint64_t;
  static __device__ __forceinline__ int order(type key) { return order_in(key); }
  static __device__ __forceinline__ int place(type key) { return place_in(key); }
  static __device__ __forceinline__ type of(int t, int place) { return key_of(t, place); }
  static __device__ __forceinline__ void of_chunk(u32x4 c, int place, type* keys) {
#pragma unroll
    for (int i = 0; i < 4; ++i) keys[i] = key_of(int(Order<F32>::of_packed(c[i])), place + i);
  }
};

// A persistent workgroup's place in a round: another one in each, so that the ends of sequences, whose positions do not
// count, fall to all workgroups (and XCDs) alike.  (4096 x 512 rows of 64 values, 53 % of which count: 127 us without.)
__device__ __forceinline__ uint32_t place_in_round(int64_t round) {
  return uint32_t((blockIdx.x + round) % gridDim.x);
}

// Up to eight alternatives of rows of up to 1024 values: each lane keeps the best of its chunks, and the lanes join
// theirs.  Keys of 32 bits are inserted one by one into a list of kKeep, an instruction a place (a median of three);
// 64-bit ones are sorted eight by eight and merged (as 32-bit ones were: 2097152 positions of 64 values, 53 % of
// which count, K = 5, 95 us, and 79 so).  Few lanes with many chunks share what is done once a row.  Five workgroups a
// unit: with 4 (116 registers) 85 us, with 6 (spills) 110.
constexpr int kFewest = 8, kBestGroups = 5120, kShortSteps = 2048;
template <typename X, bool kEntropy, int kLanes, int kChunks, int kKeep>
__global__ __launch_bounds__(kTopThreads, 5) void best_kernel(Rows r, RowOut o, Top q) {
  constexpr int kTeams = kTopThreads / kLanes, kOctet = 8 / X::kPer;  // chunks that are sorted together
  using O = Order<X>;
  using Key = ShortKey<X>;
  using K = typename Key::type;
  constexpr bool kInsert = sizeof(K) == 4;
  static_assert(kChunks % kOctet == 0 && (kInsert || kKeep == 8));
  constexpr int kEntries = kWave / kLanes * kKeep;
  __shared__ K all_entries[kTopThreads / kWave][kEntries];
  __shared__ float2 all_found[kTopThreads / kWave][kWave / kLanes];
  K* entries = all_entries[threadIdx.x / kWave];
  float2* found = all_found[threadIdx.x / kWave];
  const uint32_t per_entry = (65536u + q.K - 1) / q.K;  // (of a number below 256, the quotient by K is exact so)
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  for (int64_t round = 0; round * gridDim.x * kTeams < rows; ++round) {
    int V = r.V;
    asm volatile("" : "+s"(V));  // (as in lanes_kernel)
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int lane = thread % kLanes;
    const int64_t at = (round * gridDim.x + place_in_round(round)) * kTeams + thread / kLanes;
    const bool inside = at < rows;
    const At pos = position(r, inside ? at : rows - 1);
    const int b = pos.b, t = pos.t;
    const bool live = inside && counts(r, b, t);
    if (inside && lane == 0 && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    K best[kKeep] = {};
    Found f = {0.f, 1.f, 0.f, false};
    float x = 0.f, log_s = 0.f;
    if (__any(live)) {
      const typename X::type* values = row_of<X>(r, b, t);
      Part<X, kLanes, kChunks> part;
      part.load(values, V, lane, live);
      const int token = live && r.tokens ? take_token(r, b, t, lane == 0) : -1;
      x = token < 0 ? __uint_as_float(kNan) : X::load(values + token);
#pragma unroll
      for (int j = 0; j < kChunks; j += kOctet) {
        K keys[8];
#pragma unroll
        for (int h = 0; h < kOctet; ++h) {
          const int place = Part<X, kLanes, kChunks>::at(V, lane, j + h);
          Key::of_chunk(part.c[j + h], place, keys + h * X::kPer);
          // values that are another chunk's, or beyond the row
          if (V % X::kPer == 0 && place >= 0) continue;
          const int again = place < 0 ? X::kPer : (lane + (j + h) * kLanes) * X::kPer - place;
#pragma unroll
          for (int i = 0; i < X::kPer; ++i)
            if (i < again) keys[h * X::kPer + i] = 0;
        }
        if constexpr (kInsert) {
          insert_keys<kKeep>(best, keys, j == 0);
        } else {
          sort_keys<K, 8>(keys);
          if (j == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) best[i] = keys[i];
          } else {
            merge_keys(best, keys);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (kInsert) insert_lanes<kKeep, kLanes>(best);
      else merge_lanes<kLanes>(best);
      part.keep_packed();
      // the best is the largest value, or the row has a NaN
      f.m = live ? O::value(Key::order(best[0])) : 0.f;
      f.apart = !scales(f.m, k);
      const float M = scaled(f.m, k);
      f.s = 0.f;
      auto sums = [&](auto argument) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
          float v[X::kPer];
          part.once(V, lane, j, v);
#pragma unroll
          for (int i = 0; i < X::kPer; ++i) {
            const float a = argument(v[i]), w = exp2_fast(a);
            f.s += w;
            if (kEntropy) f.t += w * finite(a);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if (__any(f.apart)) sums([&](float v) { return f.apart ? (v - f.m) * k : fmaf(v, k, -M); });
      else sums([&](float v) { return fmaf(v, k, -M); });
      f.s = lanes_added<kLanes>(f.s);
      if (kEntropy) f.t = lanes_added<kLanes>(f.t);
      log_s = logf(f.s);
    }
    const bool none = lost(f);
    const float missing = live && none ? __uint_as_float(kNan) : -INFINITY;
    auto put = [&](int64_t to, K key, const Found& g, float log_sum, float otherwise) {
      put_id(q, to, key ? Key::place(key) : -1);
      q.logprobs[to] = key ? logprob(g, O::value(Key::order(key)), k, r.inv_temp, log_sum) : otherwise;
    };
    auto entry = [&](int j) { return live && !none && Key::order(best[j]) > O::kNone ? best[j] : 0; };
    if constexpr (kKeep <= 2) {
#pragma unroll
      for (int j = 0; j < kKeep; ++j)
        if (inside && j < q.K && j % kLanes == lane) put(at * q.K + j, entry(j), f, log_s, missing);
    } else {
      // Through LDS, from where neighbouring lanes store neighbouring entries and work out their log-probabilities.
      // (2097152 rows of 64 values of which none counts, all, K = 5: 32 and 101 us, and 51 and 110 with each entry stored by
      // the lane that has it; K = 1: 23 and 78, and 20 and 74.)
      const int own = thread % kWave / kLanes;
      if (lane == 0) found[own] = {f.m, !live ? 0.f : none ? missing : log_s};
#pragma unroll
      for (int j = 0; j < kKeep; ++j)
        if (j < q.K && j % kLanes == lane) entries[own * q.K + j] = entry(j);
      meet<kWave>();
      const int64_t first = at - own;
      const int n = int(min(rows - first, int64_t(kWave / kLanes))) * q.K;
      for (int i = thread % kWave; i < n; i += kWave) {
        const float2 of = found[i * per_entry >> 16];
        put(first * q.K + i, entries[i], {of.x, 0.f, 0.f, !scales(of.x, k)}, of.y, of.y != of.y ? of.y : -INFINITY);
      }
      meet<kWave>();
    }
    if (lane == 0 && live) put_values<kEntropy>(r, o, f, x, k, log_s, at);
    else if (lane == 0 && inside) leave_nothing(o, at);
  }
}

// kLanes lanes of a wavefront a row, a chunk each, whose values each lane puts in order; the best of the lanes' best is
// the row's next one.
template <typename X, bool kEntropy, int kLanes>
__global__ __launch_bounds__(kTopThreads) void short_kernel(Rows r, RowOut o, Top q) {
  constexpr int kTeams = kTopThreads / kLanes;
  using O = Order<X>;
  using Key = ShortKey<X>;
  const int lane = threadIdx.x % kLanes;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e;
  const int V = max(r.V, X::kPer);  // (a chunk at least, with nothing behind the row)
  for (int64_t round = 0; round * gridDim.x * kTeams < rows; ++round) {
    const int64_t at = (round * gridDim.x + place_in_round(round)) * kTeams + threadIdx.x / kLanes;
    const bool inside = at < rows;
    const At pos = position(r, inside ? at : rows - 1);
    const int b = pos.b, t = pos.t;
    const bool live = inside && counts(r, b, t);
    if (inside && lane == 0 && t == 0 && r.lengths) held_length(r.lengths[b], r.T, r.status);
    const typename X::type* values = row_of<X>(r, b, t);
    Part<X, kLanes, 1> part;
    if (r.V >= X::kPer) {
      part.load(values, V, lane, live);
    } else {
      float v[X::kPer];
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) v[i] = live && lane == 0 && i < r.V ? X::load(values + i) : -INFINITY;
      part.c[0] = X::pack(v);
    }
    const int token = live && r.tokens ? take_token(r, b, t, lane == 0) : -1;
    const float x = token < 0 ? __uint_as_float(kNan) : X::load(values + token);
    const Stats s = part_stats<kEntropy, kLanes>(part, V, lane, k);
    const Found f = {s.m, s.s, s.t, true};
    const bool none = lost(f);
    const float log_s = logf(f.s);
    typename Key::type keys[X::kPer];
    {
      float v[X::kPer];
      part.once(V, lane, 0, v);
      const int place = Part<X, kLanes, 1>::at(V, lane, 0);
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) {
        const int order = O::of(v[i]);
        keys[i] = order > O::kNone && live && !none ? Key::of(order, place + i) : 0;
      }
    }
    sort_keys<typename Key::type, X::kPer>(keys);
    typename Key::type kept = 0;
    for (int j = 0; j < q.K; ++j) {
      const typename Key::type best = lanes_most<kLanes>(keys[0]);
      if (j % kLanes == lane) kept = best;
      const bool mine = keys[0] == best;
#pragma unroll
      for (int i = 0; i < X::kPer - 1; ++i) keys[i] = mine ? keys[i + 1] : keys[i];
      keys[X::kPer - 1] = mine ? 0 : keys[X::kPer - 1];
      if (j % kLanes != kLanes - 1 && j != q.K - 1) continue;
      if (inside && lane <= j % kLanes) {
        const int64_t to = at * q.K + (j - j % kLanes + lane);
        put_id(q, to, kept ? Key::place(kept) : -1);
        q.logprobs[to] = kept          ? logprob(f, O::value(Key::order(kept)), k, r.inv_temp, log_s)
                         : live && none ? __uint_as_float(kNan)
                                        : -INFINITY;
      }
    }
    if (lane == 0 && live) put_values<kEntropy>(r, o, f, x, k, log_s, at);
    else if (lane == 0 && inside) leave_nothing(o, at);
  }
}

// ---- gradient ---------------------------------------------------------------------------------

// kThreads threads a row: the softmax's part from one reading of the row, then the entries' and the token's places
// written over with what they get beside it.
template <typename X, bool kEntropy, int kThreads>
__global__ __launch_bounds__(kThreads <= kWave ? kTopThreads : kThreads) void top_gradient_kernel(Rows r, Top q, TopGiven v) {
  constexpr bool kAlone = kThreads > kWave;
  constexpr int kTeams = kAlone ? 1 : kTopThreads / kThreads;
  __shared__ float sums[kAlone ? kThreads / kWave : 1];
  const int team = threadIdx.x / kThreads, thread = threadIdx.x % kThreads;
  const int64_t rows = int64_t(r.B) * r.T;
  const float k = r.inv_temp * kLog2e, scale = r.g_scale * r.inv_temp;
  for (int64_t group = blockIdx.x; group * kTeams < rows; group += gridDim.x) {
    const int64_t at = kAlone ? row_of_group(group, rows) : turned(group, (rows + kTeams - 1) / kTeams) * kTeams + team;
    if (at >= rows) continue;
    const At pos = position(r, at);
    const int b = pos.b, t = pos.t;
    if (!counts(r, b, t)) {
      write_zeros<X>(r, b, t, thread, kThreads);
      continue;
    }
    using Row = Span<X, kThreads <= kWave ? 16 : kLine>;
    const Row row(row_of<X>(r, b, t), r.V);
    typename X::type* g = gradient_of<X>(r, b, t);
    const float4 state = v.state[at];
    const float d_lp = v.d_lp ? v.d_lp[at] : 0.f, d_H = kEntropy ? v.d_entropy[at] : 0.f;
    const int token = r.tokens && v.d_lp ? take_token(r, b, t, false) : -1;
    auto entry = [&](int j) {
      const int64_t id = load_id(q.ids, q.long_ids, at * q.K + j);
      return id >= 0 && id < r.V ? int(id) : -1;
    };
    float sum = 0.f;
    for (int j = thread; j < q.K; j += kThreads) sum += entry(j) < 0 ? 0.f : v.d_top[at * q.K + j];
#pragma unroll
    for (int d = 1; d < (kAlone ? kWave : kThreads); d <<= 1) sum += __shfl_xor(sum, d);
    if constexpr (kAlone) {
      if (thread % kWave == 0) sums[thread / kWave] = sum;
      __syncthreads();
      sum = 0.f;
      for (int w = 0; w < kThreads / kWave; ++w) sum += sums[w];
    }
    // (a wrong token makes the row NaN)
    const float all = r.tokens && v.d_lp && token < 0 ? __uint_as_float(kNan) : sum + d_lp;
    const Slope f = slope_of(state.y * from_scaled(state.x, k), state.z, all, d_H, scale);
    write_gradient<X, kEntropy, kThreads>(row, g, thread, state.x, k, f);
    meet<kThreads>();  // (what it has stored comes before what follows)
    auto over = [&](int id, float d) {
      const float a = (X::load(row.x + id) - state.x) * k;
      X::store(g + id, scale * d + gradient_at<kEntropy>(a, f));
    };
    if (thread == 0 && token >= 0) over(token, d_lp);
    meet<kThreads>();
    for (int j = thread; j < q.K; j += kThreads) {
      const int id = entry(j);
      if (id >= 0) over(id, v.d_top[at * q.K + j] + (id == token ? d_lp : 0.f));
    }
    meet<kThreads>();
  }
}

// ---- launches ---------------------------------------------------------------------------------

template <typename X, bool kEntropy>
hipError_t launch_top(const TopCall& c) {
  const Rows& r = c.rows;
  const int64_t rows = int64_t(r.B) * r.T;
  const int chunks = (r.V + X::kPer - 1) / X::kPer;
  auto groups_of = [](int64_t units, int at_a_time) {
    const int64_t groups = (units + at_a_time - 1) / at_a_time;
    return int(groups < kMostGroups ? groups : kMostGroups);
  };
  // (lists no longer than they have to be, where their length is what keys cost)
  auto best = [&](auto lanes, auto keep) {
    constexpr int kLanes = decltype(lanes)::value;
    const int groups = std::min(groups_of(rows, kTopThreads / kLanes), kBestGroups);
    best_kernel<X, kEntropy, kLanes, 4, decltype(keep)::value><<<groups, kTopThreads, 0, c.stream>>>(r, c.out, c.top);
    return hipGetLastError();
  };
#define BEST(lanes)                                                                          \
  if (chunks <= lanes * 4) {                                                                 \
    const std::integral_constant<int, lanes> n;                                              \
    if constexpr (X::kPer == 8) {                                                            \
      if (c.top.K <= 2) return best(n, std::integral_constant<int, 2>());                    \
      if (c.top.K <= 5) return best(n, std::integral_constant<int, 5>());                    \
    }                                                                                        \
    return best(n, std::integral_constant<int, kFewest>());                                  \
  }
  if (c.top.K <= kFewest && r.V >= X::kPer) { BEST(2) BEST(4) BEST(8) BEST(16) BEST(32) }
#undef BEST
  // (K steps for 64 / lanes rows: 21846 rows of 285 values, K = 171, took 197 us, and 125 by top_kernel)
#define SHORT(lanes)                                                                                          \
  if (chunks <= lanes && (c.top.K * lanes <= kShortSteps || r.V < X::kPer)) {                                  \
    short_kernel<X, kEntropy, lanes>                                                                          \
        <<<std::min(groups_of(rows, kTopThreads / lanes), kLaneGroups), kTopThreads, 0, c.stream>>>(r, c.out, c.top); \
    return hipGetLastError();                                                                                 \
  }
  SHORT(2) SHORT(4) SHORT(8) SHORT(16) SHORT(32) SHORT(64)
#undef SHORT
  // the longest part
  const int64_t most = r.V / c.split.parts + (c.split.parts > 1 ? 64 : 0);
  const int whole = int(most / X::kPer);
  Split split = c.split;
  split.tiles = 1;
  auto go = [&](auto kernel, int threads) {
    const int teams = threads <= kWave ? kTopThreads / threads : 1, waves = std::max(threads, kTopThreads * (teams > 1)) / kWave;
    // (not multiples of 32 keys: the parts begin at other banks)
    const Room room = c.top.K <= 128 ? Room{192, 258} : teams == 1 && c.top.K < 256 ? Room{192, 258} : Room{256, kMostKeys};
    static_assert(4 * kMostKeys > TB_TOP_MOST);
    const size_t bytes = size_t(waves) * (room.keys * sizeof(uint64_t) + room.hits * kHitBytes);
    if (bytes > kPlainLds) {
      const hipError_t e = grant_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes);
      if (e != hipSuccess) return e;
    }
    const int64_t units = teams > 1 ? 1 : rows * split.parts;
    for (split.first = 0; split.first < units; split.first += kMostGroups)  // (a workgroup for each)
      kernel<<<groups_of(teams > 1 ? rows : units - split.first, teams), waves * kWave, bytes, c.stream>>>(r, c.out, c.top, split,
                                                                                                         room);
    return hipGetLastError();
  };
  auto need = [&](int threads) { return (whole + threads - 1) / threads; };
#define HELD(threads, n, step) \
  if (need(threads) <= n) return go(top_kernel<X, kEntropy, threads, n, step>, threads);
  if (c.split.parts == 1) {
    // Rows of a wavefront: where the lanes' groups of chunks are less than twice the alternatives, so that what K of
    // their largest reach lets most values through, the bound is that of the values themselves.
    const int groups = std::min(whole, 4 * kWave);
    split.by_values = 2 * c.top.K > groups;
    if (c.top.K <= 128 || (c.top.K <= 256 && whole <= 4 * kWave)) { HELD(64, 2, 2) HELD(64, 4, 2) HELD(64, 6, 2) HELD(64, 8, 2) }
    HELD(256, 4, 2) HELD(256, 6, 2) HELD(256, 8, 2)
    // (one row of 50257 values takes 8.5 us by 512 threads and 9.6 by 256; 16384 rows 267 us and 223)
    if (c.top.K < 512 && rows >= kManyRows) {
      HELD(256, 10, 2) HELD(256, 12, 2) HELD(256, 14, 2) HELD(256, 16, 2) HELD(256, 18, 2) HELD(256, 20, 2) HELD(256, 22, 2)
      HELD(256, 24, 2) HELD(256, 26, 2)
    }
  }
  if (c.top.K >= 512 || rows < kManyRows) {
    HELD(512, 6, 4) HELD(512, 8, 2) HELD(512, 10, 2) HELD(512, 12, 2) HELD(512, 14, 2) HELD(512, 16, 2)
  }
#undef HELD
  // tiles that differ by up to 64 values
  constexpr int kTileThreads = 256, kTile = 24;  // (as many chunks as leave registers for three workgroups a unit)
  split.tiles = (whole + kTile * kTileThreads - 1) / (kTile * kTileThreads);
  auto chunks_of = [&] { return (whole / split.tiles + 64 / X::kPer + 2 + kTileThreads - 1) / kTileThreads; };  // the longest's
  if (chunks_of() > kTile) ++split.tiles;
  const int each = chunks_of();
#define TILED(n) \
  if (each <= n) return go(top_kernel<X, kEntropy, kTileThreads, n, 2, true>, kTileThreads);
  TILED(14) TILED(16) TILED(18) TILED(20) TILED(22) TILED(kTile)
#undef TILED
  return hipErrorInvalidValue;  // (not reached)
}

template <typename X, bool kEntropy>
hipError_t launch_top_gradient(const TopCall& c) {
  const Rows& r = c.rows;
  const int64_t rows = int64_t(r.B) * r.T;
  const int chunks = (r.V + X::kPer - 1) / X::kPer;
  auto go = [&](auto kernel, int threads) {
    const int teams = threads <= kWave ? kTopThreads / threads : 1;
    const int64_t groups = (rows + teams - 1) / teams;
    kernel<<<int(groups < kMostGroups ? groups : kMostGroups), threads * teams, 0, c.stream>>>(r, c.top, c.given);
    return hipGetLastError();
  };
  if (chunks <= 32) return go(top_gradient_kernel<X, kEntropy, 8>, 8);
  if (chunks <= 512) return go(top_gradient_kernel<X, kEntropy, 64>, 64);
  if (chunks <= 2048) return go(top_gradient_kernel<X, kEntropy, 256>, 256);
  return go(top_gradient_kernel<X, kEntropy, 512>, 512);
}

}  // namespace

template <typename X>
hipError_t top_of(const TopCall& c) {
  hipError_t e = c.entropy ? launch_top<X, true>(c) : launch_top<X, false>(c);
  if (e != hipSuccess || c.split.parts == 1) return e;
  const int64_t rows = int64_t(c.rows.B) * c.rows.T;
  const int groups = int(rows < kMostGroups ? rows : kMostGroups);
  if (c.entropy) join_kernel<X, true><<<groups, kTopThreads, 0, c.stream>>>(c.rows, c.out, c.top, c.split);
  else join_kernel<X, false><<<groups, kTopThreads, 0, c.stream>>>(c.rows, c.out, c.top, c.split);
  return hipGetLastError();
}
template <typename X>
hipError_t top_gradient_of(const TopCall& c) {
  return c.entropy ? launch_top_gradient<X, true>(c) : launch_top_gradient<X, false>(c);
}

}  // namespace loss
}  // namespace tb
