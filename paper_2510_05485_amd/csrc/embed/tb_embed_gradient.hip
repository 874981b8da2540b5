// The gradient of a lookup in its table: positions are sorted by their tokens, in the order of the positions
// where tokens are equal, and each token's rows are added up.
//
//   part kernels    (many positions) positions by some bits of their tokens: counts, their sums, entries
//   sort_kernel     a workgroup for each value of these bits picks its positions out of all (or out of its part),
//                   sorts them, and fills the rows of tokens that do not come up with zeros: most of what is
//                   written in many vocabularies
//   sum_kernel      equal slices of the sorted positions, whatever tokens they hold; a token inside a slice is done
//   join_kernel     tokens that go over the end of a slice
#include "tb_embed.h"

namespace tb {
namespace embed {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int64_t kMostGroups = 1 << 22;
constexpr int kListed = 512;  // positions that a wavefront keeps between its two passes

// ---- tokens -----------------------------------------------------------------------------------

// The token of a position, or -1 for one that does not count or is outside the table (told by the threads with `tell`).
__device__ __forceinline__ int token_of(const Rows& r, uint32_t n, bool tell) {
  const At pos = loss::position(r, n);
  if (tell && pos.t == 0 && r.lengths) loss::held_length(r.lengths[pos.b], r.T, r.status);
  if (!loss::counts(r, pos.b, pos.t)) return -1;
  const int64_t id = loss::load_id(r.tokens, r.long_tokens, pos.b * r.token_seq + pos.t);
  if (id >= 0 && id < r.V) return int(id);
  if (tell && r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
  return -1;
}
__device__ __forceinline__ int digit_of(const Buckets& by, int token) { return (token >> by.low) & ((1 << by.bits) - 1); }
// a token's row among those of its bucket, and back
__device__ __forceinline__ int row_in(const Buckets& by, int token) {
  return (token >> (by.low + by.bits)) << by.low | (token & ((1 << by.low) - 1));
}
__device__ __forceinline__ int64_t token_in(const Buckets& by, int digit, int row) {
  return (int64_t(row >> by.low) << by.bits | digit) << by.low | (row & ((1 << by.low) - 1));
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// Sum of the values of the threads before, and of all (part: one a wavefront).
__device__ __forceinline__ int block_scan(int v, int* part, int* all) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int sum = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int u = __shfl_up(sum, d);
    if (lane >= d) sum += u;
  }
  __syncthreads();
  if (lane == kWave - 1) part[wave] = sum;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  *all = total;
  return before + sum - v;
}

// ---- parts of many positions ------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void part_count_kernel(Gradient c) {
  extern __shared__ int count[];
  const int digits = 1 << c.by.bits;
  for (int d = threadIdx.x; d < digits; d += kThreads) count[d] = 0;
  __syncthreads();
  const int64_t rows = int64_t(c.r.B) * c.r.T, from = int64_t(blockIdx.x) * c.block, to = min(from + c.block, rows);
  for (int64_t n = from + threadIdx.x; n < to; n += kThreads) {
    const int token = token_of(c.r, uint32_t(n), true);
    if (token >= 0) atomicAdd(&count[digit_of(c.by, token)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kThreads) c.counts[int64_t(d) * c.blocks + blockIdx.x] = count[d];
}

// A workgroup a digit: where each block's positions begin among those of the digit, and how many these are.
__global__ __launch_bounds__(kThreads) void part_sums_kernel(Gradient c) {
  __shared__ int part[kWaves];
  int32_t* counts = c.counts + int64_t(blockIdx.x) * c.blocks;
  int before = 0;
  for (int from = 0; from < c.blocks; from += kThreads) {
    const int i = from + threadIdx.x;
    int all;
    const int mine = i < c.blocks ? counts[i] : 0, at = block_scan(mine, part, &all);
    if (i < c.blocks) counts[i] = before + at;
    before += all;
  }
  if (threadIdx.x == 0) c.totals[blockIdx.x] = before;
}

// Where the digits' positions begin, in `begin` [digits + 1]: sums of the totals.
__device__ __forceinline__ void digit_begins(const Gradient& c, int* begin, int* part) {
  const int digits = 1 << c.by.bits;
  int before = 0;
  for (int from = 0; from < digits; from += kThreads) {
    const int i = from + threadIdx.x;
    int all;
    const int at = block_scan(i < digits ? c.totals[i] : 0, part, &all);
    if (i < digits) begin[i] = before + at;
    before += all;
  }
  if (threadIdx.x == 0) begin[digits] = before;
  __syncthreads();
}

// Entries to their digits, in the order of the positions: every wavefront has a run of the block's positions, whose
// digits it counts first.  Lanes with equal digits find one another by the digits' bits.
__global__ __launch_bounds__(kThreads) void part_kernel(Gradient c) {
  extern __shared__ int next[];  // [wave][digit], and the digits' beginnings
  __shared__ int part[kWaves];
  const int digits = 1 << c.by.bits, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int* begin = next + kWaves * digits;
  for (int d = threadIdx.x; d < kWaves * digits; d += kThreads) next[d] = 0;
  digit_begins(c, begin, part);
  const int64_t rows = int64_t(c.r.B) * c.r.T, first = int64_t(blockIdx.x) * c.block, end = min(first + c.block, rows);
  const int run = c.block / kWaves;
  const int64_t from = first + int64_t(wave) * run, to = min(from + run, end);
  for (int64_t n = from + lane; n < to; n += kWave) {
    const int token = token_of(c.r, uint32_t(n), false);
    if (token >= 0) atomicAdd(&next[wave * digits + digit_of(c.by, token)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kThreads) {
    int at = begin[d] + c.counts[int64_t(d) * c.blocks + blockIdx.x];
    for (int w = 0; w < kWaves; ++w) {
      const int n = next[w * digits + d];
      next[w * digits + d] = at;
      at += n;
    }
  }
  __syncthreads();
  int* mine = next + wave * digits;
  for (int64_t i = from; i < to; i += kWave) {
    const int64_t n = i + lane;
    const int token = n < to ? token_of(c.r, uint32_t(n), false) : -1, digit = digit_of(c.by, token);
    uint64_t same = __ballot(token >= 0);
    for (int b = 0; b < c.by.bits; ++b) {
      const bool set = digit >> b & 1;
      const uint64_t with = __ballot(set);
      same &= set ? with : ~with;
    }
    int at = 0;
    if (token >= 0) at = mine[digit];
    wave_fence();
    const int before = lanes_before(same);
    if (token >= 0 && before == 0) mine[digit] = at + __popcll(same);
    wave_fence();
    if (token >= 0) c.parted[at + before] = {uint32_t(token), uint32_t(n)};
  }
}

// ---- sorted positions -------------------------------------------------------------------------

// Zeros for a row of D values, by `lanes` threads.
template <typename X>
__device__ __forceinline__ void write_zeros(typename X::type* row, int D, int lane, int lanes) {
  if (D < X::kPer) {
    for (int i = lane; i < D; i += lanes) X::store(row + i, 0.f);
    return;
  }
  for (int i = lane * X::kPer; i < D; i += lanes * X::kPer)
    *reinterpret_cast<u32x4_any*>(row + min(i, D - X::kPer)) = u32x4{};
}

// Workgroup d: the positions whose token has the digit d.  Two passes over the positions (each wavefront has a run of
// them), or over a list of those that were found: how many of each token each wavefront has, then each one's place.
// kParted: the positions are those of the digit's part.
template <typename X, bool kParted>
__global__ __launch_bounds__(kThreads) void sort_kernel(Gradient c) {
  extern __shared__ int next[];  // [wave][row]: how many, then where the next one goes
  __shared__ Entry listed[kWaves][kListed];
  __shared__ int part[kWaves];
  const int digit = blockIdx.x, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, buckets = c.by.rows;
  for (int i = threadIdx.x; i < kWaves * buckets; i += kThreads) next[i] = 0;
  int64_t first = 0, end = int64_t(c.r.B) * c.r.T;
  if constexpr (kParted) {
    int before = 0, mine = 0, all;
    for (int d = threadIdx.x; d < (1 << c.by.bits); d += kThreads) {
      const int n = c.totals[d];
      if (d < digit) before += n;
      if (d == digit) mine = n;
    }
    block_scan(before, part, &all);
    first = all;
    block_scan(mine, part, &all);
    end = first + all;
  }
  __syncthreads();
  const int64_t run = ((end - first + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int64_t from = min(first + wave * run, end), to = min(from + run, end);
  int below = 0, seen = 0;
  // entry(i): the token at place i, or -1, and its position
  auto entry = [&](int64_t i, uint32_t* position, bool tell) {
    if constexpr (kParted) {
      const Entry e = c.parted[i];
      *position = e.position;
      return int(e.token);
    } else {
      *position = uint32_t(i);
      return token_of(c.r, uint32_t(i), tell);
    }
  };
  constexpr int kAhead = 4;
  for (int64_t i = from; i < to; i += kAhead * kWave) {
    int token[kAhead];
    uint32_t position[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t n = i + a * kWave + lane;
      token[a] = n < to ? entry(n, &position[a], digit == 0) : -1;
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int d = digit_of(c.by, token[a]);
      const bool mine = token[a] >= 0 && d == digit;
      if (!kParted) below += token[a] >= 0 && d < digit;
      const uint64_t mask = __ballot(mine);
      if (mask == 0) continue;
      if (mine) {
        atomicAdd(&next[wave * buckets + row_in(c.by, token[a])], 1);
        const int slot = seen + lanes_before(mask);
        if (slot < kListed) listed[wave][slot] = {uint32_t(token[a]), position[a]};
      }
      seen += __popcll(mask);
    }
  }
  if constexpr (!kParted) {
    int all;
    block_scan(below, part, &all);
    first = all;
  }
  __syncthreads();
  // where each row's and wavefront's positions begin; rows without any
  int64_t before = first;
  for (int i = 0; i < buckets; i += kThreads) {
    const int row = i + threadIdx.x;
    int mine = 0, all;
    if (row < buckets)
      for (int w = 0; w < kWaves; ++w) mine += next[w * buckets + row];
    int at = int(before) + block_scan(mine, part, &all);
    before += all;
    if (row < buckets) {
      for (int w = 0; w < kWaves; ++w) {
        const int n = next[w * buckets + row];
        // (a row without positions is marked for the zeros below)
        next[w * buckets + row] = mine ? at : -1;
        at += n;
      }
    }
  }
  if (digit == (1 << c.by.bits) - 1 && threadIdx.x == 0) *c.valid = int(before);
  __syncthreads();
  if (!c.accumulate) {
    const int chunks = (c.D + X::kPer - 1) / X::kPer;
    int lanes = kThreads;
    while (lanes > 1 && lanes / 2 >= chunks) lanes /= 2;
    typename X::type* out = static_cast<typename X::type*>(c.r.g);
    for (int row = threadIdx.x / lanes; row < buckets; row += kThreads / lanes) {
      if (next[row] >= 0) continue;
      const int64_t token = token_in(c.by, digit, row);
      if (token < c.r.V) write_zeros<X>(out + token * c.r.g_pos, c.D, threadIdx.x % lanes, lanes);
    }
  }
  __syncthreads();
  // lanes with the token of the first of them, then those of the next
  int* mine = next + wave * buckets;
  auto place = [&](int token, uint32_t position) {
    const int row = token >= 0 ? row_in(c.by, token) : -1;
    uint64_t left = __ballot(token >= 0);
    while (left) {
      const int r0 = __builtin_amdgcn_readlane(row, __ffsll(static_cast<unsigned long long>(left)) - 1);
      const uint64_t same = __ballot(row == r0);
      const int at = mine[r0];
      wave_fence();
      if (row == r0) {
        const int k = lanes_before(same);
        c.sorted[at + k] = {uint32_t(token), position};
        if (k == 0) mine[r0] = at + __popcll(same);
      }
      wave_fence();
      left &= ~same;
    }
  };
  if (seen <= kListed) {
    for (int i = 0; i < seen; i += kWave) {
      const Entry e = i + lane < seen ? listed[wave][i + lane] : Entry{~0u, 0};
      place(int(e.token), e.position);
    }
    return;
  }
  for (int64_t i = from; i < to; i += kWave) {
    uint32_t position = 0;
    const int token = i + lane < to ? entry(i + lane, &position, false) : -1;
    place(token >= 0 && digit_of(c.by, token) == digit ? token : -1, position);
  }
}

// ---- sums -------------------------------------------------------------------------------------

// The columns of a team's lane: a chunk of kPer values, or one value each of rows without a whole chunk.  The last chunk
// of a row ends with it, and holds values of the one before, which are written by that one.
template <typename X, bool kWide>
struct Columns {
  static constexpr int kPer = kWide ? X::kPer : 1;
  int first, skip;  // columns from `first` on; `skip` of them are another chunk's
  bool any;
  __device__ __forceinline__ Columns(int chunk, int D) {
    first = chunk * kPer;
    any = first < D;
    skip = any && kWide ? max(first - (D - kPer), 0) : 0;
    first -= skip;
  }
  static __device__ __forceinline__ u32x4 load(const typename X::type* at) {
    if constexpr (kWide) return *reinterpret_cast<const u32x4_any*>(at);
    u32x4 u = {};
    u[0] = __float_as_uint(X::load(at));
    return u;
  }
  static __device__ __forceinline__ void add(u32x4 u, float* sum) {
    if constexpr (kWide) {
      float v[X::kPer];
      X::unpack(u, v);
#pragma unroll
      for (int i = 0; i < X::kPer; ++i) sum[i] += v[i];
    } else {
      sum[0] += __uint_as_float(u[0]);
    }
  }
};

// A final sum of a lane's columns, scaled (and added to what is there), rounded once.
template <typename X, typename Out, bool kWide>
__device__ __forceinline__ void put_row(const Gradient& c, int64_t token, const Columns<X, kWide>& at, const float* sum) {
  constexpr int kPer = Columns<X, kWide>::kPer;
  typename Out::type* to = static_cast<typename Out::type*>(c.r.g) + token * c.r.g_pos + at.first;
  if (kWide && at.skip == 0) {
    float v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = sum[i] * c.scale;
#pragma unroll
    for (int i = 0; i < kPer; i += Out::kPer) {
      u32x4_any* p = reinterpret_cast<u32x4_any*>(to + i);
      if (c.accumulate) {
        float old[Out::kPer];
        Out::unpack(*p, old);
#pragma unroll
        for (int j = 0; j < Out::kPer; ++j) v[i + j] += old[j];
      }
      *p = Out::pack(v + i);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i < at.skip) continue;
    float v = sum[i] * c.scale;
    if (c.accumulate) v += Out::load(to + i);
    Out::store(to + i, v);
  }
}

template <int kPer>
__device__ __forceinline__ void store_partial(float* to, const float* sum) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = sum[i];
}

// kLanes lanes a slice and kLanes chunks of columns (a tile).
template <typename X, typename Out, int kLanes, bool kWide>
__global__ __launch_bounds__(kThreads) void sum_kernel(Gradient c, int tiles) {
  using C = Columns<X, kWide>;
  constexpr int kTeams = kThreads / kLanes, kAhead = 8, kPer = C::kPer;
  const int lane = threadIdx.x % kLanes;
  const int64_t valid = *c.valid, units = c.slices * tiles;
  for (int64_t unit = int64_t(blockIdx.x) * kTeams + threadIdx.x / kLanes; unit < units; unit += int64_t(gridDim.x) * kTeams) {
    const int64_t slice = unit / tiles, from = slice * c.slice, to = min(from + c.slice, valid);
    if (from >= to) continue;
    const C at(int(unit - slice * tiles) * kLanes + lane, c.D);
    const bool before = from > 0 && c.sorted[from - 1].token == c.sorted[from].token;
    const bool behind = to < valid && c.sorted[to].token == c.sorted[to - 1].token;
    float sum[kPer] = {};
    uint32_t token = c.sorted[from].token;
    bool head = before;
    auto done = [&](bool tail) {
      if (!at.any) return;
      if (head || tail) store_partial<kPer>(c.partial + (slice * 2 + !head) * c.D + at.first, sum);
      else put_row<X, Out, kWide>(c, token, at, sum);
    };
    for (int64_t i = from; i < to; i += kAhead) {
      Entry e[kAhead];
      u32x4 u[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) e[a] = c.sorted[min(i + a, to - 1)];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const At pos = loss::position(c.r, e[a].position);
        u[a] = at.any && i + a < to ? C::load(loss::row_of<X>(c.r, pos.b, pos.t) + at.first) : u32x4{};
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (i + a >= to) break;
        if (e[a].token != token) {
          done(false);
          head = false;
          token = e[a].token;
#pragma unroll
          for (int j = 0; j < kPer; ++j) sum[j] = 0.f;
        }
        C::add(u[a], sum);
      }
    }
    done(behind);
  }
}

// Tokens that go over the end of a slice: the workgroup takes some slices in which such a token begins, one after
// the other; its teams add up the slices' partial sums, a run of them each, and the first team what the teams have.
template <typename X, typename Out, int kLanes, bool kWide>
__global__ __launch_bounds__(kThreads) void join_kernel(Gradient c, int tiles) {
  using C = Columns<X, kWide>;
  constexpr int kTeams = kThreads / kLanes, kPer = C::kPer, kAhead = 4;
  __shared__ float sums[kTeams][kLanes * kPer];
  const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
  const int64_t valid = *c.valid, slices = (valid + c.slice - 1) / c.slice;
  const int64_t units = slices * tiles;
  auto token_at = [&](int64_t i) { return c.sorted[i].token; };
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t slice = unit / tiles, from = slice * c.slice, to = from + c.slice;
    if (to >= valid) continue;
    const uint32_t token = token_at(to - 1);
    if (token_at(to) != token) continue;
    if (token_at(from) == token && from > 0 && token_at(from - 1) == token) continue;  // (it begins before)
    // the slices that it goes on through: the last one whose first entry it has
    int64_t last = slice + 1;
    for (;;) {
      const int64_t i = last + 1 + threadIdx.x % kWave;
      const uint64_t with = __ballot(i < slices && token_at(i * c.slice) == token);
      const int n = with == ~uint64_t(0) ? kWave : __ffsll(static_cast<unsigned long long>(~with)) - 1;
      last += n;
      if (n < kWave) break;
    }
    const C at(int(unit - slice * tiles) * kLanes + lane, c.D);
    float sum[kPer] = {};
    if (at.any) {
      const int64_t many = last - slice + 1, run = (many + kTeams - 1) / kTeams;
      const int64_t lo = slice + team * run, hi = min(lo + run, last + 1);
      for (int64_t s = lo; s < hi; s += kAhead) {
        float v[kAhead][kPer];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          const int64_t i = min(s + a, hi - 1);
          const float* p = c.partial + (i * 2 + (i == slice)) * c.D + at.first;
#pragma unroll
          for (int j = 0; j < kPer; ++j) v[a][j] = p[j];
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
          if (s + a < hi) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) sum[j] += v[a][j];
          }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) sums[team][lane * kPer + j] = sum[j];
    __syncthreads();
    if (team == 0 && at.any) {
      for (int w = 1; w < kTeams; ++w)
#pragma unroll
        for (int j = 0; j < kPer; ++j) sum[j] += sums[w][lane * kPer + j];
      put_row<X, Out, kWide>(c, token, at, sum);
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------

template <typename X, typename Out, int kLanes, bool kWide>
hipError_t launch_sums(const Gradient& c) {
  constexpr int kPer = Columns<X, kWide>::kPer, kTeams = kThreads / kLanes;
  const int chunks = (c.D + kPer - 1) / kPer, tiles = (chunks + kLanes - 1) / kLanes;
  const int64_t groups = (c.slices * tiles + kTeams - 1) / kTeams;
  sum_kernel<X, Out, kLanes, kWide><<<int(groups < kMostGroups ? groups : kMostGroups), kThreads, 0, c.stream>>>(c, tiles);
  if (c.slices > 1) {
    const int64_t joins = c.slices * tiles < 2048 ? c.slices * tiles : 2048;
    join_kernel<X, Out, kLanes, kWide><<<int(joins), kThreads, 0, c.stream>>>(c, tiles);
  }
  return hipGetLastError();
}

template <typename X, typename Out>
hipError_t launch(const Gradient& c) {
  const int digits = 1 << c.by.bits;
  const size_t next = size_t(kWaves) * c.by.rows * sizeof(int);
  if (c.parted) {
    const size_t lds = size_t(digits) * sizeof(int);
    part_count_kernel<<<c.blocks, kThreads, lds, c.stream>>>(c);
    part_sums_kernel<<<digits, kThreads, 0, c.stream>>>(c);
    part_kernel<<<c.blocks, kThreads, (kWaves + 1) * lds + sizeof(int), c.stream>>>(c);
    sort_kernel<Out, true><<<digits, kThreads, next, c.stream>>>(c);
  } else {
    sort_kernel<Out, false><<<digits, kThreads, next, c.stream>>>(c);
  }
  if (const hipError_t e = hipGetLastError()) return e;
  if (c.slices == 0) return hipSuccess;  // (no positions: zeros are all)
  const int chunks = (c.D + X::kPer - 1) / X::kPer;
  if (c.D < X::kPer) return launch_sums<X, Out, 8, false>(c);
  if (chunks <= 2) return launch_sums<X, Out, 2, true>(c);
  if (chunks <= 8) return launch_sums<X, Out, 8, true>(c);
  if (chunks <= 32) return launch_sums<X, Out, 32, true>(c);
  return launch_sums<X, Out, 64, true>(c);
}

}  // namespace

hipError_t run_gradient(const Gradient& c) {
  switch (c.type) {
    case TB_FLOAT32: return launch<F32, F32>(c);
    case TB_BFLOAT16: return c.out_type == TB_FLOAT32 ? launch<BF16, F32>(c) : launch<BF16, BF16>(c);
    default: return c.out_type == TB_FLOAT32 ? launch<F16, F32>(c) : launch<F16, F16>(c);
  }
}

}  // namespace embed
}  // namespace tb
