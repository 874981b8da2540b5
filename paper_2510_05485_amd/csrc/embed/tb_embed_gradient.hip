// The gradient of a lookup in its table: positions are sorted by their tokens, in the order of the positions
// where tokens are equal, and each token's rows are added up.  No atomic adds to values: the order of a sum is that of the
// positions, cut into slices.
//
//   ready_kernel    the tokens of all positions as the sort reads them (beyond 1024 positions: every workgroup of the sort
//                   reads them all, and working them out each time took 30 of 74 us at 32768 positions)
//   part kernels    (beyond 65536 positions) positions by some bits of their tokens: counts, their sums, entries
//   sort_kernel     a workgroup for each value of these bits picks its positions out of all (or out of its part),
//                   sorts them, and fills the rows of tokens that do not come up with zeros: most of what is
//                   written in many vocabularies
//   sum_kernel      equal slices of the sorted positions, whatever tokens they hold: a token that half of the positions
//                   have is no slower than many.  A token inside a slice is done
//   join_kernel     tokens that go over the end of a slice
//
// Bound by HBM where there is much to move, else by four launches of 3 to 8 us.  On one MI355X, among other calls: 32 x
// 1024 positions (62 % of which count) of 50257 tokens distributed like words, D = 2048, bfloat16, 79 to 87 us for 290 MB: 5 to read
// the tokens, 37 to 42 for the sort (17 of them without its 175 MB of zeros), 32 for the sums, 8 for 500 joins.  2097152 positions of 64 tokens, D =
// 64: 72 us: 25 for the parts, 30 for the sums of 142 MB, 8 for the joins.  Two positions: 9 us.  Not fast:
// tokens that go over the end of a slice in narrow tables, a workgroup of 512 threads each (2097152 positions of 5 million
// rows, D = 16: 576 of 950 us).
#include "tb_embed.h"

namespace tb {
namespace embed {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostGroups = 1 << 22;

// ---- tokens -----------------------------------------------------------------------------------

// The tokens of kN positions, `step` apart from n on: -1 at places from `end` on, at positions that do not count, and
// for tokens outside the table (told by the threads with `tell`).  All requests are under way together, tokens of
// positions that do not count among them.
template <int kN>
__device__ __forceinline__ void tokens_of(const Rows& r, int64_t n, int step, int64_t end, bool tell, int* token) {
  int64_t id[kN];
  int length[kN], t[kN];
  uint8_t mask[kN];
#pragma unroll
  for (int a = 0; a < kN; ++a) {
    const int64_t at = min(n + a * step, end - 1);
    const At pos = loss::position(r, at);
    t[a] = pos.t;
    id[a] = loss::load_id(r.tokens, r.long_tokens, pos.b * r.token_seq + pos.t);
    length[a] = r.lengths ? r.lengths[pos.b] : r.T;
    mask[a] = r.mask ? r.mask[at] : 1;
  }
#pragma unroll
  for (int a = 0; a < kN; ++a) {
    const bool there = n + a * step < end, live = there && t[a] < length[a] && mask[a] != 0;
    const bool fits = id[a] >= 0 && id[a] < r.V;
    if (tell && there && t[a] == 0 && r.lengths) loss::held_length(length[a], r.T, r.status);
    if (tell && live && !fits && r.status) atomicOr(r.status, TB_DEV_TOKEN_RANGE);
    token[a] = live && fits ? int(id[a]) : -1;
  }
}
__device__ __forceinline__ int digit_of(const Buckets& by, int token) { return (token >> by.low) & ((1 << by.bits) - 1); }
// a token's row among those of its bucket, and back
__device__ __forceinline__ int row_in(const Buckets& by, int token) {
  return (token >> (by.low + by.bits)) << by.low | (token & ((1 << by.low) - 1));
}
__device__ __forceinline__ int64_t token_in(const Buckets& by, int digit, int row) {
  return (int64_t(row >> by.low) << by.bits | digit) << by.low | (row & ((1 << by.low) - 1));
}
// how many workgroups share a digit
__host__ __device__ inline int ranges_of(const Buckets& by) { return (by.rows + by.held - 1) / by.held; }
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// Sum of the values of the threads before, and of all (part: one a wavefront).
template <int kThreads>
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
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  *all = total;
  return before + sum - v;
}

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

// The tokens of all positions, -1 for none: what every workgroup of the sort reads.
constexpr int kReadyPer = 4;  // positions of a thread
__global__ __launch_bounds__(kThreads) void ready_kernel(Gradient c) {
  const int64_t rows = int64_t(c.r.B) * c.r.T, from = int64_t(blockIdx.x) * (kReadyPer * kThreads) + threadIdx.x;
  int token[kReadyPer];
  tokens_of<kReadyPer>(c.r, from, kThreads, rows, true, token);
#pragma unroll
  for (int a = 0; a < kReadyPer; ++a)
    if (from + a * kThreads < rows) c.tokens[from + a * kThreads] = token[a];
}

// ---- parts of many positions ------------------------------------------------------------------

constexpr int kHeld = kPartBlock / kThreads;  // positions of a thread

__global__ __launch_bounds__(kThreads) void part_count_kernel(Gradient c) {
  extern __shared__ int count[];
  const int digits = 1 << c.by.bits;
  const int64_t from = int64_t(blockIdx.x) * kPartBlock, rows = int64_t(c.r.B) * c.r.T;
  int token[kHeld];
  tokens_of<kHeld>(c.r, from + threadIdx.x, kThreads, rows, true, token);
#pragma unroll
  for (int a = 0; a < kHeld; ++a)
    if (from + threadIdx.x + a * kThreads < rows) c.tokens[from + threadIdx.x + a * kThreads] = token[a];
  for (int d = threadIdx.x; d < digits; d += kThreads) count[d] = 0;
  __syncthreads();
#pragma unroll
  for (int a = 0; a < kHeld; ++a)
    if (token[a] >= 0) atomicAdd(&count[digit_of(c.by, token[a])], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kThreads) c.counts[int64_t(d) * c.blocks + blockIdx.x] = count[d];
}

// A workgroup a digit: where each block's positions begin among those of the digit, and how many these are.  Where a
// digit is a token, one without positions has a row of zeros.
template <typename Out>
__global__ __launch_bounds__(kThreads) void part_sums_kernel(Gradient c) {
  __shared__ int part[kThreads / kWave];
  int32_t* counts = c.counts + int64_t(blockIdx.x) * c.blocks;
  int before = 0;
  for (int from = 0; from < c.blocks; from += kThreads) {
    const int i = from + threadIdx.x;
    int all;
    const int mine = i < c.blocks ? counts[i] : 0, at = block_scan<kThreads>(mine, part, &all);
    if (i < c.blocks) counts[i] = before + at;
    before += all;
  }
  if (threadIdx.x == 0) c.totals[blockIdx.x] = before;
  if (threadIdx.x == 0 && blockIdx.x == 0) *c.joins = 0;
  if (c.by.rows == 1 && before == 0 && !c.accumulate && int(blockIdx.x) < c.r.V)
    write_zeros<Out>(static_cast<typename Out::type*>(c.r.g) + blockIdx.x * c.r.g_pos, c.D, threadIdx.x, kThreads);
}

// Entries to their digits, in the order of the positions: every wavefront has a run of the block's positions, whose
// digits it counts first.  Lanes with equal digits find one another by the digits' bits.
__global__ __launch_bounds__(kThreads) void part_kernel(Gradient c, Entry* to) {
  constexpr int kWaves = kThreads / kWave;
  extern __shared__ int next[];  // [wave][digit], and the digits' beginnings
  __shared__ int part[kWaves];
  const int digits = 1 << c.by.bits, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int* begin = next + kWaves * digits;
  const int64_t from = int64_t(blockIdx.x) * kPartBlock + wave * (kPartBlock / kWaves) + lane, rows = int64_t(c.r.B) * c.r.T;
  int token[kHeld];
#pragma unroll
  for (int a = 0; a < kHeld; ++a) {
    const int t = c.tokens[min(from + a * kWave, rows - 1)];
    token[a] = from + a * kWave < rows ? t : -1;
  }
  for (int d = threadIdx.x; d < kWaves * digits; d += kThreads) next[d] = 0;
  int before = 0;  // (the digits' beginnings: sums of their totals)
  for (int i = 0; i < digits; i += kThreads) {
    const int d = i + threadIdx.x;
    int all;
    const int at = block_scan<kThreads>(d < digits ? c.totals[d] : 0, part, &all);
    if (d < digits) begin[d] = before + at;
    before += all;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *c.valid = before;
  __syncthreads();
  int* mine = next + wave * digits;
#pragma unroll
  for (int a = 0; a < kHeld; ++a)
    if (token[a] >= 0) atomicAdd(&mine[digit_of(c.by, token[a])], 1);
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
#pragma unroll
  for (int a = 0; a < kHeld; ++a) {
    const int digit = digit_of(c.by, token[a]);
    uint64_t same = __ballot(token[a] >= 0);
    for (int b = 0; b < c.by.bits; ++b) {
      const bool set = digit >> b & 1;
      const uint64_t with = __ballot(set);
      same &= set ? with : ~with;
    }
    int at = 0;
    if (token[a] >= 0) at = mine[digit];
    wave_fence();
    const int k = lanes_before(same);
    if (token[a] >= 0 && k == 0) mine[digit] = at + __popcll(same);
    wave_fence();
    if (token[a] >= 0) to[at + k] = {uint32_t(token[a]), uint32_t(from + a * kWave)};
  }
}

// ---- sorted positions -------------------------------------------------------------------------

constexpr int kSortThreads = 512, kListed = 384;  // positions that a wavefront keeps between its two passes

// Workgroup d: the positions whose token has the digit d.  Two passes over the positions (each wavefront has a run of
// them), or over a list of those that were found: how many of each token each wavefront has, then each one's place.
// The positions are read from the caller's tensors (few of them), from what ready_kernel has left, or from the digit's
// part.  What it takes is the latency of its reads, sixteen of which are under way for each lane, and then the zeros.
// Of tables of more than two million rows (kRanges) a digit has more than the counters hold: each of its workgroups takes a
// range of its rows, and reads the digit's part.
enum From { kTokens, kReady, kPart, kRanges };
template <typename X, int kFrom>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(Gradient c) {
  constexpr bool kParted = kFrom == kPart || kFrom == kRanges;
  constexpr int kThreads = kSortThreads, kWaves = kThreads / kWave;
  extern __shared__ int next[];  // [wave][row]: how many, then where the next one goes
  __shared__ Entry listed[kWaves][kListed];
  __shared__ int part[kWaves];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  int digit = blockIdx.x, low_row = 0, buckets = c.by.rows;
  if constexpr (kFrom == kRanges) {
    const int ranges = ranges_of(c.by);
    digit = blockIdx.x / ranges;
    low_row = int(blockIdx.x - digit * ranges) * c.by.held;
    buckets = min(c.by.held, c.by.rows - low_row);
  }
  auto in_range = [&](int token) { return kFrom != kRanges || uint32_t(row_in(c.by, token) - low_row) < uint32_t(buckets); };
  for (int i = threadIdx.x; i < kWaves * buckets; i += kThreads) next[i] = 0;
  int64_t first = 0, end = int64_t(c.r.B) * c.r.T;
  if constexpr (kParted) {
    int before = 0, mine = 0, all;
    for (int d = threadIdx.x; d < (1 << c.by.bits); d += kThreads) {
      const int n = c.totals[d];
      if (d < digit) before += n;
      if (d == digit) mine = n;
    }
    block_scan<kThreads>(before, part, &all);
    first = all;
    block_scan<kThreads>(mine, part, &all);
    end = first + all;
  } else if (digit == 0 && threadIdx.x == 0) {
    *c.joins = 0;
  }
  __syncthreads();
  const int64_t run = ((end - first + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int64_t from = min(first + wave * run, end), to = min(from + run, end);
  int below = 0, seen = 0;
  // tokens at kN places from `i` on, and their positions; -1 for none
  auto entries = [&](int64_t i, auto count, int* token, uint32_t* position, bool tell) {
    constexpr int kN = decltype(count)::value;
    if constexpr (kParted) {
#pragma unroll
      for (int a = 0; a < kN; ++a) {
        const Entry e = c.parted[min(i + a * kWave, to - 1)];
        token[a] = i + a * kWave < to ? int(e.token) : -1;
        position[a] = e.position;
      }
    } else {
      if constexpr (kFrom == kTokens) tokens_of<kN>(c.r, i, kWave, to, tell, token);
#pragma unroll
      for (int a = 0; a < kN; ++a) {
        position[a] = uint32_t(i + a * kWave);
        if constexpr (kFrom == kReady) {
          const int t = c.tokens[min(i + a * kWave, to - 1)];
          token[a] = i + a * kWave < to ? t : -1;
        }
      }
    }
  };
  constexpr int kAhead = kFrom == kTokens ? 2 : 16;  // (kDirectMost positions are two for each lane)
  for (int64_t i = from; i < to; i += kAhead * kWave) {
    int token[kAhead];
    uint32_t position[kAhead];
    entries(i + lane, std::integral_constant<int, kAhead>(), token, position, kFrom == kTokens && digit == 0);
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int d = digit_of(c.by, token[a]);
      const bool mine = token[a] >= 0 && d == digit && in_range(token[a]);
      if (!kParted) below += token[a] >= 0 && d < digit;
      if (kFrom == kRanges) below += token[a] >= 0 && row_in(c.by, token[a]) < low_row;
      const uint64_t mask = __ballot(mine);
      if (mask == 0) continue;
      // (lanes with the first one's token are counted together: 64 additions to one place of LDS take as many turns, and
      // 200000 positions of one token took 494 us so)
      const int row = mine ? row_in(c.by, token[a]) - low_row : -1, leader = __ffsll(static_cast<unsigned long long>(mask)) - 1;
      const int row0 = __builtin_amdgcn_readlane(row, leader);
      const uint64_t alike = __ballot(row == row0);
      if (mine) {
        if (row != row0 || lane == leader) atomicAdd(&next[wave * buckets + row], row != row0 ? 1 : __popcll(alike));
        const int slot = seen + lanes_before(mask);
        if (slot < kListed) listed[wave][slot] = {uint32_t(token[a]), position[a]};
      }
      seen += __popcll(mask);
    }
  }
  if constexpr (kFrom != kPart) {
    int all;
    block_scan<kThreads>(below, part, &all);
    first = kParted ? first + all : all;
  }
  __syncthreads();
  // where each row's and wavefront's positions begin; rows without any
  int64_t before = first;
  for (int i = 0; i < buckets; i += kThreads) {
    const int row = i + threadIdx.x;
    int mine = 0, all;
    if (row < buckets)
      for (int w = 0; w < kWaves; ++w) mine += next[w * buckets + row];
    int at = int(before) + block_scan<kThreads>(mine, part, &all);
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
  if (!kParted && digit == (1 << c.by.bits) - 1 && threadIdx.x == 0) *c.valid = int(before);
  __syncthreads();
  if (!c.accumulate) {
    const int chunks = (c.D + X::kPer - 1) / X::kPer;
    int lanes = kThreads;
    while (lanes > 1 && lanes / 2 >= chunks) lanes /= 2;
    typename X::type* out = static_cast<typename X::type*>(c.r.g);
    for (int row = threadIdx.x / lanes; row < buckets; row += kThreads / lanes) {
      if (next[row] >= 0) continue;
      const int64_t token = token_in(c.by, digit, row + low_row);
      if (token < c.r.V) write_zeros<X>(out + token * c.r.g_pos, c.D, threadIdx.x % lanes, lanes);
    }
  }
  __syncthreads();
  // lanes with the token of the first of them, then those of the next
  int* mine = next + wave * buckets;
  auto place = [&](int token, uint32_t position) {
    const int row = token >= 0 ? row_in(c.by, token) - low_row : -1;
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
  constexpr int kAgain = 8;
  for (int64_t i = from; i < to; i += kAgain * kWave) {
    int token[kAgain];
    uint32_t position[kAgain];
    entries(i + lane, std::integral_constant<int, kAgain>(), token, position, false);
#pragma unroll 1
    for (int a = 0; a < kAgain; ++a) {
      int t = -1;
      uint32_t p = 0;
#pragma unroll
      for (int j = 0; j < kAgain; ++j)
        if (j == a) {
          t = token[j];
          p = position[j];
        }
      place(t >= 0 && digit_of(c.by, t) == digit && in_range(t) ? t : -1, p);
    }
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

// A lane's value among those of its team's lanes.
template <int kLanes>
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) {
  if constexpr (kLanes == kWave) return uint32_t(__builtin_amdgcn_readlane(int(v), lane));
  return uint32_t(__shfl(int(v), lane, kLanes));
}

// kLanes lanes a slice and kLanes chunks of columns (a tile).  Each lane reads an entry, of as many as there are lanes at
// a time, the next ones while the rows of these are on their way.
template <typename X, typename Out, int kLanes, bool kWide>
__global__ __launch_bounds__(kThreads) void sum_kernel(Gradient c, int tiles) {
  using C = Columns<X, kWide>;
  constexpr int kTeams = kThreads / kLanes, kAhead = kLanes < 8 ? kLanes : 8, kPer = C::kPer;
  const int lane = threadIdx.x % kLanes;
  const int64_t rows = int64_t(c.r.B) * c.r.T, units = c.slices * tiles;
  for (int64_t unit = int64_t(blockIdx.x) * kTeams + threadIdx.x / kLanes; unit < units; unit += int64_t(gridDim.x) * kTeams) {
    const int64_t slice = unit / tiles, from = slice * c.slice;
    const int tile = int(unit - slice * tiles);
    // (what lies behind the sorted positions is read, too, but not used: all of it is under way together)
    Entry e = c.sorted[min(from + lane, rows - 1)];
    const Entry previous = c.sorted[max(from - 1, int64_t(0))], following = c.sorted[min(from + c.slice, rows - 1)];
    const int64_t valid = *c.valid, to = min(from + c.slice, valid);
    if (from >= to) continue;
    const C at(tile * kLanes + lane, c.D);
    float sum[kPer] = {};
    uint32_t token = of_lane<kLanes>(e.token, 0);
    bool head = from > 0 && previous.token == token;
    auto done = [&](bool tail) {
      if (!at.any) return;
      if (head || tail) store_partial<kPer>(c.partial + (slice * 2 + !head) * c.D + at.first, sum);
      else put_row<X, Out, kWide>(c, token, at, sum);
    };
    for (int64_t group = from; group < to; group += kLanes) {
      const Entry now = e;
      e = c.sorted[min(group + kLanes + lane, rows - 1)];
      const int many = int(min(to - group, int64_t(kLanes)));
      for (int i = 0; i < many; i += kAhead) {
        u32x4 u[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          const At pos = loss::position(c.r, of_lane<kLanes>(now.position, min(i + a, many - 1)));
          u[a] = at.any ? C::load(loss::row_of<X>(c.r, pos.b, pos.t) + at.first) : u32x4{};
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          if (i + a >= many) break;
          const uint32_t next = of_lane<kLanes>(now.token, i + a);
          if (next != token) {
            done(false);
            head = false;
            token = next;
#pragma unroll
            for (int j = 0; j < kPer; ++j) sum[j] = 0.f;
          }
          C::add(u[a], sum);
        }
      }
    }
    const bool behind = to < valid && following.token == token;
    done(behind);
    // (in any order: each one is joined by itself)
    if (behind && !head && tile == 0 && lane == 0) c.join_from[atomicAdd(c.joins, 1)] = int32_t(slice);
  }
}

constexpr int kJoinThreads = 512;
// A token that goes over the end of a slice, and a tile of its columns: the workgroup's teams add up the slices'
// partial sums, a run of them each, and the first team what the teams have.
template <typename X, typename Out, int kLanes, bool kWide>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(Gradient c, int tiles) {
  using C = Columns<X, kWide>;
  constexpr int kTeams = kJoinThreads / kLanes, kPer = C::kPer, kAhead = 8;
  __shared__ float sums[kTeams][kLanes * kPer];
  const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
  const int64_t valid = *c.valid, slices = (valid + c.slice - 1) / c.slice;
  const int64_t units = int64_t(*c.joins) * tiles;
  auto token_at = [&](int64_t i) { return c.sorted[i].token; };
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t entry = unit / tiles, slice = c.join_from[entry];
    const uint32_t token = token_at((slice + 1) * c.slice);
    // the last slice that it goes on through, whose first entry it has: one by one, and in steps of 64 where it has
    // all that a wavefront looks at
    int64_t last = slice + 1;
    auto steps = [&](int step) {
      const int64_t i = last + int64_t(step) * (1 + threadIdx.x % kWave);
      const uint64_t with = __ballot(i < slices && token_at(i * c.slice) == token);
      const int n = with == ~uint64_t(0) ? kWave : __ffsll(static_cast<unsigned long long>(~with)) - 1;
      last += int64_t(n) * step;
      return n == kWave;
    };
    if (steps(1)) {
      while (steps(kWave)) {
      }
      steps(1);
    }
    const C at(int(unit - entry * tiles) * kLanes + lane, c.D);
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
    const int64_t joins = c.slices * tiles < 1024 ? c.slices * tiles : 1024;
    join_kernel<X, Out, kLanes, kWide><<<int(joins), kJoinThreads, 0, c.stream>>>(c, tiles);
  }
  return hipGetLastError();
}

template <typename X, typename Out>
hipError_t launch(const Gradient& c) {
  const int digits = 1 << c.by.bits;
  const size_t next = size_t(kSortThreads / kWave) * c.by.held * sizeof(int);
  if (c.blocks) {
    const size_t lds = size_t(digits) * sizeof(int);
    const bool sorted = c.by.rows == 1;  // (a digit is a token)
    part_count_kernel<<<c.blocks, kThreads, lds, c.stream>>>(c);
    part_sums_kernel<Out><<<digits, kThreads, 0, c.stream>>>(c);
    part_kernel<<<c.blocks, kThreads, (kThreads / kWave + 1) * lds, c.stream>>>(c, sorted ? c.sorted : c.parted);
    const int ranges = ranges_of(c.by);
    if (ranges > 1) sort_kernel<Out, kRanges><<<digits * ranges, kSortThreads, next, c.stream>>>(c);
    else if (!sorted) sort_kernel<Out, kPart><<<digits, kSortThreads, next, c.stream>>>(c);
  } else if (c.tokens) {
    const int64_t rows = int64_t(c.r.B) * c.r.T;
    ready_kernel<<<int((rows + kReadyPer * kThreads - 1) / (kReadyPer * kThreads)), kThreads, 0, c.stream>>>(c);
    sort_kernel<Out, kReady><<<digits, kSortThreads, next, c.stream>>>(c);
  } else {
    sort_kernel<Out, kTokens><<<digits, kSortThreads, next, c.stream>>>(c);
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
