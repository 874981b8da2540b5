// What the kernels of the losses share: arguments, rows of logits in chunks of 16 bytes, sums over
// wavefronts and workgroups.
#pragma once

#include <hip/hip_bfloat16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tensorloss.h"

namespace tb {
namespace loss {

constexpr int kWave = 64;
constexpr float kLowest = -3.402823466e38f;
constexpr float kExtreme = 1e37f;  // stands for the reference of values all below it, whose product with log2(e) is finite
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// What a row's workgroup does behind the softmax statistics.
enum Op { kScore, kPolicy, kDistill, kGiven };  // (kGiven: the gradient alone)

struct Rows {
  const void* x;
  int64_t x_seq, x_pos;
  void* g;  // null: no gradient
  int64_t g_seq, g_pos;
  const void* tokens;
  int64_t token_seq;
  const int32_t* lengths;
  const uint8_t* mask;
  int32_t* status;
  int B, T, V;
  uint32_t t_magic, t_shift;  // of the division by T
  int long_tokens;
  float inv_temp;
  float g_scale;
};

// Positions are numbered b T + t.  n / T = (umulhi(n, magic) + n) >> shift for n < 2^31 with shift =
// ceil(log2 T) and magic = floor(2^32 (2^shift - T) / T) + 1 (Granlund and Montgomery 1994).
struct At {
  int b, t;
};

struct RowOut {  // per position, any may be null
  float *logprobs, *entropy;
  double* exact;  // log-probabilities (kScore) whose logarithm is not rounded to 32 bits
  float4* state;  // reference logit (the largest, or one near it), sum of exponentials, entropy, log-probability
  float *d_logprobs, *d_entropy;
  double* partial;  // [workgroup][4]: the weighted terms of its rows
};

// How positions are averaged.  A weight is one over a total, which every workgroup adds up from `parts`
// numbers: positions of the sequences (or, for TB_MEAN_TOKENS, of any parts), or sequences that have some.
struct Mean {
  const float* weight;  // [B]: the weights themselves, or null
  const int32_t* n;     // [parts], or null: the lengths, and T without these
  int parts, average;
};

struct Policy {
  const float *old_lp, *ref_lp, *advantages;
  int each;
  float low, high, kl_coef, entropy_coef;
};

struct Teacher {
  const void *ids, *logits;
  int K, long_ids, type;
  float tau;
};

struct Given {  // the backward pass: cotangents of lp and H (or of the row's divergence)
  const float4* state;
  const float *d_lp, *d_entropy, *upstream;
  int64_t d_seq, d_pos;
};

// ---- types ------------------------------------------------------------------------------------

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Accesses of 16 bytes to rows, which are arrays of values: at any address of a value, and at multiples of 16.
typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));
typedef u32x4 u32x4_at16 __attribute__((aligned(16), may_alias));

struct F32 {
  template <int kFirst>
  static __device__ __forceinline__ float upper(const u32x4* c);  // of the first kFirst chunks
  static constexpr uint32_t kNone = 0xFF800000u;  // -inf
  using type = float;
  static constexpr int kPer = 4;  // values of a chunk
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void unpack(u32x4 c, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(c[i]);
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(v[i]);
    return c;
  }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct BF16 {
  template <int kFirst>
  static __device__ __forceinline__ float upper(const u32x4* c);  // of the first kFirst chunks
  static constexpr uint32_t kNone = 0xFF80FF80u;  // -inf
  using type = uint16_t;
  static constexpr int kPer = 8;
  static __device__ __forceinline__ uint32_t round2(float a, float b) {  // to nearest, ties to even
    const bf16x2 r = __builtin_convertvector(f32x2{a, b}, bf16x2);
    uint32_t u;
    __builtin_memcpy(&u, &r, 4);
    return u;
  }
  static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
  static __device__ __forceinline__ void store(uint16_t* p, float v) { *p = uint16_t(round2(v, v)); }
  static __device__ __forceinline__ void unpack(u32x4 c, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(c[i] << 16);
      v[2 * i + 1] = __uint_as_float(c[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = round2(v[2 * i], v[2 * i + 1]);
    return c;
  }
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct F16 {
  template <int kFirst>
  static __device__ __forceinline__ float upper(const u32x4* c);  // of the first kFirst chunks
  static constexpr uint32_t kNone = 0xFC00FC00u;  // -inf
  using type = _Float16;
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float load(const _Float16* p) { return float(*p); }
  static __device__ __forceinline__ void store(_Float16* p, float v) { *p = _Float16(v); }
  static __device__ __forceinline__ void unpack(u32x4 c, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f16x2 h;
      const uint32_t u = c[i];
      __builtin_memcpy(&h, &u, 4);
      v[2 * i] = float(h[0]);
      v[2 * i + 1] = float(h[1]);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x2 h = {_Float16(v[2 * i]), _Float16(v[2 * i + 1])};  // to nearest, ties to even
      uint32_t u;
      __builtin_memcpy(&u, &h, 4);
      c[i] = u;
    }
    return c;
  }
};

// The largest of three; instruction and all, since the compiler would first quiet signalling NaNs, one
// instruction a value (such a value makes the row NaN in any case).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The largest of packed values, as signed integers that order values from 0 on like the values themselves
// and any of them behind those below 0 (which come the other way round).
typedef short i16x2 __attribute__((ext_vector_type(2)));
template <int kFirst>
__device__ __forceinline__ i16x2 upper_pair(const u32x4* c) {
  i16x2 top = {-32768, -32768};
#pragma unroll
  for (int k = 0; k < kFirst; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = c[k][i];
      i16x2 v;
      __builtin_memcpy(&v, &u, 4);
      top = __builtin_elementwise_max(top, v);
    }
  return top;
}
template <int kFirst>
__device__ __forceinline__ float F32::upper(const u32x4* c) {
  int top = INT32_MIN;
#pragma unroll
  for (int k = 0; k < kFirst; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, int(c[k][i]));
  return __int_as_float(top);
}
template <int kFirst>
__device__ __forceinline__ float BF16::upper(const u32x4* c) {
  const i16x2 top = upper_pair<kFirst>(c);
  return __uint_as_float(uint32_t(uint16_t(max(top[0], top[1]))) << 16);
}
template <int kFirst>
__device__ __forceinline__ float F16::upper(const u32x4* c) {
  const i16x2 top = upper_pair<kFirst>(c);
  const short most = max(top[0], top[1]);
  _Float16 h;
  __builtin_memcpy(&h, &most, 2);
  return float(h);
}

// 2^x; the hardware's instruction is within one unit in the last place, and gives 0 below 2^-126 (a
// probability that no type of gradient holds beside one of its row's others)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- rows -------------------------------------------------------------------------------------

// A row's values in the order of memory: `head` values up to the first address that is a multiple of
// kAlign, `chunks` chunks of 16 bytes, and the rest.  Head and rest are at most kEdge values together;
// chunk i and the i-th of them are thread i's (of a workgroup, or of the lanes that share a row).
// Lines of 128 bytes where a wavefront or more reads a row (its request of 1 KB then touches eight lines
// and not nine: 2 % less time on rows of 50257 values), 16 bytes where a few lanes do.
constexpr int kLine = 128;
template <typename X, int kAlign>
struct Span {
  using T = typename X::type;
  static constexpr int kEdge = kAlign / int(sizeof(T)) - 1 + X::kPer - 1;
  const T* x;
  int V, head, chunks;
  __device__ __forceinline__ Span(const T* row, int values) : x(row), V(values) {
    head = int((-reinterpret_cast<uintptr_t>(row)) & (kAlign - 1)) / int(sizeof(T));
    if (head > values) head = values;
    chunks = (values - head) / X::kPer;
  }
  __device__ __forceinline__ int at(int chunk) const { return head + chunk * X::kPer; }
  __device__ __forceinline__ u32x4 chunk(int i) const { return *reinterpret_cast<const u32x4_at16*>(x + at(i)); }
  // the j-th value of head and rest, or -1
  __device__ __forceinline__ int edge(int j) const {
    if (j < head) return j;
    const int i = j + chunks * X::kPer;
    return i < V ? i : -1;
  }
  // which of `threads` writes value i of the gradient
  __device__ __forceinline__ int owner(int i, int threads) const {
    const int c = (i - head) / X::kPer;
    return (i < head ? i : c < chunks ? c : i - chunks * X::kPer) % threads;
  }
};
template <typename X>
using Line = Span<X, kLine>;

template <typename X>
__device__ __forceinline__ const typename X::type* row_of(const Rows& r, int b, int t) {
  return static_cast<const typename X::type*>(r.x) + b * r.x_seq + t * r.x_pos;
}
template <typename X>
__device__ __forceinline__ typename X::type* gradient_of(const Rows& r, int b, int t) {
  return static_cast<typename X::type*>(r.g) + b * r.g_seq + t * r.g_pos;
}
__device__ __forceinline__ int64_t load_id(const void* ids, int wide, int64_t i) {
  return wide ? static_cast<const int64_t*>(ids)[i] : int64_t(static_cast<const int32_t*>(ids)[i]);
}

__device__ __forceinline__ int held_length(int length, int T, int32_t* status) {
  if (length >= 0 && length <= T) return length;
  if (status) atomicOr(status, TB_DEV_LENGTH_RANGE);
  return length < 0 ? 0 : T;
}
__device__ __forceinline__ At position(const Rows& r, int64_t at) {
  const uint32_t n = uint32_t(at), b = (__umulhi(n, r.t_magic) + n) >> r.t_shift;
  return {int(b), int(n - b * uint32_t(r.T))};
}
__device__ __forceinline__ int clamped(int length, int T) { return min(max(length, 0), T); }
__device__ __forceinline__ bool counts(const Rows& r, int b, int t) {
  if (r.lengths && t >= r.lengths[b]) return false;
  return !r.mask || r.mask[int64_t(b) * r.T + t] != 0;
}

// ---- sums -------------------------------------------------------------------------------------

template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int d = kWave / 2; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = kWave / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// Sum over a wavefront, all lanes active: four steps inside rows of 16 lanes, then each row's into the next
// ones'; the last lane has all of it.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ float dpp_or(float old, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}
__device__ __forceinline__ float full_wave_sum(float v) {
  v += dpp_or<0xB1>(0.f, v);          // quad_perm [1, 0, 3, 2]
  v += dpp_or<0x4E>(0.f, v);          // quad_perm [2, 3, 0, 1]
  v += dpp_or<0x141>(0.f, v);         // row_half_mirror
  v += dpp_or<0x140>(0.f, v);         // row_mirror
  v += dpp_or<0x142, 0xa>(0.f, v);    // row_bcast:15 into rows 1 and 3
  v += dpp_or<0x143, 0xc>(0.f, v);    // row_bcast:31 into rows 2 and 3
  return last_lane(v);
}
__device__ __forceinline__ float full_wave_max(float v) {
  v = fmaxf(v, dpp_or<0xB1>(v, v));
  v = fmaxf(v, dpp_or<0x4E>(v, v));
  v = fmaxf(v, dpp_or<0x141>(v, v));
  v = fmaxf(v, dpp_or<0x140>(v, v));
  v = fmaxf(v, dpp_or<0x142, 0xa>(v, v));
  v = fmaxf(v, dpp_or<0x143, 0xc>(v, v));
  return last_lane(v);
}
// Sum of 32-bit integers over a wavefront, all lanes active.
__device__ __forceinline__ int full_wave_sum(int v) {
  auto step = [](int a, int b) { return a + b; };
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false));
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false));
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false));
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false));
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  v = step(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(v, kWave - 1);
}

// Softmax statistics of a part of a row, of a = (x - m) k with k = log2(e) / temperature: the largest
// value m (the lowest finite one at least, so that no difference of two -inf is formed), s = sum 2^a,
// and for the entropy t = sum 2^a a.
struct Stats {
  float m, s, t;
};

// a without -inf, whose product with its weight 0 would be NaN; all below -1000 alike, where weights are 0, so
// that a product with a cotangent is not infinite either
__device__ __forceinline__ float finite(float a) { return fmaxf(a, -1e3f); }

template <bool kEntropy>
__device__ __forceinline__ Stats joined(const Stats& p, const Stats& q, float k) {
  Stats r;
  r.m = fmaxf(p.m, q.m);
  const float dp = (p.m - r.m) * k, dq = (q.m - r.m) * k;
  const float ep = exp2_fast(dp), eq = exp2_fast(dq);
  r.s = ep * p.s + eq * q.s;
  r.t = kEntropy ? ep * (p.t + finite(dp) * p.s) + eq * (q.t + finite(dq) * q.s) : 0.f;
  return r;
}

}  // namespace loss
}  // namespace tb
