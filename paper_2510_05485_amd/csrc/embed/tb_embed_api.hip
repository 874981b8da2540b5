// Entry points of the embeddings: argument checks, workspace, launches.  Nothing here allocates, synchronises or
// keeps state between calls.
#include <algorithm>

#include "tb_embed.h"

namespace tb {
namespace embed {
namespace {

size_t value_bytes(int type) { return type == TB_FLOAT32 ? 4 : 2; }
bool type_known(int type) { return type >= TB_FLOAT32 && type <= TB_FLOAT16; }
bool positions_fit(int64_t B, int64_t T) { return B >= 0 && T >= 0 && B * T < INT32_MAX; }

constexpr size_t kAlign = 256;
size_t aligned(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
int log2_up(int64_t n) {
  int b = 0;
  while ((int64_t(1) << b) < n) ++b;
  return b;
}

// Up to so many positions every workgroup of the sort reads all tokens (without the zeros 7 us for 4096 positions and 17 for
// 32768); more are parted first (three launches of 5 to 12 us, and what is sorted then is a part).
constexpr int64_t kScanMost = 65536;
// Up to so many they read them from the caller's tensors, beyond from what a launch before has left.
constexpr int64_t kDirectMost = 1024;
constexpr int kMostPartBits = 11, kMostRows = 1024;

struct Plan {
  Buckets by;
  int blocks, slice;  // blocks 0: not parted
  int64_t slices;
  size_t tokens, sorted, parted, counts, totals, valid, join_from, partial, bytes;
};
Plan plan_of(int64_t B, int64_t T, int V, int D) {
  Plan p = {};
  const int64_t rows = B * T;
  const bool many = rows > kScanMost;
  // Few positions: 128 values at least of neighbouring rows to one bucket, 512 buckets where there are so many rows.
  // Many: a bucket for every token where there are few, so that nothing is left to sort
  p.by.low = D < 128 && !(many && V <= 1 << kMostPartBits) ? log2_up((128 + D - 1) / D) : 0;
  const int64_t groups = (int64_t(V) + (1 << p.by.low) - 1) >> p.by.low;
  p.by.bits = std::min(many && V <= 1 << kMostPartBits ? kMostPartBits : 9, log2_up(groups));
  const int most_rows = kMostRows >> p.by.low;
  while ((groups >> p.by.bits) + 1 > most_rows && !(many && p.by.bits == kMostPartBits)) ++p.by.bits;
  p.by.rows = int((groups + (1 << p.by.bits) - 1) >> p.by.bits) << p.by.low;
  p.by.held = std::min(p.by.rows, kMostRows);  // (fewer than a digit's in tables of more than 2 million rows)
  if (many) p.blocks = int((rows + kPartBlock - 1) / kPartBlock);
  // slices of 16 to 256 positions, about 4096 wavefronts of 512 columns together (32768 positions, D = 2048: 86.3 us with
  // 2048 wavefronts, 86.9 with 4096, 103 with 8192; 2097152, D = 64: 79, 72 and 78)
  const int64_t columns = (D + 511) / 512, each = D < 512 ? std::max(1, 512 / D) : 1;
  p.slice = 16;
  while (p.slice < 256 && (rows / p.slice) * columns / each > 4096) p.slice *= 2;
  p.slices = (rows + p.slice - 1) / p.slice;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t from = at;
    at += aligned(n);
    return from;
  };
  p.tokens = take(rows > kDirectMost ? 4 * rows : 0);
  p.sorted = take(sizeof(Entry) * rows);
  p.parted = take(p.blocks && p.by.rows > 1 ? sizeof(Entry) * rows : 0);
  p.counts = take(size_t(4) * p.blocks << p.by.bits);
  p.totals = take(p.blocks ? size_t(4) << p.by.bits : 0);
  p.valid = take(8);
  p.join_from = take(4 * p.slices);
  p.partial = take(p.slices > 1 ? size_t(8) * p.slices * D : 0);
  p.bytes = at;
  return p;
}

// The bytes from the first to behind the last value of rows, or false if they do not fit 63 bits.
bool extent(int64_t B, int64_t T, int64_t seq, int64_t pos, int64_t width, size_t bytes, int64_t* n) {
  if (seq < 0 || pos < 0) return false;
  __int128 last = __int128(B - 1) * seq + __int128(T - 1) * pos + width;
  last *= bytes;
  if (last > INT64_MAX) return false;
  *n = int64_t(last);
  return true;
}
bool pointer_ok(const void* p, size_t bytes) { return p && reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Positions into `r`; B and T are there.
int take_positions(const tb_positions_t* at, int64_t B, int64_t T, int V, int32_t* status, Rows* r) {
  if (!pointer_ok(at->tokens, 1) || (at->token_bytes != 4 && at->token_bytes != 8) || at->token_stride < 0 ||
      !pointer_ok(at->tokens, at->token_bytes))
    return TB_ERR_INVALID_ARG;
  r->tokens = at->tokens;
  r->token_seq = at->token_stride;
  r->long_tokens = at->token_bytes == 8;
  r->lengths = at->lengths;
  r->mask = at->mask;
  r->status = status;
  r->B = int(B);
  r->T = int(T);
  r->V = V;
  loss::set_division(*r);
  return TB_OK;
}
template <typename T>
T* in(void* workspace, size_t offset) {
  return reinterpret_cast<T*>(static_cast<char*>(workspace) + offset);
}
int done(hipError_t e) { return e == hipSuccess ? TB_OK : TB_ERR_HIP; }

}  // namespace
}  // namespace embed
}  // namespace tb

using namespace tb::embed;

extern "C" size_t tensorembed_workspace_bytes(int32_t B, int32_t T, int32_t V, int32_t D) {
  if (!positions_fit(B, T) || V < 1 || D < 1 || D > TB_WIDTH_MOST) return 0;
  return plan_of(B, T, V, D).bytes + kAlign;
}

extern "C" int tensorembed_lookup(const tb_table_t* table, const tb_positions_t* at, int32_t B, int32_t T, float scale,
                                  void* embeddings, int32_t* status, void* hip_stream) {
  if (!table || !at || !positions_fit(B, T) || table->V < 1 || table->D < 1 || table->D > TB_WIDTH_MOST ||
      !type_known(table->type))
    return TB_ERR_INVALID_ARG;
  const size_t size = value_bytes(table->type);
  int64_t span = 0, all = 0;
  if (!extent(1, table->V, 0, table->row_stride, table->D, size, &span) || !pointer_ok(table->data, size))
    return TB_ERR_INVALID_ARG;
  if (B == 0 || T == 0) return TB_OK;
  if (!extent(1, int64_t(B) * T, 0, table->D, table->D, size, &all) || !pointer_ok(embeddings, size)) return TB_ERR_INVALID_ARG;
  const char *x = static_cast<const char*>(table->data), *y = static_cast<const char*>(embeddings);
  if (x < y + all && y < x + span) return TB_ERR_INVALID_ARG;
  Lookup c = {};
  if (int rc = take_positions(at, B, T, table->V, status, &c.r)) return rc;
  c.r.x = table->data;
  c.r.x_pos = table->row_stride;
  c.r.g = embeddings;
  c.D = table->D;
  c.type = table->type;
  c.scale = scale;
  c.stream = static_cast<hipStream_t>(hip_stream);
  return done(run_lookup(c));
}

extern "C" int tensorembed_gradient(const tb_embedding_rows_t* rows, const tb_positions_t* at,
                                    const tb_table_gradient_t* grad, int32_t* status, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  if (!rows || !at || !grad || !positions_fit(rows->B, rows->T) || grad->V < 1 || rows->D < 1 || rows->D > TB_WIDTH_MOST ||
      !type_known(rows->type) || (grad->type != rows->type && grad->type != TB_FLOAT32))
    return TB_ERR_INVALID_ARG;
  const size_t size = value_bytes(rows->type), out_size = value_bytes(grad->type);
  int64_t span = 0, all = 0;
  if (!extent(1, grad->V, 0, grad->row_stride, rows->D, out_size, &span) || !pointer_ok(grad->data, out_size) ||
      (grad->V > 1 && grad->row_stride < rows->D))
    return TB_ERR_INVALID_ARG;
  const bool empty = rows->B == 0 || rows->T == 0;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign) return TB_ERR_WORKSPACE;
  const Plan p = plan_of(rows->B, rows->T, grad->V, rows->D);
  if (workspace_bytes < p.bytes) return TB_ERR_WORKSPACE;
  const int64_t rows_of = int64_t(rows->B) * rows->T;
  Gradient c = {};
  if (empty) {  // (every token is without positions)
    c.r.V = grad->V;
  } else {
    if (!pointer_ok(rows->data, size) ||
        !extent(rows->B, rows->T, rows->seq_stride, rows->pos_stride, rows->D, size, &all))
      return TB_ERR_INVALID_ARG;
    const char *x = static_cast<const char*>(rows->data), *y = static_cast<const char*>(grad->data);
    if (x < y + span && y < x + all) return TB_ERR_INVALID_ARG;
    if (int rc = take_positions(at, rows->B, rows->T, grad->V, status, &c.r)) return rc;
    c.r.x = rows->data;
    c.r.x_seq = rows->seq_stride;
    c.r.x_pos = rows->pos_stride;
  }
  c.r.g = grad->data;
  c.r.g_pos = grad->row_stride;
  c.D = rows->D;
  c.type = rows->type;
  c.out_type = grad->type;
  c.accumulate = grad->accumulate != 0;
  c.scale = grad->scale;
  c.by = p.by;
  c.tokens = rows_of > kDirectMost ? in<int32_t>(workspace, p.tokens) : nullptr;
  c.sorted = in<Entry>(workspace, p.sorted);
  c.parted = in<Entry>(workspace, p.parted);
  c.counts = in<int32_t>(workspace, p.counts);
  c.totals = in<int32_t>(workspace, p.totals);
  c.valid = in<int32_t>(workspace, p.valid);
  c.joins = c.valid + 1;
  c.join_from = in<int32_t>(workspace, p.join_from);
  c.partial = in<float>(workspace, p.partial);
  c.blocks = p.blocks;
  c.slice = p.slice;
  c.slices = p.slices;
  c.stream = static_cast<hipStream_t>(hip_stream);
  if (empty && c.accumulate) return TB_OK;
  return done(run_gradient(c));
}
