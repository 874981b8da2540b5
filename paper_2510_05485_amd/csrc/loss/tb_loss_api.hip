// Entry points of the losses: argument checks, workspace, launches.  Nothing here allocates,
// synchronises or keeps state between calls.
#include "tb_loss_host.h"

namespace tb {
namespace loss {
namespace {

hipError_t run_rows(Op op, Call& c) {
  return c.type == TB_FLOAT32 ? rows_of<F32>(op, c) : c.type == TB_BFLOAT16 ? rows_of<BF16>(op, c) : rows_of<F16>(op, c);
}
hipError_t run_gradient(Op op, const Call& c) {
  return c.type == TB_FLOAT32    ? gradient_of<F32>(op, c)
         : c.type == TB_BFLOAT16 ? gradient_of<BF16>(op, c)
                                 : gradient_of<F16>(op, c);
}

size_t value_bytes(int type) { return type == TB_FLOAT32 ? 4 : 2; }

constexpr size_t kAlign = 256;
size_t aligned(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

struct Workspace {
  size_t counts, weight, more, partial, state, lp, d_sequence, bytes;
};
Workspace workspace_of(int64_t B, int64_t T) {
  Workspace w;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t from = at;
    at += aligned(n);
    return from;
  };
  w.counts = take(4 * (B > kCountParts ? B : kCountParts));
  w.weight = take(4 * B);
  w.more = take(8 * 4 * kMoreSums);
  const int64_t groups = B * T < kMostGroups ? B * T : kMostGroups;
  w.partial = take(8 * 4 * size_t(groups > B ? groups : B));
  w.state = take(16 * B * T);  // (of pairs only, as what follows)
  w.lp = take(8 * B * T);
  w.d_sequence = take(4 * B);
  w.bytes = at;
  return w;
}
bool positions_fit(int64_t B, int64_t T) { return B >= 0 && T >= 0 && B * T < INT32_MAX; }

// The bytes from the first to behind the last value.
bool extent(int64_t seq, int64_t pos, const tb_logits_t& l, size_t bytes, int64_t* n) {
  if (seq < 0 || pos < 0) return false;
  __int128 last = __int128(l.B - 1) * seq + __int128(l.T - 1) * pos + l.V;
  last *= bytes;
  if (last > INT64_MAX) return false;
  *n = int64_t(last);
  return true;
}

int check(const tb_logits_t* l, const tb_positions_t* at, bool tokens, const tb_gradient_t* g, Call* c) {
  if (!l || !at || l->V < 1 || !positions_fit(l->B, l->T) || l->type < TB_FLOAT32 || l->type > TB_FLOAT16 ||
      !(l->temperature > 0.f) || !(l->temperature < INFINITY))
    return TB_ERR_INVALID_ARG;
  Rows& r = c->rows;
  r = {};
  r.B = l->B;
  r.T = l->T;
  r.V = l->V;
  c->type = l->type;
  if (l->B == 0 || l->T == 0) return TB_OK;
  const size_t size = value_bytes(l->type);
  int64_t span = 0, g_span = 0;
  if (!l->data || reinterpret_cast<uintptr_t>(l->data) % size || !extent(l->seq_stride, l->pos_stride, *l, size, &span))
    return TB_ERR_INVALID_ARG;
  if (tokens && (!at->tokens || (at->token_bytes != 4 && at->token_bytes != 8) || at->token_stride < 0 ||
                 reinterpret_cast<uintptr_t>(at->tokens) % at->token_bytes))
    return TB_ERR_INVALID_ARG;
  r.x = l->data;
  r.x_seq = l->seq_stride;
  r.x_pos = l->pos_stride;
  r.tokens = tokens ? at->tokens : nullptr;
  r.token_seq = at->token_stride;
  r.long_tokens = at->token_bytes == 8;
  r.lengths = at->lengths;
  r.mask = at->mask;
  while ((uint64_t(1) << r.t_shift) < uint32_t(r.T)) ++r.t_shift;
  r.t_magic = uint32_t((((uint64_t(1) << r.t_shift) - uint32_t(r.T)) << 32) / uint32_t(r.T) + 1);
  r.inv_temp = 1.f / l->temperature;
  r.g_scale = 1.f;
  if (!(r.inv_temp * kLog2e < INFINITY) || r.inv_temp == 0.f) return TB_ERR_INVALID_ARG;
  if (!g) return TB_OK;
  if (!g->data || reinterpret_cast<uintptr_t>(g->data) % size || !extent(g->seq_stride, g->pos_stride, *l, size, &g_span))
    return TB_ERR_INVALID_ARG;
  // rows of the gradient that overlap one another: one stride has to hold what the other one steps over
  const int64_t inner = l->T > 1 ? g->pos_stride : l->V, outer = l->B > 1 ? g->seq_stride : INT64_MAX;
  const bool rows_then_seqs = inner >= l->V && __int128(outer) >= __int128(l->T - 1) * inner + l->V;
  const bool seqs_then_rows = l->T > 1 && l->B > 1 && g->seq_stride >= l->V &&
                              __int128(g->pos_stride) >= __int128(l->B - 1) * g->seq_stride + l->V;
  if (!rows_then_seqs && !seqs_then_rows) return TB_ERR_INVALID_ARG;
  const bool same = g->data == l->data && (l->B == 1 || g->seq_stride == l->seq_stride) &&
                    (l->T == 1 || g->pos_stride == l->pos_stride);
  const char *x = static_cast<const char*>(l->data), *y = static_cast<const char*>(g->data);
  if (!same && x < y + g_span && y < x + span) return TB_ERR_INVALID_ARG;
  r.g = g->data;
  r.g_seq = g->seq_stride;
  r.g_pos = g->pos_stride;
  r.g_scale = g->scale;
  return TB_OK;
}

int check_workspace(const Rows& r, void* workspace, size_t bytes) {
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign || bytes < workspace_of(r.B, r.T).bytes)
    return TB_ERR_WORKSPACE;
  return TB_OK;
}
template <typename T>
T* in(void* workspace, size_t offset) {
  return reinterpret_cast<T*>(static_cast<char*>(workspace) + offset);
}
// What a mean divides by is added up by every workgroup while its row is on its way, from the lengths, from
// the mask of few positions, or from the numbers that a launch counts in a mask; where that is too much for so
// many workgroups, launches before leave the counts, or the weights.  Policy losses in bfloat16, us:
//   sequences x positions x values    lengths in each workgroup   weights from two launches
//   1024 x 8 x 5000 (8 million)        41.5                        41.6
//   2048 x 8 x 5000 (34 million)      104.9                        91.2
//   8000 x 8 x 5000                   539                         272
//   512 x 16 x 50257 (4 million)      281.6                       288.1
//   8000 x 64 x 64 (16 million)        49.3                        45.1
//   positions x values                mask in each workgroup      counts from a launch
//   1024 x 5000                        12.1                        13.6
//   2048 x 1000, x 5000                11.9, 18.3                  13.0, 18.7
//   4096 x 1000, x 5000                15.0, 31.4                  14.8, 26.4
constexpr int kMostParts = 8192, kMostMasked = 2048;
constexpr int64_t kMostReads = 1 << 23;  // of lengths (or counts), by all workgroups together
hipError_t set_mean(Op op, Call& c, int average, const Workspace& w, void* workspace) {
  const Rows& r = c.rows;
  const bool few = r.B <= kMostParts && r.B * workgroups_of(op, c) <= kMostReads;
  int32_t* n = in<int32_t>(workspace, w.counts);
  c.mean = {nullptr, nullptr, r.B, average};
  if (average == TB_SUM || (!r.mask && !r.lengths)) return hipSuccess;
  if (r.mask && (average == TB_MEAN_TOKENS || r.B == 1)) {  // (one sequence's mean is that of its positions)
    c.mean = {nullptr, nullptr, 0, TB_MEAN_TOKENS};
    if (r.B * r.T <= kMostMasked) return hipSuccess;
    c.mean = {nullptr, n, kCountParts, TB_MEAN_TOKENS};
    return run_part_counts(r, n, c.stream);
  }
  if (!r.mask && few) return hipSuccess;
  if (r.mask) c.mean.n = n;
  const hipError_t e = run_counts(r, n, c.stream);
  if (e != hipSuccess || few) return e;
  c.mean.weight = in<float>(workspace, w.weight);
  return run_weights(r.B, average, n, in<float>(workspace, w.weight), c.stream);
}
int done(hipError_t e) { return e == hipSuccess ? TB_OK : TB_ERR_HIP; }
bool average_known(int a) { return a >= TB_MEAN_TOKENS && a <= TB_SUM; }
bool empty(const Rows& r) { return r.B == 0 || r.T == 0; }

int check_teacher(const tb_teacher_t* q, bool rows) {
  if (!q || q->K < 1 || q->K > TB_TEACHER_MOST || (q->id_bytes != 4 && q->id_bytes != 8) || q->type < TB_FLOAT32 ||
      q->type > TB_FLOAT16 || !average_known(q->average) || (rows && (!q->ids || !q->logits)))
    return TB_ERR_INVALID_ARG;
  if (rows && (reinterpret_cast<uintptr_t>(q->ids) % q->id_bytes || reinterpret_cast<uintptr_t>(q->logits) % value_bytes(q->type)))
    return TB_ERR_INVALID_ARG;
  return TB_OK;
}
Teacher teacher_of(const tb_teacher_t& q, const Rows& r) {
  Teacher t = {};
  t.ids = q.ids;
  t.logits = q.logits;
  t.K = q.K;
  t.long_ids = q.id_bytes == 8;
  t.type = q.type;
  t.tau = 1.f / r.inv_temp;
  return t;
}

}  // namespace
}  // namespace loss
}  // namespace tb

using namespace tb::loss;

extern "C" size_t tensorloss_workspace_bytes(int32_t B, int32_t T) {
  return positions_fit(B, T) ? workspace_of(B, T).bytes + kAlign : 0;
}

extern "C" int tensorloss_token_logprobs(const tb_logits_t* logits, const tb_positions_t* at, float* logprobs,
                                         float* entropy, float* row_state, int32_t* status, void* hip_stream) {
  Call c = {};
  if (int rc = check(logits, at, true, nullptr, &c)) return rc;
  if (empty(c.rows)) return TB_OK;
  if (!logprobs) return TB_ERR_INVALID_ARG;
  c.rows.status = status;
  c.out.logprobs = logprobs;
  c.out.entropy = entropy;
  c.out.state = reinterpret_cast<float4*>(row_state);
  c.entropy = entropy != nullptr;
  c.stream = static_cast<hipStream_t>(hip_stream);
  return done(run_rows(kScore, c));
}

extern "C" int tensorloss_token_logprobs_grad(const tb_logits_t* logits, const tb_positions_t* at,
                                              const float* row_state, const float* d_logprobs, const float* d_entropy,
                                              int64_t d_seq_stride, int64_t d_pos_stride, const float* upstream,
                                              const tb_gradient_t* grad, void* hip_stream) {
  Call c = {};
  if (!grad) return TB_ERR_INVALID_ARG;
  if (int rc = check(logits, at, true, grad, &c)) return rc;
  if (empty(c.rows)) return TB_OK;
  if (!row_state || !d_logprobs) return TB_ERR_INVALID_ARG;
  c.given = {reinterpret_cast<const float4*>(row_state), d_logprobs, d_entropy, upstream, d_seq_stride, d_pos_stride};
  c.entropy = d_entropy != nullptr;
  c.stream = static_cast<hipStream_t>(hip_stream);
  return done(run_gradient(kScore, c));
}

extern "C" int tensorloss_policy(const tb_logits_t* logits, const tb_positions_t* at, const tb_policy_t* policy,
                                 const tb_gradient_t* grad, float* terms, float* logprobs, float* row_state,
                                 float* d_logprobs, float* d_entropy, int32_t* status, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  Call c = {};
  if (int rc = check(logits, at, true, grad, &c)) return rc;
  if (!policy || !terms || !average_known(policy->average) || !(policy->clip_low >= 0.f) || !(policy->clip_high >= 0.f) ||
      !(policy->kl_coef >= 0.f) || policy->entropy_coef != policy->entropy_coef)
    return TB_ERR_INVALID_ARG;
  c.stream = static_cast<hipStream_t>(hip_stream);
  const Rows& r = c.rows;
  if (!empty(r) && (!policy->old_logprobs || !policy->advantages || !logprobs || (policy->kl_coef != 0.f && !policy->ref_logprobs)))
    return TB_ERR_INVALID_ARG;
  if (int rc = check_workspace(r, workspace, workspace_bytes)) return rc;
  const Workspace w = workspace_of(r.B, r.T);
  double *partial = in<double>(workspace, w.partial), *more = in<double>(workspace, w.more);
  if (empty(r)) return done(run_terms(0, partial, more, terms, 4, c.stream));
  c.rows.status = status;
  c.out = {logprobs, nullptr, nullptr, reinterpret_cast<float4*>(row_state), d_logprobs, d_entropy, partial};
  c.policy = {policy->old_logprobs, policy->ref_logprobs, policy->advantages, policy->each, policy->clip_low,
              policy->clip_high, policy->kl_coef, policy->entropy_coef};
  c.entropy = policy->entropy_coef != 0.f;
  if (set_mean(kPolicy, c, policy->average, w, workspace) != hipSuccess || run_rows(kPolicy, c) != hipSuccess)
    return TB_ERR_HIP;
  return done(run_terms(c.groups, partial, more, terms, 4, c.stream));
}

extern "C" int tensorloss_preference(const tb_logits_t* logits, const tb_positions_t* at,
                                     const tb_preference_t* preference, const tb_gradient_t* grad, float* terms,
                                     float* sequence_logprobs, float* margins, float* row_state, float* d_sequence,
                                     int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Call c = {};
  if (int rc = check(logits, at, true, grad, &c)) return rc;
  if (!preference || preference->kind < TB_PAIR_SIGMOID || preference->kind > TB_PAIR_IPO || !(preference->beta > 0.f) ||
      !(preference->beta < INFINITY) || !(preference->label_smoothing >= 0.f) || !(preference->label_smoothing <= 0.5f) ||
      (preference->label_smoothing != 0.f && preference->kind != TB_PAIR_SIGMOID) || c.rows.B % 2 || !terms)
    return TB_ERR_INVALID_ARG;
  c.stream = static_cast<hipStream_t>(hip_stream);
  Rows& r = c.rows;
  if (r.B > 0 && (!sequence_logprobs || !margins)) return TB_ERR_INVALID_ARG;
  if (!empty(r) && !preference->ref_logprobs) return TB_ERR_INVALID_ARG;
  if (int rc = check_workspace(r, workspace, workspace_bytes)) return rc;
  const Workspace w = workspace_of(r.B, r.T);
  float4* state = row_state ? reinterpret_cast<float4*>(row_state) : in<float4>(workspace, w.state);
  if (!d_sequence) d_sequence = in<float>(workspace, w.d_sequence);
  void* g = r.g;
  if (!empty(r)) {
    r.g = nullptr;
    r.status = status;
    c.out = {nullptr, nullptr, in<double>(workspace, w.lp), state, nullptr, nullptr, nullptr};
    if (run_rows(kScore, c) != hipSuccess) return TB_ERR_HIP;
  }
  const Pairs pairs = {preference->ref_logprobs, in<double>(workspace, w.lp), terms, sequence_logprobs, margins, d_sequence,
                       in<double>(workspace, w.partial), preference->kind, preference->beta, preference->label_smoothing};
  if (run_pairs(r, pairs, c.stream) != hipSuccess) return TB_ERR_HIP;
  if (!g || empty(r)) return TB_OK;
  r.g = g;
  r.status = nullptr;
  c.given = {state, d_sequence, nullptr, nullptr, 1, 0};
  return done(run_gradient(kScore, c));
}

extern "C" int tensorloss_distill(const tb_logits_t* logits, const tb_positions_t* at, const tb_teacher_t* teacher,
                                  const tb_gradient_t* grad, float* terms, float* row_loss, float* row_state,
                                  float* d_row, int32_t* status, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
  Call c = {};
  if (int rc = check(logits, at, false, grad, &c)) return rc;
  const Rows& r = c.rows;
  if (int rc = check_teacher(teacher, !empty(r))) return rc;
  if (!terms || (!empty(r) && !row_loss)) return TB_ERR_INVALID_ARG;
  c.stream = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_workspace(r, workspace, workspace_bytes)) return rc;
  const Workspace w = workspace_of(r.B, r.T);
  double *partial = in<double>(workspace, w.partial), *more = in<double>(workspace, w.more);
  if (empty(r)) return done(run_terms(0, partial, more, terms, 1, c.stream));
  c.rows.status = status;
  c.out = {row_loss, nullptr, nullptr, reinterpret_cast<float4*>(row_state), d_row, nullptr, partial};
  c.teacher = teacher_of(*teacher, r);
  if (set_mean(kDistill, c, teacher->average, w, workspace) != hipSuccess || run_rows(kDistill, c) != hipSuccess)
    return TB_ERR_HIP;
  return done(run_terms(c.groups, partial, more, terms, 1, c.stream));
}

extern "C" int tensorloss_distill_grad(const tb_logits_t* logits, const tb_positions_t* at, const tb_teacher_t* teacher,
                                       const float* row_state, const float* d_row, const float* upstream,
                                       const tb_gradient_t* grad, void* hip_stream) {
  Call c = {};
  if (!grad) return TB_ERR_INVALID_ARG;
  if (int rc = check(logits, at, false, grad, &c)) return rc;
  const Rows& r = c.rows;
  if (int rc = check_teacher(teacher, !empty(r))) return rc;
  if (empty(r)) return TB_OK;
  if (!row_state || !d_row) return TB_ERR_INVALID_ARG;
  c.teacher = teacher_of(*teacher, r);
  c.given = {reinterpret_cast<const float4*>(row_state), d_row, nullptr, upstream, r.T, 1};
  c.stream = static_cast<hipStream_t>(hip_stream);
  return done(run_gradient(kDistill, c));
}
