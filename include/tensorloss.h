/*
 * tensorloss.h -- C ABI of the losses over a policy's logits (same library as tensorbleu.h).
 *
 * What a training loop does with the rewards that tensorbleu.h computes: log-probabilities of the
 * sampled tokens, the likeliest tokens beside them, the clipped policy loss, the loss of paired log ratios,
 * and the distillation of a teacher's best logits, each with its gradient in the logits.
 *
 * Notation: row r = (sequence b, position t) of the logits holds V values x; z = x / temperature,
 * p = softmax(z), lp = z[token] - log sum exp z, H = -sum p log p.
 *
 * Conventions that hold for every entry point
 *   - Data pointers are DEVICE pointers owned by the caller; the structs are HOST memory, read during
 *     the call only.  Nothing is allocated, kept or synchronised; work goes to `hip_stream`.
 *   - Logits and gradients: rows of V consecutive values, row (b, t) at data + b*seq_stride +
 *     t*pos_stride (elements; a row needs no alignment beyond its type's).  The rows of a gradient
 *     must not overlap.  The gradient may be written over the logits (same pointer and strides);
 *     any other overlap of the two is refused.
 *   - Arrays over positions are contiguous [B, T]; tokens may have a row stride of their own.
 *   - Position (b, t) counts iff t < lengths[b] (or lengths is NULL) and mask[b, t] is not 0 (or mask
 *     is NULL).  What stands at other positions -- logits, tokens, values -- has no part in anything,
 *     whatever it is; log-probabilities, entropies and gradients there are 0.
 *   - Arithmetic is in float32, sums over positions in float64; gradients are rounded once to the
 *     logits' type.  The order of a row's sum goes by the row's length and by its address modulo 128.
 *   - A logit of -inf is a token that cannot be: it has probability 0 and, unless it is the position's
 *     own token, gradient 0.  A row that has no finite logit, or one of +inf or NaN, has no
 *     distribution: its values are NaN.  Finite logits may be of any size.
 *   - Results do not depend on the order in which workgroups run.
 *   - Problems that the host can see come back as tb_status_t before any work is enqueued.  A token
 *     (or teacher's) id outside [0, V) makes the values of its row NaN and sets TB_DEV_TOKEN_RANGE, a
 *     length outside [0, T] is clamped and sets TB_DEV_LENGTH_RANGE in *status (int32, may be NULL;
 *     cleared by the caller); every access stays in bounds.
 *   - B * T == 0 is no error: sums over nothing are 0.
 */
#ifndef TENSORLOSS_H
#define TENSORLOSS_H

#include "tensorbleu.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { TB_FLOAT32 = 0, TB_BFLOAT16 = 1, TB_FLOAT16 = 2 } tb_type_t;

typedef struct tb_logits {
  const void* data;
  int64_t seq_stride, pos_stride; /* in elements */
  int32_t B, T, V;                /* V in 1..TB_VALUES_MOST; B*T below 2^31 - 1 */
  int32_t type;                   /* tb_type_t */
  float temperature;              /* > 0, and log2(e) / temperature finite in float32 */
} tb_logits_t;

/* The end of a row and a workgroup behind it are still a number of 32 bits. */
enum { TB_VALUES_MOST = 0x7FFFFE00 };

typedef struct tb_positions {
  const void* tokens;    /* [B, T], row b at tokens + b*token_stride */
  int64_t token_stride;  /* in elements */
  int32_t token_bytes;   /* 4 or 8 */
  const int32_t* lengths; /* [B] or NULL */
  const uint8_t* mask;    /* [B, T] or NULL */
} tb_positions_t;

typedef struct tb_gradient {
  void* data;                     /* of the logits' type */
  int64_t seq_stride, pos_stride; /* in elements */
  float scale;                    /* the gradient is that of scale * loss */
} tb_gradient_t;

/* What the backward pass needs of a row: a reference logit m, the sum of exp(z - m / temperature), the
 * entropy (0 where it was not asked for), the log-probability of the token.  float32 [B, T, 4]. */
enum { TB_ROW_STATE = 4 };

/* Log-probabilities of the tokens, and entropies where `entropy` is not NULL: float32 [B, T].
 * row_state: NULL, or float32 [B, T, 4] for the backward pass. */
int tensorloss_token_logprobs(const tb_logits_t* logits, const tb_positions_t* at, float* logprobs,
                              float* entropy, float* row_state, int32_t* status, void* hip_stream);

/* Gradient of  scale * upstream * sum over positions (d_logprobs lp + d_entropy H)  in the logits.
 * d_logprobs: float32, for position (b, t) at d_logprobs[b*d_seq_stride + t*d_pos_stride]; d_entropy
 * alike, or NULL; upstream: one float32 on the device, or NULL for 1.  row_state as the forward pass
 * left it for the same logits. */
int tensorloss_token_logprobs_grad(const tb_logits_t* logits, const tb_positions_t* at,
                                   const float* row_state, const float* d_logprobs,
                                   const float* d_entropy, int64_t d_seq_stride,
                                   int64_t d_pos_stride, const float* upstream,
                                   const tb_gradient_t* grad, void* hip_stream);

typedef struct tb_top {
  void* ids;          /* [B, T, K], of id_bytes 4 or 8 */
  float* logprobs;    /* [B, T, K] (not used by the gradient) */
  int32_t id_bytes, K; /* K in 1..min(V, TB_TOP_MOST) */
} tb_top_t;

enum { TB_TOP_MOST = 1024 };

/* The K likeliest tokens of every position in descending order of their logits, equal ones (0 and -0 among
 * them) by their ids, with their log-probabilities.  Logits of -inf are none of them: entries that are not
 * there, and all of a position that does not count, have the id -1 and the log-probability -inf.  A row
 * without a distribution has ids of -1 and log-probabilities of NaN.
 * Beside them the log-probabilities of the tokens (logprobs NULL: at->tokens is not read) and entropies (NULL
 * for none): float32 [B, T].  row_state: NULL, or float32 [B, T, 4] for the backward pass.
 * workspace: of tensorloss_top_workspace_bytes (NULL where that is 0). */
int tensorloss_top_logprobs(const tb_logits_t* logits, const tb_positions_t* at, const tb_top_t* top,
                            float* logprobs, float* entropy, float* row_state, int32_t* status,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gradient of scale * sum over positions of (sum_k d_top_k lp(ids_k) + d_logprobs lp + d_entropy H) in the
 * logits, ids and row_state as the forward pass left them for the same logits.  Entries with an id outside
 * [0, V) have no part in it; no id comes twice.  d_top: float32 [B, T, K]; d_logprobs (NULL: tokens are not
 * read) and d_entropy (or NULL): float32 [B, T].  The gradient may not overlap the logits. */
int tensorloss_top_logprobs_grad(const tb_logits_t* logits, const tb_positions_t* at, const tb_top_t* top,
                                 const float* row_state, const float* d_top, const float* d_logprobs,
                                 const float* d_entropy, const tb_gradient_t* grad, void* hip_stream);

/* Workspace of the forward pass, 256-byte aligned device memory that needs no initialisation: 0 for most
 * shapes (and for invalid arguments), some bytes for rows so long that workgroups share them. */
size_t tensorloss_top_workspace_bytes(int32_t B, int32_t T, int32_t V, int32_t type, int32_t K);

/* How positions are averaged: weight w of a position that counts is 1/N (N: positions that count),
 * 1/(S n_b) (n_b: those of its sequence, S: sequences that have any), or 1. */
typedef enum { TB_MEAN_TOKENS = 0, TB_MEAN_SEQUENCES = 1, TB_SUM = 2 } tb_average_t;

typedef struct tb_policy {
  const float* old_logprobs; /* [B, T], of the policy that sampled */
  const float* ref_logprobs; /* [B, T], of the reference; may be NULL where kl_coef is 0 */
  const float* advantages;   /* [B], or [B, T] with each != 0 */
  int32_t each;
  int32_t average;           /* tb_average_t */
  float clip_low, clip_high; /* the ratio is held to [1 - clip_low, 1 + clip_high] */
  float kl_coef, entropy_coef;
} tb_policy_t;

/* Clipped policy loss.  With ratio = exp(lp - old), kl = exp(ref - lp) - (ref - lp) - 1:
 *   loss = sum w (-min(ratio A, clip(ratio) A) + kl_coef kl - entropy_coef H).
 * A position is clipped, and its first term without gradient, iff A > 0 and ratio > 1 + clip_high, or
 * A < 0 and ratio < 1 - clip_low.
 * terms float32 [4]: loss, sum w kl, sum w [clipped], sum w H (kl and H where their coefficients are
 * not 0, else 0).  logprobs float32 [B, T].
 * grad: NULL for none.  For a backward pass later (tensorloss_token_logprobs_grad): row_state
 * [B, T, 4], d_logprobs and d_entropy [B, T] receive d loss / d lp and d loss / d H (each may be NULL). */
int tensorloss_policy(const tb_logits_t* logits, const tb_positions_t* at, const tb_policy_t* policy,
                      const tb_gradient_t* grad, float* terms, float* logprobs, float* row_state,
                      float* d_logprobs, float* d_entropy, int32_t* status, void* workspace,
                      size_t workspace_bytes, void* hip_stream);

typedef enum { TB_PAIR_SIGMOID = 0, TB_PAIR_HINGE = 1, TB_PAIR_IPO = 2 } tb_pair_t;

typedef struct tb_preference {
  const float* ref_logprobs; /* [B, T], of the reference */
  int32_t kind;              /* tb_pair_t */
  float beta;                /* > 0 */
  float label_smoothing;     /* in [0, 1/2], TB_PAIR_SIGMOID only */
} tb_preference_t;

/* Loss of paired log ratios: sequence i < B/2 is preferred to sequence i + B/2 (B is even).  With
 * d_b = sum over positions of (lp - ref), for TB_PAIR_IPO their mean (0 of none), and the margin
 * h = d_i - d_{i+B/2}:
 *   SIGMOID  (1 - e) log(1 + exp(-beta h)) + e log(1 + exp(beta h)),  e = label_smoothing
 *   HINGE    max(0, 1 - beta h)
 *   IPO      (h - 1 / (2 beta))^2
 * averaged over the pairs.  terms float32 [3]: loss, share of pairs with h > 0, mean margin.
 * sequence_logprobs float32 [B]: sum of lp; margins float32 [B/2].
 * grad NULL: for a backward pass later, row_state [B, T, 4] and d_sequence [B] (d loss / d lp of each
 * position of a sequence) are filled where not NULL. */
int tensorloss_preference(const tb_logits_t* logits, const tb_positions_t* at,
                          const tb_preference_t* preference, const tb_gradient_t* grad, float* terms,
                          float* sequence_logprobs, float* margins, float* row_state,
                          float* d_sequence, int32_t* status, void* workspace,
                          size_t workspace_bytes, void* hip_stream);

typedef struct tb_teacher {
  const void* ids;    /* [B, T, K], of id_bytes 4 or 8 */
  const void* logits; /* [B, T, K] of type `type` */
  int32_t id_bytes, type, K; /* K in 1..TB_TEACHER_MOST */
  int32_t average;    /* tb_average_t */
} tb_teacher_t;

enum { TB_TEACHER_MOST = 1024 };

/* Distillation from a teacher's K best logits.  q = softmax(teacher logits / temperature) over a
 * position's K entries; row_loss = temperature^2 sum q (log q - lp[id]); loss = sum w row_loss.
 * An entry of -inf is none (its id is not read); a position without entries has row_loss and gradient
 * 0 and still enters the average.  Entries with the same id add up in the gradient.
 * terms float32 [1]: the loss.  row_loss float32 [B, T].  `at`: tokens are not read.
 * grad: NULL for none; row_state [B, T, 4] and d_row [B, T] (d loss / d row_loss) for a backward pass
 * later (tensorloss_distill_grad) are filled where not NULL. */
int tensorloss_distill(const tb_logits_t* logits, const tb_positions_t* at, const tb_teacher_t* teacher,
                       const tb_gradient_t* grad, float* terms, float* row_loss, float* row_state,
                       float* d_row, int32_t* status, void* workspace, size_t workspace_bytes,
                       void* hip_stream);

/* Gradient of scale * upstream * sum over positions of d_row row_loss in the logits. */
int tensorloss_distill_grad(const tb_logits_t* logits, const tb_positions_t* at,
                            const tb_teacher_t* teacher, const float* row_state, const float* d_row,
                            const float* upstream, const tb_gradient_t* grad, void* hip_stream);

/* Workspace of the losses for B sequences of T positions: 256-byte aligned device memory, contents
 * need no initialisation (0 on invalid arguments). */
size_t tensorloss_workspace_bytes(int32_t B, int32_t T);

#ifdef __cplusplus
}
#endif
#endif /* TENSORLOSS_H */
