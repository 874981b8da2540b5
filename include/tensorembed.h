/*
 * tensorembed.h -- C ABI of embeddings of token ids (same library as tensorbleu.h).
 *
 * The other end of a policy over token ids than tensorloss.h: rows of a table by ids, scaled, and the gradient
 * of that in the table by sorted ids.
 *
 *   embedding of position n   = scale * table[token n]
 *   gradient of row v         = scale * sum over positions n with token v of rows n
 *
 * Conventions that hold for every entry point
 *   - Data pointers are DEVICE pointers owned by the caller; the structs are HOST memory, read during
 *     the call only.  Nothing is allocated, kept or synchronised; work goes to `hip_stream`.
 *   - Rows are D consecutive values at any address of a value; their strides are in elements.
 *   - Positions are those of tensorloss.h: (b, t) counts iff t < lengths[b] (or lengths is NULL) and
 *     mask[b, t] is not 0 (or mask is NULL).  What stands at other positions has no part in anything,
 *     whatever it is; their embeddings are 0.
 *   - Sums are in float32 in an order that positions, their number, V and D fix: results do not depend on the
 *     order in which workgroups run.  Every value is rounded once, to the type of what it is written to.
 *   - Problems that the host can see come back as tb_status_t before any work is enqueued.  A token outside
 *     [0, V) has an embedding of NaN and no part in a gradient, and sets TB_DEV_TOKEN_RANGE; a length
 *     outside [0, T] is clamped and sets TB_DEV_LENGTH_RANGE in *status (int32, may be NULL; cleared by
 *     the caller); every access stays in bounds.
 */
#ifndef TENSOREMBED_H
#define TENSOREMBED_H

#include "tensorloss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tb_table {
  const void* data;   /* row v at data + v*row_stride */
  int64_t row_stride;
  int32_t V, D;       /* V >= 1, D in 1..TB_WIDTH_MOST */
  int32_t type;       /* tb_type_t */
} tb_table_t;

enum { TB_WIDTH_MOST = 1 << 20 };

/* embeddings: [B, T, D] of the table's type, contiguous. */
int tensorembed_lookup(const tb_table_t* table, const tb_positions_t* at, int32_t B, int32_t T, float scale,
                       void* embeddings, int32_t* status, void* hip_stream);

typedef struct tb_embedding_rows {
  const void* data;               /* row (b, t) at data + b*seq_stride + t*pos_stride; rows may overlap */
  int64_t seq_stride, pos_stride;
  int32_t B, T, D;
  int32_t type;
} tb_embedding_rows_t;

typedef struct tb_table_gradient {
  void* data;          /* row v at data + v*row_stride; row_stride >= D where V > 1 */
  int64_t row_stride;
  int32_t V;
  int32_t type;        /* that of the rows, or TB_FLOAT32 */
  float scale;
  int32_t accumulate;  /* 0: every row is written.  Otherwise rows of tokens that come up are added to, and no
                          other one is read or written */
} tb_table_gradient_t;

/* The gradient may not overlap the rows. */
int tensorembed_gradient(const tb_embedding_rows_t* rows, const tb_positions_t* at,
                         const tb_table_gradient_t* grad, int32_t* status, void* workspace,
                         size_t workspace_bytes, void* hip_stream);

/* Workspace of the gradient: 256-byte aligned device memory, contents need no initialisation (0 on invalid
 * arguments). */
size_t tensorembed_workspace_bytes(int32_t B, int32_t T, int32_t V, int32_t D);

#ifdef __cplusplus
}
#endif
#endif /* TENSOREMBED_H */
