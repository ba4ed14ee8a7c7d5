/*
 * deepreduce_losses.h -- the losses of a data-parallel training step, as
 * calls of the library whose codec (deepreduce.h) sends the step's gradient.
 *
 *  - dr_top_logits: a teacher's logits, row by row, into the K largest and
 *    one entry that stands for all others.  The payload is 8 K + 4 bytes a
 *    row, and it determines a distribution over K + 1 outcomes.
 *  - dr_distill_forward, dr_distill_backward, dr_distill_step: a student's
 *    divergence from such payloads and its gradient.
 *  - dr_balance_forward, dr_balance_backward: per-expert counts and the
 *    balance loss of a router, and its gradient.
 *
 * The conventions of deepreduce.h hold: device pointers unless the name ends
 * in _h, calls asynchronous on `stream`, arguments checked on the host before
 * anything is launched (DR_EINVAL launches nothing), all memory the caller's,
 * scratch from `ws` (256-byte aligned, dr_losses_workspace_bytes() bytes,
 * undefined between calls, not shared by calls that run concurrently), no
 * state kept between calls, no host synchronisation, nothing that a graph
 * capture would refuse.  Results do not depend on the order in which blocks
 * run: the same inputs give the same bits.
 *
 * A launch counts its threads in 32 bits: calls that would need more are
 * EINVAL (some 10^11 numbers; 2^24 rows of a distillation, however short, 2^23
 * to 2^25 of dr_top_logits, 2^24 groups of a balance loss).
 *
 * Logits.  A matrix of rows x cols numbers of one type, each row contiguous,
 * rows `row_stride` numbers apart; any alignment that suits the type.  -inf
 * masks a column.  +inf and NaN are outside the contract: the outputs of that
 * row (that group, for the balance loss) are then unspecified, no other
 * output changes, and every kernel ends.
 */
#ifndef DEEPREDUCE_LOSSES_H
#define DEEPREDUCE_LOSSES_H

#include "deepreduce.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Number types of matrices and index types. */
#define DR_TYPE_F32 0u
#define DR_TYPE_BF16 1u
#define DR_TYPE_F16 2u
#define DR_INDEX_I32 0u
#define DR_INDEX_I64 1u

#define DR_MAX_TOP 256u      /* most logits dr_top_logits keeps of a row */
#define DR_MAX_TEACHER 1024u /* most entries of a teacher's row */
#define DR_MAX_EXPERTS 1024u /* most experts of a router */
#define DR_MAX_COLS (1ull << 31) /* fewer columns than this */
#define DR_DISTILL_STATS 8u  /* floats that dr_distill_forward saves per row */

typedef struct {
    const void *data;
    uint64_t rows;       /* fewer than 2^31 */
    uint64_t cols;       /* 1 .. DR_MAX_COLS - 1 */
    uint64_t row_stride; /* numbers from one row's start to the next one's, >= cols */
    uint32_t type;       /* DR_TYPE_* */
} dr_logits;

/* A teacher's payload: per row k columns with their logits, and the entry
 * that stands for the rest.  Columns are distinct within a row (a column
 * given twice leaves that row's loss and gradient unspecified); one outside
 * [0, cols) is no entry, and its logit is not used. */
typedef struct {
    const void *idx;     /* columns, row r at r * idx_stride */
    const void *val;     /* logits (not divided by the temperature), row r at r * val_stride */
    const float *rest;   /* per row, ln of the sum of exp(logit / temperature) over the columns not kept;
                            null, or -inf in a row: the kept ones are the whole distribution */
    uint64_t idx_stride; /* >= k */
    uint64_t val_stride; /* >= k */
    uint32_t k;          /* 1 .. DR_MAX_TEACHER */
    uint32_t idx_type;   /* DR_INDEX_* */
    uint32_t val_type;   /* DR_TYPE_* */
} dr_teacher;

/* Scratch bytes sufficient for any call below on a matrix of at most rows x
 * cols numbers with at most k kept logits (0 for an argument out of its
 * range). */
DR_EXPORT size_t dr_losses_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t k);

/* ---------------------------------------------------------------------- */
/* A teacher's logits into a payload                                       */
/* ---------------------------------------------------------------------- */

/* For each row: idx_out and val_out (rows x k, contiguous) receive the
 * columns and values of the k largest logits, by value descending, of equal
 * values the lowest column first.  -inf is never kept: places left over hold
 * column -1 and value -inf.  rest_out (nullable, one per row) receives ln of
 * the sum of exp(logit / temperature) over the columns not kept (a float's
 * largest or lowest where that is beyond it), -inf if that sum is 0.  EINVAL:
 * k outside 1 .. DR_MAX_TOP, temperature not finite or not above 0, a null
 * pointer, workspace too small. */
DR_EXPORT dr_status dr_top_logits(const dr_logits *logits_h, uint32_t k, float temperature, int32_t *idx_out,
                                  float *val_out, float *rest_out, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------- */
/* Distillation from a teacher's top logits                                */
/* ---------------------------------------------------------------------- */

/* With t the temperature, v_k the teacher's logits and z the student's row:
 *   p = softmax over (v_0 / t, ..., v_{k-1} / t, rest)
 *   q = softmax(z / t), q_rest = the sum of q over the columns not kept
 *   loss = w (sum_k p_k (ln p_k - ln q_k) + p_rest (ln p_rest - ln q_rest)),
 * terms with p = 0 being 0.  w is the row's weight (null: 1); fold the mean's
 * 1 / n and distillation's customary t^2 into it.  A row of weight 0 is not
 * read at all, whatever it holds: loss, saved numbers and gradient are 0.  A
 * teacher's row without entries has p_rest = q_rest = 1 and loss 0 if its
 * rest is finite (+inf if the student's row is all -inf).  Where rest is -inf
 * or null, a teacher's row without entries, or with logits of -inf alone, is
 * no distribution, and has loss 0 and gradient 0.  A student's row that gives
 * a kept column no probability (its logit is -inf) has loss +inf and a finite
 * gradient.  One entry per row and rest null is the cross entropy with that
 * column as the label.
 *
 * stats_out (nullable, rows x DR_DISTILL_STATS, contiguous) receives what the
 * backward pass reads: m = the row's largest logit, 1 / S with S = sum_j
 * exp((z_j - m) / t), m' = the largest logit not kept, (q_rest - p_rest) / S'
 * with S' the sum of exp((z_j - m') / t) over the columns not kept (0 if S' is
 * 0), M = the largest of (v_k / t, rest), 1 / sum exp((v_k / t, rest) - M), and
 * zeros. */
DR_EXPORT dr_status dr_distill_forward(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                                       const float *weight, float *loss_out, float *stats_out, void *ws,
                                       size_t ws_bytes, void *stream);

/* The gradient at the student's logits, in their type:
 *   (u w / t) (q_j - p_j) for a kept column,
 *   (u w / t) q_j (1 - p_rest / q_rest) for another one, which is
 *   (u w / t) (q_rest - p_rest) times its share of the columns not kept,
 * u the loss's gradient of the row, upstream[r * upstream_stride] (null: 1; a
 * stride of 0 takes one number for all rows).  A row with w = 0 or u = 0 is
 * not read and receives zeros.  stats is what dr_distill_forward saved with
 * the same student, teacher, temperature and weight.  grad_out has the
 * student's rows and columns, rows grad_stride numbers apart; it may be the
 * student's own matrix (same pointer and stride), otherwise the two must not
 * overlap. */
DR_EXPORT dr_status dr_distill_backward(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                                        const float *weight, const float *upstream, uint64_t upstream_stride,
                                        const float *stats, void *grad_out, uint64_t grad_stride, void *stream);

/* Both directions at once, for a program that knows its rows' weights before
 * the loss: loss_out as by dr_distill_forward, grad_out as by
 * dr_distill_backward with u = 1. */
DR_EXPORT dr_status dr_distill_step(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                                    const float *weight, float *loss_out, void *grad_out, uint64_t grad_stride,
                                    void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------- */
/* Balance loss of a router                                                */
/* ---------------------------------------------------------------------- */

/* A router's rows (tokens) in groups of group_rows consecutive ones (the last
 * may be shorter), each group balanced by itself: one group for a batch as a
 * whole, one per sequence for sequences.  E = cols experts, k chosen per row.
 * row_mask (nullable, one byte per row): a row whose byte is 0 is padding; it
 * counts nowhere, its logits may hold anything, its gradient is 0. */
typedef struct {
    const void *idx;     /* chosen experts, row r at r * idx_stride; one outside [0, E) was dropped and is not
                            counted.  Not used by dr_balance_backward (may be null there) */
    uint64_t idx_stride; /* >= k */
    uint32_t k;          /* 1 .. E */
    uint32_t idx_type;   /* DR_INDEX_* */
    const uint8_t *row_mask;
    uint64_t group_rows; /* 1 .. 2^31 - 1 */
} dr_routes;

/* For group g with n_g valid rows and G groups in all (ceil(rows /
 * group_rows)):
 *   counts_out[g E + e] = the choices of expert e,  rows_out[g] = n_g,
 *   prob_out[g E + e] = P_ge = the mean of softmax(z)_e over the valid rows,
 *   loss_out[0] = coef / G sum_g sum_e f_ge P_ge, f_ge = E counts_ge / (k n_g).
 * A group without valid rows has zeros.  A row whose logits are all -inf is
 * valid and adds nothing to P.  prob_out may be null.  EINVAL: cols above
 * DR_MAX_EXPERTS, rows * k above 2^31 - 1, k above cols, coef not finite, a
 * null pointer, workspace too small. */
DR_EXPORT dr_status dr_balance_forward(const dr_logits *router_h, const dr_routes *routes_h, float coef,
                                       int32_t *counts_out, int32_t *rows_out, float *prob_out, float *loss_out,
                                       void *ws, size_t ws_bytes, void *stream);

/* The gradient at the router's logits, the counts taken as constants:
 *   u (coef / (G n_g)) p_j (f_gj - sum_e f_ge p_e), f_ge = E counts_ge / (k N_g)
 * with n_g = rows_in[g] this worker's valid rows and N_g = count_rows[g] the
 * rows that counts covers: pass rows_in twice for a worker's own counts, or
 * the sums over all workers for a balance over the global batch (whose loss
 * is coef / G sum_g sum_e f_ge prob_ge with the same f).  upstream: one number,
 * u (null: 1).  grad_out as for dr_distill_backward. */
DR_EXPORT dr_status dr_balance_backward(const dr_logits *router_h, const dr_routes *routes_h, float coef,
                                        const int32_t *counts, const int32_t *count_rows, const int32_t *rows_in,
                                        const float *upstream, void *grad_out, uint64_t grad_stride, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* DEEPREDUCE_LOSSES_H */
