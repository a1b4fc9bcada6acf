/*
 * zero_operators.h -- C ABI of libzeroshard's training operators: the rows of a
 * sparse student distilled from a teacher, whose fp16 gradients the shard step
 * of zero_shard.h takes.  For AMD Instinct MI355X (gfx950).
 *
 *   zero_rms_norm     root-mean-square norm with the residual's addition, rows
 *                     in the model's type and in 8 bits with scales; backward
 *   zero_route        the choice of k experts a token and their weights, the
 *                     slots ordered by expert; backward
 *   zero_distill      loss and gradient of a student's logits against a
 *                     teacher's top logits, with a hard-label term
 *
 * Mixed precision as in ZeRO (Rajbhandari et al., arXiv 1910.02054) Sec. 3.1: the
 * gradient carries the loss scale from the loss on (grad_scale below); where it
 * leaves binary16's range it becomes inf, which the shard step finds and skips on.
 *
 * Conventions, beside those of zero_shard.h (return values, zero_last_error,
 * streams, the current device):
 *   - A call takes its arguments in a record.  Array members are DEVICE pointers
 *     owned by the caller; the library keeps nothing between calls and has no
 *     workspace of its own for them: where a call needs room, the caller gives it
 *     (`workspace`, sized by the function named there) and may use it for anything
 *     else once the call's work on the stream is complete.
 *   - Calls only enqueue kernels on `stream` and can be captured into a graph.
 *     They write all of every output and read no output's old contents.
 *   - `dtype` is the type of a record's arrays declared void* (ZERO_F32,
 *     ZERO_F16, ZERO_BF16).  Arithmetic is in fp32 whatever the type, each output
 *     is rounded once, to nearest even.  A softmax's terms below 2^-126 count as 0, and so
 *     do gradients that are their multiples, whatever the loss scale.
 *   - A matrix [rows, cols] has its rows `ld` elements apart (ld >= cols; any
 *     alignment of an element, rows of whole 16-byte groups run fastest); its
 *     other elements are neither read nor written.  rows may be 0.
 *   - An output must not overlap another array of the call, but for the pairs
 *     that a call names as in place (same address, same ld).  Columns of one buffer
 *     (same ld) do not overlap.
 *   - Every array must lie inside one GPU-accessible allocation, checked on each
 *     call but while the stream is being captured (make one eager call first). That
 *     the current device can access it (its own memory, or a peer's with access enabled)
 *     is the caller's to see to.
 *   - ZERO_EINVAL means that nothing was launched.
 */
#ifndef ZERO_OPERATORS_H
#define ZERO_OPERATORS_H

#include <stdint.h>

#include "zero_shard.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ZERO_F32 0
#define ZERO_F16 1
#define ZERO_BF16 2

/* ------------------------------------------------------------------------ */
/* Root-mean-square norm                                                    */
/* ------------------------------------------------------------------------ */

#define ZERO_NORM_MAX_COLS 32768

/* h    = x + residual rounded to dtype (h = x without a residual)
 * rstd = 1 / sqrt(mean of h^2 over the row + eps)
 * y    = h * rstd * weight
 * and, for groups of `group` columns (0: the whole row; else 32, 64, 128 or 256;
 * the last group of a row may be short), from the unrounded y,
 * scale = max(largest |y| of the group, 2^-100) / 448,  q8 = e4m3(y / scale).
 * e4m3 is the OCP 8-bit float with largest value 448 and no infinities; it is
 * rounded to nearest even.  A NaN in a row makes the row's rstd, y, q8 and scales
 * NaN; an infinity makes rstd 0.  Finite rows have the rstd and y of the formula wherever fp32 holds
 * that rstd, also where squares or eps would leave fp32's range. */
typedef struct {
    int32_t dtype;       /* of x, residual, weight, h, y                            */
    int32_t group;       /* columns of one scale; 0: one scale a row                */
    int64_t rows, cols;  /* 1 <= cols <= ZERO_NORM_MAX_COLS                         */
    double eps;          /* >= 0, finite                                            */
    const void* x;
    int64_t ld_x;
    const void* residual; /* NULL: none                                             */
    int64_t ld_residual;
    const void* weight;  /* [cols]                                                  */
    void* h;             /* NULL: not wanted; may be x or residual in place; needs a residual */
    int64_t ld_h;
    void* y;             /* NULL: not wanted; may be x or residual in place         */
    int64_t ld_y;
    uint8_t* q8;         /* e4m3 codes; NULL: not wanted (then scale is NULL too)   */
    int64_t ld_q8;
    float* scale;        /* [rows, ceil(cols / group)], close together              */
    float* rstd;         /* [rows]; NULL: not wanted                                */
} zero_rms_norm_args_t;

int zero_rms_norm(const zero_rms_norm_args_t* args, void* stream);

/* The gradients: with g = dy * weight and n = h * rstd,
 *   dx = rstd * (g - n * mean over the row of (g * n)) + dh
 *   dweight = sum over the rows of dy * n.
 * dx is the gradient of x and of the residual alike.  dh is the gradient that
 * reaches h from elsewhere (the residual stream's).  The 8-bit rows' gradient is
 * dy too (rounding is passed straight through).  The rows' sum is taken in a fixed
 * order: the same call gives the same bits. */
typedef struct {
    int32_t dtype;       /* of dy, h, weight, dh, dx, dweight                       */
    int32_t pad_;
    int64_t rows, cols;
    const void* dy;
    int64_t ld_dy;
    const void* h;       /* the h of zero_rms_norm (x where it had no residual)     */
    int64_t ld_h;
    const void* weight;
    const float* rstd;   /* [rows], of zero_rms_norm                                */
    const void* dh;      /* NULL: none                                              */
    int64_t ld_dh;
    void* dx;            /* may be dy, dh or h in place                             */
    int64_t ld_dx;
    void* dweight;       /* [cols]; 0 where rows = 0                                */
    float* workspace;    /* zero_rms_norm_workspace(rows, cols) floats; NULL if 0   */
    int64_t workspace_floats;
} zero_rms_norm_backward_args_t;

int zero_rms_norm_backward(const zero_rms_norm_backward_args_t* args, void* stream);

/* Floats of workspace that zero_rms_norm_backward needs, into *floats (host): at
 * most 1024 * cols.  ZERO_EINVAL for sizes the call does not take. */
int zero_rms_norm_workspace(int64_t rows, int64_t cols, int64_t* floats);

/* ------------------------------------------------------------------------ */
/* Routing to experts                                                       */
/* ------------------------------------------------------------------------ */

#define ZERO_ROUTE_MAX_EXPERTS 1024
#define ZERO_ROUTE_MAX_K 64
#define ZERO_SCORE_SOFTMAX 0
#define ZERO_SCORE_SIGMOID 1

/* Each token takes the k experts with the largest keys, equal keys by the lowest
 * expert, in falling order:
 *   sigmoid: key = 1 / (1 + exp(-logit)) + bias
 *   softmax: key = logit + bias, the order of exp(bias) * softmax.  (Loss-free balancing as it
 *            is published adds the bias to the probability: softmax + bias.  Where biases differ
 *            that rule can choose other experts, and a bias trained for one does not serve the
 *            other.  group_top = 2 likewise adds two keys, not two probabilities.)
 * The bias balances the experts' loads: it acts on the choice alone.  An expert
 * is out where its logit or its bias is -inf: it is neither chosen nor part of a sum.
 * With groups > 1 the experts are cut into that many equal runs; a group's score
 * is the sum of its group_top (1 or 2) largest keys, and the choice is among the
 * top_groups groups of the largest scores (equal ones by the lowest group).  Keys
 * and scores that are NaN or -inf are never chosen; where no expert is left a slot
 * gets index -1 and weight 0.
 * The weight of a chosen expert is scale times its score without bias:
 *   softmax: exp(logit) / sum of exp(logit) over the experts that are in, or with
 *            renormalise over the chosen ones
 *   sigmoid: 1 / (1 + exp(-logit)), with renormalise divided by the chosen ones' sum
 *            (by 2^-126 if that is less)
 * A NaN among the logits of experts that are in makes the token's weights NaN (of
 * its slots with an expert). */
typedef struct {
    int32_t dtype;       /* of logits                                               */
    int32_t score;       /* ZERO_SCORE_*                                            */
    int64_t rows;        /* tokens; rows * k < 2^31                                 */
    int32_t experts, k;  /* k <= experts                                            */
    int32_t groups, top_groups, group_top; /* groups divides experts, at most 64; group_top = 2
                                              needs groups of two or more           */
    int32_t renormalise;
    double scale;        /* finite in fp32                                          */
    const void* logits;  /* [rows, experts]                                         */
    int64_t ld_logits;
    const float* bias;   /* [experts]; NULL: none                                   */
    int32_t* index;      /* [rows, k]                                               */
    float* weight;       /* [rows, k]                                               */
} zero_route_args_t;

int zero_route(const zero_route_args_t* args, void* stream);

/* The slots (slot t * k + i is the i-th choice of token t) ordered by expert and
 * then by slot: order[offsets[e] .. offsets[e+1]) are expert e's.  Slots without an
 * expert (an index outside [0, experts)) come in no run: order's last
 * slots - offsets[experts] entries are -1. */
typedef struct {
    const int32_t* index; /* [slots]                                                */
    int64_t slots;        /* < 2^31                                                 */
    int32_t experts, pad_;
    int32_t* offsets;     /* [experts + 1]                                          */
    int32_t* order;       /* [slots]                                                */
    int32_t* workspace;   /* zero_route_workspace(slots, experts) ints; NULL if 0   */
    int64_t workspace_ints;
} zero_route_order_args_t;

int zero_route_order(const zero_route_order_args_t* args, void* stream);

/* Ints of workspace that zero_route_order needs, into *ints (host): at most
 * 1024 * (experts + 1). */
int zero_route_workspace(int64_t slots, int32_t experts, int64_t* ints);

/* The gradient of the logits from the weights' (the choice itself has none): with
 * d_i = scale * dweight_i and s the scores,
 *   softmax:                  dlogit_e = s_e * (d_e - sum_j d_j s_j), d_e = 0 for the rest
 *   softmax, renormalised:    the same over the chosen ones, 0 for the rest
 *   sigmoid:                  dlogit_i = d_i s_i (1 - s_i), 0 for the rest; 1 - s_i is taken from
 *                             the logit, so saturated scores keep their slope
 *   sigmoid, renormalised:    d_i replaced by (d_i - sum_j d_j s_j / S) / S, S = sum_j s_j
 * Experts that are out get 0.  `index` holds no expert twice in a row. */
typedef struct {
    int32_t dtype;       /* of logits and dlogits                                   */
    int32_t score;
    int64_t rows;
    int32_t experts, k;
    int32_t renormalise, pad_;
    double scale;
    const void* logits;
    int64_t ld_logits;
    const float* bias;   /* as given to zero_route                                  */
    const int32_t* index;
    const float* dweight; /* [rows, k]; not looked at in slots without an expert    */
    void* dlogits;       /* [rows, experts]; may be logits in place                 */
    int64_t ld_dlogits;
} zero_route_backward_args_t;

int zero_route_backward(const zero_route_backward_args_t* args, void* stream);

/* ------------------------------------------------------------------------ */
/* Distillation from a teacher's top logits                                 */
/* ------------------------------------------------------------------------ */

#define ZERO_DISTILL_MAX_K 1024

/* A row's teacher is a list of at most k entries, each a token and its logit; an
 * entry is absent where its token lies outside [0, vocab) or its logit is -inf.
 * With tau the temperature, p = softmax of the present entries' logits / tau and
 * q_T = softmax of the row's student logits z / T,
 *   loss = row_weight * ( soft * tau^2 * sum_j p_j (log p_j - log q_tau[token_j])
 *                         - hard * log q_1[label] )
 * The soft term is 0 in a row without entries (and where p_j = 0), the hard term in
 * one whose label lies outside [0, vocab); a row of weight 0 has loss 0 and is not
 * looked at.  A token listed twice counts twice.  The soft term is formed from differences
 * of logits times soft * tau, so it is finite where its value is (a student masked by its
 * type's lowest value included); its logarithms' rounding, 2^-20 or so, counts tau^2 times.
 * The gradient, with u = grad_scale * row_weight (* dloss where that is given):
 *   dlogits_v = u * ( soft * tau * (q_tau[v] - sum of p_j over entries of token v)
 *                     + hard * (q_1[v] - [v = label]) )
 * each term where the row has it.
 * zero_distill_step gives both from one read of the logits (of two where a row does
 * not fit a workgroup's registers); zero_distill_loss gives the loss and, for
 * zero_distill_backward with the same record, each row's statistics. */
typedef struct {
    int32_t dtype;         /* of logits and dlogits                                 */
    int32_t teacher_dtype; /* of teacher_logits                                     */
    int64_t rows, vocab;   /* vocab in [1, 2^30]                                    */
    int32_t k, pad_;       /* entries a row, 0 <= k <= ZERO_DISTILL_MAX_K           */
    double temperature;    /* in [1e-30, 1e30]                                      */
    double soft, hard;     /* soft * temperature and hard finite in fp32            */
    double grad_scale;     /* finite in fp32; the loss scale                        */
    const void* logits;    /* [rows, vocab]                                         */
    int64_t ld_logits;
    const int32_t* teacher_index;  /* [rows, k], close together; NULL if k = 0      */
    const void* teacher_logits;    /* [rows, k]                                     */
    const int32_t* labels;         /* [rows]; NULL: no hard term                    */
    const float* row_weight;       /* [rows]; NULL: 1                               */
    float* loss;           /* [rows]; written by the step and the loss, NULL in the backward */
    float* stats;          /* [rows, 3]; written by the loss (NULL: not wanted), read by the
                              backward, NULL in the step                            */
    const float* dloss;    /* [rows], the backward's only; NULL: 1                  */
    void* dlogits;         /* [rows, vocab]; the step's and the backward's (NULL in the loss);
                              may be logits in place                                */
    int64_t ld_dlogits;
} zero_distill_args_t;

int zero_distill_step(const zero_distill_args_t* args, void* stream);
int zero_distill_loss(const zero_distill_args_t* args, void* stream);
int zero_distill_backward(const zero_distill_args_t* args, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ZERO_OPERATORS_H */
