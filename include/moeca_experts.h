/*
 * moeca_experts.h -- tokens sorted by expert and back, with their gradients
 * (Eq. 5 / 6 around the experts' products).
 *
 * A layer's branches (token, slot) are worked on expert by expert.
 * moeca_expert_sort orders them: rows of expert 0 first, then expert 1's, each
 * expert's by token and slot.  moeca_expert_rows copies the tokens' rows into
 * that order, the experts' products run on them (grouped by `offsets`, as
 * moeca_q8_matmul takes them), and moeca_expert_combine adds the weighted
 * results to their tokens.  moeca_expert_combine_grad gives the gradients of
 * that sum; the gradient of moeca_expert_rows is moeca_expert_combine without
 * weights and residual.
 *
 * Conventions.  As in moeca_q8.h: row-major, borrowed device buffers of the
 * current device, asynchronous on `stream`, arguments checked on the host
 * before anything is launched, a moeca_status back, the message of a failure
 * from moeca_last_error(NULL) on the same thread.  Nothing is allocated and
 * nothing kept between calls; calls may run at once on several streams (with a
 * workspace each) and be captured into graphs.  Buffers that a call writes must
 * not overlap its others unless stated (INVALID_ARG where the ranges do).
 * Results do not depend on the order in which blocks run.
 */
#ifndef MOECA_EXPERTS_H_
#define MOECA_EXPERTS_H_

#include "moeca.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sort N = n_tokens x n_slots branches by expert, stably.  An id outside
 * [0, n_experts) is a branch that is not sorted (an empty slot, or one served
 * from the cache): its place is -1 and it has no row.  N at most 2^30. */
typedef struct {
  const int32_t* experts;  /* [n_tokens, n_slots]                                    */
  int32_t n_tokens;        /* >= 0                                                   */
  int32_t n_slots;         /* 1 .. 16                                                */
  int32_t n_experts;       /* 1 .. 512                                               */
  int32_t* offsets;        /* [n_experts + 1]: expert e's rows are offsets[e] ..
                              offsets[e + 1] - 1; the last is the number of rows     */
  int32_t* place;          /* [n_tokens, n_slots]: the branch's row, or -1           */
  int32_t* slot;           /* [N]: the row's branch, token n_slots + slot; -1 behind
                              the last row.  May be NULL                             */
  int32_t* token;          /* [N]: the row's token; -1 behind the last.  May be NULL */
  int32_t* workspace;      /* moeca_expert_sort_workspace() values; NULL where that
                              is 0                                                   */
} moeca_expert_sort_args;
moeca_status moeca_expert_sort(const moeca_expert_sort_args* args, void* stream);
/* int32 values that moeca_expert_sort works in; -1 where a size is out of range. */
int64_t moeca_expert_sort_workspace(int32_t n_tokens, int32_t n_slots, int32_t n_experts);

/* rows[place[t, p]] <- x[t] for every branch whose place is in [0, n_rows).
 * With `count` (the last entry of offsets, on the device) the rows from *count
 * on become zeros; without it they keep what they hold.  Two branches with one
 * place leave either's row.  Rows must not overlap one another. */
typedef struct {
  const void* x;         /* [n_tokens] rows                                          */
  int64_t x_stride;      /* elements from row to row, >= width                       */
  void* rows;            /* [n_rows] rows                                            */
  int64_t rows_stride;   /* elements                                                 */
  int64_t n_rows;        /* 0 .. 2^31 - 1                                            */
  const int32_t* place;  /* [n_tokens, n_slots]                                      */
  const int32_t* count;  /* device count of rows in use, or NULL                     */
  int32_t dtype;         /* moeca_dtype of x and rows                                */
  int32_t n_tokens;      /* >= 0                                                     */
  int32_t n_slots;       /* 1 .. 16                                                  */
  int32_t width;         /* values per row, 1 .. 2^20                                */
} moeca_expert_rows_args;
moeca_status moeca_expert_rows(const moeca_expert_rows_args* args, void* stream);

/* out[t] = x[t] + sum_p weights[t, p] rows[place[t, p]]: sums in fp32, slot by
 * slot, rounded once.  A place outside [0, n_rows) adds nothing, whatever its
 * weight. */
typedef struct {
  const void* rows;      /* [n_rows] rows                                            */
  int64_t rows_stride;   /* elements                                                 */
  int64_t n_rows;        /* 0 .. 2^31 - 1                                            */
  const int32_t* place;  /* [n_tokens, n_slots]                                      */
  const float* weights;  /* [n_tokens, n_slots], or NULL: 1                          */
  const void* x;         /* [n_tokens] rows, the residual; NULL: 0                   */
  int64_t x_stride;      /* elements                                                 */
  void* out;             /* [n_tokens] rows; may be x itself (same base and stride)  */
  int64_t out_stride;    /* elements                                                 */
  int32_t dtype;         /* moeca_dtype of rows, x and out                           */
  int32_t n_tokens;      /* >= 0                                                     */
  int32_t n_slots;       /* 1 .. 16                                                  */
  int32_t width;         /* values per row, 1 .. 2^20                                */
} moeca_expert_combine_args;
moeca_status moeca_expert_combine(const moeca_expert_combine_args* args, void* stream);

/* Gradients of moeca_expert_combine for the gradient dout of its result (x's
 * own gradient is dout):
 *   drows[place[t, p]] = weights[t, p] dout[t]                (rounded once)
 *   dweights[t, p]     = sum_d dout[t, d] rows[place[t, p], d]  (fp32 sums)
 * dweights is 0 where the place is outside [0, n_rows).  Rows of drows behind
 * *count are zeros, or keep what they hold, as in moeca_expert_rows. */
typedef struct {
  const void* dout;      /* [n_tokens] rows                                          */
  int64_t dout_stride;   /* elements                                                 */
  const void* rows;      /* [n_rows] rows; may be NULL without dweights              */
  int64_t rows_stride;   /* elements                                                 */
  int64_t n_rows;        /* 0 .. 2^31 - 1                                            */
  const int32_t* place;  /* [n_tokens, n_slots]                                      */
  const float* weights;  /* [n_tokens, n_slots], or NULL: 1                          */
  const int32_t* count;  /* device count of rows in use, or NULL                     */
  void* drows;           /* [n_rows] rows, or NULL                                   */
  int64_t drows_stride;  /* elements                                                 */
  float* dweights;       /* [n_tokens, n_slots], or NULL                             */
  int32_t dtype;         /* moeca_dtype of dout, rows and drows                      */
  int32_t n_tokens;      /* >= 0                                                     */
  int32_t n_slots;       /* 1 .. 16                                                  */
  int32_t width;         /* values per row, 1 .. 2^20                                */
} moeca_expert_combine_grad_args;
moeca_status moeca_expert_combine_grad(const moeca_expert_combine_grad_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOECA_EXPERTS_H_ */
