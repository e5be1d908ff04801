/*
 * moeca_attention.h -- the attention sub-layer on packed tokens: norms of query
 * and key heads with the position rotation, and attention over sequences of
 * different lengths (Sec. 3's F_SA, without a handle).
 *
 * The stack's own attention (moeca.h) takes samples of one length.  These calls
 * take the tokens of all sequences one after another, as a fused projection
 * leaves them: a head is dim consecutive values, heads and tokens are any
 * stride apart.  Serving only: no gradients.
 *
 * Conventions.  As in moeca_experts.h.
 */
#ifndef MOECA_ATTENTION_H_
#define MOECA_ATTENTION_H_

#include "moeca.h"

#ifdef __cplusplus
extern "C" {
#endif

/* [n_tokens] tokens of `heads` heads; strides in elements, both >= 0. */
typedef struct {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
  int32_t heads;
} moeca_heads;

/* For every token and every head x of q (weight wq) and k (weight wk):
 *   y = x / sqrt(mean(x^2) + eps) * weight
 * and the first `rot` values of y are turned by the token's row of the table,
 *   (a, b) -> (a cos - b sin, b cos + a sin),
 * pair i being (y[i], y[i + rot / 2]), or (y[2 i], y[2 i + 1]) with `pairs`.
 * All in fp32, rounded once; heads whose sum of squares passes fp32's largest value
 * become 0.  A token whose position is outside
 * [0, n_positions) is left out: nothing is written for it, or zeros (`clear`).  q_out and k_out may
 * be q and k themselves (same base and strides).  With rot = 0 positions are not
 * looked at. */
typedef struct {
  moeca_heads q, k;        /* read; k.heads = 0: no keys                             */
  moeca_heads q_out, k_out;/* written; as many heads                                 */
  const float* q_weight;   /* [dim], or NULL: 1                                      */
  const float* k_weight;   /* [dim], or NULL: 1                                      */
  const float* table;      /* [n_positions, rot / 2, 2]: cos and sin, 8-byte aligned;
                              NULL with rot = 0                                      */
  const int32_t* pos;      /* [n_tokens] rows of the table, or NULL: the token's
                              number                                                 */
  int64_t n_positions;     /* 0 .. 2^31 - 1                                          */
  int32_t dtype;           /* moeca_dtype of q, k and the results                    */
  int32_t n_tokens;        /* >= 0                                                   */
  int32_t dim;             /* values per head, 1 .. 512                              */
  int32_t rot;             /* values turned, even, 0 .. dim                          */
  int32_t pairs;           /* 0 / 1                                                  */
  float eps;               /* >= 0                                                   */
  int32_t clear;           /* results in which tokens that are left out become 0: the sum
                              of 1 (q_out) and 2 (k_out), or 0                       */
} moeca_qk_norm_rope_args;
moeca_status moeca_qk_norm_rope(const moeca_qk_norm_rope_args* args, void* stream);

/* Attention of every sequence's queries over its keys:
 *   o_i = sum_j p_ij v_j,  p_i = softmax over j of (scale q_i . k_j)
 * over the sequence's keys j, with `causal` over j <= i + (keys - queries) (the
 * last query sees the last key; one new token after a prompt is a query of
 * length 1).  Query head h reads key head h / (q.heads / k.heads).  A row that
 * sees no key (a sequence without keys, the first rows of a longer query under
 * `causal`), or whose every score is -infinity, is 0 with lse = -infinity.
 *
 * Sequence b's queries are tokens q_offsets[b] .. q_offsets[b + 1] - 1, its keys
 * k_offsets[b] .. k_offsets[b + 1] - 1; offsets ascend and are clamped to the
 * tokens there are.  Without offsets all sequences are equally long.  Query
 * tokens that are not computed keep what out and lse hold, unless `clear` says
 * otherwise: those of no sequence (before q_offsets[0], from q_offsets[n_seqs]
 * on), and a sequence's behind its first max_q.
 *
 * Scores, softmax statistics and sums are fp32, the exponential in base 2; its
 * argument's error does not grow with the scores' size.  With bf16 values p is
 * rounded to bf16 before it meets v, the sum of p is not.  Keys and values behind a
 * sequence's end are never looked at, whatever they hold, nor do other sequences'
 * queries change a result; a value that is not finite may reach, by 0 x infinity,
 * rows of its own sequence that `causal` hides it from.
 * Splits of the key axis are joined in a fixed order.
 * UNSUPPORTED: above 2^30 tokens, or tiles beyond a grid's 2^31 - 1. */
typedef struct {
  moeca_heads q;             /* read                                                 */
  moeca_heads k, v;          /* read; q.heads is a multiple of k.heads = v.heads     */
  moeca_heads out;           /* written; q.heads heads; may be q itself (same base
                                and strides)                                         */
  const int32_t* q_offsets;  /* [n_seqs + 1] device, or NULL: n_queries / n_seqs each */
  const int32_t* k_offsets;  /* [n_seqs + 1] device, or NULL: n_keys / n_seqs each   */
  float* lse;                /* [n_queries, q.heads] or NULL: log of the sum of
                                exponentials of the scores                           */
  void* workspace;           /* moeca_attention_workspace() bytes, 16-byte aligned;
                                NULL where that is 0                                 */
  int32_t* status;           /* device int32 [2] of zeros, or NULL: [0] becomes
                                MOECA_ERR_TIMEOUT if one of the kernel's bounded
                                waits ran out (the output is then incomplete)        */
  int64_t n_queries;         /* query tokens                                         */
  int64_t n_keys;            /* key tokens                                           */
  int32_t n_seqs;            /* 1 .. 2^20                                            */
  int32_t max_q;             /* the longest query; 0: not known                      */
  int32_t dtype;             /* moeca_dtype of q, k, v and out                       */
  int32_t dim;               /* values per head, 1 .. 256                            */
  int32_t causal;            /* 0 / 1                                                */
  int32_t clear;             /* 1: query tokens that are not computed become 0 (lse
                                -infinity); 2: only their lse is written; 0: nothing */
  float scale;               /* > 0, scale log2(e) at most fp32's largest value      */
} moeca_attention_args;
moeca_status moeca_attention(const moeca_attention_args* args, void* stream);
/* Bytes that moeca_attention with these arguments works in (device pointers are
 * not looked at but for their alignment); -1 where sizes, types or strides would be
 * refused, or the tokens are too many. */
int64_t moeca_attention_workspace(const moeca_attention_args* args);

#ifdef __cplusplus
}
#endif
#endif /* MOECA_ATTENTION_H_ */
