/*
 * moeca_q8.h -- 8-bit rows: branch caches held in 8 bits and 8-bit expert
 * products (no counterpart in the paper, which keeps its caches in 16 bits).
 *
 * A branch cache is the largest buffer of a trajectory: T k D values a layer.
 * These calls write such rows in 8 bits as they are produced, combine (Eq. 8)
 * or read them back, and multiply 8-bit activations by 8-bit expert weights,
 * the product's rows going to the next product or to their cache slots in 8
 * bits again.  None needs a handle; none allocates.
 *
 * Format.  A row of `width` values is `width` bytes (e4m3: no infinities, NaN
 * 0x7F / 0xFF, largest 448; or e5m2: largest 57344) and ceil(width / 128)
 * scale bytes.  Scale byte s stands for 2^(s - 127) (255: NaN) and belongs to
 * 128 consecutive values, the last block to the rest of the row: value =
 * byte x scale.  Writing a block: with a its largest finite magnitude and MAX
 * the format's, the scale is the smallest power of two (at least 2^-127) with
 * a <= MAX x scale, 1 where a = 0; a value is x / scale (exact, the scale
 * being a power of two) rounded to the nearest of the format, ties to even.
 * NaN stays NaN; an infinity stays one in e5m2 and becomes NaN in e4m3.
 *
 * Conventions.  As in moeca.h: row-major, borrowed device buffers of the
 * current device, asynchronous on `stream`, a moeca_status back, the message
 * of a failure from moeca_last_error(NULL) on the same thread.  Arguments are
 * checked on the host before anything is launched.  Row lists and counts are
 * device data, read by the kernel: an entry outside its range is skipped, as
 * stated at each call, and nothing is read or written for it.  Calls may be
 * captured into a graph, run at the same time on several streams or threads,
 * and share nothing.  Buffers that a call writes must not overlap its others
 * unless stated (INVALID_ARG where the address ranges do).
 */
#ifndef MOECA_Q8_H_
#define MOECA_Q8_H_

#include "moeca.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Formats beside MOECA_F32 and MOECA_BF16. */
typedef enum { MOECA_E4M3 = 2, MOECA_E5M2 = 3 } moeca_q8_format;

/* Rows in 8 bits; as a product's output also rows of fp32 or bf16.  Rows are read
 * in pieces of 16 bytes and scales in words, the last ones to their end. */
typedef struct {
  void* q;               /* [rows] rows of `width` bytes, 16-byte aligned             */
  uint8_t* scale;        /* [rows] rows of ceil(width / 128) bytes, 4-byte aligned    */
  int64_t rows;          /* 0 .. 2^31 - 1                                             */
  int64_t q_stride;      /* bytes from row to row: a multiple of 16, >= width         */
  int64_t scale_stride;  /* bytes from row to row: a multiple of 4, >= ceil(width/128) */
  int32_t width;         /* values per row, 1 .. 2^20                                 */
  int32_t format;        /* moeca_q8_format                                           */
} moeca_q8_rows;

/* Quantise rows into a cache: cache row dst[i] <- x row src[i] for
 * 0 <= i < n (n = *count where count is given, at most args->n).  An entry
 * whose src or dst is out of its range (negative included) is skipped.  The
 * other rows of the cache, and the bytes of a row past its width, keep what
 * they hold.  Two entries with one dst leave a mix of their rows there. */
typedef struct {
  moeca_q8_rows cache;   /* written                                                   */
  const void* x;         /* [x_rows] rows of cache.width values                       */
  int64_t x_rows;        /* 0 .. 2^31 - 1                                             */
  int64_t x_stride;      /* elements from row to row, >= width (any base alignment of
                            the type; 16-byte aligned base and rows are faster)       */
  int32_t dtype;         /* moeca_dtype of x                                          */
  int32_t n;             /* entries, >= 0; without a list at most that side's rows    */
  const int32_t* src;    /* [n] rows of x, or NULL: i                                 */
  const int32_t* dst;    /* [n] rows of the cache, or NULL: i                         */
  const int32_t* count;  /* device count of entries, or NULL: n                       */
} moeca_q8_write_args;
moeca_status moeca_q8_write(const moeca_q8_write_args* args, void* stream);

/* Read cache rows back: out row i <- cache row rows[i], 0 <= i < n; a row of
 * zeros where rows[i] is out of range. */
typedef struct {
  moeca_q8_rows cache;   /* read                                                      */
  void* out;             /* [n] rows of cache.width values                            */
  int64_t out_stride;    /* elements from row to row, >= width                        */
  int32_t dtype;         /* moeca_dtype of out                                        */
  int32_t n;             /* rows of out, >= 0; without a list at most cache.rows      */
  const int32_t* rows;   /* [n] rows of the cache, or NULL: i                         */
  int32_t* status;       /* as in moeca_q8_matmul_args                                */
} moeca_q8_read_args;
moeca_status moeca_q8_read(const moeca_q8_read_args* args, void* stream);

/* Eq. 8 over an 8-bit branch cache: for token i < n_tokens
 *   out_i = x_i + g_(i / seq) * sum_p weights[i, p] h_(i, p)
 * with h_(i, p) the cache row rows[i, p], p < n_slots (a shared expert's
 * output is one more slot of weight 1).  A slot whose row is out of range
 * holds nothing: it adds nothing, whatever its weight.  h is the cache's value
 * in fp32 (exact; an infinity past fp32's largest), sums are fp32, slot by slot,
 * and the result is rounded once.  norms[i, p] = ||h_(i, p)|| over the row
 * (Eq. 9's history), 0 for a slot that holds nothing; the sum of squares is
 * fp32: rows of a norm above 1.8e19 have an infinite one, squares below 1.4e-45
 * count nothing. */
typedef struct {
  moeca_q8_rows cache;   /* read                                                      */
  const int32_t* rows;   /* [n_tokens, n_slots]                                       */
  const float* weights;  /* [n_tokens, n_slots], or NULL: 1                           */
  const void* x;         /* [n_tokens] rows, the residual; NULL: 0                    */
  int64_t x_stride;      /* elements                                                  */
  const float* gate;     /* [ceil(n_tokens / seq)] rows (AdaLN gate), or NULL: 1      */
  int64_t gate_stride;   /* elements                                                  */
  void* out;             /* [n_tokens] rows; may be x itself (same base and stride)   */
  int64_t out_stride;    /* elements                                                  */
  float* norms;          /* [n_tokens, n_slots], or NULL                              */
  int32_t dtype;         /* moeca_dtype of x and out                                  */
  int32_t n_tokens;      /* >= 0                                                      */
  int32_t n_slots;       /* 1 .. 16                                                   */
  int32_t seq;           /* tokens per gate row, >= 1 (with a gate)                   */
  int32_t* status;       /* as in moeca_q8_matmul_args                                */
} moeca_q8_combine_args;
moeca_status moeca_q8_combine(const moeca_q8_combine_args* args, void* stream);

/* Activation of a product's rows (Eq. 5's GELU). */
typedef enum { MOECA_ACT_NONE = 0, MOECA_ACT_GELU = 1, MOECA_ACT_GELU_TANH = 2 } moeca_q8_act;

/* Grouped product of 8-bit rows:
 *   out row dst[m] = act(sum_k a[m, k] b[g n_cols + c, k] + bias[g, c]), c < n_cols,
 * for the rows offsets[g] <= m < offsets[g + 1] of every group g (an expert):
 * a holds one group's rows after another's, b every group's n_cols weight
 * rows, both K = width values wide.  Sums are fp32 as the tensor core adds them,
 * truncating (relative error about 7e-8 at K = 1152 and 3e-7 at 4608, where fp32
 * with rounding has 4e-8 and 6e-8); GELU is z (1 + h) / 2 in fp32, within 6 x 2^-24 |z|
 * of the function and 0 where h rounds to -1; the result is rounded once, to out's
 * format.  Rows outside the groups are not computed.  Offsets
 * are clamped to [0, a.rows], a group that would end before it starts is
 * empty; rows that two groups claim hold either's result.  An entry of dst
 * out of [0, out.rows) drops its row; entries are distinct.  Rows of out that
 * no entry names, and bytes past a row's width, keep what they hold.
 * MOECA_ERR_UNSUPPORTED above 2^30 rows of a or b, or where (a.rows / 16 +
 * n_groups) x ceil(n_cols / 256), or (ceil(n_groups / 2) x a.rows / 224 +
 * n_groups) x ceil(n_cols / 256), passes 2^30 (tiles are counted in 32 bits,
 * and offsets that step back may claim every row again and again). */
typedef struct {
  moeca_q8_rows a;         /* activations                                             */
  moeca_q8_rows b;         /* weights: rows = n_groups x n_cols, width = a.width      */
  moeca_q8_rows out;       /* width = n_cols; format MOECA_E4M3 / E5M2 (8-bit rows), or
                              MOECA_F32 / BF16: q and q_stride (bytes) aligned to the
                              type (16 bytes: faster), scale not used                 */
  const int32_t* offsets;  /* [n_groups + 1] device, or NULL: one group of all rows   */
  const float* bias;       /* [n_groups, n_cols] device, or NULL                      */
  const int32_t* dst;      /* [a.rows] device rows of out, or NULL: m                 */
  int32_t* status;         /* device int32 [2] of zeros, or NULL: [0] becomes
                              MOECA_ERR_TIMEOUT if one of the kernel's bounded waits
                              ran out (the output is then incomplete)                 */
  int32_t n_groups;        /* 1 .. 512 (1 where offsets is NULL)                     */
  int32_t n_cols;          /* N >= 1                                                  */
  int32_t act;             /* moeca_q8_act                                            */
} moeca_q8_matmul_args;
moeca_status moeca_q8_matmul(const moeca_q8_matmul_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOECA_Q8_H_ */
