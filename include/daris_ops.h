/*
 * daris_ops.h -- operators of a generation step: the chain that one token (or a few, or a chunk of a prompt) takes through a
 * decoder block, for programs that run a generating model on a partition next to the tasks of daris.h.
 *
 *     norm -> product -> append -> attend -> product -> norm -> gated product -> product
 *
 * An operator is a descriptor that names buffers of the caller; daris_run_ops runs a list of them.  The general rules of
 * daris.h apply (status codes, nothing throws or aborts, one API thread).  In addition:
 *   - Every pointer is HIP memory of the library's GPU, aligned to its element, and stays valid until the call returns.  Channels
 *     of a row (or head) lie side by side; distances between rows and heads ("_row", "_head") count elements, may be anything
 *     that keeps distinct elements of an output apart, and default to nothing: 0 is the distance 0.
 *   - dtype is DARIS_FP32 or DARIS_BF16: the type of activations.  Sums, softmax statistics and norms are fp32; an output is rounded
 *     once.  Matrix products take what is fp32 -- queries, weights of the softmax, rows of x -- in two f16 parts (22 bits), divided by
 *     powers of two so that none overflows; bf16 queries and weights of the softmax in one, bf16 rows of x as they are.  Codes are exact.
 *     What a weight of the softmax has below 2^-35 of its row's largest (times their values' scales) is lost, in an output whose larger terms are zero, too.
 *     A row of a norm with numbers above 1e19, whose squares pass fp32, gives zeros, and scores (scale * q.k) above 1e7, which fp32 holds
 *     to the next whole number only, leave their row of attention open.
 *   - Eight bits are e4m3 numbers (OCP, no infinity, largest 448) and e8m0 scales, one byte each: 2^(byte - 127).  A group's scale is
 *     the smallest power of two, 2^-100 at least, that leaves none of its finite numbers above 448; a number that is not finite
 *     becomes the NaN code and has no part in the scale.
 *   - Counts (rows, channels, outputs, sequences) are 2^30 at most; distances are 64 bits wide and may pass 32.
 *   - Lengths and page numbers lie in device memory and change from step to step while the descriptors stay.  The kernels check
 *     them: what they say is outside a buffer is not there.
 */
#ifndef DARIS_OPS_H
#define DARIS_OPS_H

#include "daris.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { DARIS_STEP_NORM = 0, DARIS_STEP_APPEND = 1, DARIS_STEP_ATTEND = 2, DARIS_STEP_MATVEC = 3 };
enum { DARIS_PAGE_TOKENS = 64, DARIS_SCALE_TOKENS = 16 };

/*
 * Root-mean-square norm of rows, after the addition of a residual.
 *   h = x + res (res may be NULL: h = x);  sum = h in dtype (NULL: not stored; may be x or res itself)
 *   y = h / sqrt(mean(h^2) + eps) * weight, from the unrounded h
 * With scale == NULL y is of dtype.  Otherwise y is e4m3 and scale[row][width / group] (dense) holds the scales of `group` =
 * 32, 64 or 128 neighbouring channels; width is then a multiple of it.
 */
typedef struct daris_norm {
  const void* x;
  const void* res;
  const void* weight; /* [width] of dtype */
  void* sum;
  void* y;
  uint8_t* scale;
  int64_t x_row, res_row, sum_row, y_row;
  int32_t rows, width, group, dtype;
  float eps;
} daris_norm;

/*
 * A cache of keys and values in pages of DARIS_PAGE_TOKENS tokens, eight bits a number; DARIS_SCALE_TOKENS neighbouring tokens
 * of a page and head share a scale.  Dense:
 *   k [n_pages][kv_heads][64][dim]   v [n_pages][kv_heads][dim][64]   k_scale, v_scale [n_pages][kv_heads][4]
 * Token t of sequence s is token t mod 64 of page pages[s * pages_row + t / 64].  A page number outside 0 .. n_pages - 1, and
 * a token past the row's pages_row entries, stands for a page that is not there: its tokens are neither written nor attended.
 * before[s]: tokens of sequence s in front of this step's.  No page may belong to two places of the table that one call
 * writes.  dim is 64, 128 or 256.  k and v are aligned to 16 bytes, the scales, pages and before to 4.
 */
typedef struct daris_cache {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* pages;
  const int32_t* before;
  int64_t pages_row;
  int32_t n_pages, n_seqs, kv_heads, dim;
} daris_cache;

/*
 * Rows of the step, for both operators on a cache: rows row_start[s] .. row_start[s + 1] - 1 of the buffers are the new tokens
 * before[s], before[s] + 1, ... of sequence s (row_start: device int32[n_seqs + 1], not decreasing, from 0 to n_rows; rows of
 * no sequence are left alone).  row_start == NULL: n_rows == n_seqs, row s is sequence s's.
 *
 * Appends k and v [n_rows][kv_heads][dim] to the cache.  Positions are applied on the way: of the first rot_dim channels of
 * a key's head (even, 0 = none, at most dim), channels j and j + rot_dim / 2 -- or, with pairs != 0, 2j and 2j + 1 --
 * are turned by the angle whose cosine and sine are turn[position][j] and turn[position][rot_dim / 2 + j] (device
 * float[turn_rows][rot_dim]; any base or scaling for long contexts is a matter of this table; a position outside
 * it has NaN there).  q [n_rows][q_heads][dim], if not NULL, is turned the same way into q_out (of dtype; may be q itself).
 * A sixteenth that has tokens already gets the larger of its scale and the new tokens' own, its codes rounded again (exact but for
 * e4m3's subnormals).  What its places behind the last token hold stays.
 */
typedef struct daris_append {
  daris_cache cache;
  const void* k;
  const void* v;
  const void* q;
  void* q_out;
  const float* turn;
  const int32_t* row_start;
  int64_t k_row, k_head, v_row, v_head, q_row, q_head, qo_row, qo_head;
  int32_t n_rows, q_heads, dtype, turn_rows, rot_dim, pairs;
} daris_append;

/*
 * Attention of q [n_rows][q_heads][dim] over the cache, which holds the step's own tokens already: the row of position p
 * attends tokens p - window + 1 .. p of its sequence (window == 0: 0 .. p) with weights softmax(scale * q.k), |scale| <= 1e38; query head
 * h reads key head h / (q_heads / kv_heads).  out [n_rows][q_heads][dim] of dtype; a row that attends nothing gets zeros.  Tokens
 * that a row does not attend have no influence on it, NaN included.
 */
typedef struct daris_attend {
  daris_cache cache;
  const void* q;
  void* out;
  const int32_t* row_start;
  int64_t q_row, q_head, out_row, out_head;
  int32_t n_rows, q_heads, dtype, window;
  float scale;
} daris_attend;

/*
 * Products of a few rows with 4-bit weights: r[row][i] = sum_k x[row][k] * (code(i, k) - 8) * w_scale[i][k / group].
 * w [n][k / 2] bytes, the earlier k in the low half of a byte, rows w_row bytes apart; w and w_row are multiples of 16;
 * w_scale bf16 [n][k / group] dense; group 32, 64 or 128, k a multiple of it.  x is of dtype, or, with x_scale != NULL, e4m3 with
 * scales x_scale[rows][k / group] (dense), as a norm of the same group leaves them.
 * A row that holds an infinity or a NaN has outputs that are not finite (which of them is left open).  K may be shared between workgroups by the
 * partition's size, so that the last bits differ from partition to partition, but not from call to call.
 * gate == 0: y[row][i] = r[row][i].  gate != 0: n is even, y[row][i] = silu(r[row][2i]) * r[row][2i + 1], n / 2 columns.
 */
typedef struct daris_matvec {
  const void* x;
  const uint8_t* x_scale;
  const uint8_t* w;
  const uint16_t* w_scale;
  void* y;
  int64_t x_row, w_row, y_row;
  int32_t rows, n, k, group, dtype, gate;
} daris_matvec;

typedef struct daris_op {
  int32_t kind; /* DARIS_STEP_... : which member counts */
  int32_t reserved; /* 0 */
  union {
    daris_norm norm;
    daris_append append;
    daris_attend attend;
    daris_matvec matvec;
  } u;
} daris_op;

typedef int32_t daris_plan; /* handle of a planned list of operators; <0 is an error code */

/* Runs n operators one after the other on stream 0 of partition p and waits for them; each sees what those in front of it
 * wrote.  The caller's streams are synchronised first (as daris_forward does), and the results are visible to every HIP
 * stream and the host on return.  All descriptors are checked before anything is launched: DARIS_EINVAL names the first operator that is
 * wrong, and nothing has run.  Operators without rows do nothing.  Tasks may have active jobs, which go on meanwhile (those
 * that share the queue wait in line).  Attention and products keep partial results in a workspace of the partition, which grows when a call
 * needs more (DARIS_ENOMEM: nothing has run) and lives until daris_shutdown. */
daris_status daris_run_ops(const daris_op* ops, int32_t n, daris_part p);
/* The same in two parts, for a program that runs the same list step after step: daris_plan_ops checks the descriptors and keeps
 * the launches with their arguments in device memory (not the buffers, which it neither reads nor copies); daris_run_plan
 * runs them (a list of one norm 6.8 us a call in place of 8.8, of eight 18 in place of 23).  daris_free_plan gives a plan up; daris_shutdown gives up all,
 * and handles from before it are DARIS_ERANGE for good.  daris_free_plan alone may be called on another thread. */
daris_plan daris_plan_ops(const daris_op* ops, int32_t n, daris_part p);
daris_status daris_run_plan(daris_plan plan);
daris_status daris_free_plan(daris_plan plan);

#ifdef __cplusplus
}
#endif
#endif /* DARIS_OPS_H */
