/*
 * daris_ops.h -- operators of a generation step: the chain that one token (or a few, or a chunk of a prompt) takes through a
 * decoder block, for programs that run a generating model on a partition next to the tasks of daris.h.
 *
 *     norm -> product -> append -> attend -> product -> norm -> gated product -> product
 *
 * and, behind its last product, the words that come of it: drawn from given random numbers, and accepted from trees of drafted ones (see daris_tree_append and on).
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
/* ... of a step whose words are drafted (see daris_tree_append and on; 7 is none) */
enum { DARIS_STEP_TREE_APPEND = 4, DARIS_STEP_TREE_ATTEND = 5, DARIS_STEP_SAMPLE = 6, DARIS_STEP_ACCEPT = 8, DARIS_STEP_KEEP = 9, DARIS_STEP_COPY = 10 };
enum { DARIS_PAGE_TOKENS = 64, DARIS_SCALE_TOKENS = 16, DARIS_TREE_WORDS = 16, DARIS_SAMPLE_WORDS = 1 << 20 };

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

/*
 * A drafted step: the new rows of a sequence are the nodes of a tree of words that hang on its cached tokens, and all go through the model at once.
 *
 *     append (tree) -> attend (tree) -> ... -> sample -> accept -> keep
 *
 * tree [n_rows][tree_words] (dense, aligned to 8 bytes, 1 to DARIS_TREE_WORDS words a row): bit j mod 64 of word j / 64 of a row's mask is set if the row sees
 * node j of its sequence, which is the sequence's row j.  A node's own bit and those of the nodes above it make a tree, whose nodes are numbered from
 * the root on (a node behind the one that it hangs on); any other masks over the step's rows may stand there too.  Bits of rows that the sequence does not have are ignored by attention and
 * acceptance; a position counts all bits of the mask, these among them.
 *
 * Append and attend as above with these differences.  Node j lies in the cache as token before + j, but its position -- for the turning of keys and
 * queries -- is before + (the number of bits in its mask) - 1.  A row attends the cached tokens 0 .. before - 1 and the nodes of its mask, in this
 * order; window != 0: the last `window` of them.  k and v of an append have the same distances (a
 * descriptor is as large as daris_append: lists that were laid out before there were trees stay right).
 */
typedef struct daris_tree_append {
  daris_cache cache;
  const void* k;
  const void* v;
  const void* q;
  void* q_out;
  const float* turn;
  const int32_t* row_start;
  const uint64_t* tree;
  int64_t kv_row, kv_head, q_row, q_head, qo_row, qo_head;
  int32_t n_rows, q_heads, dtype, turn_rows, rot_dim, pairs, tree_words;
} daris_tree_append;

typedef struct daris_tree_attend {
  daris_attend attend;
  const uint64_t* tree;
  int32_t tree_words;
} daris_tree_attend;

/*
 * A word for each row of logits [rows][n] (n at most DARIS_SAMPLE_WORDS), drawn by the caller's random numbers.  With M a row's largest logit and T =
 * temperature[row], word i weighs exp((x_i - M) / T); what weighs less than 2^-64, and NaN and -infinity, is nothing.  In this order,
 *   top_k[row] > 0   leaves the top_k largest;
 *   top_p[row] < 1   leaves the shortest front of these, the largest first, whose weights come to top_p of the sum of them all (one word at least);
 *   min_p[row] > 0   leaves those of them that weigh min_p or more (and the largest).
 * Of equal logits the word of the lower number is the larger.  word[row] is the first word that is left, by number, at which the sum of the weights that
 * are left is more than random[row] times all of it (random in [0, 1); NaN and what is below 0 count as 0; from 1 on it is the last word).  Weights and sums are
 * doubles, within 2^-46 of themselves; top_p, and where a long row's sum passes the random number, are found with weights rounded to whole numbers, within 2^-39 of each.
 * chance[row], if not NULL, is its weight divided by that sum.  T <= 0 or NaN, and random == NULL, give the largest (and 1); a row with nothing but NaN and
 * -infinity gives -1 (and 0).  A row with +infinity is drawn among those words.  temperature == NULL is 1, the others' NULL leaves everything.  All per row: float, top_k int32.
 */
typedef struct daris_sample {
  const void* logits;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* random;
  int32_t* word;
  float* chance;
  int64_t logits_row;
  int32_t rows, n, dtype;
} daris_sample;

/*
 * Which nodes of a tree stand: answers[row] is the word that the model gave behind the row's node, words[row] the node's own.  The walk starts at a
 * sequence's node 0 (its last word, of which the cache holds no token yet) and goes from a node to the first node below it (the one of the lowest number whose mask's highest bit
 * in front of its own is that node) whose word is the node's answer and not negative, until there is none.  path[row_start[s] + j] is the j-th node of the walk, and -1 behind the last;
 * count[s] how many there are, word[s] the last one's answer: the sequence's new last word.  after[s] = before[s] + count[s] (after may be NULL, or before itself if
 * no operator that follows in the list needs the old one).  A sequence without rows has count 0 and word -1.  Rows from 64 * tree_words on are no nodes.
 */
typedef struct daris_accept {
  const uint64_t* tree;
  const int32_t* words;
  const int32_t* answers;
  const int32_t* row_start;
  const int32_t* before;
  int32_t* path;
  int32_t* count;
  int32_t* word;
  int32_t* after;
  int32_t n_rows, n_seqs, tree_words;
} daris_accept;

/*
 * Keeps the tokens of some of the step's rows: token before[s] + path[row_start[s] + j] of the cache becomes token before[s] + j, for j < count[s] (at most the
 * sequence's rows; path as daris_accept leaves it).  Entries increase and name rows of the sequence; the first that does not ends the list.  before is what it was for the
 * step's append.  A sixteenth that gets tokens has the largest scale of the tokens that it then holds, and its codes are rounded again where theirs was smaller; one that gets
 * none, and what lies behind the last kept token, stays as it is.  A token whose old or new page is not there is not moved.  No page that gets tokens may belong to two
 * places of the table.
 */
typedef struct daris_keep {
  daris_cache cache;
  const int32_t* path;
  const int32_t* count;
  const int32_t* row_start;
  int32_t n_rows;
} daris_keep;

/*
 * Copies pages of a cache, all heads' keys, values and scales: page pairs[i][0] over page pairs[i][1] (device int32[n][2]), for sequences that are continued twice and for pages
 * that gather elsewhere.  A pair with a page outside 0 .. n_pages - 1 is left out.  No page may be written twice, or read by one pair and written by another.
 * Only k, v, the scales, n_pages, kv_heads and dim of the cache count.
 */
typedef struct daris_copy {
  daris_cache cache;
  const int32_t* pairs;
  int32_t n;
} daris_copy;

typedef struct daris_op {
  int32_t kind; /* DARIS_STEP_... : which member counts */
  int32_t reserved; /* 0 */
  union {
    daris_norm norm;
    daris_append append;
    daris_attend attend;
    daris_matvec matvec;
    daris_tree_append tree_append;
    daris_tree_attend tree_attend;
    daris_sample sample;
    daris_accept accept;
    daris_keep keep;
    daris_copy copy;
  } u;
} daris_op;

typedef int32_t daris_plan; /* handle of a planned list of operators; <0 is an error code */

/* Runs n operators one after the other on stream 0 of partition p and waits for them; each sees what those in front of it
 * wrote.  The caller's streams are synchronised first (as daris_forward does), and the results are visible to every HIP
 * stream and the host on return.  All descriptors are checked before anything is launched: DARIS_EINVAL names the first operator that is
 * wrong, and nothing has run.  Operators without rows do nothing.  Tasks may have active jobs, which go on meanwhile (those
 * that share the queue wait in line).  Attention, products and sampling (12 KB for every 8192 or 16384 logits of a row) keep partial results in a workspace of the partition, which grows when a call
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
