/* ff_ops.h -- operators of language models for gfx950 (MI355X), in the same library as ff_sim.h.
 *
 * The simulator takes exeTimes from a task of every (operation type, output size) being run once on the device
 * (Section 5.1, task properties).  These are the operators of a language model's training step, beside plain matrix
 * products, that such a measurement runs: layer norm, attention and the loss over a vocabulary, each forward and
 * backward.  The vocabulary can be a shard of it, as a strategy that splits the channel dim of the output projection
 * leaves on one device.  With the operators behind them such a model answers: a paged cache of keys and values, attention
 * of new tokens over it, and the choice of the next token.
 *
 * Every call takes one record and a stream; it checks the record on the host, puts kernels on the stream and returns.
 * It allocates nothing, waits for nothing and keeps nothing, so it may be captured into a HIP graph.  All pointers in
 * the records are DEVICE pointers; the caller owns them and keeps them until the work on the stream is done.  Outputs
 * must not overlap inputs unless said so.  Calls that need scratch memory take a workspace of at least the bytes that
 * ..._workspace_bytes returns (0: none needed; the pointer may then be null); calls that overlap in time need one each.
 * Results do not depend on the order in which blocks run: the same inputs give the same bits.
 *
 * Returns FF_OK, FF_EINVAL (malformed record), FF_EWORKSPACE (workspace missing, too small or not aligned to 256 bytes),
 * FF_ERANGE (a limit below is passed) or FF_EHIP (a launch failed).
 */
#ifndef FF_OPS_H
#define FF_OPS_H

#include "ff_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FF_F32 = 0, FF_F16 = 1, FF_BF16 = 2 }; /* types of tensors; layer norm and sampling take all three, the others FF_F16 and FF_BF16 */

#define FF_OP_MAX_COLS 65536      /* layer norm: elements of a row */
#define FF_OP_MAX_HEAD_DIM 128    /* attention: elements of a head, a multiple of 8 */
#define FF_OP_MAX_LEN (1u << 28)  /* attention: positions of a sequence */
#define FF_OP_MAX_SIDE (65535u * 128) /* attention: queries of a sequence times query heads of a key head; backward: its keys, too */
#define FF_OP_MAX_ROWS (1u << 28) /* layer norm: rows */
#define FF_OP_MAX_TOKENS ((1u << 26) - 4) /* vocabulary loss: rows, words */
#define FF_OP_MAX_DIM 65536       /* vocabulary loss: elements of a token's vector */
#define FF_OP_MAX_PAGE 32768      /* paged cache: positions of a page, a power of two from 16 on */
#define FF_OP_MAX_WORDS (1u << 24) /* sampling: words of a vocabulary */
#define FF_OP_MAX_CHOICES ((1u << 22) - 1) /* sampling: rows */
/* and of the vocabulary loss, backward, rows * dim up to 2^34, and products (rows x words, rows x dim, dim x words) of fewer than 2^24 tiles, which are
 * 256 x 256 in products that large, but 128 x 128 where fewer than 512 is summed over.  attention: heads and batch up to 65535, batch * kv_heads up to 65535 * 32.
 * paged cache: the same, the positions of a table up to FF_OP_MAX_LEN; writing: new_len * kv_heads below 2^28; reading: batch * kv_heads up to 65535, kv_len below 2^28; attention: queries of a
 * sequence times query heads of a key head up to 65535 * 16, times all heads below 2^26. */

/* rows of a matrix: element (r, c) is p[r * stride + c].  stride counts elements and may be any number that keeps
 * outputs from overlapping themselves (inputs may repeat rows: stride 0). */
typedef struct {
    void* p;
    int64_t stride;
} ff_rows_t;

/* heads of a batch: element (b, h, i, d) is p[b * batch + h * head + i * pos + d]; strides count elements and are
 * multiples of 8, p is aligned to 16 bytes. */
typedef struct {
    void* p;
    int64_t batch, head, pos;
} ff_heads_t;

/* Layer norm over the elements of a row:  h = x + res (rounded to the type; res.p null: h = x, and h.p is not written),
 * mean = sum h / cols,  rstd = 1 / sqrt(sum (h - mean)^2 / cols + eps),  y = (h - mean) * rstd * weight + bias.
 * weight and bias [cols] are of the tensors' type, bias may be null; mean and rstd [rows] are float (both may be null).
 * Sums are held in 32 bits; y is rounded once.  y may be the same memory as x or res. */
typedef struct {
    uint32_t dtype, cols;
    uint64_t rows;
    float eps;
    ff_rows_t x, res, h, y;
    const void *weight, *bias;
    float *mean, *rstd;
} ff_layernorm_fwd_t;
int ff_op_layernorm_fwd(const ff_layernorm_fwd_t* a, void* stream);

/* Its backward pass from h, mean and rstd:  xh = (h - mean) * rstd,  g = dy * weight,
 * dx = rstd * (g - mean(g) - xh * mean(g * xh)) (+ dh, the gradient that reaches h past the norm; dh.p may be null),
 * dweight = sum over rows of dy * xh,  dbias = sum over rows of dy (both of the tensors' type, rounded once; either may be null).
 * dx is the gradient of x and of res alike; it may be the same memory as dy or dh. */
typedef struct {
    uint32_t dtype, cols;
    uint64_t rows;
    ff_rows_t dy, h, dh, dx;
    const void* weight;
    const float *mean, *rstd;
    void *dweight, *dbias;
    void* workspace;
    size_t workspace_bytes;
} ff_layernorm_bwd_t;
size_t ff_op_layernorm_bwd_workspace_bytes(const ff_layernorm_bwd_t* a);
int ff_op_layernorm_bwd(const ff_layernorm_bwd_t* a, void* stream);

/* Attention:  s_ij = scale * <q_i, k_j>,  o_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij), over the keys
 * that query i sees.  Query head h reads key head h / (heads / kv_heads).  Sequence b has q_lengths[b] queries and
 * kv_lengths[b] keys (int32 [batch] each, values 0 .. q_len / kv_len, others are clamped to that; null: all of them);
 * with `causal`, query i sees the keys j <= i + kv_lengths[b] - q_lengths[b], the last query all of them.  A query that sees no key, and one
 * beyond q_lengths[b], gets o = 0 and lse = -inf.  Keys and values beyond kv_lengths[b] are not read.  A value row that
 * some queries of a block of 64 keys see and others do not has to be finite (in the backward pass a key row, too), as has every query and gradient within the
 * lengths, and every key where head_dim is neither 64 nor 128.  Probabilities below 2^-126 are 0.
 * lse is float [batch][heads][q_len].  scale > 0.  Products are summed in 32 bits; the probabilities are rounded to the
 * tensors' type before they meet the values, in float16 2^8 times what they are of the row's largest. */
typedef struct {
    uint32_t dtype, batch, heads, kv_heads, q_len, kv_len, head_dim, causal;
    float scale;
    ff_heads_t q, k, v, o;
    float* lse;
    const int32_t *q_lengths, *kv_lengths;
    void* workspace;
    size_t workspace_bytes;
} ff_attention_fwd_t;
size_t ff_op_attention_fwd_workspace_bytes(const ff_attention_fwd_t* a);
int ff_op_attention_fwd(const ff_attention_fwd_t* a, void* stream);

/* Its backward pass from o and lse, the probabilities computed again:  p = exp(s - lse),  dv_j = sum_i p_ij do_i,
 * ds_ij = p_ij (<do_i, v_j> - <do_i, o_i>),  dq_i = scale * sum_j ds_ij k_j,  dk_j = scale * sum_i ds_ij q_i; dk and dv sum
 * over the query heads of a key head.  Gradients beyond the lengths, and of queries that see no key, are 0.
 * o and lse may be of more keys than the call's (a sequence's keys in pieces, the pieces' o and lse joined): dq is then this piece's
 * part of the sum.  p and ds are rounded to the tensors' type before they are multiplied, in float16 2^10 times p, and ds times a power of two, of
 * the row for dq and of the key for dk, that keeps all of them in its range. */
typedef struct {
    uint32_t dtype, batch, heads, kv_heads, q_len, kv_len, head_dim, causal;
    float scale;
    ff_heads_t dout, q, k, v, o, dq, dk, dv;
    const float* lse;
    const int32_t *q_lengths, *kv_lengths;
    void* workspace;
    size_t workspace_bytes;
} ff_attention_bwd_t;
size_t ff_op_attention_bwd_workspace_bytes(const ff_attention_bwd_t* a);
int ff_op_attention_bwd(const ff_attention_bwd_t* a, void* stream);

/* Softmax cross entropy of rows of x [rows][dim] against a vocabulary w [vocab][dim]:  z_iv = <x_i, w_v>,
 * lse_i = log sum_v exp(z_iv),  loss_i = lse_i - z_it.  The logits are made in pieces and not kept.
 * targets [rows] are int32.  A row whose target is ignore_index takes no part: loss 0, no gradient.
 * w may be words first_word .. first_word + vocab - 1 of a larger vocabulary: lse is then over those words, target_logit is
 * z_it where the target is among them and 0 elsewhere, and loss is not asked for (null); with lse joined over the shards
 * as log sum exp, and target_logit as a sum, the backward pass of each shard takes the joined lse.
 * Where loss is asked for, a target that is neither a word nor ignore_index gives a NaN.
 * loss, target_logit (either may be null) and lse are float [rows]. */
typedef struct {
    uint32_t dtype, rows, vocab, dim;
    int32_t ignore_index, first_word;
    ff_rows_t x, w;
    const int32_t* targets;
    float *loss, *lse, *target_logit;
    void* workspace;
    size_t workspace_bytes;
} ff_vocab_loss_fwd_t;
size_t ff_op_vocab_loss_fwd_workspace_bytes(const ff_vocab_loss_fwd_t* a);
int ff_op_vocab_loss_fwd(const ff_vocab_loss_fwd_t* a, void* stream);

/* Its backward pass:  g_iv = (exp(z_iv - lse_i) - [v = t_i]) * dloss_i,  dx = g w,  dw = g^T x.  dloss is float [rows], finite
 * where the row takes part; what x, dloss and lse hold in the others is not used, and they cost no products.  z is made again, in
 * pieces of the vocabulary; g is rounded to the tensors' type, in float16 to steps of 2^-39 of the largest |dloss| of all rows and no smaller ones (a loss may be
 * small, but a row that weighs 2^-k of the largest keeps probabilities from 2^(k-39) on, to 11 bits from 2^(k-29) on); sums are held in 32 bits.  Either of dx and dw may have a null pointer. */
typedef struct {
    uint32_t dtype, rows, vocab, dim;
    int32_t ignore_index, first_word;
    ff_rows_t x, w, dx, dw;
    const int32_t* targets;
    const float *dloss, *lse;
    void* workspace;
    size_t workspace_bytes;
} ff_vocab_loss_bwd_t;
size_t ff_op_vocab_loss_bwd_workspace_bytes(const ff_vocab_loss_bwd_t* a);
int ff_op_vocab_loss_bwd(const ff_vocab_loss_bwd_t* a, void* stream);

/* A paged cache of keys and values.  Position i of sequence b lies in page table[b * table_stride + i / page] at place i % page:
 * element d of head h is k[n][h][i % page][d] of that page n, pages k_stride bytes apart, everything in a page side by side; v likewise.
 * How elements are held:
 *   FF_HELD_SAME  in the tensors' type.
 *   FF_HELD_E4M3  in 8 bits (4 of exponent, 3 of fraction, no infinities), a scale for each row (the head_dim elements of a position and head);
 *                 head_dim is a multiple of 16.
 *   FF_HELD_E2M1  in 4 bits (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; the element of even number in the low half of the byte), a scale for each
 *                 32 elements of a row; head_dim is a multiple of 32.
 * A scale is a byte s and stands for 2^(s - 127), 255 for NaN: k_scale[n][h][block][i % page], pages k_scale_stride bytes apart.  Powers of two, because
 * the codes are floats, which another scale gives no more precision; so a value has one right code and is read back without a further rounding (but of
 * float16 below 2^-14).
 * page is a power of two, 16 .. FF_OP_MAX_PAGE.  k, v and their strides are multiples of 16 bytes, those of scales of 4.  Pages may lie in any order
 * and be shared by sequences; a table holds table_pages entries for each sequence, and those beyond its length are not looked at.  An entry that is no page
 * (below 0, or not below `pages`) is never followed: see each call. */
enum { FF_HELD_SAME = 0, FF_HELD_E4M3 = 1, FF_HELD_E2M1 = 2 };
typedef struct {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t* table;
    int64_t k_stride, v_stride, k_scale_stride, v_scale_stride; /* bytes */
    int64_t table_stride;                                       /* entries */
    uint32_t pages, page, table_pages, held;
} ff_cache_t;

/* Writes new keys and values: k and v [batch][kv_heads][new_len][head_dim], position i of sequence b becomes position start[b] + i of its
 * cache, for the first lengths[b] of them (clamped to 0 .. new_len; null: all).  What lies at positions below 0, behind the table or in an entry that is no page is not
 * written, nor is anything else touched.  No two of the positions written in a call may lie at the same place.
 * Held in fewer bits: the scale is the least power of two for which the block's largest value is at most 448 (E4M3) or 6 (E2M1) times it, at least 2^-127; codes are the
 * nearest, even of two as near.  Values beyond 15/16 (E4M3) or 3/4 (E2M1) of the power of two behind the type's last are held as that much.  A block in which a value is not finite has scale 255
 * and reads back as NaN. */
typedef struct {
    uint32_t dtype, batch, kv_heads, head_dim, new_len;
    ff_heads_t k, v;
    ff_cache_t cache;
    const int32_t *start, *lengths;
} ff_cache_write_t;
int ff_op_cache_write(const ff_cache_write_t* a, void* stream);

/* Reads a cache back: k and v [batch][kv_heads][kv_len][head_dim] are written whole, zeros from lengths[b] on (clamped to 0 .. kv_len and the positions of
 * the table; null: kv_len).  Positions whose entry is no page give NaN.  batch * kv_heads is at most 65535. */
typedef struct {
    uint32_t dtype, batch, kv_heads, head_dim, kv_len;
    ff_heads_t k, v;
    ff_cache_t cache;
    const int32_t* lengths;
} ff_cache_read_t;
int ff_op_cache_read(const ff_cache_read_t* a, void* stream);

/* Attention of new queries over a paged cache: as ff_op_attention_fwd with kv_lengths[b] keys of sequence b (clamped to 0 .. the positions of the table; null: all of these).
 * A query that sees a position whose entry is no page gets NaN for o and lse, no other does.  Value rows that some queries of a sequence see, and others that see any do not, have to be finite.
 * Probabilities meet the values in bfloat16 as a sum of two such numbers, in float16 rounded, 2^8 times what they are of the row's largest. */
typedef struct {
    uint32_t dtype, batch, heads, kv_heads, q_len, head_dim, causal;
    float scale;
    ff_heads_t q, o;
    ff_cache_t cache;
    float* lse;
    const int32_t *q_lengths, *kv_lengths;
    void* workspace;
    size_t workspace_bytes;
} ff_attention_paged_fwd_t;
size_t ff_op_attention_paged_fwd_workspace_bytes(const ff_attention_paged_fwd_t* a);
int ff_op_attention_paged_fwd(const ff_attention_paged_fwd_t* a, void* stream);

/* Chooses a word of each row of logits z [rows][vocab] with a given random number u[r] in [0, 1).  The words are taken in the order of their logits, the
 * largest first, equal ones in the order of their numbers; a word weighs w = exp((z - max z) / temperature), in 64 bits.  Kept are, one after the other,
 *   the first top_k words (0 or less: all),
 *   of these the shortest beginning whose weights sum to top_p of theirs, at least one word (1 or more: all),
 *   of these the words with w >= min_p, at least the first.
 * The word is the first whose running sum of weights is more than u times the sum of all that are kept (the last of them, if none); logprob is the logarithm of its
 * share of that sum.  At temperature 0 it is the first word, with logprob 0.  Words that are not next to a border of top_k, top_p, min_p or u are summed to 2^-29 of their
 * weight, so borders lie that near the exact ones.
 * Every parameter has a value for all rows, or a vector with one for each (which counts if it is not null).  -inf is the logit of a word that is never chosen beside others.  An infinite
 * logit is as good as any other largest one.  A row gives word -1 and logprob NaN where it holds a NaN or nothing but -inf, where its temperature is negative, NaN or
 * infinite, or another parameter or u is NaN; u is taken as 0 below that. */
typedef struct {
    uint32_t dtype, rows, vocab;
    ff_rows_t logits;
    const float *u, *temperatures, *top_ps, *min_ps;
    const int32_t* top_ks;
    float temperature, top_p, min_p;
    int32_t top_k;
    int32_t* words;
    float* logprob;
} ff_sample_t;
int ff_op_sample(const ff_sample_t* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif
