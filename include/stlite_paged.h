/*
 * stlite_paged.h -- serving from a paged cache after the compression pass.
 *
 * stlite_compact_kv writes a dense cache that cannot grow.  These calls keep the
 * cache in pages instead, so that a sequence can go on: with the next token, a
 * few drafted tokens, or the next screenshot.
 *
 *   stlite_paged_compact    the kept rows of the compression, straight into pages
 *   stlite_paged_append     new tokens: the per-head norm and the rotation of
 *                           queries and keys, keys and values into pages
 *   stlite_paged_attention  causal attention of the new tokens over the pages
 *
 * Conventions (pointers, streams, units, ownership, errors) are those of
 * stlite.h: the calls only enqueue work, allocate nothing, keep no state, and
 * validate every host-side argument before anything is enqueued.  The current
 * device must be the one that holds the tensors and `stream`.
 *
 * The pool.  k and v are [n_layers][n_kv_heads][n_pages][page_size][d]: a page
 * holds page_size consecutive tokens of one sequence, of one (layer, kv head).
 * page_table [n_seqs][max_pages] is shared by all layers and kv heads: token j of
 * sequence s is row j % page_size of page page_table[s][j / page_size].  A cache
 * of one layer is the same struct with n_layers = 1 and k, v at that layer.
 *
 * Lengths live on the device, so that a captured graph follows them: seq_lens[s]
 * counts the tokens of sequence s INCLUDING the new ones of this call.  The new
 * tokens are its last n_s = cu_new[s+1] - cu_new[s] ones: new token t is token
 * seq_lens[s] - n_s + t.  Lengths outside [0, max_len] are cut to it.
 *
 * What the kernels check, since the host cannot see it: a page index outside
 * [0, n_pages) is never followed.  Attention leaves the tokens of such a page
 * out, an append or a compaction drops the rows that belong there, and a new
 * token whose index would be negative (seq_lens[s] < n_s) is not stored.  So an
 * idle slot of a padded batch is a sequence of length 0.
 *
 * A page may be in several rows of the table (a shared prefix) as long as no
 * call writes to it for more than one of them.
 */
#ifndef STLITE_PAGED_H
#define STLITE_PAGED_H

#include "stlite.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of q, k, v, the pool, the norm weights and the outputs of a call. */
typedef enum stlite_dtype {
  STLITE_BF16 = 0,
  STLITE_FP16 = 1 /* IEEE half */
} stlite_dtype;

/*
 * A paged cache and the new tokens of one call.
 *
 * Limits: head_dim == 128; n_q_heads % n_kv_heads == 0, at most 128 query heads
 * per kv head; page_size 16, 32, 64, 128 or 256; n_layers * n_kv_heads <= 65535;
 * n_seqs <= 65535; 1 <= max_len <= min(2^28, max_pages * page_size); n_s <=
 * max_len; n_pages * page_size < 2^31; total_new < 2^31.
 */
typedef struct stlite_paged {
  int32_t n_layers;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t dtype;             /* stlite_dtype */
  int32_t page_size;
  int32_t n_pages;           /* of the pool, per (layer, kv head) */
  int32_t n_seqs;
  int32_t max_pages;         /* entries of a sequence in page_table */
  int32_t max_len;           /* no sequence is longer */
  int64_t total_new;         /* = cu_new[n_seqs] */
  void* k;                   /* the pools, 16-byte aligned */
  void* v;
  const int32_t* page_table; /* device [n_seqs][max_pages] */
  int32_t* seq_lens;         /* device [n_seqs]; only stlite_paged_compact writes it */
  const int32_t* cu_new;     /* device [n_seqs+1], prefix sums of the new tokens, cu_new[0] = 0 */
  const int32_t* h_cu_new;   /* host mirror of cu_new */
} stlite_paged;

/*
 * Rows of new tokens: heads x d contiguous elements per (layer, token), 16-byte
 * aligned; token i of layer l starts at data + l * layer_stride + i *
 * token_stride (elements, multiples of 8).  A slice of a fused projection is
 * such rows.
 */
typedef struct stlite_rows {
  const uint16_t* data;
  int64_t token_stride;
  int64_t layer_stride;
} stlite_rows;

/*
 * The position rotation.  Pair i of a head, 0 <= i < 64, is (x_i, x_{i+64}), or
 * (x_{2i}, x_{2i+1}) where interleaved; it turns by position * theta^(-i/64).
 * With n_axes = 1 every pair goes by the token's one position.  With n_axes = 3
 * (time, row and column of a screenshot's patches) the first sections[0] pairs go
 * by the first position, the next sections[1] by the second and the last
 * sections[2] by the third; the sections add up to 64.
 */
typedef struct stlite_rope {
  double theta;        /* finite, >= 1 */
  int32_t interleaved; /* 0 or 1 */
  int32_t n_axes;      /* 1 or 3 */
  int32_t sections[3]; /* read where n_axes == 3 */
  int32_t reserved;    /* must be 0 */
} stlite_rope;

/*
 * Checks every host-visible field of `c`.  h_page_table and h_seq_lens (host,
 * both nullable) are the values that the device arrays hold: with h_seq_lens,
 * every length must lie in [n_s, max_len]; with both, every page of a sequence's
 * tokens must lie in [0, n_pages), and a page that new tokens are stored in must
 * belong to no other sequence.
 */
stlite_status stlite_paged_validate(const stlite_paged* c, const int32_t* h_page_table,
                                    const int32_t* h_seq_lens);

/* Bytes of device workspace that stlite_paged_attention needs for `c`.  They do
 * not depend on the lengths. */
stlite_status stlite_paged_workspace_size(const stlite_paged* c, size_t* bytes);

/*
 * The kept rows of the compression into pages: for every unit u, sequence s and
 * j < B_s, row kept[u][cu_budget[s] + j] of k and v (the layout of
 * stlite_compact_kv) becomes token j of sequence s.  Exact row copies of 16-bit
 * patterns, which must be of the pool's type (the compression pass knows bf16 alone:
 * its rows belong in a bf16 pool).  seq_lens[s] becomes B_s.  p and c must agree in
 * n_layers, n_kv_heads and n_seqs, and every B_s must be at most c->max_len; the
 * new tokens (total_new, cu_new, h_cu_new) are not read.  per_layer != 0: one
 * kept list per layer, as in stlite_compact_kv_layer.  A kept index outside
 * [0, total_tokens) stores zeros.  k and v must not alias the pool.
 */
stlite_status stlite_paged_compact(const stlite_problem* p, const stlite_paged* c, const uint16_t* k,
                                   const uint16_t* v, const int32_t* kept, int32_t per_layer,
                                   void* stream);

/*
 * Stores the keys and values of the new tokens and rotates their queries.  For
 * every layer, new token i and head, with x a row of q or k:
 *   n = x * w / sqrt(mean(x^2) + eps)   where norm weights w are given, else x
 *   (y_a, y_b) = (n_a cos - n_b sin, n_b cos + n_a sin)   for every pair (a, b)
 * in fp32, rounded once; the angles are formed in 64 bits.  The q rows' y go to
 * q_out [n_layers][total_new][n_q_heads][d], the k rows' y and the v rows as they
 * are to the tokens' places in the pool.
 *   positions  int32 [n_axes][total_new]; rope and positions both NULL: no rotation
 *   q_norm, k_norm  [n_layers][d], each nullable, 16-byte aligned
 *   eps        finite, >= 0; read where a norm is
 * q->data and q_out both NULL: no queries.  q_out must not alias q, k, v or the pool;
 * k and v must not lie where the call stores other rows.
 */
stlite_status stlite_paged_append(const stlite_paged* c, const stlite_rope* rope, const int32_t* positions,
                                  const stlite_rows* q, const stlite_rows* k, const stlite_rows* v,
                                  const uint16_t* q_norm, const uint16_t* k_norm, float eps, uint16_t* q_out,
                                  void* stream);

/*
 * Causal attention of the new tokens over their sequences' pages: for every
 * layer, sequence s, new token t < n_s and query head g (kv head g / G),
 *   out = sum_{j <= m} softmax_{j <= m}(scale q . k_j) v_j,   m = seq_lens[s] - n_s + t,
 * over the tokens j that lie in valid pages; a token that sees none gets 0.
 * What the mask leaves out has no influence, NaN and infinities among it.
 *   q    [n_layers][total_new][n_q_heads][d], 16-byte aligned
 *   out  the same layout and type; 16-byte aligned, must not alias q or the pool
 *   scale  > 0, at most 2^127
 * fp32 logits, softmax statistics and sums, which stay finite for logits (scale q . k
 * log2(e)) and values of any size in fp32's range and up to 2^20 keys.  With one new
 * token per sequence the weights keep fp32's 24 bits (fp16: 22, or 2^-40 of the greatest
 * weight); with more they are rounded to the type of the call before they meet v.
 * An infinity or NaN of a value that is seen reaches the output whatever its weight (an
 * infinity of a weight that is rounded to 0 as NaN).  A logit of infinity or NaN makes
 * its token's head NaN; one of -infinity weighs nothing, and where all are, the output
 * is 0.  Rows of out belong to new tokens only: nothing behind total_new is written.
 * The workspace must not alias q, out or the pool.
 */
stlite_status stlite_paged_attention(const stlite_paged* c, const uint16_t* q, float scale, uint16_t* out,
                                     void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STLITE_PAGED_H */
