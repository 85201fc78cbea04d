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
 *   stlite_paged_read       the new tokens' rows out of the pages
 *   stlite_paged_grow       lengths, pages and places for the next new tokens
 *   stlite_paged_release    pages behind a sequence's end, back to the free ones
 *   stlite_verify_drafts    drafted tokens against the target's probabilities
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
 * A pool in 4 bits (a dtype with STLITE_KV4).  k and v are bytes, [n_layers]
 * [n_kv_heads][n_pages][page_size * 68]: a page is page_size rows of 64 bytes of codes
 * and then page_size rows of 4 scale bytes.  Block b of a row is its values 32 b to
 * 32 b + 31; value 2 i is the low half of byte i, value 2 i + 1 the high half: a sign
 * (bit 3) and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6, times 2^(scale byte - 127).  A row that
 * is stored gets for each block the least power of two of which 7 times reaches the
 * block's greatest magnitude, cut to 2^-120 .. 2^125 (fp16: 2^-14 .. 2^13), and each value
 * the nearest code, ties to the even one, beyond 6 to 6.  A block with an infinity or NaN
 * gets scale byte 255: all of its values are NaN.  (Any other byte is read as what it says,
 * its values rounded to the 16-bit type, beyond that to infinity.)  The same calls store and
 * read such a pool; what they compute, they compute of the values that the codes stand for.
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

/* Type of q, k, v, the pool, the norm weights and the outputs of a call; the pool's
 * own with STLITE_KV4. */
typedef enum stlite_dtype {
  STLITE_BF16 = 0,
  STLITE_FP16 = 1,                           /* IEEE half */
  STLITE_KV4 = 16,                           /* flag: the pool holds 4 bits */
  STLITE_BF16_KV4 = STLITE_BF16 | STLITE_KV4,
  STLITE_FP16_KV4 = STLITE_FP16 | STLITE_KV4
} stlite_dtype;

/*
 * A paged cache and the new tokens of one call.
 *
 * Limits: head_dim == 128; n_q_heads % n_kv_heads == 0, at most 128 query heads
 * per kv head; page_size 16, 32, 64, 128 or 256; n_layers * n_kv_heads <= 65535;
 * n_seqs <= 65535; 1 <= max_len <= min(2^28, max_pages * page_size); n_s <=
 * max_len (in stlite_paged_grow any number); n_pages * page_size < 2^31; total_new < 2^31.
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
  int32_t* seq_lens;         /* device [n_seqs]; compact, grow, release and verify write it */
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
 * every length must lie in [n_s, max_len] or be negative (parked, see
 * stlite_paged_grow); with both, every page of a sequence's tokens must lie in
 * [0, n_pages), and a page that new tokens are stored in must belong to no other
 * sequence, a parked one's tokens included.
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
 * its rows belong in a bf16 pool); into a 4-bit pool, their codes.  seq_lens[s] becomes B_s.
 * A parked sequence (stlite_paged_grow) stays parked, and nothing is stored for it; an empty one
 * (-1) that holds pages for all of B_s takes them instead, and is parked no more.  (So the
 * lengths of a new cache have to be set, to 0.  In a row of the table that no call has grown,
 * -1 with a page in the first entry is as good as 0.)
 * p and c must agree in n_layers, n_kv_heads and n_seqs, and every B_s must be at most
 * c->max_len; the new tokens (total_new, cu_new, h_cu_new) are not read.  per_layer != 0: one
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
 * in fp32, rounded once; the angles are formed in 64 bits.  (What goes into a 4-bit pool
 * is formed in 64 bits throughout: the codes are those of the exact y but where y lies
 * within 64 bits' rounding of a border.)  The q rows' y go to
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
 * weight); with more, and over a 4-bit pool, they are rounded to the type of the call
 * before they meet v.
 * An infinity or NaN of a value that is seen reaches the output whatever its weight (an
 * infinity of a weight that is rounded to 0 as NaN).  A logit of infinity or NaN makes
 * its token's head NaN; one of -infinity weighs nothing, and where all are, the output
 * is 0.  Rows of out belong to new tokens only: nothing behind total_new is written.
 * The workspace must not alias q, out or the pool.
 */
stlite_status stlite_paged_attention(const stlite_paged* c, const uint16_t* q, float scale, uint16_t* out,
                                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * The new tokens' rows out of the pages: k_out, v_out [n_layers][total_new][n_kv_heads][d]
 * in the call's 16-bit type, each nullable, 16-byte aligned; they must not alias the pool.
 * A row of an invalid page, or whose index would be negative, is zeros.  With cu_new the
 * prefix sums of the lengths it reads whole sequences (to move them, or to a dense cache).
 */
stlite_status stlite_paged_read(const stlite_paged* c, uint16_t* k_out, uint16_t* v_out, void* stream);

/*
 * The free pages of a pool, on the device: pages[0 .. n_free) are those that no sequence
 * holds (the next one to be given out is the last), and held[s] counts the entries of
 * page_table's row s, from its first, that sequence s holds a page in.  To begin with:
 * pages every index of the pool, n_free = n_pages, held and seq_lens 0.  No page may be
 * in the list and in a row's held entries, or in two rows', at once.  page_table is the
 * cache's, which grow and release write.
 */
typedef struct stlite_free_pages {
  int32_t* pages;  /* device [n_pages] */
  int32_t* n_free; /* device [1] */
  int32_t* held;   /* device [n_seqs] */
  int32_t* page_table; /* = the cache's page_table */
} stlite_free_pages;

/*
 * Grows every sequence by its new tokens (cu_new): seq_lens[s] += n_s, with pages from the
 * list behind the held ones where the new length needs more.  Sequences are served in
 * turn, the lowest first, each wholly or not at all: one whose pages, and those that the
 * sequences before it ask for, are more than the list has, or whose length would pass
 * max_len, is PARKED: its length becomes ~len (negative), and its pages stay as they
 * are (behind those of an empty one its row gets a -2).  To every call a parked sequence is
 * an idle slot (length 0): nothing of it is read or stored, its new tokens' outputs are 0.
 * It stays parked until a release brings it back.
 * One that needs no page is not held up by those before it.
 * One with more than max_len new tokens, which no sequence can have, is parked like any other
 * that does not fit.  The other calls refuse a batch that holds it, with nothing done: the
 * host, which knows the counts, gives them one without those tokens (n_s = 0).
 *   slots  [total_new], nullable: the row of the pool (page * page_size + row in the page)
 *          of every new token, -1 for a parked sequence's
 */
stlite_status stlite_paged_grow(const stlite_paged* c, const stlite_free_pages* pages, int32_t* slots, void* stream);

/*
 * Gives back the pages behind the sequences' ends; their entries of the page table become
 * -1.  lens [n_seqs], nullable: sequence s keeps its first min(lens[s], len) tokens, 0 to
 * end it, and is parked no more; lens[s] < 0, or NULL, leaves its length (a parked one's
 * pages behind ~len are given back too).  Pages return so that growing again takes the
 * same ones in the same places.  The new tokens (total_new, cu_new, h_cu_new) are not read.
 */
stlite_status stlite_paged_release(const stlite_paged* c, const stlite_free_pages* pages, const int32_t* lens,
                                   void* stream);

/* Type of the probabilities of stlite_verify_drafts. */
typedef enum stlite_prob { STLITE_PROB_BF16 = 0, STLITE_PROB_FP16 = 1, STLITE_PROB_FP32 = 2 } stlite_prob;

/*
 * Drafted tokens of a batch.  Sequence s has n_s = cu_new[s+1] - cu_new[s] rows: row t < n_s
 * - 1 judges its drafted token t, and the last one follows them all.  (After a call of
 * attention with n_s new tokens, a sampled one and n_s - 1 drafted ones: its rows.)
 * Limits: n_seqs <= 65535, vocab <= 2^24, total_new < 2^31.
 */
typedef struct stlite_verify {
  int32_t n_seqs;
  int32_t vocab;
  int32_t dtype;          /* stlite_prob, of target and draft */
  int32_t reserved;       /* must be 0 */
  int64_t total_new;      /* = cu_new[n_seqs] */
  const int32_t* cu_new;  /* device [n_seqs+1], cu_new[0] = 0 */
  const int32_t* h_cu_new;
  const void* target;     /* device: row i, vocab probabilities, at target + i * target_stride */
  const void* draft;      /* the same of the draft, at rows of drafted tokens; NULL: it gave each token with certainty */
  int64_t target_stride;  /* entries, >= vocab */
  int64_t draft_stride;
  const int32_t* tokens;  /* device [total_new]: row i's drafted token (a sequence's last row: not read) */
  const float* accept;    /* device [total_new]: random numbers in [0, 1), one to a drafted token */
  const float* pick;      /* device [n_seqs]: one to a sequence */
  int32_t* seq_lens;      /* device [n_seqs], nullable: lengths that count all n_s new tokens */
} stlite_verify;

stlite_status stlite_verify_workspace_size(const stlite_verify* v, size_t* bytes);

/*
 * Drafted token x of row i is accepted where accept_i q_i(x) < p_i(x) (draft NULL: q_i(x) =
 * 1), compared exactly; a token outside [0, vocab) is not.  A sequence's run ends at the
 * first one that is not, row k, and its next token comes from
 *   w_j = max(p_k(j) - q_k(j), 0)    (draft NULL: p_k(j), and 0 for the refused token)
 * or, where all are accepted, from w = p of its last row (and also where the other w are
 * all 0): the least j with w_0 + .. + w_j > pick (w_0 + .. + w_{vocab-1}), in 64-bit sums;
 * p need not add up to 1.  Entries of p and q that are negative, infinite or NaN count as
 * 0; a row without any weight gives -1.
 *   out    [total_new]: the accepted tokens, the next one, then -1
 *   n_out  [n_seqs]: accepted tokens + 1; 0 where n_s = 0
 * seq_lens[s] becomes what is right behind the accepted tokens: n_s - n_out[s] less.  A
 * negative length (a parked sequence) stays, with n_out 0 and out -1.
 * out, n_out, seq_lens and the workspace must not overlap one another or an input.
 */
stlite_status stlite_verify_drafts(const stlite_verify* v, int32_t* out, int32_t* n_out, void* workspace,
                                   size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STLITE_PAGED_H */
