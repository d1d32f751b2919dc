/*
 * fastrack_latent.h -- C ABI of the latent cache operators that serve behind the sealed channel of fastrack.h.
 *
 * A latent cache holds ONE vector per token for all heads: `latent_dim` channels, from which a matrix makes every head's keys and
 * values, and `rope_dim` channels of a key that all heads share and that turns with the position.  Such a token is a fraction of what the
 * cache of fastrack_kv.h keeps even in 8 bits, and so is what has to cross the link when pages leave; the values stay in 16 bits.
 *
 *   - A sequence's tokens are cut into blocks of `block_tokens`, and every block, the unfinished one included, has a page.  A page fills up in
 *     place; once it is full and its tokens are certain (see fastrack_latent_accept) it does not change any more, and can be sealed under one
 *     IV (chunk_bytes = page bytes makes a page one chunk of fastrack_encrypt_tag).
 *   - There are two ways to attend.  With the matrices absorbed into the queries and the answers, fastrack_latent_attention works on the
 *     cache itself: 2 * (2 latent_dim + rope_dim) operations per pair of a query's head and a token, and each token is read once for all heads
 *     (or twice, for more than 64 rows of queries at a time).  That suits single tokens and drafts.  For prompts, fastrack_latent_expand makes keys and values of every head, and
 *     fastrack_latent_prompt attends over those: 2 * (key_dim + rope_dim + value_dim) operations per pair.
 *
 * Page (fastrack_latent_page_bytes): [block_tokens][latent_dim + rope_dim] 16-bit values, tokens in order.
 *
 * Conventions are those of fastrack_kv.h: int results (FASTRACK_OK or FASTRACK_ERR_*), nothing throws or prints, device pointers d_*,
 * work is asynchronous on `stream`, calls are refused with FASTRACK_ERR_ARG unless the handle's device is current.  A handle holds constants
 * only, so it may be used from several threads and on several streams at a time; the workspace that a call is given must not be
 * shared between calls that may overlap (two captured graphs that may run at the same time want one each).  No call allocates.  Every call may be captured in a CUDA graph: lengths, page numbers,
 * positions and trees are read on the device, and only the bounds in the structs below are fixed at capture.
 */
#ifndef FASTRACK_LATENT_H
#define FASTRACK_LATENT_H

#include "fastrack_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fastrack_latent fastrack_latent;

typedef struct {
    int dtype;                  /* FASTRACK_KV_BF16 / _F16: of everything that has 16 bits */
    int heads;                  /* 1 .. 1024 */
    int latent_dim;             /* 128, 256, 384 or 512 */
    int rope_dim;               /* 32 or 64 */
    int key_dim, value_dim;     /* a head's expanded key without its shared part, and its value: 64 or 128 each */
    int block_tokens;           /* 16, 32, 64 or 128 */
    int rotary;                 /* FASTRACK_ROTARY_* : how append turns the shared keys and the queries' part; NONE leaves them */
    const double* frequencies;  /* host, rope_dim / 2: radians per position of each pair, finite; copied; NULL without rotary */
    float rotary_gain;          /* turned channels are multiplied by it (1 for none) */
    float norm_eps;             /* >= 0 */
    float softmax_scale;        /* >= 0; 0: 1 / sqrt(key_dim + rope_dim) */
} fastrack_latent_config;

/* The sequences of a call, as fastrack_kv_batch has them: the new tokens of all sequences lie packed, sequence i has rows
 * d_starts[i] .. d_starts[i+1]-1 of the inputs and answers, and they are its LAST tokens: d_lens[i] counts them.  A sequence without
 * new tokens is left alone, and so are rows that belong to no sequence.  Whatever stands in d_lens, d_starts and d_table, nothing outside the bounds below is touched. */
typedef struct {
    int n_seqs;                 /* at most 65535 */
    int total_new;              /* d_starts[n_seqs], or an upper bound of it; times heads below 2^31 */
    int max_new;                /* upper bound of the new tokens of a sequence; at most total_new; times heads at most 2^30 */
    int max_len;                /* upper bound of d_lens; at most 2^30 */
    int pool_pages;             /* pages in d_pool; a table entry outside 0 .. pool_pages - 1 is an absent page: what is stored to it is
                                   dropped, and attention passes over its tokens */
    int table_stride;           /* entries in a row of d_table; at least max_len / block_tokens, rounded up */
    void* d_pool;               /* [pool_pages][page bytes], 16-byte aligned */
    const int32_t* d_table;     /* [n_seqs][table_stride]: page of each block */
    const int32_t* d_lens;      /* [n_seqs] tokens held, the new ones included */
    const int32_t* d_starts;    /* [n_seqs + 1] */
    const int64_t* d_positions; /* [total_new] position of each new token (append with rotary only; may differ from its place in the cache) */
} fastrack_latent_batch;

/* A handle for one shape of cache on the current device.  Copies the configuration; allocates 1 KiB of device memory.
 * FASTRACK_ERR_ARG for a configuration outside the ranges above. */
FASTRACK_API int fastrack_latent_create(const fastrack_latent_config* config, fastrack_latent** out);
FASTRACK_API void fastrack_latent_destroy(fastrack_latent* latent);    /* NULL is allowed; synchronises the device */
FASTRACK_API size_t fastrack_latent_page_bytes(const fastrack_latent* latent); /* 0 for NULL */
FASTRACK_API int fastrack_latent_last_cuda_error(const fastrack_latent* latent);
FASTRACK_API uint64_t fastrack_latent_launch_count(const fastrack_latent* latent);

/* Stores the new tokens.  With a norm weight, the latent x becomes x / sqrt(mean(x^2) + norm_eps) * weight (sums in 32 bits, rounded once);
 * with d_norm_weight NULL it is stored as it is.  The shared key is turned as the configuration says (see fastrack_rotary).
 *   latent, key     rows of latent_dim and rope_dim values; only their token strides count
 *   d_norm_weight   [latent_dim] 16-bit values, 16-byte aligned, or NULL
 *   q, q_out        both NULL, or [token][head] rows of rope_dim values that are turned in the same launch (they may be the same). */
FASTRACK_API int fastrack_latent_append(fastrack_latent* latent, const fastrack_latent_batch* batch, const fastrack_kv_rows* latents,
                                        const fastrack_kv_rows* key, const void* d_norm_weight, const fastrack_kv_rows* q,
                                        const fastrack_kv_rows* q_out, void* stream);

/* Bytes that fastrack_latent_attention needs as workspace for such a batch (the bounds in the struct count, not the device's values; some 40 MB); 0 for bad
 * arguments. */
FASTRACK_API size_t fastrack_latent_attention_workspace(const fastrack_latent* latent, const fastrack_latent_batch* batch);

/* Attention of the new tokens over the cache (append them first), in the latent space.  With c_t and r_t the two parts of token t:
 *     out = sum_t p_t c_t,  p = softmax_t(softmax_scale * (q . c_t + q_rope . r_t)).
 * New token j of the n of a sequence of length L stands at place L - n + j.
 *   d_parents NULL: it sees the tokens up to its own place.
 *   d_parents [total_new]: the new tokens are a tree.  d_parents[start + j] is the index among the sequence's new tokens of j's parent,
 *               less than j; anything else makes j a root.  A token sees all tokens before the new ones, itself and its ancestors.  max_new is
 *               at most FASTRACK_LATENT_TREE_MOST.
 * Absent pages' tokens are seen by nobody.  A query that sees nothing (or nothing but scores of -infinity) gets out = 0 and lse = -inf.
 * What a query does not see has no part in its answer, whatever stands there.  A token that it sees and that holds infinities or NaN makes the
 * answer NaN, unless its score is -infinity: then it does not count, but the channels that are not finite may come out NaN.
 *   q, out      rows of latent_dim values; q_rope rows of rope_dim values (turned)
 *   d_lse       [total_new][heads] float, natural logarithm of the sum of exponentials; may be NULL
 *   d_workspace 16-byte aligned, fastrack_latent_attention_workspace bytes, with no requirement on its contents.
 * The result is the same in every run. */
enum { FASTRACK_LATENT_TREE_MOST = 1024 };
FASTRACK_API int fastrack_latent_attention(fastrack_latent* latent, const fastrack_latent_batch* batch, const fastrack_kv_rows* q,
                                           const fastrack_kv_rows* q_rope, const fastrack_kv_rows* out, float* d_lse, const int32_t* d_parents,
                                           void* d_workspace, size_t workspace_bytes, void* stream);

/* Keys and values of every head for all tokens that the sequences hold: token t of sequence i goes to row d_key_starts[i] + t,
 *     k_out[row][h] = W[h][0 .. key_dim) c_t,  v_out[row][h] = W[h][key_dim .. key_dim + value_dim) c_t.
 * Products are summed in 32 bits and rounded once.  Tokens of absent pages give zeros.  Rows that no token belongs to are left alone, and so is
 * what would lie at or behind row total_keys, or in front of row 0.
 *   d_weights     [heads][key_dim + value_dim][latent_dim], 16-byte aligned
 *   d_key_starts  [n_seqs]: first row of each sequence
 * Only n_seqs, max_len, pool_pages, table_stride, d_pool, d_table and d_lens of the batch count. */
FASTRACK_API int fastrack_latent_expand(fastrack_latent* latent, const fastrack_latent_batch* batch, const void* d_weights, const fastrack_kv_rows* k_out,
                                        const fastrack_kv_rows* v_out, const int32_t* d_key_starts, int total_keys, void* stream);

/* Bytes that fastrack_latent_prompt needs as workspace (the bounds in the struct count): for answers in parts, where there are too few heads, sequences and
 * new tokens to fill the device; else 0, and 0 for bad arguments. */
FASTRACK_API size_t fastrack_latent_prompt_workspace(const fastrack_latent* latent, const fastrack_latent_batch* batch);

/* Attention of the new tokens over expanded keys and values (rows as fastrack_latent_expand writes them; total_keys rows) with the shared keys
 * from the pages:
 *     out = sum_t p_t v_t[h],  p = softmax_t(softmax_scale * (q . k_t[h] + q_rope . r_t)),
 * over the tokens up to the query's own place, without absent pages' and without those whose row lies outside 0 .. total_keys - 1.  q rows have
 * key_dim values, out rows value_dim.  Empty rows, d_lse, and what a query does not see are as above.  The result is the same in every run.
 *   d_workspace 16-byte aligned, fastrack_latent_prompt_workspace bytes, with no requirement on its contents; NULL if that is 0. */
FASTRACK_API int fastrack_latent_prompt(fastrack_latent* latent, const fastrack_latent_batch* batch, const fastrack_kv_rows* q,
                                        const fastrack_kv_rows* q_rope, const fastrack_kv_rows* k, const fastrack_kv_rows* v,
                                        const int32_t* d_key_starts, int total_keys, const fastrack_kv_rows* out, float* d_lse, void* d_workspace,
                                        size_t workspace_bytes, void* stream);

/* Keeps of a drafted tree what the model agrees with.  Row 0 of a sequence's new tokens is certain (the token that the last step ended with);
 * from there on, as long as one of the row's children holds the token that the model chose behind the row, the first such child is accepted.
 * The accepted rows' vectors move together in the pages (row k of the path to the place L - n + k), and the length becomes
 * L - n + accepted.  Drafts that were appended at positions L - n + depth are then where they belong.
 *   d_parents   [total_new] as for fastrack_latent_attention (a root other than row 0 is never accepted), or NULL: row j's parent is j - 1
 *   d_tokens    [total_new] token of each new row (row 0's does not count); d_choices [total_new] the model's choice behind each
 *   d_path      [total_new] out: the accepted rows of each sequence, from its start on, then -1
 *   d_n_accepted, d_next, d_lens_out  [n_seqs] out: accepted rows, the choice behind the last one, the new length (d_lens_out may be the
 *               batch's d_lens).  A sequence without new tokens gets 0, -1 and its length.
 * max_new is at most FASTRACK_LATENT_TREE_MOST. */
typedef struct {
    const int32_t* d_parents;
    const int32_t* d_tokens;
    const int32_t* d_choices;
    int32_t* d_path;
    int32_t* d_n_accepted;
    int32_t* d_next;
    int32_t* d_lens_out;
} fastrack_latent_acceptance;
FASTRACK_API int fastrack_latent_accept(fastrack_latent* latent, const fastrack_latent_batch* batch, const fastrack_latent_acceptance* acceptance,
                                        void* stream);

#ifdef __cplusplus
}
#endif
#endif
