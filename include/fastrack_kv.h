/*
 * fastrack_kv.h -- C ABI of the key-value cache operators that serve behind the sealed channel of fastrack.h.
 *
 * A model that answers through the channel keeps the keys and values of earlier tokens in device memory.  What does not
 * fit there leaves over the same PCIe link as everything else, and may lie in host memory only sealed.  So the cache is
 * made of pages that suit the link and the seal:
 *
 *   - A sequence's tokens are cut into blocks of `block_tokens`.  A full block is held in 8 bits, in one page: the codes
 *     of K and V of all kv heads and one scale per head for K and one for V.  It is quantised once, when its last token
 *     arrives, and never changes after that: a page can be sealed under one IV (chunk_bytes = page bytes makes a page
 *     one chunk of fastrack_encrypt_tag) and brought back bit for bit.
 *   - The unfinished last block stays in the 16-bit type, in a row of the `tail` buffer that belongs to the sequence.
 *
 * Page (fastrack_kv_page_bytes, a multiple of 128):
 *     K codes  [kv_heads][block_tokens][head_dim]  1 byte each
 *     V codes  [kv_heads][block_tokens][head_dim]  1 byte each
 *     scales   [kv_heads][2]                       float: K's, V's
 *     padding, never read or written
 * A code c stands for scale * c, c a signed 8-bit integer in -127 .. 127 (FASTRACK_KV_INT8) or a float of 4 exponent and 3
 * fraction bits (FASTRACK_KV_E4M3).  scale = amax / 127 or amax / 448, amax the largest magnitude of the block and head;
 * a block with amax < 2^-100 is held as zeros with scale 0.  A NaN or infinity in a block makes that block's scale (head
 * and K or V) NaN or infinite, and every answer that weighs the block NaN: it does not pass unseen.
 * Row of the tail buffer (fastrack_kv_tail_bytes): [kv_heads][2: K, V][block_tokens][head_dim] 16-bit values.  There a NaN or infinity
 * counts for the queries that see its token: K's makes their scores what it makes them, V's shows in its channels.
 *
 * Conventions are those of fastrack.h: int results (FASTRACK_OK or FASTRACK_ERR_*), nothing throws or prints, device
 * pointers d_*, work is asynchronous on `stream`, calls are refused with FASTRACK_ERR_ARG unless the handle's device is
 * current.  A handle holds constants only (no scratch), so it may be used from several threads and on several streams at
 * a time; the workspace that a call is given must not be shared between calls that may overlap.  No call allocates.  Every call may be captured in a CUDA graph: lengths, page
 * numbers and positions are read on the device, and only the bounds in the structs below are fixed at capture.
 */
#ifndef FASTRACK_KV_H
#define FASTRACK_KV_H

#include "fastrack.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FASTRACK_KV_BF16 = 0, FASTRACK_KV_F16 = 1 };     /* type of q, k, v, the answers and the tail */
enum { FASTRACK_KV_INT8 = 0, FASTRACK_KV_E4M3 = 1 };    /* what a full block is held in */
enum {
    FASTRACK_ROTARY_NONE = 0,
    FASTRACK_ROTARY_HALF = 1,                           /* pair i = channels (i, i + rotary_dim / 2) */
    FASTRACK_ROTARY_INTERLEAVED = 2                     /* pair i = channels (2 i, 2 i + 1) */
};
enum {
    FASTRACK_FREQ_PLAIN = 0,
    FASTRACK_FREQ_LINEAR = 1,                           /* every frequency divided by the factor */
    FASTRACK_FREQ_BASE = 2,                             /* the base raised so that the slowest pair is slowed by the factor */
    FASTRACK_FREQ_RAMP = 3                              /* slow pairs divided by the factor, fast ones left, a ramp between */
};

typedef struct fastrack_kv fastrack_kv;

typedef struct {
    int dtype;                  /* FASTRACK_KV_BF16 / _F16 */
    int format;                 /* FASTRACK_KV_INT8 / _E4M3 */
    int q_heads, kv_heads;      /* 1 .. 1024, q_heads a multiple of kv_heads; q head h reads kv head h / (q_heads / kv_heads) */
    int head_dim;               /* 64, 96 or 128 */
    int block_tokens;           /* 16, 32, 64 or 128 */
    int rotary;                 /* FASTRACK_ROTARY_* */
    int rotary_dim;             /* channels that are turned, from the first on: a multiple of 16, at most head_dim; 0 without rotary */
    const double* frequencies;  /* host, rotary_dim / 2: radians per position of each pair, finite; copied */
    float rotary_gain;          /* turned channels are multiplied by it (1 for none) */
    float softmax_scale;        /* >= 0; 0: 1 / sqrt(head_dim) */
} fastrack_kv_config;

/* The sequences of a call.  The new tokens of all sequences lie packed: sequence i has rows d_starts[i] .. d_starts[i+1]-1
 * of q, k and v, and they are its LAST tokens: d_lens[i] counts them.  The same struct serves the append of the tokens and
 * the attention of their queries.  A sequence without new tokens is left alone.  q, k, v, their positions and the answers have
 * total_new rows. */
typedef struct {
    int n_seqs;                 /* at most 65535 */
    int total_new;              /* d_starts[n_seqs], or an upper bound of it; times q_heads below 2^31 */
    int max_new;                /* upper bound of the new tokens of a sequence; at most total_new; times q_heads at most 2^30 */
    int max_len;                /* upper bound of d_lens; at most 2^30 */
    int pool_pages;             /* pages in d_pool; a table entry outside 0 .. pool_pages - 1 is an absent page: what is appended to
                                   it is dropped, and attention passes over its tokens */
    int table_stride;           /* entries in a row of d_table; at least max_len / block_tokens */
    void* d_pool;               /* [pool_pages][page bytes], 16-byte aligned */
    void* d_tail;               /* [n_seqs][tail bytes], 16-byte aligned */
    const int32_t* d_table;     /* [n_seqs][table_stride]: page of each full block */
    const int32_t* d_lens;      /* [n_seqs] tokens held, the new ones included */
    const int32_t* d_starts;    /* [n_seqs + 1] */
    const int64_t* d_positions; /* [total_new] position of each new token (rotary only; may differ from its place in the cache) */
} fastrack_kv_batch;

/* Rows of 16-bit vectors: token t, head h at data + t * token_stride + h * head_stride values, head_dim values in one
 * piece.  data is 16-byte aligned and the strides are multiples of 8 values. */
typedef struct {
    void* data;
    int64_t token_stride, head_stride;
} fastrack_kv_rows;

/* A handle for one shape of cache on the current device.  Copies the configuration; allocates 1 KiB of device memory.
 * FASTRACK_ERR_ARG for a configuration outside the ranges above. */
FASTRACK_API int fastrack_kv_create(const fastrack_kv_config* config, fastrack_kv** out);
FASTRACK_API void fastrack_kv_destroy(fastrack_kv* kv);            /* NULL is allowed; synchronises the device */
FASTRACK_API size_t fastrack_kv_page_bytes(const fastrack_kv* kv); /* 0 for NULL */
FASTRACK_API size_t fastrack_kv_tail_bytes(const fastrack_kv* kv); /* 0 for NULL */
FASTRACK_API int fastrack_kv_last_cuda_error(const fastrack_kv* kv);
FASTRACK_API uint64_t fastrack_kv_launch_count(const fastrack_kv* kv);

/* Frequencies base^(-2 i / rotary_dim) of the pairs i = 0 .. rotary_dim / 2 - 1, changed for a context `factor` times as
 * long as the `original_len` positions that the model was trained on, as FASTRACK_FREQ_* says.  RAMP: a pair that makes
 * more than 32 turns in original_len positions is left, one that makes fewer than 1 is divided by the factor, and between
 * the two the share follows the turns; *gain is then 0.1 ln(factor) + 1, otherwise 1.  Host only.
 * frequencies: rotary_dim / 2 doubles out; gain may be NULL.  factor >= 1, base > 1, rotary_dim even and >= 2 (>= 4 for BASE). */
FASTRACK_API int fastrack_rotary_frequencies(int rotary_dim, double base, int scaling, double factor, double original_len,
                                             double* frequencies, float* gain);

/* Rotary positions: pair (a, b) of a token at position p becomes gain * (a cos w - b sin w, b cos w + a sin w), w = p * frequency.
 * inverse != 0 turns by -w (the gain stays): that is the gradient of the input from the gradient of the output.
 * The angle is formed modulo one turn in 64-bit fixed point: at position p it is off by at most 2^-32 + |p| 2^-63 of a turn (for
 * frequencies up to a turn per position), which is 2^-31 up to p = 2^31 and 2^-23 at 2^40.
 * Channels from rotary_dim on are copied.  in == out (same strides) is allowed; other overlap is not checked.
 * `heads` need not be the configuration's.  tokens == 0 or heads == 0: nothing is done. */
FASTRACK_API int fastrack_rotary(fastrack_kv* kv, int64_t tokens, int heads, const fastrack_kv_rows* in, const fastrack_kv_rows* out,
                                 const int64_t* d_positions, int inverse, void* stream);

/* Appends the new tokens: K is turned as the configuration says, V is taken as it is; blocks that get complete are quantised
 * into their pages (from the unrounded turned values), the rest goes to the tail.  q (may be NULL): turned into q_out in the
 * same launch. */
FASTRACK_API int fastrack_kv_append(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* k, const fastrack_kv_rows* v,
                                    const fastrack_kv_rows* q, const fastrack_kv_rows* q_out, void* stream);

/* The values held, in the 16-bit type: token t of sequence i goes to row i * max_len + t of k_out and v_out (kv_heads heads);
 * rows from the sequence's length up to max_len, and those of absent pages, become zeros. */
FASTRACK_API int fastrack_kv_read(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* k_out,
                                  const fastrack_kv_rows* v_out, void* stream);

/* Bytes that fastrack_kv_attention needs as workspace for such a batch (the bounds in the struct count, not the device's
 * values); 0 for bad arguments.  With weights it grows with max_new * max_len (4 bytes per q head and 16 to 64 tokens): long prompts
 * are best taken in pieces of some thousand tokens. */
FASTRACK_API size_t fastrack_kv_attention_workspace(const fastrack_kv* kv, const fastrack_kv_batch* batch, int with_mass);

/* Attention of the new tokens over the cache (append them first).  Query j of the n new ones of a sequence of length L stands at
 * place i = L - n + j and sees the tokens t <= i, with window > 0 only those t > i - window (a window of max_len or more hides
 * nothing), without absent pages:
 *     out = sum_t p_t v_t,  p = softmax_t(softmax_scale * q . k_t).
 * A query that sees nothing gets out = 0 and lse = -inf.  What a query does not see has no part in its answer, whatever stands there.  What it
 * sees counts by its share of the answer: the weights, of 11 bits (bf16) or 22 (f16), are held down to 2^-25 of the largest weight times
 * scale of V.
 *   d_lse       [total_new][q_heads] float, natural logarithm of the sum of exponentials; may be NULL.
 *   d_mass_in, d_mass_out  [n_seqs][kv_heads][mass_stride] float; both NULL, or both set (they may be the same).  For every block of a
 *               sequence, the unfinished one included: out = in + the sum of p over the block's tokens, the sequence's new
 *               queries and the q heads of the kv head.  The entries behind a sequence's last block are left alone.
 *               mass_stride >= ceil(max_len / block_tokens).
 *   d_workspace 16-byte aligned, fastrack_kv_attention_workspace bytes, with no requirement on its contents.
 * The result does not depend on the other sequences' contents, and is the same in every run. */
FASTRACK_API int fastrack_kv_attention(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* q, const fastrack_kv_rows* out,
                                       float* d_lse, int window, const float* d_mass_in, float* d_mass_out, int mass_stride,
                                       void* d_workspace, size_t workspace_bytes, void* stream);

/* Eviction by accumulated weight.  A full block's score is the sum of its weights over the kv heads (added in 64 bits, rounded to
 * float).  Of a sequence with more than `budget` full blocks, the full - budget blocks with the least scores leave, among equals
 * the lowest index first, a NaN counting as more than any number; the first keep_first and the last keep_last full blocks and the
 * unfinished one never leave (so fewer may go than the budget asks).  The rest move up in order.
 * Pages are not touched: seal or free those that d_evicted lists.
 *   d_table, d_lens, d_mass -> d_table_out, d_lens_out, d_mass_out: pairwise the same pointer (in place) or apart.  Entries behind
 *   the last block become -1 (table) and 0 (mass).  d_evicted [n_seqs][table_stride]: pages that left, in block order, then -1.
 *   d_n_evicted [n_seqs]. */
typedef struct {
    int n_seqs, table_stride, mass_stride;      /* strides: at least ceil(length / block_tokens) of every sequence */
    int budget, keep_first, keep_last;          /* >= 0 */
    const int32_t* d_table;
    const int32_t* d_lens;
    const float* d_mass;
    int32_t* d_table_out;
    int32_t* d_lens_out;
    float* d_mass_out;
    int32_t* d_evicted;
    int32_t* d_n_evicted;
} fastrack_kv_eviction;
FASTRACK_API int fastrack_kv_evict(fastrack_kv* kv, const fastrack_kv_eviction* eviction, void* stream);

#ifdef __cplusplus
}
#endif
#endif
