/*
 * The operators of a decoder step beside the any-precision products of apgemv.h, for AMD MI355X (gfx950): rotation of q and k and
 * the append of k and v to a paged cache held in 4 bits, attention of new tokens over that cache, causal attention over packed
 * prompts, and the verification of tokens that a model at fewer bits has drafted.
 *
 * Conventions are those of apgemv.h: activations are binary16, every function returns an ap_status and neither throws, aborts nor
 * prints, arguments are checked before the first HIP call, work is enqueued on `stream` (a hipStream_t; NULL = the default stream),
 * nothing is allocated or synchronised, and results do not depend on the order in which workgroups run.
 *
 * Sizes: head_dim is 64 or 128 (AP_ERR_SHAPE otherwise); heads is a multiple of kv_heads, and head i uses key head i / (heads /
 * kv_heads).  Rows of head_dim values are contiguous and 16-byte aligned; tokens and heads may have any strides that keep them so.
 * Up to 4096 heads, 1024 key heads, 2^31 - 256 tokens, 2^20 sequences.
 *
 * What the device reads as data (slots, positions, page numbers, lengths, starts) cannot be checked on the host.  No value of it
 * makes a kernel read or write outside the arrays described here; each function says what it makes of values out of range.
 */
#ifndef APDECODE_H
#define APDECODE_H

#include "apgemv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* binary16 rows: head h of token t starts at data + t * token_stride + h * head_stride (in elements, multiples of 8) */
typedef struct {
    void *data; /* device, 16-byte aligned */
    int64_t token_stride, head_stride;
} ap_heads;

/*
 * A paged cache.  A page holds page_tokens tokens of every key head, and a token's place is its slot: page * page_tokens + place in
 * the page.  Keys and values are held as 16 evenly spaced values per token and head: low + scale * code with low the least of the
 * head_dim values, scale = (greatest - least) / 15 rounded to binary16, and code the nearest of 0..15 (ties to even).  Of a row
 * with an infinity or a NaN every value reads back as NaN.  head_dim / 2 + 4 bytes per token, head and side.
 *
 * What 4 bits cost: on normally distributed rows (1000 keys) the result of attention is 13 % (head_dim 64) to 14 % (128) of its norm away from that over
 * the unrounded keys and values, 9 to 10 % each from keys and values.  One step serves a whole row: where one channel of the keys is 8
 * times the others it is 34 to 38 %.  Whether a model bears that is for its user to measure; there is no wider format.
 *
 * Page and head are contiguous: key codes of the page's tokens, value codes, then (low, scale) pairs of the keys and of the values.
 */
typedef struct {
    void *data;    /* device, ap_cache_size bytes, 256-byte aligned, caller-owned; needs no initialisation */
    int64_t pages; /* pages * page_tokens < 2^40 */
    int page_tokens; /* 16, 32, 64, 128 or 256 */
    int kv_heads;    /* 1 .. 1024 */
    int head_dim;
} ap_cache;

/* Bytes of the cache that c describes; c->data is not looked at. */
ap_status ap_cache_size(const ap_cache *c, size_t *bytes);

/*
 * Rotates q and k and appends k and v to the cache, in one launch.
 *   q, k, v    tokens rows of heads (q) and c->kv_heads (k, v) heads; q.data may be NULL (no queries), heads is then ignored
 *   slots      device, one per token: where its k and v go; a slot outside the cache (-1 by custom) keeps the token out of it.  Two
 *              tokens with one slot leave a mixture there
 *   rotary     device, rotary_rows x rot_dim binary32: row p holds the rot_dim / 2 cosines, then the sines of position p; NULL = no
 *              rotation
 *   positions  device, one per token (with rotary); the rotated channels of a token whose position is outside the table become NaN
 *   rot_dim    channels that are rotated, a multiple of 16 up to head_dim; the others stay
 *   interleaved 0: channel i turns with channel i + rot_dim / 2; 1: channel 2i with 2i + 1
 *   q_out, k_out  the rotated rows; may be q and k themselves (same addresses and strides).  k_out.data may be NULL.  The cache
 *              holds k as rounded there
 * x1' = x1 cos - x2 sin and x2' = x2 cos + x1 sin in binary32, every product and sum rounded by itself, then rounded to binary16.
 */
typedef struct {
    ap_heads q, k, v, q_out, k_out;
    int heads;
    int64_t tokens;
    const int64_t *slots, *positions;
    const float *rotary;
    int64_t rotary_rows;
    int rot_dim, interleaved;
} ap_append;
ap_status ap_cache_append(const ap_cache *c, const ap_append *a, void *stream);

/* The values that slots of the cache stand for, rounded to binary16 (at most 65504): k_out, v_out device, tokens x kv_heads x
 * head_dim, contiguous and 16-byte aligned; zeros for a slot outside the cache. */
ap_status ap_cache_read(const ap_cache *c, const int64_t *slots, int64_t tokens, void *k_out, void *v_out, void *stream);

/*
 * Attention of new tokens (tokens * heads / 16 + sequences * kv_heads < 2^24) over the cache: out[i] = sum_j softmax_j(scale * q[i] . k[j]) v[j].
 *   q          tokens rows of heads heads; the tokens of a sequence are adjacent
 *   q_starts   device, sequences + 1: sequence s has the tokens q_starts[s] .. q_starts[s + 1] - 1; not descending (a sequence
 *              whose two starts descend or leave 0 .. tokens has no tokens).  NULL: tokens / sequences each
 *   lengths    device, sequences: the keys of a sequence, its new tokens included (they have been appended): token i of n sees the
 *              first lengths[s] - n + 1 + i keys.  A token that sees none gets zeros.  Lengths above max_length are taken as
 *              max_length
 *   tables     device, sequences x table_width page numbers; a page outside the cache holds no keys
 *   max_length host's bound of the lengths, up to table_width * page_tokens and 2^30: decides how the work is divided
 *   out        device, tokens x heads x head_dim, contiguous, 16-byte aligned; only the tokens of q_starts are written
 *   work       device, ap_attention_cached_size bytes, 16-byte aligned; may be NULL where that is 0
 * Scores, softmax and sums are binary32; the weights of the values, times their steps, have 16 bits.  Long sequences are divided among workgroups and
 * joined by a second launch.
 */
typedef struct {
    ap_heads q;
    int heads;
    int64_t tokens;
    int sequences;
    const int32_t *q_starts, *lengths, *tables;
    int64_t table_width, max_length;
    float scale;
    void *out, *work;
    size_t work_bytes;
} ap_cached;
ap_status ap_attention_cached_size(const ap_cache *c, const ap_cached *a, size_t *bytes);
ap_status ap_attention_cached(const ap_cache *c, const ap_cached *a, void *stream);

/*
 * Causal attention over packed sequences: sequence s has the queries q_starts[s] .. q_starts[s + 1] - 1 and the keys k_starts[s] ..
 * k_starts[s + 1] - 1 (device, sequences + 1 each, not descending; a sequence whose two starts descend or leave the rows has none);
 * its last query sees its last key.  Query i of n sees the first m - n + 1 + i of m keys; one that sees none gets zeros, as does
 * one whose scores are all -inf.  What a query does not see does not reach it, NaN and infinities included.
 *   q; k, v    tokens rows of heads heads (tokens * heads < 2^31 - 256, tokens * heads / 128 + sequences * kv_heads < 2^24); keys (up to
 *              2^30) rows of kv_heads heads, their token strides in 0 .. 2^24 (AP_ERR_SHAPE otherwise)
 *   out        device, tokens x heads x head_dim, contiguous, 16-byte aligned; only the tokens of q_starts are written
 *   work       device, ap_attention_prompt_size bytes, 16-byte aligned; may be NULL where that is 0
 * Scores, softmax and sums are binary32; the weights of the values are rounded to binary16.  Where the rows are too few for the
 * card the keys are divided among workgroups and joined by a second launch.
 */
typedef struct {
    ap_heads q, k, v;
    int heads, kv_heads, head_dim;
    int64_t tokens, keys;
    int sequences;
    const int32_t *q_starts, *k_starts;
    float scale;
    void *out, *work;
    size_t work_bytes;
} ap_prompt;
ap_status ap_attention_prompt_size(const ap_prompt *a, size_t *bytes);
ap_status ap_attention_prompt(const ap_prompt *a, void *stream);

/*
 * Verification of drafted tokens.  Sequence s has counts[s] drafts (drafts each where counts is NULL; a count outside 0..drafts is
 * taken as the nearest).  Draft i is accepted while uniform[i] * draft[i][x] < target[i][x] for its token x (binary32).
 * accepted[s] = n is how many are; the token after them is the one with the greatest w[v] / noise[v], the lowest of equals, among
 * those with w[v] > 0 and noise[v] >= 0 (-1 if there is none), where w = target[n] - draft[n] after a refusal (or target[n] where
 * no token has more than its draft) and w = target[n] after all counts[s] drafts.  With uniform numbers in [0, 1) and noise from
 * the exponential distribution the tokens are distributed as the target's own.
 *   target     device, sequences x (drafts + 1) x vocabulary probabilities;  draft  device, sequences x drafts x vocabulary
 *              binary32, or binary16 where half != 0; contiguous; vocabulary < 2^31
 *   drafted    device, sequences x drafts; a token outside the vocabulary is refused
 *   uniform    device, sequences x drafts binary32;  noise  device, sequences x vocabulary binary32
 *   tokens     device, sequences x (drafts + 1): the accepted drafts, the token after them, then -1
 *   accepted   device, sequences
 *   work       device, ap_verify_size bytes, 16-byte aligned; may be NULL where that is 0
 */
typedef struct {
    const void *target, *draft;
    int half;
    int sequences, drafts;
    int64_t vocabulary;
    const int64_t *drafted;
    const float *uniform, *noise;
    const int32_t *counts;
    int64_t *tokens;
    int32_t *accepted;
    void *work;
    size_t work_bytes;
} ap_verification;
ap_status ap_verify_size(const ap_verification *a, size_t *bytes);
ap_status ap_verify(const ap_verification *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* APDECODE_H */
