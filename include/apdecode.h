/*
 * The operators of a decoder step beside the any-precision products of apgemv.h, for AMD MI355X (gfx950): rotation of q and k and
 * the append of k and v to a paged cache held in 4 bits, attention of new tokens over that cache, causal attention over packed
 * prompts, and the verification of tokens that a model at fewer bits has drafted; and what a step needs around them: attention of
 * sequences that share a prefix, the norms around a block, sampling from logits.
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
 *              whose two starts descend or leave 0 .. tokens has no tokens, nor has one that begins before the end of an earlier
 *              one).  NULL: tokens / sequences each
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
 * k_starts[s + 1] - 1 (device, sequences + 1 each, not descending; a sequence whose two starts descend or leave the rows has none, nor
 * has one any queries that begins in q_starts before the end of an earlier one); its last query sees its last key.  Query i of n sees the first m - n + 1 + i of m keys; one that sees none gets zeros, as does
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

/*
 * Attention of new tokens over the cache where sequences share prefixes: out[i] = sum_j softmax_j(scale * q[i] . k[j]) v[j] over the keys of the
 * sequence's prefix and its own.  A prefix is read once for all rows of its sequences.
 *   own        as for ap_attention_cached: q, the sequences' own keys (lengths and tables count from the first one behind the prefix), max_length
 *              the bound of their number, out, work (ap_attention_shared_size bytes).  tables may be NULL where max_length is 0
 *   prefixes   up to 2^20, (tokens * heads / 8 + (sequences + prefixes + 512) * kv_heads) < 2^24, tokens * heads < 2^24
 *   prefix_starts device, prefixes + 1: prefix p belongs to the sequences prefix_starts[p] .. prefix_starts[p + 1] - 1; not descending (a prefix
 *              whose two starts descend or leave 0 .. sequences has no sequences, nor has one whose sequences' tokens do in q_starts, or begin before the end
 *              of an earlier prefix's).  Sequences before the first and behind the last have no prefix.  NULL: sequences / prefixes each
 *   prefix_lengths device, prefixes: their keys, all of which every token of their sequences sees; above max_prefix taken as max_prefix
 *   prefix_tables  device, prefixes x prefix_width page numbers; may be NULL where max_prefix is 0
 *   max_prefix host's bound of prefix_lengths, up to prefix_width * page_tokens and 2^30: decides how the work is divided
 * A token that sees no key at all gets zeros.  A prefix need not fill its last page; pages may be shared in any way.  Scores, softmax and sums are
 * binary32.  Where prefixes have more than 64 rows per key head on average, their values enter the products as ap_cache_read gives them, rounded to
 * binary16; else, and for the sequences' own keys, as in ap_attention_cached.
 */
typedef struct {
    ap_cached own;
    int prefixes;
    const int32_t *prefix_starts, *prefix_lengths, *prefix_tables;
    int64_t prefix_width, max_prefix;
} ap_shared;
ap_status ap_attention_shared_size(const ap_cache *c, const ap_shared *a, size_t *bytes);
ap_status ap_attention_shared(const ap_cache *c, const ap_shared *a, void *stream);

/*
 * The end of one block of a decoder layer and the start of the next, in one launch:
 *   y = post ? norm(x) * post_weight + post_bias : x,   r = residual + scale * gate * y rounded to the residual's type,   out = norm(r) * weight + bias
 * with norm(a) = a / sqrt(mean(a^2) + eps), or (centred) (a - mean(a)) / sqrt(mean((a - mean(a))^2) + eps).
 *   tokens, columns  up to 2^31 - 256 rows of up to 32768 values, which are contiguous; rows may have any stride (in elements; 0 = the same row for all, of
 *              what is read; |stride| >= columns of what is written)
 *   x          binary16, the block's output; NULL = none (r = residual; gate, post and scale are not looked at)
 *   residual   binary32, or binary16 where half != 0; NULL = none (r = scale * gate * y); x and residual are not both NULL
 *   gate       binary16; NULL = 1.  A gate per channel has stride 0
 *   weight, bias, post_weight, post_bias  binary16, columns values; NULL = 1 and 0
 *   residual_out  r, of the residual's type; may be the residual itself (same address and stride); NULL = not wanted
 *   out        binary16; may be x itself (same address and stride); NULL = not wanted
 * Sums over a row are binary32 for up to 32 values and binary64 beyond; each value is computed in binary32 and rounded once, the norm of r starts from r as it is rounded.
 */
typedef struct {
    const void *data; /* device, aligned to its type */
    int64_t stride;   /* elements from row to row, |stride| < 2^40 */
} ap_rows;
typedef struct {
    ap_rows x, residual, gate, residual_out, out;
    int64_t tokens, columns;
    int half, post, centred;
    const void *weight, *bias, *post_weight, *post_bias;
    float scale, eps;
} ap_normed;
ap_status ap_norm(const ap_normed *a, void *stream);

/*
 * Tokens from logits and random numbers.  With t = temperature[r], the weight of token v of row r is exp((x[v] - max x) / t); tokens are ordered by
 * descending logit, equal ones by ascending number.  Of the first top_k of them (all where top_k[r] < 1), the shortest beginning whose weights reach
 * top_p of those' sum (all where top_p[r] is not below 1), of these the ones whose weight is at least min_p (where min_p[r] is above 0; the first one in
 * any case) are kept.  probabilities = weight / sum of the kept, 0 for the others, and tokens[r] is the first token, by number, at which the kept weights up to it pass
 * uniform[r] * their sum (the last kept one where none does: a uniform number not below 1, or NaN).
 *   t not above 0 (or NaN): the first token alone.  A logit that is NaN counts as -inf, which is never kept; where one is +inf only such are.  A row
 *   that keeps nothing has the token -1 and probabilities of 0.
 *   logits     device, rows x vocabulary binary32, or binary16 where half != 0; rows up to 2^21, vocabulary up to 2^20, contiguous in a row, stride elements
 *              from row to row
 *   uniform, temperature, top_p, min_p  device, rows binary32;  top_k  device, rows int32;  each but uniform may be NULL: 1, 1, 0 and 0
 *   tokens     device, rows
 *   probabilities device, rows x vocabulary contiguous binary32, or binary16 where half_probabilities != 0; not in the logits' memory; NULL = not wanted
 *   work       not used: ap_sample_size gives 0 for every call
 * Weights are binary64 and their sums 64-bit fixed point, exact in any order: what is kept and which token is drawn does not depend on how the work is
 * divided.  A weight below 2^-42 of the greatest (2^-62 of it times the vocabulary) may count as nothing in the sums.
 */
typedef struct {
    const void *logits;
    int64_t stride;
    int half, half_probabilities;
    int64_t rows, vocabulary;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int64_t *tokens;
    void *probabilities;
    void *work;
    size_t work_bytes;
} ap_sampling;
ap_status ap_sample_size(const ap_sampling *a, size_t *bytes);
ap_status ap_sample(const ap_sampling *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* APDECODE_H */
