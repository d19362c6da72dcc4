/*
 * focused_attention.h - C ABI of the attention operators of the focused convolution library for AMD MI355X (gfx950): a key/value
 * cache in 8 bits, attention over it, and attention over the blocks that a score selects.
 *
 * A focused convolution computes where a mask says that the input matters; fc_focused_attention is the same for attention: a cheap
 * score labels blocks of the cache, the labels become ordered lists on the device, and the unchanged arithmetic runs on the listed
 * blocks only.  fc_cache_attention is its counterpart without labels.
 *
 * The cache
 *   - A block is 64 consecutive tokens of one sequence.  The cache is a pool of blocks; row b of `table` ([batch][table_width],
 *     device) holds the pool's numbers of the blocks of sequence b in order.  An entry outside [0, blocks) is a block that is not there:
 *     its tokens are written nowhere, read as zeros (fc_kv_read) and attended to by nobody.
 *   - Keys and values are E4M3 codes (FC_FP8) with one scale for each block, head, and kind (key or value).  The scale is a power of two,
 *     2^e with the least e of [-64, 120] for which no finite value of the block exceeds 448 * 2^e; code = value / scale, rounded
 *     to the nearest, ties to even.  (The format's relative precision does not depend on the scale, so a power of two gives nothing away, and
 *     scaling is exact.)  NaN and infinities become NaN.
 *   - Tokens appended to a block that already holds some keep its scale or raise it; raising rounds the codes that are there again
 *     (exact except below 2^-6 in units of the new scale).
 *   - A block's sketch is made when its 64th token is written: the sums of the keys' codes over the 64 tokens (NaN counts as zero), a = the largest
 *     magnitude among its channels, 2^f the least power of two with a <= 127 * 2^f, sketch = round(sum / 2^f) to nearest even, and
 *     its weight 2^f / 64 * scale.
 *   - The layout is the library's own (fc_kv_cache_bytes gives its size); nothing has to be cleared before the first use.
 *     A block in use by several sequences is fine as long as nobody appends to it.
 *
 * Sequences
 *   - lengths[b] (device) counts the tokens of sequence b with the new ones, which are its last; rows starts[b] .. starts[b + 1] of the call's
 *     tensors (device, [batch + 1]) are its new tokens.  starts NULL: max_new rows for every sequence, tokens = batch * max_new.
 *     Without rows (tokens 0) there is nothing to do, whatever max_new is.
 *   - Rows with no position (more new tokens than the length) are dropped by fc_kv_append, read as zeros, and attend to nothing.
 *   - Bounds known to the host: max_new >= every sequence's new tokens, max_len >= every length.  What the device's arrays say beyond
 *     these bounds, beyond `tokens` or beyond the table is cut off, so wrong contents give wrong results and never an access out of range.
 *     Work is laid out by the bounds: batch, max_new and heads that come to more workgroups than a launch holds (2^32 threads) give FC_ERR_RANGE.
 *
 * Attention
 *   - Query head h reads key/value head h / (heads / kv_heads).  Row i of the n new tokens of a sequence has position
 *     p = length - n + i and attends to positions 0 .. p with FC_CAUSAL, to all of the length without.
 *   - out = sum_t softmax_t(scale * q.k_t) v_t with keys and values as the cache holds them.  Products of stored values accumulated
 *     in 32 bits; softmax in 32 bits; weights rounded to 11 bits (f16) for their product with the values, steps of 2^-30 of the largest at
 *     least; one rounding to the output type.
 *   - What a row does not attend to has no influence on it, NaN included.  A row that attends to nothing is +0.0 with lse = -infinity, and so is one
 *     whose scores are all -infinity (a query of infinity against keys of one sign).
 *   - lse, where it is wanted: log(sum_t exp(scale * q.k_t)) in 32 bits, [tokens][heads].
 *
 * Selection (fc_focused_attention; FC_CAUSAL is implied)
 *   - For each row and key head, own = p / 64: blocks 0 .. first - 1, blocks own - last + 1 .. own (last >= 1), and of the others up to own
 *     the `top` with the largest score, ties to the lowest number.
 *   - score = float(sum over the group's heads and the channels of q8 * sketch) * weight, q8 = round(q / 2^g) to nearest even, 2^g the least power of
 *     two (g of [-126, 120]) with |q| <= 127 * 2^g over the group's heads (not-finite values count as zero).  The sum is of whole numbers, so a
 *     selection does not depend on the order of summation.  A group has at most 32767 heads, a sequence's bound is at most 32768 blocks (FC_ERR_RANGE).
 *   - selected: [tokens][kv_heads][first + last + top], block numbers of the sequence, ascending, -1 behind the last.
 *
 * Conventions are those of focused_conv.h: device pointers, a stream, nothing allocated and no waiting, argument errors found before
 * anything is launched, launches only (calls can be captured after one eager call).  q, k, v: any strides of rows and heads, channels
 * next to each other, aligned to their element; the other pointers 16 bytes.
 */
#ifndef FOCUSED_ATTENTION_H
#define FOCUSED_ATTENTION_H

#include "focused_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    FC_CAUSAL = 1u /* a row attends to no position after its own; FC_WORKSPACE_READY (4) as for convolutions */
};

enum { FC_KV_BLOCK = 64 };        /* tokens of a block */
enum { FC_KV_MAX_HEAD_DIM = 256 };
enum { FC_MAX_SELECTED = 1024 };  /* first + last + top */

typedef struct {
    int32_t blocks, kv_heads, head_dim;                 /* the cache: blocks of the pool, heads, channels of a head (1 .. 256) */
    int32_t batch, tokens, max_new, max_len, table_width; /* sequences, rows of q / k / v, bounds, entries of a table row */
    int32_t heads;                                      /* query heads, a multiple of kv_heads */
    int32_t dtype;                                      /* of q, k, v and out: FC_BF16 or FC_F16 */
    uint32_t flags;                                     /* FC_CAUSAL, FC_WORKSPACE_READY */
    int32_t first, last, top;                           /* selection */
    float scale;                                        /* of the products q.k, finite */
    int32_t reserved;                                   /* zero */
    int64_t q_row, q_head, k_row, k_head, v_row, v_head; /* strides in elements, >= 0 */
} fc_attention_desc;

/* Bytes of a cache (fields blocks, kv_heads, head_dim). */
int32_t fc_kv_cache_bytes(const fc_attention_desc *d, size_t *bytes);

/* Rounds the new tokens' keys and values into the cache.  Fields read: the cache's, the sequences', dtype, strides of k and v.
 * k, v: [tokens][kv_heads][head_dim].  No two sequences may append to the same block. */
int32_t fc_kv_append(const fc_attention_desc *d, void *cache, const void *k, const void *v, const int32_t *table,
                     const int32_t *lengths, const int32_t *starts, void *stream);

/* The last starts[b + 1] - starts[b] tokens of every sequence as 32-bit values: k, v [tokens][kv_heads][head_dim] (either may be NULL).
 * (A bf16 value above 2^128 - 2^123 rounds up to a code for 2^128 and reads as infinity.) */
int32_t fc_kv_read(const fc_attention_desc *d, const void *cache, const int32_t *table, const int32_t *lengths, const int32_t *starts,
                   float *k, float *v, void *stream);

/* Bytes of workspace for the two calls below (zero: none is needed).  With FC_WORKSPACE_READY in flags the caller vouches that the workspace's
 * counters are zero, as a workspace that was zeroed once has them, and from then on after every completed call of one of these functions with
 * this descriptor: it saves the launch that clears them (fc_cache_attention; the selection of fc_focused_attention clears them beside its work). */
int32_t fc_cache_attention_workspace_bytes(const fc_attention_desc *d, size_t *bytes);
int32_t fc_focused_attention_workspace_bytes(const fc_attention_desc *d, size_t *bytes);

/* q [tokens][heads][head_dim] (strides), out [tokens][heads][head_dim] dense, lse [tokens][heads] or NULL. */
int32_t fc_cache_attention(const fc_attention_desc *d, const void *cache, const void *q, const int32_t *table, const int32_t *lengths,
                           const int32_t *starts, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream);
int32_t fc_focused_attention(const fc_attention_desc *d, const void *cache, const void *q, const int32_t *table, const int32_t *lengths,
                             const int32_t *starts, void *out, float *lse, int32_t *selected, void *workspace, size_t workspace_bytes,
                             void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FOCUSED_ATTENTION_H */
