/*
 * hv_fp8_cache.h -- a cache of keys and values held in 8 bits, and attention over it.
 *
 * What stands between a decoder's projections on verified 8-bit weights (hv_fp8.h):
 * new tokens' keys and values go to pages of a cache, and the tokens' queries are
 * answered from there, one at a time or whole prompts.
 *
 * Format.  A cache is a pool of pages of `page_tokens` tokens each, for every key
 * head.  Codes are OCP E4M3 as in hv_fp8.h.  16 consecutive tokens of a page
 * and head are a block and share a scale, one for their keys and one for their
 * values.  A scale is a power of two from 2^-126 to 2^127 (a 32-bit number of which
 * only the exponent is read); the value of a code is the code's number times it.
 * Keys lie token by token, values of a block dimension by dimension, as the matrix
 * unit reads them:
 *   k_codes [pages][kv_heads][page_tokens][head_dim]
 *   v_codes [pages][kv_heads][page_tokens / 16][head_dim][16]
 *   k_scales, v_scales [pages][kv_heads][page_tokens / 16]
 * Pages and heads of the codes may lie any multiple of 16 bytes apart that keeps
 * them from overlapping; the rest is contiguous.  Codes are 16-byte aligned.
 *
 * Batches.  A call serves `count` sequences.  Sequence i has, with this call's new
 * tokens, lengths[i] tokens; the new ones are the last of them and take the rows
 * starts[i] to starts[i + 1] - 1 of the call's matrices, no row of two sequences, so a token in row t has
 * the position lengths[i] - starts[i + 1] + t.  The token at position p of sequence
 * i lies in page pages[i][p / page_tokens].  All three are device memory that the
 * call's kernels read, so a captured call takes what they hold when it is replayed.
 * What they may not hold is dealt with as follows, and nothing out of bounds is read
 * or written: a sequence of no rows, and one whose rows are not within the
 * call's, is left out (its rows, like those that belong to no sequence, are neither read nor
 * written); tokens at negative positions, behind the table's last column or in a page that
 * does not exist (any negative number may stand for none) are not in the cache: they are
 * neither written nor seen.
 *
 * Every call is asynchronous on `stream` and queues kernels only, so it may be
 * captured in a HIP graph.  All pointers but those to the two descriptions are
 * device pointers of the device that is current; the descriptions are read before the call
 * returns.  Strides count elements.  Rows of the wider
 * matrices need no alignment beyond that of their element type; 16-byte aligned ones
 * are read faster.  Inputs and outputs must not overlap.  A call with no elements to write
 * does nothing.  Results do not depend on the stream or on what runs beside, and are equal
 * bit for bit from call to call.
 *
 * Common errors: HV_ERR_INVALID_ARG for an unknown type, a NULL or misaligned pointer,
 * strides that overlap, a head_dim that is no multiple of 16 from 16 to 256, a
 * page_tokens that is no multiple of 16 from 16 to 65536, or sizes past the limits (pages
 * 2^31 - 1, kv_heads 65535, sequences 65536, columns * page_tokens 2^30, tokens * heads
 * 2^30, strides 2^40, all of an operand 2^62); HV_ERR_HIP.
 */
#ifndef HV_FP8_CACHE_H
#define HV_FP8_CACHE_H

#include "hv_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HV_FP8_CACHE_BLOCK 16 /* tokens of a head that share a scale */

typedef struct {
    uint8_t* k_codes;
    float* k_scales;
    uint8_t* v_codes;
    float* v_scales;
    uint64_t pages, kv_heads, page_tokens, head_dim;
    uint64_t k_page, k_head; /* bytes between the keys of neighbouring pages, and heads */
    uint64_t v_page, v_head;
} hv_fp8_cache;

typedef struct {
    const int32_t* starts;  /* [count + 1] */
    const int32_t* lengths; /* [count] */
    const int32_t* pages;   /* [count][columns], rows ld_pages apart */
    uint64_t count, columns, ld_pages;
} hv_fp8_batch;

/* Writes the new tokens' keys and values.
 * A block's scale is the smallest power of two (at least 2^-126) under which the finite
 * new values written to it have codes of at most 448, or the scale that it had if that is
 * larger and the block holds earlier tokens of the sequence.  Where it grows, the
 * earlier tokens' codes are rounded to it.  (The scale being a power of two, that
 * changes only codes that get below 2^-6, by at most half of the new scale's 2^-9.)
 * A new value's code is value / scale rounded to the nearest E4M3 number, ties to
 * even; a NaN or an infinity becomes a NaN code and leaves the rest of its block alone.
 * Slots of a block behind its last new token stay as they are and hold nothing.
 * No page may be written by two sequences in one call, nor by two columns of one.
 *   k, v: [tokens][kv_heads][head_dim] of the type, the dimensions of a head adjacent. */
hv_status hv_fp8_cache_write(const hv_fp8_cache* cache, const hv_fp8_batch* batch, hv_type type, const void* k,
                             uint64_t k_token, uint64_t k_head, const void* v, uint64_t v_token, uint64_t v_head,
                             uint64_t tokens, hipStream_t stream);

/* Scratch bytes hv_fp8_attention needs; 0 where it needs none, and for sizes that it refuses.
 * `capacity`: columns * page_tokens of the batch. */
size_t hv_fp8_attention_workspace_bytes(uint64_t sequences, uint64_t capacity, uint64_t tokens, uint64_t heads,
                                        uint64_t kv_heads, uint64_t head_dim, uint32_t window, uint32_t sinks);

/* Attention of the batch's new tokens over the cache, in which they are already:
 *   out[t][h] = sum over visible positions j of w_j v_j,
 *   w = softmax over them of scale * (q[t][h] . k_j),
 * with the keys and values of key head h / (heads / kv_heads).  A token at position
 * p sees the positions j <= p that are in the cache; with a window, of these only the
 * last `window` (p - j < window) and the first `sinks` (j < sinks).  A token that sees
 * nothing gets zeros.  What a token does not see does not change its output, whatever it
 * holds (NaN included).
 * Products of q and codes and of weights and codes are added in 32 bits, the softmax
 * is in 32 bits; a weight is rounded to the type before its product, relative to its row's
 * largest, and the result once.  Finite scores of any size are kept apart as far as 32 bits do.  Scores beyond 32 bits,
 * their sums before the key scale, and `scale` times a key scale beyond them give NaN or, where all of a token's scores are
 * minus infinity, zeros; values whose sums, by weights of up to 2^8 that are divided by theirs at the end,
 * are beyond 32 bits give infinities or NaN.  For HV_BF16, values (codes times their scale) below 2^-126 are rounded to
 * multiples of 2^-133.
 *   type: HV_BF16 or HV_F16, of q and out.
 *   q, out: [tokens][heads][head_dim], the dimensions of a head adjacent; kv_heads divides heads.
 *   scale: positive and finite, at least 2^-126.
 *   window: 0 for none; sinks count only beside a window.
 *   workspace: >= hv_fp8_attention_workspace_bytes(...), 256-byte aligned; NULL where that is 0.
 *              Scratch: calls that share one must share a stream.
 * For HV_F16, a weight is rounded together with its block's value scale, relative to the largest weight
 * and the largest scale of what the token sees: products of the two below 2^-18 begin to lose bits, below 2^-29 all.
 * Errors: HV_ERR_INVALID_ARG also for another type, heads that are no multiple of kv_heads, or another
 * scale; HV_ERR_WORKSPACE for a missing, short or misaligned workspace. */
hv_status hv_fp8_attention(const hv_fp8_cache* cache, const hv_fp8_batch* batch, hv_type type, const void* q,
                           uint64_t q_token, uint64_t q_head, uint64_t tokens, uint64_t heads, float scale,
                           uint32_t window, uint32_t sinks, void* out, uint64_t out_token, uint64_t out_head,
                           void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HV_FP8_CACHE_H */
