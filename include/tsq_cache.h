/*
 * tsq_cache.h — C ABI of the serving side of the library (gfx950): a key/value cache held in 8 or 4 bits, in
 * blocks, and the operators that fill and read it.  It is where the keys and values of a split model live
 * on the machine that goes on with it: tsq_decompress_batch restores what the other side sent as rows
 * [tokens x kv_heads*head_dim], tsq_cache_append stores such rows, tsq_cache_attend reads them, and
 * tsq_cache_gather gives them back as rows that tsq_compress_batch sends on.
 *
 * Conventions are those of tsq.h: pointers named d_* are device pointers, `stream` is a hipStream_t as
 * void*, calls only enqueue and never synchronize, errors are return codes, the library allocates no
 * device memory.  A call whose kernels would have 2^32 threads or more is TSQ_ERR_UNSUPPORTED, and nothing of it
 * is enqueued.  Calls keep no state between them: any number of them may run at once on different
 * streams, as long as no two write the same memory.
 *
 * One cache is the keys and values of one layer: `blocks` blocks of `block_tokens` tokens.  A request owns
 * a list of blocks (a row of the block table); token t of a request lies in its block t / block_tokens at
 * place t % block_tokens.  A slot is block * block_tokens + place.
 */
#ifndef TSQ_CACHE_H
#define TSQ_CACHE_H

#include "tsq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    uint32_t blocks;        /* blocks of the cache, >= 1; blocks * block_tokens < 2^31                */
    uint32_t block_tokens;  /* tokens of a block: 16, 32, 64 or 128                                  */
    uint32_t q_heads;       /* query heads, a multiple of kv_heads, <= 1024                          */
    uint32_t kv_heads;      /* key and value heads, >= 1                                             */
    uint32_t head_dim;      /* elements of a head: 64, 128 or 256                                    */
    int32_t  dtype;         /* tsq_dtype of queries, keys, values and outputs                        */
    uint32_t max_blocks;    /* entries of a row of the block table: the most blocks of a request     */
    uint32_t reserved;      /* 0                                                                     */
} tsq_cache_config;

typedef struct tsq_cache tsq_cache;   /* opaque, host memory, never written after tsq_cache_create   */

/*
 * Device memory of one cache (the caller's; any bytes to begin with: what no token was stored to is
 * never used).  All 16-byte aligned.
 *   d_k       int8  [blocks][kv_heads][block_tokens][head_dim]
 *   d_v       int8  [blocks][kv_heads][head_dim][block_tokens]
 *   d_k_scale f32   [blocks][kv_heads]      a key is code * scale
 *   d_v_scale f32   [blocks][kv_heads]
 * Of a cache in 4 bits:
 *   d_k, d_v  uint8 [blocks][kv_heads][block_tokens][head_dim / 2]: byte j has element 2j in its low four bits,
 *             element 2j + 1 in its high ones.  Codes 0 .. 7 are 0, 0.5, 1, 1.5, 2, 3, 4, 6; 8 .. 15 the same with
 *             the sign turned
 *   d_k_scale, d_v_scale  uint8 [blocks][kv_heads][head_dim / 32][block_tokens]: scale s of 32 elements of a token
 *             says that they are code * 2^(s - 127), or NaN where s is 255
 */
typedef struct {
    void *d_k, *d_v, *d_k_scale, *d_v_scale;
} tsq_cache_memory;

typedef struct {
    uint64_t code_bytes;    /* of d_k, and of d_v                                                    */
    uint64_t scale_bytes;   /* of d_k_scale, and of d_v_scale                                        */
} tsq_cache_sizes;

/*
 * Host only; INVALID_ARG / UNSUPPORTED / NO_MEMORY without touching *out.  tsq_cache_create makes a cache in 8 bits,
 * tsq_cache_create_bits one in `bits`, 8 or 4.  All functions below take either; what is said of one alone is marked.
 */
tsq_status tsq_cache_create(const tsq_cache_config *cfg, tsq_cache **out);
tsq_status tsq_cache_create_bits(const tsq_cache_config *cfg, uint32_t bits, tsq_cache **out);
void       tsq_cache_destroy(tsq_cache *cache);
tsq_status tsq_cache_memory_sizes(const tsq_cache *cache, tsq_cache_sizes *out);

/*
 * Block tables, slots and positions of one step, from the requests' lengths.  Request r has
 * d_lengths[r] tokens in the cache and brings d_new[r] more; d_new[r] = -1 says that it is done, and its
 * blocks go back.  All integers are 32 bits signed where not said otherwise.
 *   requests         <= 4096
 *   d_new, d_lengths [requests]
 *   d_table          [requests][max_blocks]: entries before ceil(length / block_tokens) are the request's
 *                    blocks (read); those of its new blocks are written; the others are left as they are
 *   d_ring           [blocks] the free blocks, used in a ring: block number i that was ever taken or given
 *                    back is at i % blocks
 *   d_counters       int64 [2]: how many blocks were ever taken from the ring, and ever put into it
 *                    (begin with the free blocks in d_ring[0 .. n) and counters {0, n})
 *   capacity         entries of d_positions and d_slots
 * Written:
 *   d_lengths_out    [requests] lengths after the step (0 for requests that are done)
 *   d_counters_out   int64 [2]
 *   d_starts         [requests + 1] first row of each request among the step's new tokens, and their sum
 *   d_positions      [capacity] each new token's position in its request; -1 past the last token
 *   d_slots          [capacity] each new token's slot; -1 past the last token
 *   d_status         one word: TSQ_OK, or why the step cannot be taken: TSQ_ERR_CAPACITY (not enough free
 *                    blocks, a request longer than max_blocks blocks, more tokens than capacity) or
 *                    TSQ_ERR_INVALID_ARG (a length < 0 or past max_blocks blocks, d_new < -1, counters
 *                    that no ring of this size can have).  Then lengths and counters are copied, starts are
 *                    0, positions and slots are -1, and table and ring stay as they were.
 * New blocks are taken in the order of the requests; blocks given back by a call are free from the next
 * call on.  d_lengths_out, d_counters_out must not be d_lengths, d_counters.
 */
tsq_status tsq_cache_schedule(const tsq_cache *cache, uint32_t requests, const void *d_new, const void *d_lengths,
                              void *d_table, void *d_ring, const void *d_counters, uint32_t capacity,
                              void *d_lengths_out, void *d_counters_out, void *d_starts, void *d_positions,
                              void *d_slots, void *d_status, void *stream);

/*
 * RMS norm of every head of the queries and the keys, then the rotation by position:
 *   x' = x / sqrt(mean(x^2) + eps) * weight          (weight NULL: x' = x, eps not used)
 *   (a, b) -> (a cos - b sin, b cos + a sin)          for every pair (a, b) of the first `rotary` elements
 * in binary32, rounded once.  pairs: TSQ_PAIRS_HALVES: elements i and i + rotary/2; TSQ_PAIRS_NEIGHBOURS:
 * elements 2i and 2i+1; both turn by angle i.
 *   d_q, d_k         rows of q_heads (kv_heads) heads, head after head; *_stride: elements from one row to
 *                    the next, a multiple of 8; 16-byte aligned.  Outputs may be the inputs themselves
 *                    (same pointer and stride) but not overlap them otherwise
 *   d_q_weight, d_k_weight  [head_dim] of the cache's dtype, 16-byte aligned, or NULL
 *   d_angles         f32 [angle_rows][rotary]: row p holds the cosines of position p's rotary/2 angles,
 *                    then their sines; 16-byte aligned
 *   rotary           a multiple of 16, 16 <= rotary <= head_dim
 *   d_positions      int32 [tokens].  A row of a negative position is not written (see
 *                    tsq_cache_schedule); one past angle_rows becomes NaN
 * tokens 0 is a call that does nothing.
 */
typedef enum { TSQ_PAIRS_HALVES = 0, TSQ_PAIRS_NEIGHBOURS = 1 } tsq_pairs;
tsq_status tsq_cache_norm_rotate(const tsq_cache *cache, uint32_t tokens, const void *d_q, uint64_t q_stride,
                                 const void *d_k, uint64_t k_stride, const void *d_positions, const void *d_angles,
                                 uint32_t angle_rows, uint32_t rotary, int32_t pairs, const void *d_q_weight,
                                 const void *d_k_weight, float eps, void *d_q_out, uint64_t q_out_stride,
                                 void *d_k_out, uint64_t k_out_stride, void *stream);

/*
 * The same, where a position has a place on each of several axes (time, height and width of an image or a film):
 * pair i turns by its angle i at the place on axis d_axis[i].
 *   axes             1 .. 4
 *   d_positions      int32 [axes][tokens].  A row with a negative place on any axis is not written; one with a place
 *                    past angle_rows on any axis becomes NaN
 *   d_axis           uint8 [rotary / 2], 8-byte aligned; a pair of an axis that there is not becomes NaN
 */
tsq_status tsq_cache_norm_rotate_axes(const tsq_cache *cache, uint32_t tokens, const void *d_q, uint64_t q_stride, const void *d_k,
                                      uint64_t k_stride, uint32_t axes, const void *d_positions, const void *d_axis,
                                      const void *d_angles, uint32_t angle_rows, uint32_t rotary, int32_t pairs,
                                      const void *d_q_weight, const void *d_k_weight, float eps, void *d_q_out,
                                      uint64_t q_out_stride, void *d_k_out, uint64_t k_out_stride, void *stream);

/*
 * Stores rows of keys and values.  In 8 bits: for each block and head that gets tokens, with s the scale it has (0 if
 * the first of them goes to place 0: what a block held before is forgotten) and m the largest magnitude
 * among the new elements:
 *   s' = max(s, m / 127)         (m / 127 below 2^-126 counts as 0; a NaN or infinity among the new
 *                                elements makes s' NaN, and the block's head then reads as NaN)
 *   codes already there become round(code * (s / s')), new ones round(x * (1 / s')), ties to even
 * in binary32.  An element that is stored and not recoded is within s'/2 of its value.
 * In 4 bits: for each 32 elements of a token, with m the largest magnitude among them, e is the least exponent with
 *   m <= 7 * 2^e         (0 if m is 0; -23 <= e <= 13 for binary16, -120 <= e <= 125 for bfloat16)
 * and each element becomes the nearest code * 2^e, of two the one with an even code, 6 * 2^e if it is larger than
 * that: within 2^e / 4 of values up to 2 * 2^e, 2^e / 2 up to 4 * 2^e, 2^e above (but for magnitudes of binary16 above
 * 7 * 2^13 and of bfloat16 above 7 * 2^125).  A NaN or infinity among a token's keys or values of a head makes all of
 * them, keys and values, read as NaN.  A token does not change others.
 *   d_k, d_v         rows of kv_heads heads, strides as in tsq_cache_norm_rotate
 *   d_slots          int32 [tokens]: where each row goes; negative, or past the cache: the row is skipped.
 *                    In 8 bits the tokens of one block must be consecutive rows at consecutive places (as
 *                    tsq_cache_schedule makes them): each such run is stored as one.  In 4 bits they may be in any
 *                    order, but none twice (its place would get parts of both)
 */
tsq_status tsq_cache_append(const tsq_cache *cache, const tsq_cache_memory *memory, uint32_t tokens, const void *d_k,
                            uint64_t k_stride, const void *d_v, uint64_t v_stride, const void *d_slots, void *stream);

/*
 * Reads tokens back: rows d_starts[r] .. d_starts[r+1] - 1 receive the last tokens of request r, up to its
 * d_lengths[r], as code * scale rounded to the cache's dtype (exact in 4 bits).  Rows before a request's first token, and
 * blocks that the table does not hold (an entry outside the cache, or past max_blocks), read as NaN.
 *   requests         <= 65535
 *   d_table          int32 [requests][max_blocks];  d_starts int32 [requests + 1];  d_lengths int32 [requests]
 *   tokens           rows of d_k_out and d_v_out; rows that no request has are not written
 */
tsq_status tsq_cache_gather(const tsq_cache *cache, const tsq_cache_memory *memory, uint32_t requests,
                            const void *d_table, const void *d_starts, const void *d_lengths, uint32_t tokens,
                            void *d_k_out, uint64_t k_out_stride, void *d_v_out, uint64_t v_out_stride, void *stream);

/*
 * Attention of the queries in rows d_starts[r] .. d_starts[r+1] - 1 over the cache of request r, for all
 * requests.  Query i of the n that request r has stands at position p = d_lengths[r] - n + i and sees the
 * tokens t < d_lengths[r] with
 *   causal: t <= p          window > 0: t > p - window
 * out = sum of softmax(scale * q.k) v over them, and lse the natural logarithm of the softmax's
 * denominator.  A query that sees nothing gets zeros and an lse of -inf.  Out and lse of a query are NaN if
 * it sees a token of a block whose scale of keys or values is NaN for its head (in 4 bits: a token that is marked
 * as NaN), or of a table entry outside the cache, or if its request is longer than max_blocks blocks.  Query head j
 * reads kv head j / (q_heads / kv_heads).  Scales are as tsq_cache_append leaves them: 0, NaN, or at least 2^-126, and
 * in 4 bits within its exponents, or 255 in all of a token's groups, keys and values.
 *   d_q, d_out       rows of q_heads heads, strides as in tsq_cache_norm_rotate; must not overlap
 *   requests         <= 65535
 *   tokens           rows of d_q, d_out and d_lse; rows that no request has are not written
 *   max_new, max_length  the most queries of a request, and the longest length: they choose how the work is
 *                    split and size the workspace; larger requests are computed too, only slower
 *   scale            finite, > 0
 *   causal           0 or 1;  window: 0 for none
 *   d_lse            f32 [tokens][q_heads] or NULL
 *   d_ws             tsq_cache_attend_workspace_bytes() bytes for the same numbers, 256-byte aligned; needs
 *                    no reset; one call at a time.  NULL where the size is 0
 * A call may cover a part of a step's requests (d_table, d_starts and d_lengths from the first of them on;
 * rows stay those of the whole step).  Requests with up to 64 rows of a kv head (queries times query heads
 * of one kv head; 32 rows for head_dim 256) and those with more go to different kernels: max_new says which
 * a call needs.  Where the requests have a quarter of max_new queries on average, or less, both run one
 * after the other; otherwise one takes all requests.  The workspace holds the pieces that long requests are
 * cut into, for rows of the first kind of 8192 tokens or less each: it grows with max_length, which should
 * not be far above the longest request's.
 * Products are exact in binary32 sums: codes are whole numbers, and queries keep their bits, but for
 * elements of bfloat16 queries below 2^-27 of the largest of their head, which lose low bits.  scale times
 * a scale of keys is taken in binary32 and should be a normal number.  Weights of the values are rounded
 * to 11 bits; softmax statistics and all sums are binary32.
 * In 4 bits queries, keys and values are exact in either type; scores, and the sums of weights, at most 1 each, times
 * values of bfloat16 have to stay within binary32's range, and products of weights and values below 2^-126 may count as
 * 0.  A part of the work whose queries see marked tokens, or scales of bfloat16 values below 2^-19 or above 2^12, may be done
 * twice (2.3 to 2.8 times as long).
 */
tsq_status tsq_cache_attend(const tsq_cache *cache, const tsq_cache_memory *memory, uint32_t requests, const void *d_table,
                            const void *d_starts, const void *d_lengths, uint32_t tokens, uint32_t max_new,
                            uint32_t max_length, const void *d_q, uint64_t q_stride, float scale, int32_t causal,
                            uint32_t window, void *d_out, uint64_t out_stride, void *d_lse, void *d_ws, void *stream);
size_t     tsq_cache_attend_workspace_bytes(const tsq_cache *cache, uint32_t requests, uint32_t tokens, uint32_t max_new,
                                            uint32_t max_length, uint32_t window);

#ifdef __cplusplus
}
#endif

#endif
