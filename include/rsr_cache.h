/*
 * rsr_cache.h - what stands between the weight products of a decoder's step: the paged cache of keys and
 * values, and the attention of a step's new tokens over it.
 *
 * The products of rsr.h make queries, keys and values of the new tokens (several vectors per call cost far
 * less than several calls, which is why a step verifies a whole tree of drafted tokens at once).  The
 * functions here take them from there to the vectors of the next product:
 *
 *   rsr_tree_masks      parents of drafted trees -> who sees whom, and how deep a token hangs
 *   rsr_tree_attention  softmax(scale * q . k) . v over a request's cached tokens and its new ones
 *   rsr_cache_slots     lengths -> block tables, slots of the tokens that are kept, the pages that stay free
 *   rsr_cache_append    keys and values of the kept tokens -> their slots
 *
 * A drafted token enters the cache only when it is kept: until then its key and value are read from where the
 * product left them, rounded to the type of the cache exactly as rsr_cache_append rounds them, so that a tree
 * verified in one step sees what the same tokens decoded one by one would see.
 *
 * Conventions as in rsr.h: plain C types, HOST / DEVICE stated per pointer, RSR_OK or a negative rsr_status,
 * message through rsr_last_error(), no exceptions.  All calls are asynchronous on `stream`, allocate nothing,
 * keep nothing from one call to the next and may be captured in a HIP graph.  The device that holds the
 * buffers must be current.  Lengths live on the device and are not seen by the host: a length, page or slot
 * out of range there is left out as stated below, and never leads outside the buffers.  (rsr_cache_slots alone is not
 * told how long the list of free pages is; rsr_cache_slots_bounded is.)
 */
#ifndef RSR_CACHE_H_
#define RSR_CACHE_H_

#include <stdint.h>

#include "rsr.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { RSR_F32 = 0, RSR_F16 = 1, RSR_BF16 = 2 };

/*
 * A paged cache of one layer.  Token t of a request lies at offset t % page_size of the page that entry
 * t / page_size of the request's block table names.  A slot is page * page_size + offset.
 *
 *   k, v        DEVICE, 16-byte aligned; owned by the caller.  Element (page, head, offset, d) is at
 *               page * page_stride + head * head_stride + offset * token_stride + d (in elements), in both.
 *               Strides are multiples of 8, page_stride below 2^31 and token_stride below 2^24.  Pages of
 *               [kv_heads][page_size][head_dim] are read fastest.
 *   dtype       RSR_F16 or RSR_BF16
 *   pages       >= 1, pages * page_size < 2^31
 *   page_size   a power of two, 8 .. 1024
 *   kv_heads    1 .. 1024
 *   head_dim    a multiple of 8, 8 .. 256
 */
typedef struct rsr_cache_t {
  void *k, *v;
  int64_t page_stride, head_stride, token_stride;
  int32_t dtype, pages, page_size, kv_heads, head_dim;
  int32_t reserved;
} rsr_cache_t;

/*
 * The requests of a step.  The rows of q, k, v and out are the new tokens of the requests, one request's
 * behind the other's: request r has the rows start[r] .. start[r+1]-1.
 *
 *   requests   0 .. 65535
 *   tokens     rows in q, k, v and out (0 .. 2^31-1)
 *   max_new    no request has more new tokens (what goes beyond is left out); 1 .. 65535, at most 64 with a mask
 *   max_pages  length of a row of `table`.  The host sees no lengths: how rsr_tree_attention shares out its work goes by
 *              requests, max_new and the tokens that max_pages could name, and tables far wider than what is held cost
 *              time (up to twice as much: see there).
 *   table      DEVICE [requests][max_pages] int32, the block tables.  An entry outside 0 .. pages-1 stands for a
 *              page that is not there: its tokens are not seen (pages that were given up).
 *   held       DEVICE [requests] int32, tokens in the cache (taken as 0 if negative, and as what the table
 *              can name if more)
 *   start      DEVICE [requests+1] int32
 *   mask       DEVICE [tokens] uint64 or NULL.  Bit j of a token's mask: it sees new token j of its request.
 *              Bits of tokens that the request does not have mean nothing.  A token sees itself only if its own
 *              bit is set.  NULL: a chain, token i sees new tokens 0 .. i.
 */
typedef struct rsr_step_t {
  const int32_t *table, *held, *start;
  const uint64_t *mask;
  int32_t requests, tokens, max_new, max_pages;
} rsr_step_t;

/*
 * rsr_tree_attention - for new token i of request r and query head a, with key head b = a / (heads / kv_heads):
 *   out[start[r]+i][a] = sum_p w_p v_p / sum_p w_p,   w_p = exp(scale * <q[start[r]+i][a], k_p>)
 * over the cached tokens of the request on pages that are there and the new tokens that i sees.  A token that
 * sees nothing gets zeros; what it does not see does not touch it, infinities and NaN included.  A seen key or
 * value that is not finite makes the results that it enters not finite (infinite or NaN), whatever the sign of
 * the score; so does a score beyond the range of float.
 *
 *   q        DEVICE, row t at q + t * q_stride elements: [heads][head_dim]
 *   k, v     DEVICE, row t at k + t * kv_stride: [kv_heads][head_dim]; rounded to the type of the cache
 *   out      DEVICE, row t at out + t * out_stride: [heads][head_dim], overwritten; rows of no request are left
 *            alone.  Must not overlap the inputs.
 *   dtype    of q, k, v and out: RSR_F32 or the type of the cache
 *   heads    a multiple of kv_heads, at most 64 * kv_heads
 *   scale    finite
 *   strides  at least a row's elements, below 2^31; rows and pointers 16-byte aligned
 *   workspace  DEVICE, rsr_tree_attention_workspace bytes, 256-byte aligned, zero before its first use; calls leave it
 *            ready for the next one.  Calls that share it must not overlap.  More requests, max_new, max_pages or heads never
 *            need fewer bytes: what is enough for a program's largest step over a cache is enough for all of them.
 *
 * Statistics and sums are held in 32 bits.  Float queries and weights are carried through the matrix cores as sums of
 * three bfloat16 (all their 24 bits) or two float16 (22 bits).  With 16-bit activations the weights are rounded to
 * that type before they meet the values: the error of the result is 1.4 times that of its own rounding (bfloat16
 * 2.3e-3 for 1.7e-3, float16 2.8e-4 for 2.1e-4 of its norm).
 * The order of additions is fixed for given lengths, sizes and max_pages of a step: the same call gives the same bits.  A request
 * alone, in another batch or with a wider table may differ by rounding.
 * More than 64 rows (new tokens times query heads) per key head: with tables for some 32768 tiles of 32 tokens and 64 rows, over all
 * key heads, workgroups take 128 or 256 rows together, which pays over long caches alone.  (5 key heads, 64 tokens with four query
 * heads each over 2000 tokens: 21 us with a table for up to 32768 tokens, 41 with one for 131072.  Eight requests of 32 such tokens: 28 us
 * with tables for 2000 tokens, 46 from 32768 on.  One token over 500, 20 key heads: 12 and 14.)
 * Errors: RSR_ERR_INVALID_ARGUMENT, RSR_ERR_UNSUPPORTED (tables that could name more than some 2^47 tokens of all key heads),
 * RSR_ERR_HIP (launch failure).
 */
int64_t rsr_tree_attention_workspace(const rsr_cache_t *cache, const rsr_step_t *step, int heads); /* bytes, or a negative status; HOST only */
int rsr_tree_attention(const rsr_cache_t *cache, const rsr_step_t *step, const void *q, int64_t q_stride, const void *k,
                       const void *v, int64_t kv_stride, void *out, int64_t out_stride, int dtype, int heads, float scale,
                       void *workspace, int64_t workspace_bytes, void *stream);

/*
 * rsr_cache_slots - pages and slots for the next add[r] tokens of every request.  A request that holds held[r]
 * tokens has ceil(held[r] / page_size) pages in its table; the pages it needs beyond those are taken from the end of
 * the list of free pages, requests in order.
 *
 *   held, add    DEVICE [requests] int32 (negative: 0)
 *   table        DEVICE [requests][max_pages] int32, in and out: the new entries are written, no others
 *   page_size    as in rsr_cache_t
 *   free_pages   DEVICE int32, its first free_count[0] entries are free pages; not written.  The list must have that many.
 *   free_count   DEVICE int32 [1]
 *   free_left    DEVICE int32 [1] out: free_count[0] minus the pages needed; negative if there were too few.
 *                The free list of the next call is free_pages up to free_left[0].
 *   slots        DEVICE [max_slots] int32 out: the slots of the added tokens, requests in order; -1 for a token
 *                that gets none (no page was left, or the table is full) and behind the last token
 *   start        DEVICE [requests+1] int32 out: where a request's slots begin (at most max_slots, and 2^31-1)
 *   now          DEVICE [requests] int32 out: held[r] and those of the added tokens that the request's pages have room
 *                for (places on a page that it gave up count as room); at most 2^31-1
 * No output may overlap an input or another output.  requests 0 .. 65535, max_pages >= 1, max_slots >= 0.
 *
 * rsr_cache_slots_bounded - the same with the length of the list: a free_count[0] above max_free (>= 0) is taken as max_free.
 */
int rsr_cache_slots(const int32_t *held, const int32_t *add, int requests, int32_t *table, int max_pages, int page_size,
                    const int32_t *free_pages, const int32_t *free_count, int32_t *free_left, int32_t *slots, int64_t max_slots,
                    int32_t *start, int32_t *now, void *stream);
int rsr_cache_slots_bounded(const int32_t *held, const int32_t *add, int requests, int32_t *table, int max_pages, int page_size,
                            const int32_t *free_pages, int64_t max_free, const int32_t *free_count, int32_t *free_left, int32_t *slots,
                            int64_t max_slots, int32_t *start, int32_t *now, void *stream);

/*
 * rsr_cache_append - writes keys and values of `count` tokens into the cache, rounded to its type (to the nearest, ties to even).
 *   k, v    DEVICE [nrows], row t at k + t * stride elements: [kv_heads][head_dim]; dtype RSR_F32 or the type of
 *           the cache; rows and pointers 16-byte aligned
 *   rows    DEVICE [count] int32 or NULL: token i is row rows[i] (NULL: row i); nothing is written for a row
 *           outside 0 .. nrows-1
 *   slots   DEVICE [count] int32: where token i goes; nothing is written for a slot outside the cache.  Slots that
 *           are there must differ.
 */
int rsr_cache_append(const rsr_cache_t *cache, const void *k, const void *v, int64_t stride, int64_t nrows, int dtype,
                     const int32_t *rows, const int32_t *slots, int64_t count, void *stream);

/*
 * rsr_tree_masks - masks and depths of drafted trees.
 *   parent  DEVICE [tokens] int32: the token, counted within the request, that a drafted token hangs on; anything
 *           but an earlier token of the request (-1, say) makes it hang on the request's last cached token
 *   start   DEVICE [requests+1] int32, as in rsr_step_t
 *   mask    DEVICE [tokens] uint64 out: the token itself and all that it hangs on, directly or not
 *   depth   DEVICE [tokens] int32 out: how many drafted tokens it hangs on (its position is held + depth)
 * Trees have at most 64 tokens; those beyond get mask 0 and depth -1.  Rows of no request are left alone.
 */
int rsr_tree_masks(const int32_t *parent, const int32_t *start, int requests, int tokens, uint64_t *mask, int32_t *depth, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* RSR_CACHE_H_ */
