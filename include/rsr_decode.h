/*
 * rsr_decode.h - what a decoder's step does on both sides of its attention (rsr_cache.h), so that it stays on the device
 * from the rows that the q/k/v products give to the keys and values that enter the cache:
 *
 *   rsr_head_rotate   norms of the queries' and keys' heads, and their rotation by the tokens' positions
 *   rsr_sample        scores of the next tokens -> a token for every row: temperature, top-k, top-p, min-p
 *   rsr_tree_keep     the path of a drafted tree that the chosen tokens agree with -> rows and counts for
 *                     rsr_cache_slots and rsr_cache_append, and the tokens that were found
 *
 * Conventions as in rsr_cache.h: plain C types, HOST / DEVICE stated per pointer, RSR_OK or a negative rsr_status, message
 * through rsr_last_error(), no exceptions.  All calls are asynchronous on `stream`, allocate nothing, keep nothing from one
 * call to the next and may be captured in a HIP graph.  The device that holds the buffers must be current.  What lies on the
 * device (positions, parameters, trees) is not seen by the host: a value out of range there does what is stated below, and
 * never leads outside the buffers.
 */
#ifndef RSR_DECODE_H_
#define RSR_DECODE_H_

#include <stdint.h>

#include "rsr_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * How heads are normed and rotated.
 *
 *   frequency   DEVICE [rotated / 2] double, 8-byte aligned: the angle of pair j grows by frequency[j] (in radians) from one position to
 *               the next
 *   q_weight,   DEVICE [head_dim] float, 4-byte aligned, or NULL (ones): the norm's weights, the same for all heads of the queries
 *   k_weight    and of the keys
 *   eps         of the norm; finite, >= 0
 *   norm        1: heads are normed before they are rotated; 0: they are not, and weights and eps mean nothing
 *   head_dim    a multiple of 8, 8 .. 256
 *   rotated     a multiple of 8, 0 .. head_dim: so many of a head's first dimensions are rotated
 *   pairs       what belongs together: 0: dimensions j and j + rotated / 2; 1: dimensions 2j and 2j + 1
 */
typedef struct rsr_rotary_t {
  const double *frequency;
  const float *q_weight, *k_weight;
  float eps;
  int32_t norm, head_dim, rotated, pairs;
  int32_t reserved;
} rsr_rotary_t;

/*
 * rsr_head_rotate - for every head x of every row of q and k
 *   y = x * weight / sqrt(mean(x^2) + eps)     (or y = x)
 *   (y_a, y_b) -> (y_a cos t - y_b sin t, y_a sin t + y_b cos t),   t = position[row] * frequency[j], for pair j = (a, b)
 * in 32 bits, with one rounding at the end to the type of the result.  (Where squares leave the range of float their mean is taken in 64
 * bits.)  The angle's whole turns are taken off in 64 bits, with what those lose: a far position is rotated as exactly as a near one.
 * A value that is not finite touches its own head alone (its pair, without a norm).  A head of zeros with eps 0 is not finite.
 *
 *   q, k         DEVICE, row t at q + t * q_stride elements: [heads][head_dim], k: [kv_heads][head_dim]
 *   dtype        of q and k: RSR_F32, RSR_F16 or RSR_BF16
 *   position     DEVICE [tokens] int32 (any; negative ones rotate the other way)
 *   tokens       0 .. 2^31 - 1
 *   heads, kv_heads   0 .. 65535, not both 0; without heads q and q_out (k and k_out) mean nothing
 *   q_out, k_out DEVICE, rows as those of q and k, with strides of their own; q_out may be q, and k_out k, with the same stride and
 *                type; otherwise no output may overlap an input or the other
 *   out_dtype    of q_out and k_out: RSR_F32, RSR_F16 or RSR_BF16
 *   strides      at least a row's elements; rows and pointers 16-byte aligned
 */
int rsr_head_rotate(const rsr_rotary_t *rotary, const void *q, int64_t q_stride, int heads, const void *k, int64_t k_stride, int kv_heads, int dtype,
                    const int32_t *position, int64_t tokens, void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, int out_dtype,
                    void *stream);

/*
 * rsr_sample - a token for every row of scores.  In row r, with the parameters of that row and scores x_0 .. x_(columns-1):
 *   w_i = exp((x_i - max x) / temperature); tokens in order of their scores, the highest first, of equal ones the lowest first
 *   1. the first top_k tokens
 *   2. of these as many of the first as have together at least top_p of the weight of these
 *   3. of these those with w_i >= min_p
 * kept = how many these are; token = the first of them behind which the sum of weights is above uniform times the weight of all of
 * them; probability = its weight divided by that of all of them.  So uniform numbers from [0, 1) give every kept token with its
 * probability, and 0 the likeliest.
 *
 *   logits       DEVICE, row r at logits + r * stride elements, of dtype RSR_F32, RSR_F16 or RSR_BF16; aligned as its elements
 *   rows         0 .. 2^24
 *   columns      1 .. 2^22
 *   stride       >= columns
 *   temperature  DEVICE [rows] float or NULL (1).  0, a negative one or NaN: the highest score, whatever the other parameters say.
 *   top_k        DEVICE [rows] int32 or NULL.  0 or negative: all.
 *   top_p        DEVICE [rows] float or NULL.  1 and more, or NaN: all; 0 or negative: the first token.
 *   min_p        DEVICE [rows] float or NULL.  0, negative or NaN: all; more than 1: as 1.
 *   uniform      DEVICE [rows] float, taken into 0 .. 1 - 2^-24 (NaN: 0)
 *   token        DEVICE [rows] int32 out
 *   probability  DEVICE [rows] float out, or NULL
 *   kept         DEVICE [rows] int32 out, or NULL
 *   workspace    DEVICE, rsr_sample_workspace bytes, 256-byte aligned, zero before its first use; calls leave it ready for the
 *                next one.  Calls that share it must not overlap.  More rows or columns never need fewer bytes.
 * No output may overlap an input, the workspace or another output.
 * A score of minus infinity is no token's: it is never chosen and not counted.  A row without another score has token -1,
 * probability 0 and kept 0; a row with NaN has token -1, probability NaN and kept 0.  With scores of plus infinity only these
 * tokens have weight, all the same.
 * Weights and sums are held in 64 bits: a weight is off by some 2^-39 of itself (2^-34 where thousands of different scores lie
 * next to each other), a sum of weights by no more than that of itself, however many they are: a border of a sum falls between the
 * tokens between which it falls exactly unless it is that near to one.  A row's results depend on nothing but its own scores and
 * parameters, and in their last bits on where in 16 bytes it begins; not on other rows, nor on the order in which workgroups come.
 * Errors: RSR_ERR_INVALID_ARGUMENT, RSR_ERR_HIP (launch failure).
 */
int64_t rsr_sample_workspace(int64_t rows, int64_t columns); /* bytes, or a negative status; HOST only */
int rsr_sample(const void *logits, int64_t rows, int64_t columns, int64_t stride, int dtype, const float *temperature, const int32_t *top_k,
               const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *probability, int32_t *kept, void *workspace,
               int64_t workspace_bytes, void *stream);

/*
 * rsr_tree_keep - what a verified step has found.  The trees are those of rsr_tree_masks: request r has the tokens start[r] ..
 * start[r+1]-1, of which the first was decided before the step and the others are guesses.  Its path begins with the first token; from
 * a token it goes on to the guess that hangs on it and is the token that was chosen behind it (of several the first), and ends
 * where there is none.
 *
 *   drafted  DEVICE [tokens] int32: the tokens of the trees
 *   chosen   DEVICE [tokens] int32: the token that was chosen behind each (negative: none, the path ends there)
 *   parent   DEVICE [tokens] int32, as in rsr_tree_masks, or NULL: chains, token i hangs on token i - 1
 *   start    DEVICE [requests+1] int32
 *   rows     DEVICE [tokens] int32 out: the rows on the paths, requests in order, and -1 behind the last
 *   found    DEVICE [tokens] int32 out: what was chosen behind each of these, and -1 behind the last.  The last one of a
 *            request is the first token of its next tree.
 *   add      DEVICE [requests] int32 out: rows of the request (0 if it has no tokens)
 *   first    DEVICE [requests+1] int32 out: where a request's rows begin (at most tokens)
 * requests 0 .. 65535.  Trees have at most 64 tokens; those beyond are not looked at.  No output may overlap an input or
 * another output.  With rsr_cache_slots (add, max_slots = tokens) and rsr_cache_append (rows, count = tokens) the kept tokens enter
 * the cache without the host knowing how many they are.
 */
int rsr_tree_keep(const int32_t *drafted, const int32_t *chosen, const int32_t *parent, const int32_t *start, int requests, int tokens, int32_t *rows,
                  int32_t *found, int32_t *add, int32_t *first, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* RSR_DECODE_H_ */
