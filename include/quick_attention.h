/*
 * quick_attention.h -- between the projections of an attention layer in
 * libquick.so: rotary positions, a paged cache of keys and values in 4 bits,
 * and attention over it.
 *
 * Conventions are those of quick.h: status codes, caller-owned buffers,
 * everything validated before anything is enqueued, asynchronous on `stream`
 * (hipStream_t as void*, NULL = default stream).  All pointers are device
 * pointers.  No entry point allocates, waits or keeps anything, so all may be
 * called while a stream is captured.  Element types (QUICK_F16, QUICK_BF16,
 * QUICK_F32) are those of quick_mx.h.
 *
 * Cache.  A page holds the keys and values of 64 consecutive tokens of one
 * sequence.  Each head of a token is cut into blocks of 32 channels in the
 * microscaled format of quick_mx.h (a byte s, the scale 2^(s - 127), and
 * 4-bit codes), rounded as by quick_mxfp4_quantize: 4.25 bits a value.
 *   cache  uint8 [pages][heads][68 * D], 16-byte aligned; of token t of the
 *          page, 0 <= t < 64:
 *     keys' codes     at 0:      byte t * D/2 + c/2 holds channels c, c + 1
 *                                (c even, the lower one in the low nibble)
 *     keys' scales    at 32 * D: byte 64 * (c/32) + 4 * (t % 16) + t / 16
 *     values' codes   at 34 * D: with w = min(D, 128) / 16 channels of a lane,
 *                                c' = c % 128 and t' = t % 4, byte
 *                                (c/128) * 4096 + (t/4) * 32 * w +
 *                                ((c'/w) * 4 + t') * w/2 + (c' % w) / 2
 *     values' scales  at 66 * D: byte 64 * (c/32) + 16 * ((t % 16) / 4) +
 *                                4 * (t / 16) + t % 4
 * In this order a lane's loads of codes are operands of the matrix
 * instruction: its 16 bytes of keys are one block, those of values the same
 * channels of four tokens.  A slot is 64 * page + t.
 * heads <= QUICK_KV4_MAX_HEADS, D = 64, 128 or 256 (UNSUPPORTED otherwise),
 * 1 <= pages < 2^25 (SHAPE).
 */
#ifndef QUICK_ATTENTION_H
#define QUICK_ATTENTION_H

#include <stddef.h>
#include <stdint.h>

#include "quick.h"
#include "quick_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Tokens of a cache page, most heads of a cache and most sequences of a call. */
#define QUICK_KV4_PAGE 64
#define QUICK_KV4_MAX_HEADS 1024
#define QUICK_KV4_MAX_SEQS 4096

/* Rotary positions: of every head, the pairs (a, b) of the first R channels
 * turn by an angle that grows with the token's position,
 *   a' = factor * (a cos - b sin),  b' = factor * (b cos + a sin),
 *   angle = positions[t] * freqs[i],  pair i: channels i and i + R/2, or with
 *   `interleaved` 2 i and 2 i + 1;
 * the other D - R channels are copied.  With `inverse` the angle is negated:
 * with factor 1 the inverse, and for any factor the transpose, which takes the
 * gradient of the result to that of x.
 *   x          [T][H][D] of `dtype` (f16, bf16 or f32), token t and head h at
 *              t * x_token + h * x_head elements, channels consecutive
 *   positions  int32 [T]; freqs f64 [R/2]; the angle is taken in 64 bits
 *   out        as x, with strides of its own; may be x itself with x's
 *              strides, must not overlap it otherwise
 * Elements aligned to their size; 16-byte alignment of x, out and their
 * strides with R/2 (interleaved: R) and D multiples of 16 bytes is faster.
 * Sums are binary32, rounded once.  R even, 0 <= R <= D <= 4096, H <= 65535,
 * T < 2^24 (SHAPE).  T == 0 is a valid no-op.
 * Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_rotary(const void* x, int dtype, int64_t x_token, int64_t x_head, int64_t T, int64_t H, int64_t D,
                 const int32_t* positions, const double* freqs, int64_t R, int interleaved, int inverse, float factor,
                 void* out, int64_t out_token, int64_t out_head, void* stream);

/* Writes token i's keys and values, rounded, to slot slots[i] of the cache.
 *   k, v   [T][heads][D] of `dtype` (QUICK_F16 or QUICK_BF16), 16-byte
 *          aligned, token t and head h at t * *_token + h * *_head elements,
 *          the strides multiples of 8
 *   slots  int32 [T]; one outside 0 .. 64 * pages - 1 (a padded token's -1,
 *          say) is passed over.  Slots of a call have to differ: of two equal
 *          ones the slot keeps parts of either
 * Other slots keep their bytes.  T < 2^24 and ceil(T / (2048 / D)) * heads < 2^24
 * (SHAPE).  T == 0 is a valid no-op.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, HIP. */
int quick_kv4_write(const void* k, const void* v, int dtype, int64_t k_token, int64_t k_head, int64_t v_token,
                    int64_t v_head, const int32_t* slots, int64_t T, int64_t heads, int64_t D, void* cache,
                    int64_t pages, void* stream);

/* k, v [T][heads][D] of `dtype` (f16, bf16 or f32; 16-byte aligned) = the
 * values that slots[i] holds, rounded where the type cannot hold them (a scale
 * of 255 gives NaN); zero for a slot outside the cache.  Either may be NULL.
 * Limits and errors as quick_kv4_write. */
int quick_kv4_read(const void* cache, int64_t pages, const int32_t* slots, int64_t T, int64_t heads, int64_t D,
                   int dtype, void* k, void* v, void* stream);

typedef struct quick_attention {
    int64_t T;           /* rows of q                                          */
    int64_t q_heads;     /* heads of q, a multiple of `heads`                  */
    int64_t heads;       /* heads of the cache                                 */
    int64_t D;           /* channels of a head                                 */
    int64_t pages;       /* pages of the cache                                 */
    int64_t seqs;        /* sequences                                          */
    int64_t table_width; /* page ids of a sequence in the table                */
    int64_t most;        /* most queries of a sequence; more are taken as so
                            many of its first ones                             */
    int64_t q_token, q_head;     /* strides of q in elements, multiples of 8   */
    int64_t window;      /* tokens that a query sees at most, 0 = all (causal) */
    int causal;          /* nonzero: a query sees no token behind its own      */
    float scale;         /* of the scores                                      */
} quick_attention_t;

/* out = softmax(scale * q . K^T) . V over the tokens of q's sequence that the
 * query sees; query head h reads cache head h / (q_heads / heads).
 *   q        [T][q_heads][D] of `dtype` (QUICK_F16 or QUICK_BF16), 16-byte
 *            aligned
 *   table    int32 [seqs][table_width]: token j of sequence b is in page
 *            table[b][j / 64]; tokens of a page outside the cache are not seen
 *   lengths  int32 [seqs]: tokens of the sequence in the cache, its queries'
 *            own among them; taken as 0 .. 64 * table_width
 *   offsets  int32 [seqs + 1]: the queries of sequence b are the rows
 *            offsets[b] .. offsets[b+1] - 1 of q; values that break the order or
 *            leave 0 .. T are clamped.  NULL: row b is that of sequence b
 * Query i of n stands at position p = lengths[b] - n + i: it sees the tokens
 * j <= p (causal), of those the last `window`, or all of them (not causal).
 * A row that sees nothing is zero, its lse -inf.  What a row does not see does
 * not enter it, NaN and infinities included, and slots behind lengths[b] may
 * hold anything.
 *   out      [T][q_heads][D] of `dtype`, 16-byte aligned, contiguous, must not
 *            overlap q; rows that belong to no sequence keep their values
 *   lse      f32 [T][q_heads], log of the sum of exp(scaled scores); NULL = none
 * Products are those of q and of the cached keys and values as `dtype` holds
 * them (a block whose scale it cannot hold, above 2^13 with f16 and 2^125 with
 * bf16, counts as NaN);
 * scores, softmax and sums are binary32 (a sum of values whose magnitudes add up
 * to 2^128 or more may be infinite), the weights of the values are rounded to
 * `dtype`, the result once more.  Deterministic.
 * workspace: 16-byte aligned, of quick_kv4_attention_workspace_bytes() (0: may
 * be NULL); calls that share one must be ordered.
 * `most` chooses the kernels for all sequences of a call: prompts beside many
 * single tokens are faster as two calls, of their rows each.
 * T < 2^24, q_heads / heads <= 64, seqs <= QUICK_KV4_MAX_SEQS, table_width <
 * 2^24, T * q_heads * D < 2^40, most >= 1, window >= 0 and without `causal` 0
 * (SHAPE).  T == 0 or seqs == 0 is a valid no-op.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, WORKSPACE, HIP. */
int quick_kv4_attention(const quick_attention_t* a, const void* q, int dtype, const void* cache, const int32_t* table,
                        const int32_t* lengths, const int32_t* offsets, void* out, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream);
size_t quick_kv4_attention_workspace_bytes(const quick_attention_t* a);

#ifdef __cplusplus
}
#endif

#endif /* QUICK_ATTENTION_H */
