/*
 * quick_moe.h -- what surrounds the grouped products of a mixture-of-experts
 * layer in libquick.so: routing tokens to experts, and joining the experts'
 * rows again.
 *
 * Conventions are those of quick.h: status codes, caller-owned buffers,
 * everything validated before anything is enqueued, asynchronous on `stream`
 * (hipStream_t as void*, NULL = default stream).  All pointers are device
 * pointers.  No entry point allocates, waits or keeps anything.  Element
 * types (QUICK_F16, QUICK_BF16, QUICK_F32) are those of quick_mx.h.
 */
#ifndef QUICK_MOE_H
#define QUICK_MOE_H

#include <stddef.h>
#include <stdint.h>

#include "quick.h"
#include "quick_grouped.h"
#include "quick_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QUICK_SCORE_SOFTMAX 0
#define QUICK_SCORE_SIGMOID 1

/* Most experts a token goes to, and most groups of experts. */
#define QUICK_MAX_TOPK 16
#define QUICK_MAX_GROUPS 64

typedef struct quick_route {
    int score;           /* QUICK_SCORE_SOFTMAX or QUICK_SCORE_SIGMOID         */
    int topk;            /* experts a token goes to, 1..16                     */
    int groups;          /* groups of E / groups consecutive experts; 1 = none */
    int topk_groups;     /* groups that stay, 1..groups                        */
    int group_best;      /* a group's score: the sum of its 1 or 2 best choices*/
    int renormalize;     /* nonzero: a token's weights are divided by their sum*/
    float scale;         /* factor of the weights                              */
} quick_route_t;

/* Experts and weights of every token, and the routed rows sorted by expert.
 *   logits   [T][E] of `dtype`, aligned to its element
 *   bias     f32 [E], added to the scores for the choice alone; NULL = none
 *   s        softmax over the row, or sigmoid, in binary32.  A logit of -inf
 *            (an expert that is masked) has s = 0, also in a row that has
 *            nothing else; a NaN or +inf gives what the formula gives
 *   c        s + bias (softmax without bias and group_best 1: in the order of
 *            the logits, which is that of s); a NaN is taken as -inf
 * The topk_groups groups with the largest scores stay, and in them the topk
 * largest c are chosen, equal ones by the lower index.
 *   ids      int32 [T][topk], in descending order of c
 *   weights  f32 [T][topk]: s of the chosen, / their sum (0 if that is 0) with
 *            renormalize, * scale
 *   offsets  int32 [E+1], rows int32 [T*topk]: the routed rows as the grouped
 *            products take them, an expert's rows in the order of the tokens
 *   slots    int32 [T][topk]: the routed row of each (token, choice)
 * T <= 2^30, T * topk < 2^31, E <= QUICK_MAX_EXPERTS, E a multiple of groups, topk <=
 * topk_groups * E / groups (SHAPE otherwise).  T == 0 writes offsets alone.
 * Deterministic.  workspace: 16-byte aligned, of
 * quick_moe_route_workspace_bytes() (0: may be NULL); calls that share one
 * must be ordered.
 * Errors: INVALID_ARG, SHAPE, ALIGNMENT, WORKSPACE, HIP. */
int quick_moe_route(const void* logits, int dtype, int64_t T, int64_t E, const quick_route_t* route,
                    const float* bias, int32_t* ids, float* weights, int32_t* offsets, int32_t* rows,
                    int32_t* slots, void* workspace, size_t workspace_bytes, void* stream);
size_t quick_moe_route_workspace_bytes(int64_t T, int64_t E, int64_t topk);

/* out[t] = residual[t] + sum over j < topk of weights[t][j] * y[slots[t][j]].
 *   y        [R][D] of `dtype` (QUICK_F16 or QUICK_BF16), aligned to 2 bytes
 *            (16, with D a multiple of 8, is faster); slots int32 [T][topk]: a
 *            slot outside 0..R-1 adds nothing; weights f32 [T][topk]
 *   residual [T][D] of `dtype`; NULL = none
 *   out      [T][D] of `dtype`; may be residual, must not overlap y
 * Sums are binary32 in the order of j, rounded once.  1 <= topk <=
 * QUICK_MAX_TOPK; R <= 2^31 - 1, T * (D / 2048 rounded up; / 256 where that
 * speed is not met) < 2^24 (SHAPE beyond).  T == 0 is a valid no-op.
 * Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_moe_combine(const void* y, int dtype, int64_t R, int64_t D, const int32_t* slots, const float* weights,
                      int64_t T, int64_t topk, const void* residual, void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QUICK_MOE_H */
