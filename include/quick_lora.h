/*
 * quick_lora.h -- low-rank adapters of many requests beside a projection that
 * they share (libquick.so).
 *
 * Conventions are those of quick.h: status codes, caller-owned buffers,
 * everything validated before anything is enqueued, asynchronous on `stream`
 * (hipStream_t as void*, NULL = default stream).  All pointers are device
 * pointers.  No entry point allocates, waits or keeps anything, so all may be
 * called while a stream is captured.  Element types (QUICK_F16, QUICK_BF16)
 * are those of quick_mx.h.
 */
#ifndef QUICK_LORA_H
#define QUICK_LORA_H

#include <stddef.h>
#include <stdint.h>

#include "quick.h"
#include "quick_grouped.h"
#include "quick_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QUICK_LORA_MAX_RANK 128

/* The tokens in the order of their adapters, for all projections of a step.
 *   ids      int32 [T]: the adapter of each token; one outside 0..E-1 means
 *            none
 *   offsets  int32 [E+1], rows int32 [T]: adapter e has the tokens rows[r] for
 *            offsets[e] <= r < offsets[e+1], in their order; tokens without
 *            one follow from offsets[E] on, in theirs
 * 1 <= E <= QUICK_MAX_EXPERTS, T < 2^24 (SHAPE).  T == 0 writes offsets alone.
 * Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_lora_group(const int32_t* ids, int64_t T, int64_t E, int32_t* offsets, int32_t* rows, void* stream);

/* For offsets[e] <= r < offsets[e+1] and t = rows[r]:
 *   out[t] = y[t] + scales[e] * (x[t] . A_e^T) . B_e^T,
 * and out[t] = y[t] for r from offsets[E] on.
 *   x        [T][K] of `dtype` (QUICK_F16 or QUICK_BF16), row t at t * ldx
 *   a        [E][rank][K], b [E][N][rank], of `dtype`, contiguous
 *   scales   f32 [E]; NULL = 1
 *   offsets  int32 [E+1], rows int32 [R] as quick_lora_group writes them;
 *            values that break that order are clamped, a row outside 0..T-1 is
 *            passed over.  Rows of out that are not listed keep their values; a
 *            row may be listed once
 *   y, out   [T][N] of `dtype`, row t at t * ldy and t * ldo; out may be y with
 *            ldo == ldy (rows without an adapter are not touched then), must
 *            not overlap it otherwise, nor x, a and b
 * Adapters of lower ranks in one call are padded with zeros.
 * x . A^T is summed in binary32, times the scale rounded to `dtype`, as operand
 * of the second product, whose sums are binary32, y's value among them, and
 * rounded once.  Deterministic.
 * All pointers 16-byte aligned (scales, offsets, rows: 4), K, N, rank and the
 * strides multiples of 8; ldx >= K, ldy, ldo >= N.
 * workspace: 16-byte aligned, of quick_lora_workspace_bytes(); calls that share
 * one must be ordered.
 * rank <= QUICK_LORA_MAX_RANK, E <= QUICK_MAX_EXPERTS, T < 2^24, R <= T, K and
 * N <= 2^20 (SHAPE).  R == 0 is a valid no-op.
 * Errors: INVALID_ARG, SHAPE, ALIGNMENT, WORKSPACE, HIP. */
int quick_lora_add(const void* x, int64_t ldx, int dtype, int64_t T, int64_t K, int64_t N, int64_t E, int64_t rank,
                   const void* a, const void* b, const float* scales, const int32_t* offsets, const int32_t* rows,
                   int64_t R, const void* y, int64_t ldy, void* out, int64_t ldo, void* workspace,
                   size_t workspace_bytes, void* stream);
size_t quick_lora_workspace_bytes(int64_t R, int64_t K, int64_t E, int64_t rank);

#ifdef __cplusplus
}
#endif

#endif /* QUICK_LORA_H */
