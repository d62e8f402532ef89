/*
 * quick_mx.h -- microscaled 4-bit floating point (MXFP4) in libquick.so:
 * quantisation, its inverse, and products with weights in that format.
 *
 * Format (OCP microscaling formats, version 1.0): 32 consecutive channels of
 * a row share one scale, 2^(s - 127) with the byte s (s = 255 means NaN); each
 * value is a 4-bit code, sign * {0, 0.5, 1, 1.5, 2, 3, 4, 6}, codes 0..7, bit
 * 3 the sign.  A matrix of R rows and K channels is
 *   codes   uint8 [R][K/2], channel 2i of a row in the low nibble of byte i
 *   scales  uint8 [R][K/32]
 * Products read activations in that form and weights in a packed form
 * (quick_mxfp4_pack), in which a lane's 16-byte load is its operand of the
 * gfx950 matrix instruction, which multiplies the codes and applies both
 * scales itself.
 *
 * Conventions are those of quick.h: status codes, caller-owned buffers,
 * everything validated before anything is enqueued, asynchronous on `stream`
 * (hipStream_t as void*, NULL = default stream).  All pointers are device
 * pointers.  No entry point allocates, waits or keeps anything, so all may be
 * called while a stream is captured.
 * K must be a positive multiple of 32 (SHAPE otherwise), any number of rows
 * and columns is accepted within these limits (SHAPE beyond):
 * rows <= 2^24, K <= 2^22, N <= 2^24; for quantisation and its inverse rows *
 * (K / 8192 rounded up) < 2^24; for a product rows * K < 2^33 activations,
 * N * K < 2^33 weights of one matrix, at most 2^22 rows of y, and at most 2^22
 * tiles of the size that the call is given: a dense product keeps that with
 * (M + 64) * (N + 128) <= 2^34, one over experts with (R / 32 + E) * (N + 128)
 * <= 2^28.
 */
#ifndef QUICK_MX_H
#define QUICK_MX_H

#include <stddef.h>
#include <stdint.h>

#include "quick.h"
#include "quick_fused.h"
#include "quick_grouped.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of activations and results. */
#define QUICK_F16 0
#define QUICK_BF16 1
#define QUICK_F32 2

/* codes, scales = x, rounded.  With a = max |x| over a block and e the
 * exponent of a as an 8-bit biased binary32 exponent, s = max(e - 2, 0), and
 * each code is x * 2^(127 - s) rounded to the nearest representable value
 * (ties to the even code), magnitudes above 6 becoming 6.  A block with a NaN
 * or an infinity gets s = 255 and codes 0.
 *   x       [rows][K] of `dtype` (QUICK_F16, QUICK_BF16, QUICK_F32), 16-byte
 *           aligned, row r at r * ldx elements; ldx >= K, and ldx * element
 *           size a multiple of 16
 *   codes   [rows][K/2], 16-byte aligned; scales [rows][K/32]
 * rows == 0 is a valid no-op.  Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_mxfp4_quantize(const void* x, int dtype, int64_t ldx, int64_t rows, int64_t K, void* codes, void* scales,
                         void* stream);

/* y [rows][K] of `dtype` = the values of codes and scales, rounded to nearest
 * even where the type cannot hold them (a scale of 255 gives NaN).
 * codes and y 16-byte aligned.  Errors as quick_mxfp4_quantize. */
int quick_mxfp4_dequantize(const void* codes, const void* scales, int dtype, int64_t rows, int64_t K, void* y,
                           void* stream);

/* Bytes of one packed N x K weight matrix and of its packed scales (the
 * columns are padded to 16, the channels to 128 and, for the scales, to 512).
 * Any output pointer may be NULL.  Errors: SHAPE. */
int quick_mxfp4_packed_sizes(int64_t N, int64_t K, size_t* packed_bytes, size_t* scales_bytes);

/* Lays E weight matrices out for the products (once, when weights are
 * loaded).  Output column n of a matrix is row n of codes [E][N][K/2] and
 * scales [E][N][K/32].  With `gate_up` nonzero (N a multiple of 32) the first
 * N/2 rows are a gate projection and the others the matching up projection,
 * in the order that QUICK_ACT_SILU_GATE needs.
 * codes and packed 16-byte, packed_scales 4-byte aligned; scales any.
 *   packed         unit (n/16, k/128) of 1 KiB, units of one column tile
 *                  consecutive: lane 16 * ((k % 128) / 32) + n % 16 holds the
 *                  16 code bytes of its column's 32 channels
 *   packed_scales  unit (n/16, k/512) of 256 bytes: byte 4 * lane + (k % 512)
 *                  / 128 is the scale of that lane's 32 channels
 * Padding is zero.  Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_mxfp4_pack(const void* codes, const void* scales, int64_t E, int64_t N, int64_t K, int gate_up,
                     void* packed, void* packed_scales, void* stream);

/* y[M][N] = x . W^T (+ bias), or with QUICK_ACT_SILU_GATE y[M][N/2] =
 * silu(gate) * up of weights packed with gate_up (then N % 32 == 0, SHAPE).
 * The products of codes and scales are exact; sums are binary32 and rounded
 * once, after the epilogue.  Deterministic.  A NaN scale makes the results
 * that it enters NaN.
 *   codes, scales           activations [M][K/2] (16-byte aligned), [M][K/32]
 *                           (4-byte aligned)
 *   packed, packed_scales   from quick_mxfp4_pack (16- and 4-byte aligned)
 *   bias                    of y's type, [N] in the logical column order (gate
 *                           columns first), 2-byte aligned; NULL = none
 *   y                       `dtype` QUICK_F16 or QUICK_BF16, 8-byte aligned;
 *                           must not overlap the inputs
 * M == 0 is a valid no-op.  Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_mxfp4_gemm(const void* codes, const void* scales, const void* packed, const void* packed_scales, void* y,
                     int dtype, int64_t M, int64_t N, int64_t K, const void* bias, int activation, void* stream);

/* The same with 16-bit activations x [M][K] of y's type, quantised as by
 * quick_mxfp4_quantize on the way (the results are those of the two calls, up
 * to the order of the sums):
 * inside the product's launch for few rows, otherwise into the workspace.
 * x: 16-byte aligned, contiguous.  workspace: 16-byte aligned, of
 * quick_mxfp4_linear_workspace_bytes() (0 when none is needed: may be NULL);
 * calls that share one must be ordered.  Errors as quick_mxfp4_gemm, and
 * WORKSPACE. */
int quick_mxfp4_linear(const void* x, const void* packed, const void* packed_scales, void* y, int dtype, int64_t M,
                       int64_t N, int64_t K, const void* bias, int activation, void* workspace,
                       size_t workspace_bytes, void* stream);
size_t quick_mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);

/* The product over experts: y[r] = x[rows[r]] . W_e^T (+ bias_e) for
 * offsets[e] <= r < offsets[e+1], epilogue as above; one launch.  rows,
 * offsets, T, R and E as in quick_w4a16_grouped_gemm (rows NULL: row r reads
 * x[r]); values that break that contract are clamped, and rows that no expert
 * owns are left as they were.  packed and packed_scales: the experts' back to
 * back, as quick_mxfp4_pack writes them; bias [E][N].
 * R == 0 is a valid no-op.  Errors: INVALID_ARG, SHAPE, ALIGNMENT, HIP. */
int quick_mxfp4_grouped_gemm(const void* codes, const void* scales, const int32_t* rows, const int32_t* offsets,
                             const void* packed, const void* packed_scales, void* y, int dtype, int64_t T, int64_t R,
                             int64_t E, int64_t N, int64_t K, const void* bias, int activation, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QUICK_MX_H */
