/*
 * wq_mx.h -- C ABI of microscaled (MX) matrices and of the decoder linears that
 * multiply them, in the same library as wq.h (libwq.so; status codes, error
 * messages and the conventions of every entry point are shared with it).
 *
 * The paper's models hold their weights in 4 bits (Table 1), one scale to a
 * group (wq.h).  MX is such a format whose products the matrix cores form
 * directly: a row's blocks of WQ_MX_BLOCK consecutive elements share a scale
 * that is a power of two, and the elements are small floating-point numbers:
 *
 *   WQ_MX_FP4  E2M1: sign, 2 exponent bits, 1 mantissa bit; 0, 0.5, 1, 1.5, 2,
 *              3, 4, 6 and their negatives.
 *   WQ_MX_FP8  E4M3: sign, 4 exponent bits, 3 mantissa bits; up to 448, no
 *              infinities, 0x7F and 0xFF are NaN.
 *
 * A matrix [rows][cols] is two arrays:
 *   codes   [rows][cols / 2] bytes (FP4: element 2i in bits 0..3 of byte i,
 *           element 2i + 1 in bits 4..7) or [rows][cols] bytes (FP8); 16-byte
 *           aligned.
 *   scales  [rows][WQ_MX_SCALE_STRIDE(cols)] bytes, 16-byte aligned: byte b of a
 *           row belongs to elements 32 b .. 32 b + 31 and is E8M0, 2^(byte - 127),
 *           255 being NaN.  Bytes from cols / 32 on are padding, never written
 *           and of any value.
 * An element stands for its code's value times its block's scale.
 */
#ifndef WQ_MX_H
#define WQ_MX_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"
#include "wq_logits.h" /* WQ_DTYPE_* */

#ifdef __cplusplus
extern "C" {
#endif

#define WQ_MX_FP4 4
#define WQ_MX_FP8 8
#define WQ_MX_BLOCK 32
#define WQ_MX_SCALE_STRIDE(cols) (((int64_t)(cols) + 511) / 512 * 16)

#define WQ_MX_MAX_ROWS ((int64_t)1 << 24)
#define WQ_MX_MAX_COLS ((int64_t)1 << 20)

/*
 * wq_mx_quantize -- values to an MX matrix.
 *
 *   v = x[r][c]                                    gated = 0
 *   v = silu(x[r][c]) * x[r][cols + c]             gated = 1 (x has 2 * cols
 *       columns, the gate and up projections; silu(a) = a / (1 + exp(-a)); in
 *       fp32, within 2^-20 * |v| + 2^-148 * (1 + |up|) of the exact value, but
 *       silu of a below -87 may come out as -0)
 *   scale   of a block: the smallest power of two, at least 2^-127, with which
 *           max |v| / scale does not pass the type's largest value (6 or 448)
 *   element v / scale rounded to nearest, ties to even
 *
 * So an element differs from v / scale by at most half a step of its type.  A
 * block that holds a NaN or an infinity gets the scale NaN and elements 0.  In a
 * block of zeros the scale is 2^-127.
 *
 *   x        [rows][cols] (or [rows][2 * cols]), rows x_stride elements apart (a
 *            multiple of 8); 16-byte aligned.
 *   rows     1 .. WQ_MX_MAX_ROWS; cols a multiple of 32, 32 .. WQ_MX_MAX_COLS.
 *   dtype    WQ_DTYPE_* of x.
 *   format   WQ_MX_FP4 or WQ_MX_FP8.
 * The outputs must not overlap x or each other.
 * Errors: INVALID_ARG, UNSUPPORTED (dtype, format, cols % 32), MISALIGNED, HIP.
 */
wq_status wq_mx_quantize(const void* x, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t cols, int64_t x_stride,
                         int64_t dtype, int64_t gated, int64_t format, void* stream);

/*
 * wq_mx_dequantize -- what an MX matrix stands for, rounded once to `dtype`
 * (nearest, ties to even; too large a value becomes an infinity).
 *
 *   out      [rows][cols], rows out_stride elements apart (a multiple of 8);
 *            16-byte aligned.
 * Sizes and errors as for wq_mx_quantize.
 */
wq_status wq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, void* out, int64_t rows, int64_t cols,
                           int64_t out_stride, int64_t format, int64_t dtype, void* stream);

/*
 * wq_mx_linear_workspace_size -- bytes of device workspace that wq_mx_linear
 * needs for these sizes (0 when none).  Pure host function.
 */
wq_status wq_mx_linear_workspace_size(int64_t N, int64_t K, int64_t M, int64_t x_format, size_t* bytes);

/*
 * wq_mx_linear -- y[m][n] = sum_k x[m][k] * w[n][k] of two MX matrices, from one
 * token to whole prompts.
 *
 *   w_codes, w_scales  [N][K], WQ_MX_FP4.
 *   x_codes, x_scales  [M][K], x_format WQ_MX_FP4 or WQ_MX_FP8.
 *   y        [M][N] of `dtype` (WQ_DTYPE_F16 or WQ_DTYPE_BF16), rows y_stride
 *            elements apart, aligned to its elements; written.
 *   N, M     1 .. WQ_MX_MAX_ROWS; K a multiple of 32, 32 .. WQ_MX_MAX_COLS.
 *   workspace  of at least the bytes that wq_mx_linear_workspace_size reports,
 *            16-byte aligned, owned by the caller, used only while the work
 *            queued by this call runs (calls on one stream may share it); may
 *            be NULL when that size is 0.
 * The matrix cores add eight neighbouring products at a time.  With x in 8 bits
 * they drop of each what lies more than 13 binary places below the largest of
 * the eight (12 beside a weight of 0.5); with x in 4 bits nothing.  These sums
 * they scale and add in fp32, where a step of 128 may leave out 2^-19 of what is
 * added up; y is rounded once.  Per element the result is within
 *
 *     e * |y| + (f + K * 2^-26) * sum_k |x[m][k] w[n][k]| + t
 *
 * of the exact value, f = 2^-9 for x in 8 bits, 2^-15 in 4 bits, e = 2^-11 and
 * t = 2^-25 for binary16, 2^-8 and 2^-126 for bfloat16, while the sums stay in
 * fp32's range; for random codes the error before y's rounding is about 2^-17 of
 * that sum.  The same call gives the same bits each time; how a sum is cut into
 * parts, and with it its last bits, also depends on M and N.  A NaN element or
 * scale makes every result NaN that it takes part in.
 * y must not overlap any input or the workspace.
 * Errors: INVALID_ARG, UNSUPPORTED (x_format, dtype, K % 32), MISALIGNED, HIP.
 */
wq_status wq_mx_linear(const uint8_t* w_codes, const uint8_t* w_scales, const uint8_t* x_codes, const uint8_t* x_scales,
                       void* y, int64_t N, int64_t K, int64_t M, int64_t y_stride, int64_t x_format, int64_t dtype,
                       void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_MX_H */
