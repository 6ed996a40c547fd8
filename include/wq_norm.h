/*
 * wq_norm.h -- C ABI of the work between two layers of a decoder: the residual's
 * addition and the root-mean-square norm of the sum, for any number of tokens,
 * in the same library as wq.h (libwq.so; status codes, error messages and the
 * conventions of every entry point are shared with it).
 *
 * The paper's compiler fuses kernels at the graph level (Sec. 2.3).  Here the
 * addition, the norm and the rounding of the next linear's input are one pass:
 *
 *   s[c]     = x[c] + residual[c]               (x[c] without a residual)
 *   total[c] = s[c] rounded to `dtype`
 *   v[c]     = s[c] / sqrt(mean_j s[j]^2 + eps) * weight[c]
 *   out[c]   = v[c] rounded to `dtype`, and / or v as an MX matrix (wq_mx.h)
 *
 * All of it in fp32, each result rounded once: the norm is that of s, not of
 * total.  Squares that pass fp32's range on either side are formed of scaled
 * numbers, so that in fp32 arithmetic a row's v are within
 *
 *     2^-18 * |v| + 2^-149 * (1 + |weight|)
 *
 * of the exact values, whatever the size of finite s and of eps.  A row of zeros
 * with eps = 0 is 0 / 0, NaN.  Where s holds an infinity, v is NaN there and 0
 * elsewhere; where it holds a NaN, all of v is NaN.
 */
#ifndef WQ_NORM_H
#define WQ_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"
#include "wq_logits.h" /* WQ_DTYPE_* */
#include "wq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WQ_NORM_MAX_ROWS ((int64_t)1 << 21)
#define WQ_NORM_MAX_DIM ((int64_t)32768)

/* One call.  All pointers are DEVICE pointers owned by the caller, 16-byte
 * aligned; those marked optional may be NULL. */
typedef struct wq_norm_call {
    const void* x;        /* [rows][dim], rows x_stride elements apart */
    const void* residual; /* [rows][dim], residual_stride apart; optional */
    const void* weight;   /* [dim] */
    void* total;          /* [rows][dim], total_stride apart; optional; may be x or residual itself (with its stride) */
    void* out;            /* [rows][dim], out_stride apart; optional; may be x or residual itself (with its stride) */
    uint8_t* codes;       /* the MX result of type `format` (wq_mx.h); optional */
    uint8_t* scales;      /* with codes */
    int64_t rows, dim;    /* dim a multiple of 32 */
    int64_t x_stride, residual_stride, total_stride, out_stride; /* multiples of 8, at least dim; of used arrays */
    int64_t dtype;        /* WQ_DTYPE_* of x, residual, weight, total and out */
    int64_t format;       /* WQ_MX_* of codes */
    float eps;            /* finite, >= 0 */
} wq_norm_call;

/*
 * wq_add_rmsnorm -- the above.
 *
 *   call  HOST struct, read during the call only.  At least one of out and
 *         codes is given.
 * A block of the MX result that holds a NaN or an infinity is handled as
 * wq_mx_quantize handles it.  Outputs must not overlap each other, weight, or
 * (but for total or out in the place of x or of residual) an input.
 * Errors: INVALID_ARG, UNSUPPORTED (dtype, format, dim), MISALIGNED, HIP.
 */
wq_status wq_add_rmsnorm(const wq_norm_call* call, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_NORM_H */
