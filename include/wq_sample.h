/*
 * wq_sample.h -- C ABI of the choice of a decoder's next word by chance, from
 * random numbers that the caller gives, in the same library as wq.h (libwq.so;
 * status codes, error messages and the conventions of every entry point are
 * shared with it).
 *
 * The engine's OpenAI-style requests (Sec. 2.1) name a temperature and a share
 * of the probability to choose from.  For each row (one sequence) with logits
 * x, in exact arithmetic:
 *
 *   order   words by x, the largest first, of equal ones the lowest word first
 *   w       = exp((x - max x) / temperature)
 *   top-k   the first top_k words of the order stay
 *   top-p   of these the shortest beginning stays whose sum of w reaches top_p
 *           of theirs; the first word always stays
 *   min-p   of these the words with w >= min_p stay
 *   token   the first of the words that stay, by their number, up to which
 *           their sum of w passes random * (the sum of all that stay)
 *   share   the token's w over that sum
 *
 * With a temperature of 0 (or below, or NaN) the token is the first word of the
 * order, its share 1.  A logit that is NaN or -infinity takes no part; where
 * all are, the token is -1 and its share 0.  Where the largest logit is
 * +infinity, w is 1 for the words that have it and 0 for the others.
 *
 * The device holds w as multiples of 2^-s, s = min(51, 62 - ceil(log2(vocab)))
 * (2^-45 for 128256 words), formed in fp64, and adds them as whole numbers: the
 * token is the exact one unless random, top_p or min_p lies within a few of these
 * steps per word of a border (always where the words that weigh anything are of
 * one logit: shares of the sum are taken exactly), and is the same whatever order
 * the hardware runs in.
 *
 * Time: a histogram of at most 1/64 of a logit's distance from the best ones tells
 * where the cut is; up to 4096 words of its bin are listed.  Where the bin has
 * more, one workgroup reads the row again and again: thousands of equal logits at
 * the cut, and from about 170000 words on also top-p cuts in the middle of a broad
 * row (262144 normal logits, temperature 2 / 3 of their deviation, top-p 0.95:
 * 0.62 ms; at temperature 1 / 3 of it and top-p 0.9 0.04 ms).
 */
#ifndef WQ_SAMPLE_H
#define WQ_SAMPLE_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"
#include "wq_logits.h" /* WQ_DTYPE_* */

#ifdef __cplusplus
extern "C" {
#endif

#define WQ_SAMPLE_MAX_ROWS ((int64_t)65535)
#define WQ_SAMPLE_MAX_VOCAB ((int64_t)1 << 20)

/* One batch.  All pointers are DEVICE pointers owned by the caller; those marked
 * optional may be NULL. */
typedef struct wq_sample_call {
    const void* logits;       /* [rows][vocab], rows logits_stride elements apart; aligned to its elements */
    const float* random;      /* [rows], in [0, 1): below 0 or NaN counts as 0; 1 and above: the last word that stays */
    const float* temperature; /* [rows]; optional: 1 */
    const int32_t* top_k;     /* [rows], 0 or below: all; optional: all */
    const float* top_p;       /* [rows], 1 or above or NaN: all; 0 or below: the first word; optional: all */
    const float* min_p;       /* [rows], 0 or below or NaN: all; above 1 counts as 1; optional: all */
    int32_t* token;           /* [rows], written */
    float* share;             /* [rows], written; optional */
    int64_t rows, vocab, logits_stride;
    int64_t dtype;            /* WQ_DTYPE_* of logits */
} wq_sample_call;

/*
 * wq_sample_logits_workspace_size -- bytes of device workspace that
 * wq_sample_logits needs for these sizes (0 when none).  Pure host function.
 */
wq_status wq_sample_logits_workspace_size(int64_t rows, int64_t vocab, int64_t dtype, size_t* bytes);

/*
 * wq_sample_logits -- the above.
 *
 *   call       HOST struct, read during the call only.
 *   workspace  of at least the bytes that wq_sample_logits_workspace_size
 *              reports, 16-byte aligned, owned by the caller, used only while
 *              the work queued by this call runs (calls on one stream may
 *              share it); may be NULL when that size is 0.
 * token and share must not overlap each other, an input or the workspace.
 * Errors: INVALID_ARG, UNSUPPORTED (dtype), MISALIGNED, HIP.
 */
wq_status wq_sample_logits(const wq_sample_call* call, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_SAMPLE_H */
