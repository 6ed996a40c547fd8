/*
 * wq_logits.h -- C ABI of the step between a decoder's logits and its next
 * token, in the same library as wq.h (libwq.so; status codes, error messages
 * and the conventions of every entry point are shared with it).
 *
 * The engine generates under a grammar, masking the words that it does not
 * allow (Sec. 2.1, Sec. 2.2), and its OpenAI-style requests carry penalties for
 * repeated words and biases for single ones (Sec. 2.1).  For each row (one
 * sequence) and word w, in fp32 and in this order, every operation rounded by
 * itself:
 *
 *   x = logits[w]
 *   x = x > 0 ? x / repetition : x * repetition    if w is in the row's history
 *   x = x - frequency * c                           c = times w was generated
 *   x = x - presence                                if c > 0
 *   x = x + bias                                    if the row lists w
 *   x = -infinity                                   if the mask does not allow w
 *
 * out[w] is x rounded once to the logits' type, and token the word with the
 * largest x among the allowed ones (the lowest such word; a NaN never wins; -1
 * when there is none).
 */
#ifndef WQ_LOGITS_H
#define WQ_LOGITS_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of values. */
#define WQ_DTYPE_F16 0  /* IEEE binary16 */
#define WQ_DTYPE_BF16 1 /* bfloat16 */
#define WQ_DTYPE_F32 2

#define WQ_LOGITS_MAX_ROWS ((int64_t)65535)
#define WQ_LOGITS_MAX_VOCAB ((int64_t)1 << 24)
#define WQ_LOGITS_MAX_HISTORY ((int64_t)1 << 24)
#define WQ_LOGITS_MAX_BIAS ((int64_t)1 << 16)

/*
 * What to do with one batch of logits.  All pointers are DEVICE pointers owned
 * by the caller; those marked optional may be NULL.
 */
typedef struct wq_logits_call {
    const void* logits;          /* [rows][vocab], rows logits_stride elements apart */
    void* out;                   /* [rows][vocab], out_stride apart; may be logits itself (with its stride) */
    int32_t* token;              /* [rows]; optional */
    const uint32_t* mask;        /* [rows][ceil(vocab / 32)], mask_stride words apart: bit w % 32 of word
                                    w / 32 set where w is allowed; optional: all are */
    const int32_t* history;      /* [rows][history_size]: the row's prompt, then what it generated; optional */
    const int32_t* history_lens; /* [rows] words of the history; optional: history_size */
    const int32_t* prompt_lens;  /* [rows] words of it that are the prompt; optional: 0 */
    const float* repetition;     /* [rows], above 0; optional: 1 */
    const float* frequency;      /* [rows]; optional: 0 */
    const float* presence;       /* [rows]; optional: 0 */
    const int32_t* bias_ids;     /* [rows][bias_size] words; of one listed twice the later entry holds; optional */
    const float* bias_values;    /* [rows][bias_size]; with bias_ids */
    const int32_t* bias_lens;    /* [rows] entries used; optional: bias_size */
    int64_t rows, vocab;
    int64_t logits_stride, out_stride, mask_stride;
    int64_t history_size, bias_size;
    int64_t dtype;               /* WQ_DTYPE_* of logits and out */
} wq_logits_call;

/*
 * wq_process_logits_workspace_size -- bytes of device workspace that
 * wq_process_logits needs for these sizes (0 when none).  Pure host function.
 */
wq_status wq_process_logits_workspace_size(int64_t rows, int64_t vocab, int64_t dtype, size_t* bytes);

/*
 * wq_process_logits -- the above.
 *
 *   call       HOST struct, read during the call only.  Pointers are aligned to
 *              their elements (any row may start anywhere).
 *   workspace  of at least the bytes that wq_process_logits_workspace_size
 *              reports, 16-byte aligned, owned by the caller, used only while
 *              the work queued by this call runs (calls on one stream may
 *              share it); may be NULL when that size is 0 or token is NULL.
 * Lengths below 0 count as 0 and those above the list's size as its size;
 * words outside [0, vocab) in a history or a bias list are ignored.  out and
 * token must not overlap any input (but out may be logits).
 * Errors: INVALID_ARG, UNSUPPORTED (dtype), MISALIGNED, HIP.
 */
wq_status wq_process_logits(const wq_logits_call* call, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_LOGITS_H */
