/*
 * wq_window.h -- C ABI of causal attention with a sliding window and sinks over
 * the paged KV cache, for prompts and for single tokens, in the same library as
 * wq.h (libwq.so; status codes, error messages and the conventions of every
 * entry point are shared with it).
 *
 * The engine keeps every sequence's keys and values in a paged cache (Sec. 2.2;
 * attention over it: Sec. 2.3).  A conversation that runs on for ever is held
 * to a window of its last tokens and a few first ones that stay visible, so
 * that the pages between can be given back (wq_cache.h).  Sequence s has L_s
 * tokens in the cache, of which the last n_s are new and ask.  The one at
 * position p sees the tokens
 *
 *     V(p) = { t : t <= p and (t < sinks or t > p - window) }
 *
 * and for query head h, with kv head h / G (G = num_q_heads / num_kv_heads),
 *
 *     a_t = scale * sum_d q[d] K_t[d],   o = sum_{t in V(p)} softmax(a)_t V_t .
 *
 * A window of max_seq_len or more is plain causal attention.  With window = 0
 * and sinks = 0 nothing is visible and the outputs are zero.
 *
 * Cache, block_table and seq_lens are laid out as in wq_attention.h, the
 * values IEEE binary16 or bfloat16.  Only table entries are read whose page
 * holds a token that one of the sequence's new tokens sees; the others may be
 * anything, so freed pages need no page behind them.
 *
 * Numerics: products of 16-bit values are exact, scores, softmax and sums are
 * fp32; the weights exp(a - m) are rounded to the values' type for the matrix
 * cores that multiply them by V, and the output once.  A sequence whose new tokens
 * have at most 16 rows per kv head (n_s * G; unless it is the only one of a call
 * with max_query_len * G above 16) has what a weight's rounding took multiplied as
 * well; in the others a weight is rounded once, by a relative 2^-11 (bfloat16:
 * 2^-8) or, in binary16, by up to 2^-32 of the row's largest weight.  Per element
 * the result is within
 *
 *     e * sum_t w_t |V_t[d]| + f * sum_{t in V(p)} |V_t[d]| + 1e-6
 *
 * of the exact value, e = 3e-3 for binary16 and 2e-2 for bfloat16, f = 2^-32 for
 * binary16, 2^-43 up to those 16 rows, and 0 for bfloat16, when
 * scale * sum_d |q[d] K_t[d]| <= 60 for every token.
 * Infinities and NaN in a cached token, or in the unused part of a page, reach
 * only outputs whose query sees that token.
 *
 * Lengths, starts and table entries are on the device and cannot be checked
 * before the launch.  The kernels read nothing outside the arrays described.
 * A sequence whose length is negative or above max_seq_len or max_pages_per_seq
 * * page_size, or that has more new tokens than tokens or than
 * max_query_len, gets NaN in all its outputs; one that sees a page outside
 * [0, num_pages) gets NaN in every output that depends on it and perhaps in
 * others of its own; one whose q_starts lie outside [0, num_tokens] or fall
 * is left out.  Other sequences are unaffected.
 */
#ifndef WQ_WINDOW_H
#define WQ_WINDOW_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"
#include "wq_logits.h" /* WQ_DTYPE_F16, WQ_DTYPE_BF16 */

#ifdef __cplusplus
extern "C" {
#endif

#define WQ_WINDOW_MAX_GROUP 16               /* num_q_heads / num_kv_heads */
#define WQ_WINDOW_MAX_KV_HEADS 256
#define WQ_WINDOW_MAX_PAGE_SIZE 1024         /* a power of two */
#define WQ_WINDOW_MAX_SEQ_LEN ((int64_t)1 << 24)
#define WQ_WINDOW_MAX_SEQS ((int64_t)1 << 16)
#define WQ_WINDOW_MAX_TOKENS ((int64_t)1 << 22)

/*
 * wq_window_attention_workspace_size -- bytes of device workspace that
 * wq_window_attention needs for these sizes (0 when none).  Pure host function.
 */
wq_status wq_window_attention_workspace_size(int64_t num_seqs, int64_t num_tokens, int64_t max_query_len,
                                             int64_t num_q_heads, int64_t num_kv_heads, int64_t head_dim,
                                             int64_t max_seq_len, int64_t window, int64_t sinks, size_t* bytes);

/*
 * wq_window_attention -- the above.
 *
 *   q             [num_tokens][num_q_heads][head_dim], rows q_stride elements
 *                 apart (a multiple of 8, at least num_q_heads * head_dim, so
 *                 that they may lie in the QKV projection's output); 16-byte
 *                 aligned.
 *   out           likewise with out_stride; written.
 *   k_cache, v_cache  [num_pages][num_kv_heads][page_size][head_dim]; 16-byte
 *                 aligned.
 *   block_table   [num_seqs][max_pages_per_seq] int32, seq_lens [num_seqs]
 *                 int32, L_s with the new tokens.
 *   q_starts      [num_seqs + 1] int32: the new tokens of sequence s are rows
 *                 [q_starts[s], q_starts[s + 1]); NULL for one each
 *                 (num_tokens == num_seqs).
 *   num_seqs      1 .. WQ_WINDOW_MAX_SEQS; num_tokens 1 ..
 *                 WQ_WINDOW_MAX_TOKENS.
 *   max_query_len an upper bound of the n_s, 1 .. num_tokens.
 *   num_q_heads   a multiple of num_kv_heads, at most WQ_WINDOW_MAX_GROUP
 *                 times it.
 *   head_dim      64 or 128.
 *   page_size     a power of two, 1 .. WQ_WINDOW_MAX_PAGE_SIZE.
 *   max_seq_len   an upper bound of the L_s, 1 .. WQ_WINDOW_MAX_SEQ_LEN; it
 *                 sizes the launch, so a tight bound is faster.
 *   window, sinks 0 .. 2^30.
 *   scale         finite; usually 1 / sqrt(head_dim).
 *   dtype         WQ_DTYPE_F16 or WQ_DTYPE_BF16: the type of q, out and the
 *                 caches.
 *   workspace     of at least the bytes that wq_window_attention_workspace_size
 *                 reports, 16-byte aligned, owned by the caller, used only
 *                 while the work queued by this call runs (calls on one stream
 *                 may share it); may be NULL when that size is 0.
 * out must not overlap any input or the workspace.
 * Errors: INVALID_ARG, UNSUPPORTED (head_dim, group, page_size, dtype),
 *         MISALIGNED, HIP.
 */
wq_status wq_window_attention(const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                              const int32_t* block_table, const int32_t* seq_lens, const int32_t* q_starts,
                              uint16_t* out, int64_t num_seqs, int64_t num_tokens, int64_t max_query_len,
                              int64_t num_q_heads, int64_t num_kv_heads, int64_t head_dim, int64_t q_stride,
                              int64_t out_stride, int64_t page_size, int64_t num_pages,
                              int64_t max_pages_per_seq, int64_t max_seq_len, int64_t window, int64_t sinks,
                              float scale, int64_t dtype, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_WINDOW_H */
