/*
 * wq_cache.h -- C ABI of the work that keeps a paged key-value cache, in the
 * same library as wq.h (libwq.so; status codes, error messages and the
 * conventions of every entry point are shared with it).
 *
 * The engine manages sequences in a paged KV cache (Sec. 2.2).  Here that is
 *   caches       any number of arrays [num_pages][num_kv_heads][page_size]
 *                [head_dim] of 16-bit values, one for the keys and one for
 *                the values of each layer, as wq_attention.h and wq_window.h
 *                read them.  One page number stands for the same place in all.
 *   block_table  [num_seqs][max_pages_per_seq] int32: entry e of row s is
 *                the page of tokens [e page_size, (e + 1) page_size) of
 *                sequence s; a negative entry is no page.
 *   refs         [num_pages] int32: how many table entries hold the page.  A
 *                page with refs <= 0 is free.
 * All of it lives on the device and is changed there, in stream order, so a
 * decoding loop needs no copy of it on the host and can be captured.  Free
 * pages are handed out lowest number first, and every result below is the
 * same whatever order the hardware runs in.
 *
 * Values that the kernels read from device memory (lengths, table entries,
 * page numbers, sequence numbers) cannot be checked before the launch.  One
 * that lies outside its range is skipped; nothing is read or written outside
 * the arrays described here.
 */
#ifndef WQ_CACHE_H
#define WQ_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "wq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WQ_CACHE_MAX_ARRAYS ((int64_t)256)      /* caches of one call */
#define WQ_CACHE_MAX_KV_HEADS ((int64_t)256)
#define WQ_CACHE_MAX_HEAD_DIM ((int64_t)1024)   /* a multiple of 8 */
#define WQ_CACHE_MAX_PAGE_SIZE ((int64_t)1024)  /* a power of two */
#define WQ_CACHE_MAX_PAGES ((int64_t)1 << 24)
#define WQ_CACHE_MAX_SEQS ((int64_t)1 << 16)
#define WQ_CACHE_MAX_TOKENS ((int64_t)1 << 26)  /* new tokens of one call */

/*
 * wq_cache_append -- write the keys and values of new tokens to their slots.
 *
 *   k_new, v_new  [num_tokens][num_kv_heads][head_dim] 16-bit values, the
 *                 rows of tokens k_stride / v_stride elements apart (a
 *                 multiple of 8, at least num_kv_heads * head_dim), so that
 *                 they may lie in the QKV projection's output; 16-byte aligned.
 *   k_cache, v_cache  16-byte aligned, written.
 *   seq_lens      [num_seqs] int32, the lengths with the new tokens.
 *   q_starts      [num_seqs + 1] int32: the new tokens of sequence s are rows
 *                 [q_starts[s], q_starts[s + 1]), its last ones in order;
 *                 NULL for one new token per sequence (num_tokens ==
 *                 num_seqs).
 * A token whose table entry is no page (negative, or num_pages and above) is
 * not written.
 * Errors: INVALID_ARG, UNSUPPORTED (head_dim, page_size), MISALIGNED, HIP.
 */
wq_status wq_cache_append(const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
                          const int32_t* block_table, const int32_t* seq_lens, const int32_t* q_starts,
                          int64_t num_seqs, int64_t num_tokens, int64_t num_kv_heads, int64_t head_dim,
                          int64_t k_stride, int64_t v_stride, int64_t page_size, int64_t num_pages,
                          int64_t max_pages_per_seq, void* stream);

/*
 * wq_cache_copy_pages -- copy page src[i] to page dst[i] in every cache.
 *
 *   caches     HOST array of num_caches device pointers (1 ..
 *              WQ_CACHE_MAX_ARRAYS), read during the call only.
 *   page_bytes bytes of one page of one cache, a positive multiple of 16.
 *   src, dst   [count] int32 on the device; a pair with a number outside
 *              [0, num_pages) is skipped.  No page may be in dst twice or in
 *              both lists (the pages concerned then hold either content).
 *   count      0 .. num_pages.
 * Errors: INVALID_ARG, MISALIGNED, HIP.
 */
wq_status wq_cache_copy_pages(void* const* caches, int64_t num_caches, int64_t page_bytes, int64_t num_pages,
                              const int32_t* src, const int32_t* dst, int64_t count, void* stream);

/*
 * wq_page_workspace_size -- bytes of device workspace that wq_cache_reserve,
 * wq_cache_fork and wq_cache_compact need at most for a pool of num_pages
 * pages and num_seqs table rows.  Pure host function.
 */
wq_status wq_page_workspace_size(int64_t num_pages, int64_t num_seqs, size_t* bytes);

/*
 * wq_cache_reserve -- give sequences that grow the pages they lack.
 *
 * For every sequence s, in order, each entry e from ceil(old_lens[s] /
 * page_size) up to, not including, ceil(new_lens[s] / page_size) that holds
 * no page gets the lowest free page left, with a reference count of 1.  Lengths
 * below 0 count as 0, those beyond the table's row as the row's end.
 *   shortfall  int32 on the device, written: 0, or how many pages too few are
 *              free (at most INT32_MAX); then nothing else has been changed.
 *   workspace  of at least the bytes that wq_page_workspace_size reports,
 *              16-byte aligned, owned by the caller, used only while the
 *              work queued by this call runs (calls on one stream may share it).
 * Errors: INVALID_ARG, UNSUPPORTED (page_size), MISALIGNED, HIP.
 */
wq_status wq_cache_reserve(int32_t* block_table, int32_t* refs, const int32_t* old_lens, const int32_t* new_lens,
                           int64_t num_seqs, int64_t page_size, int64_t num_pages, int64_t max_pages_per_seq,
                           int32_t* shortfall, void* workspace, size_t workspace_bytes, void* stream);

/*
 * wq_cache_free -- take pages from sequences.
 *
 * For each listed sequence s of length L, every page is given up of whose
 * tokens none is below `sinks` or, when window > 0, visible through a window of
 * `window` tokens to the token that comes next (t + window > L): its entry
 * becomes -1 and its reference count falls by one.  window = 0 and sinks = 0
 * give up all pages.
 *   seqs  [count] int32 on the device; a number outside [0, num_seqs) is
 *         skipped.  count 0 .. num_seqs.
 *   window, sinks  0 .. 2^30.
 * Errors: INVALID_ARG, UNSUPPORTED (page_size), MISALIGNED, HIP.
 */
wq_status wq_cache_free(int32_t* block_table, int32_t* refs, const int32_t* seq_lens, const int32_t* seqs,
                        int64_t count, int64_t window, int64_t sinks, int64_t num_seqs, int64_t page_size,
                        int64_t num_pages, int64_t max_pages_per_seq, void* stream);

/*
 * wq_cache_fork -- make sequence dst[i] a copy of sequence src[i].
 *
 * Full pages are shared: row dst[i] gets the entries of row src[i], and their
 * reference counts rise by one.  A last page that is only partly filled is
 * copied instead, the filled part in every cache, to the lowest free page left
 * (the forks in order).  Entries past it become -1, and seq_lens[dst[i]] =
 * seq_lens[src[i]].  What row dst[i] held before is overwritten, so its
 * pages are given up first (wq_cache_free).
 *   src, dst   [count] int32 on the device.  A sequence may be forked several
 *              times; none may be in dst twice or in both lists.  A pair with
 *              a number outside [0, num_seqs), or whose length does not fit the
 *              table's row, is skipped.
 *   count      0 .. num_seqs.
 *   shortfall, workspace  as for wq_cache_reserve.
 *   caches     as for wq_cache_copy_pages, pages of num_kv_heads x page_size
 *              x head_dim 16-bit values.
 * Errors: INVALID_ARG, UNSUPPORTED (head_dim, page_size), MISALIGNED, HIP.
 */
wq_status wq_cache_fork(void* const* caches, int64_t num_caches, int32_t* block_table, int32_t* refs,
                        int32_t* seq_lens, const int32_t* src, const int32_t* dst, int64_t count,
                        int64_t num_seqs, int64_t num_kv_heads, int64_t head_dim, int64_t page_size,
                        int64_t num_pages, int64_t max_pages_per_seq, int32_t* shortfall, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * wq_cache_compact -- move the pages in use to the lowest numbers.
 *
 * With n pages in use, the i-th page in use at n or above moves to the i-th
 * free page below n, in every cache; new_table and new_refs are the table and
 * the counts with the new numbers, and live = n.  The pages from n on can then
 * be given back.  new_table may be block_table and new_refs may be refs; they
 * must not overlap otherwise.
 * Errors: INVALID_ARG, MISALIGNED, HIP.
 */
wq_status wq_cache_compact(void* const* caches, int64_t num_caches, int64_t page_bytes, const int32_t* block_table,
                           const int32_t* refs, int32_t* new_table, int32_t* new_refs, int32_t* live,
                           int64_t num_seqs, int64_t num_pages, int64_t max_pages_per_seq, void* workspace,
                           size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WQ_CACHE_H */
