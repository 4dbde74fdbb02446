/*
 * paged_cache.h -- C ABI of the cache of keys and values that new tokens are decoded against: which pages of a pool belong to which request, and keys and values on their way
 * into the pages.
 *
 * The cache (DEVICE, 16-byte aligned, contiguous; the caller owns it):
 *   k_cache, v_cache : [num_pages][num_kv_heads][page_size][head_dim], bf16, or e4m3 (OCP, finite, no infinities) that stands for the value times scale[head]
 * Token t of a request lies in row t % page_size of page table[request][t / page_size]; its slot is the number page * page_size + row.
 *
 * Requests (DEVICE, int32, 4-byte aligned): request i is row i of every array; an idle one has length 0 and nothing new.
 *   kv_len    : [num_requests] tokens in the cache
 *   held      : [num_requests] pages that belong to the request: the first `held` entries of its row of the table, kv_len <= held * page_size
 *   table     : [num_requests][max_pages]; entries from `held` on are never read
 *   free_pages: [num_pages] a stack of the pages that belong to nobody, its top at num_free - 1
 *   num_free  : [1]
 * What these hold is not known to the host, so nothing in them is an error: lengths and counts out of their range count as the nearest that is in it, and a page number that is none makes
 * the slots of its tokens -1.
 *
 * A step of a server: paged_cache_extend for the tokens that come in, paged_cache_write for their keys and values in every layer, attention over the cache (paged_attn.h),
 * and, where drafted tokens were rejected or requests end, paged_cache_truncate.  A request that paged_cache_extend did not serve (`granted` 0) is as it was, and its last cached tokens are none of this
 * step's: nothing may be dropped for the step, so with drafts it is verified with a count of 0, (new - 1) * granted (draft_verify.h); its rows are in q_start all the same, and what is computed from them means nothing.
 *
 * The calls are asynchronous on `hip_stream`, keep nothing, allocate nothing and may be captured into a graph.  Results do not depend on timing.  Scratch space is the caller's `workspace` (DEVICE
 * memory, 256-byte aligned, of paged_cache_workspace_bytes; its contents need not survive, and calls that may run at the same time need one each).
 * Return CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef PAGED_CACHE_H_
#define PAGED_CACHE_H_

#include "chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PAGED_CACHE_MAX_REQUESTS 65536
#define PAGED_CACHE_MAX_PAGE_SIZE 65536

/* What a number in the cache is held as. */
enum { PAGED_CACHE_BF16 = 0, PAGED_CACHE_E4M3 = 1 };

typedef struct {
  int32_t num_requests; /* 1 .. PAGED_CACHE_MAX_REQUESTS, else CHUNK_ATTN_UNSUPPORTED (below 1: CHUNK_ATTN_INVALID_ARG) */
  int32_t max_pages;    /* pages that a request can have, >= 1; max_pages * page_size < 2^31 */
  int32_t page_size;    /* tokens to a page, 1 .. PAGED_CACHE_MAX_PAGE_SIZE, any number */
  int32_t num_pages;    /* pages of the pool, >= 1 */
} paged_cache_desc;

int paged_cache_validate(const paged_cache_desc* desc);
int paged_cache_workspace_bytes(const paged_cache_desc* desc, size_t* bytes);

/*
 * Pages and slots for the tokens that come in: new_tokens [num_requests] (negative: 0).  Request i has use for max(0, ceil((kv_len + new) / page_size) - held) pages.  Requests are
 * served in their order: one that needs pages gets them, off the top of the stack, if those before it and it together need no more than there are; one that needs none is always served.
 * Not served, and without a claim on pages, is a request that would be longer than max_pages * page_size, or whose rows do not all fit in max_rows.
 *   q_start     : [num_requests + 1] sums of new_tokens before each request, at most max_rows: rows q_start[i] .. q_start[i + 1] - 1 of the tensors of new tokens are request i's
 *   slots       : [max_rows] int64, 8-byte aligned: the slot of each row; -1 for rows of requests that are not served and for rows behind the last request
 *   granted     : [num_requests] 1 if the request is served, else 0; or null
 *   kv_len_out, held_out, num_free_out: the state behind the call (may each be its input, and may overlap nothing else); of a request that is not served as before
 *   table       : new pages are entered.  free_pages is read.
 */
int paged_cache_extend(const paged_cache_desc* desc, const int32_t* new_tokens, const int32_t* kv_len, const int32_t* held, int32_t* table, const int32_t* free_pages,
                       const int32_t* num_free, int32_t* kv_len_out, int32_t* held_out, int32_t* num_free_out, int32_t* q_start, int64_t* slots, int32_t max_rows,
                       int32_t* granted, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Tokens off the end of requests: drop [num_requests] (negative: 0; kv_len or more: all, the request has ended).  Pages that hold none of the tokens left go back on the stack, in
 * the order of the requests and of their tables; those that would not fit the stack (pages given back twice) are lost.  The table is read, and stays as it is.  *_out as above.
 * It knows no holders: a page that several requests hold goes onto the stack once for each that gives it back, and then to two others.  Requests that share pages (full ones, of a common prompt: the
 * attention reads them as any) are therefore dropped down to the shared tokens and no further, where the caller sets their kv_len and held to 0; the last holder gives the shared pages back.
 */
int paged_cache_truncate(const paged_cache_desc* desc, const int32_t* drop, const int32_t* kv_len, const int32_t* held, const int32_t* table, int32_t* free_pages,
                         const int32_t* num_free, int32_t* kv_len_out, int32_t* held_out, int32_t* num_free_out, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

/*
 * Keys and values of new tokens to their slots: k, v bf16, row r, head h at r * stride + h * head_dim (strides in elements, >= num_kv_heads * head_dim; 2-byte aligned), slots [rows] int64.
 * Rows whose slot is negative or >= num_pages * page_size are skipped; rows of the cache that no slot names stay as they are.  Where two rows have the same slot, what is left there is of
 * either, piece by piece.  cache_type PAGED_CACHE_E4M3: k_scale, v_scale [num_kv_heads] float32, > 0; the float32 quotient of the value and the scale is rounded to the nearest (ties to
 * even), what is past 448 to 448; signs are kept, of zeros too, and NaN stays NaN.  PAGED_CACHE_BF16: copied, k_scale and v_scale are not read and may be null.
 * head_dim 64, 96, 128 or 256, else CHUNK_ATTN_UNSUPPORTED; rows >= 0, rows * num_kv_heads * head_dim <= 2^35 - 2^11.  The cache may overlap nothing else.
 */
int paged_cache_write(int32_t rows, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages, int32_t cache_type, const void* k, int64_t k_stride,
                      const void* v, int64_t v_stride, const int64_t* slots, const float* k_scale, const float* v_scale, void* k_cache, void* v_cache, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAGED_CACHE_H_ */
