/*
 * paged_attn.h -- C ABI of the attention of new tokens over a paged cache of keys and values (paged_cache.h): the single-token form of chunk_attn.h's attention, for one or a few new tokens of
 * each of many sequences.
 *
 * Sequence i has kv_len[i] tokens in the cache, of which its last n = q_start[i + 1] - q_start[i] are new: rows q_start[i] .. q_start[i + 1] - 1 of q.  New token j attends to tokens
 * t = 0 .. kv_len - n + j of its own sequence and to nothing else.  The result is exact softmax attention, O = softmax(scale * Q K^T + mask) V; a row that sees no token (kv_len < n)
 * has o = 0 and lse = -inf; rows of a request that paged_cache_extend did not serve take its last cached tokens for new ones, and mean nothing.  Query head h uses key/value head h / (num_q_heads / num_kv_heads).
 *
 * Tensors (DEVICE; the caller owns them):
 *   q, o     : bf16, row r, head h at r * stride + h * head_dim (strides in elements, >= num_q_heads * head_dim; 2-byte aligned); rows behind q_start[num_seqs] are not read, and left as they are
 *   lse      : [num_q_heads][total_q] float32, natural-log sum of exp of the scaled scores; or null
 *   k_cache, v_cache, table: as in paged_cache.h; k_scale, v_scale [num_kv_heads] float32, > 0 (PAGED_CACHE_E4M3; else not read)
 *   kv_len   : [num_seqs] int32;  q_start: [num_seqs + 1] int32, in increasing order from 0
 * What kv_len, q_start and table hold is not known to the host, so nothing in them is an error: lengths count as at most max_pages * page_size, rows outside [0, total_q) as not there (n counts the
 * others), and tokens on a page whose number is none, which no row sees, as masked; a row that starts which do not increase give to several sequences holds what any of them leaves there.
 * What lies in the cache where a row sees nothing (other rows of a page, tokens behind it) does not reach it, whatever it is; a value that is not finite in a key that it sees leaves its dimension not
 * finite (an infinity may become NaN).
 *
 * Any number of new tokens is right; many of them (hundreds) read a sequence's keys and values once for every 128 rows of a key/value head (32 for head dimension 256), and are
 * faster with chunk_attn_fwd.  Scores, softmax and sums are float32; weights go into the products with values as two bf16 terms, with e4m3 values as one float16 term; a result is rounded once.
 * Results do not depend on timing; the walk over the keys is cut where the lengths of all sequences say, so a sequence's last bits may depend on the others' lengths.
 *
 * The calls are asynchronous on `hip_stream`, keep nothing, allocate nothing and may be captured into a graph: lengths and tables are read on the device, so a replay follows them.  Scratch space
 * is the caller's `workspace` (DEVICE memory, 256-byte aligned, of paged_attn_workspace_bytes; its contents need not survive, and calls that may run at the same time need one each).  Outputs may overlap nothing else.
 * Return CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef PAGED_ATTN_H_
#define PAGED_ATTN_H_

#include "paged_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t num_q_heads;  /* 1 .. 16384, else CHUNK_ATTN_UNSUPPORTED */
  int32_t num_kv_heads; /* > 0, divides num_q_heads */
  int32_t head_dim;     /* 64, 96, 128 or 256 */
  int32_t num_seqs;     /* 1 .. PAGED_CACHE_MAX_REQUESTS */
  int32_t total_q;      /* rows of q and o, >= 0 (0: nothing to do); total_q * num_q_heads < 2^31 */
  int32_t page_size;    /* 1 .. PAGED_CACHE_MAX_PAGE_SIZE */
  int32_t num_pages;    /* pages of the pool; num_pages * num_kv_heads * page_size < 2^31 */
  /* entries of a row of the table; max_pages * page_size <= 2^30, and with the rows of all sequences, R = total_q * num_q_heads / num_kv_heads:
   * (num_seqs + R / 32) * max_pages * page_size <= 2^37 */
  int32_t max_pages;
  int32_t cache_type;   /* PAGED_CACHE_BF16 or PAGED_CACHE_E4M3 */
  float softmax_scale;  /* finite, > 0; normally 1/sqrt(head_dim) */
} paged_attn_desc;

int paged_attn_validate(const paged_attn_desc* desc);

/* Scratch size: float32 partial results of sequences that are cut. */
int paged_attn_workspace_bytes(const paged_attn_desc* desc, size_t* bytes);

int paged_attn_fwd(const paged_attn_desc* desc, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                   const int32_t* table, const int32_t* kv_len, const int32_t* q_start, void* o, int64_t o_stride, float* lse, void* workspace, size_t workspace_bytes,
                   void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAGED_ATTN_H_ */
