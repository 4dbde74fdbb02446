/*
 * chunk_rope.h -- C ABI of the rotary positions of the chunk-attention library.
 *
 * The rows of a chunk sit at positions that follow from its segment table (chunk_attn.h): query row q_start + i of a
 * segment with context length C = kv_len - q_len is at position C + i of its sequence, and its key belongs into key row
 * kv_start + C + i.  These calls rotate queries and keys by their positions on the way from the projection that made them to the
 * buffers chunk_attn_fwd reads, and gradients on the way back.  With x the rows of one head, f_j the frequencies, p the position:
 *
 *   forward:   y_a = m (x_a cos(p f_j) - x_b sin(p f_j)),   y_b = m (x_b cos(p f_j) + x_a sin(p f_j))
 *   backward:  d_a = m (g_a cos(p f_j) + g_b sin(p f_j)),   d_b = m (g_b cos(p f_j) - g_a sin(p f_j))     (the transpose)
 *
 * for the pairs (a, b) of the first rotary_dim elements of the head: (j, j + rotary_dim / 2), or (2 j, 2 j + 1) where
 * `interleaved` is set; the elements behind them are copied.  Angles are reduced in 64 bits, products are formed in 32, and a result
 * is rounded to bf16 once.
 *
 * Tensors (DEVICE pointers, bf16 unless noted), `heads` rows of head_dim elements next to each other for each token, tokens a
 * stride apart (in elements; at least heads * head_dim, so that views of a fused projection will do):
 *   q, q_out, dq, dq_out : [total_q][num_q_heads][head_dim]
 *   k, dk_out            : [total_q][num_kv_heads][head_dim]   keys of the chunk's own tokens
 *   k_out, dk            : [total_kv][num_kv_heads][head_dim]  rows of the attention's keys; dk is float32 where dk_is_f32 is set
 *                          (chunk_attn_bwd_f32kv)
 * Rows of k_out that belong to no token of the chunk (context, gaps) stay as they are, and those of dk are not read.  In the backward of a split
 * sequence a slice's own rows of dk are complete once every later slice has added to them, which is when this call wants them.
 * Either tensor may be left out together with its output (both null).  q_out may be q (dq_out dq) with the same stride, and k_out k (dk_out dk) where
 * besides every segment has key rows = query rows (kv_start + C = q_start) and dk is bf16, else CHUNK_ATTN_INVALID_ARG; apart from that an output
 * must overlap nothing else.  Tensors need no more alignment than their type's; 16-byte aligned rows are faster.
 *
 * The calls are asynchronous on `hip_stream`, use no workspace, keep nothing and may be captured into a graph.  Segment table and
 * frequencies are HOST memory, read during the call; they travel as kernel arguments, 192 segments to a launch.
 * Returns CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef CHUNK_ROPE_H_
#define CHUNK_ROPE_H_

#include "chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t rotary_dim;        /* even, 2 .. head_dim of the chunk */
  int32_t interleaved;       /* 0: pairs (j, j + rotary_dim / 2); 1: pairs (2 j, 2 j + 1) */
  const double* frequencies; /* HOST array, rotary_dim / 2 finite angles per position, in radians */
  float magnitude;           /* m above: finite, normally 1 */
} chunk_rope_desc;

/*
 * Frequencies f_j = base^(-2 j / R), R = rotary_dim, and the usual ways to stretch them over contexts `factor` (s) times longer:
 *   CHUNK_ROPE_LINEAR   f_j / s
 *   CHUNK_ROPE_BASE     base * s^(R / (R - 2)) in the place of base (R > 2): the first pair keeps its frequency, the last one's is divided by s
 *   CHUNK_ROPE_RAMP     g f_j + (1 - g) f_j / s with g = clamp((n_j - low) / (high - low), 0, 1), where n_j = original_length f_j / 2 pi is how often
 *                       pair j turns over the original context: fast pairs keep their frequency, slow ones are stretched
 * Writes rotary_dim / 2 values to the HOST array `frequencies`.  CHUNK_ATTN_INVALID_ARG for an odd or non-positive rotary_dim, a base that is not finite and > 1,
 * a factor that is not finite and >= 1, an unknown kind, or a ramp without original_length > 0 and high > low >= 0.
 */
enum { CHUNK_ROPE_PLAIN = 0, CHUNK_ROPE_LINEAR = 1, CHUNK_ROPE_BASE = 2, CHUNK_ROPE_RAMP = 3 };
int chunk_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length,
                           double low_rotations, double high_rotations, double* frequencies);

int chunk_rope_fwd(const chunk_attn_desc* desc, const chunk_rope_desc* rope, const void* q, int64_t q_stride, const void* k,
                   int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* hip_stream);

int chunk_rope_bwd(const chunk_attn_desc* desc, const chunk_rope_desc* rope, const void* dq, int64_t dq_stride, const void* dk,
                   int64_t dk_stride, int32_t dk_is_f32, void* dq_out, int64_t dq_out_stride, void* dk_out, int64_t dk_out_stride,
                   void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CHUNK_ROPE_H_ */
