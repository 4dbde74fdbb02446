/*
 * fused_norm.h -- C ABI of the norms around a block, with its gate and residual scale.
 *
 * What lies between the output y of a block (attention, or what follows it) and the next block's input, in one pass over the rows:
 *
 *   r' = residual_scale * r + block_scale * a(g) * N(y; w_post)          h = N(r'; w_pre)
 *
 * with N(x; w) = x w / sqrt(mean(x^2) + eps) over a row and a(g) the gate: g itself, sigmoid(g) or g sigmoid(g).  Every part may be left out
 * (null): no w_post, N(y) is y; no gate, a(g) is 1; no r or no y, its term is 0 (one of the two has to be there); no w_pre, there is no
 * h (and h is null); residual_out may be null where h is wanted only.  With rows of one head each this is the norm and gate of a linear attention's output.
 *
 * The backward starts from what the forward has left in residual_out, forming the row's statistics again while it has the row in registers:
 *
 *   t  = d_residual_out + gradient of N at r' applied to d_h             (d_h is there where w_pre is, and only there; d_residual_out may be null beside it)
 *   d_residual = residual_scale * t,   d_gate = block_scale * t * N(y; w_post) * a'(g),   dy = gradient of N at y applied to block_scale * a(g) * t
 *   d_pre_weight = sum over rows of d_h r' / rms(r'),   d_post_weight = sum over rows of block_scale * a(g) * t * y / rms(y)
 *
 * Any output may be null, and is then not formed.  All arithmetic is in float32, sums over rows run in a fixed order (results are bit-reproducible), every result
 * is rounded once; the forward's h is that of r' before it is rounded.
 *
 * Tensors are DEVICE pointers, rows x cols, rows a stride apart (in elements, >= cols); y, gate, h and their gradients are bf16; residual,
 * residual_out, d_residual_out and d_residual bf16, or float32 where residual_is_f32 is set; weights [cols] bf16, or float32 where
 * weight_is_f32 is set; gradients of weights [cols] float32.  No more alignment than the type's is needed; 16-byte aligned rows are faster.
 * An output may be one of the call's inputs of the same type with the same address and stride (residual_out = residual, d_residual = d_residual_out,
 * dy = y, ...); apart from that outputs must overlap nothing.
 *
 * The calls are asynchronous on `hip_stream`, allocate and keep nothing, and may be captured into a graph.  The backward needs a workspace where it forms
 * gradients of weights: DEVICE memory, 16-byte aligned, of fused_norm_bwd_workspace_bytes (calls that may run at the same time need one each).
 * rows >= 0, 1 <= cols <= FUSED_NORM_MAX_COLS (else CHUNK_ATTN_UNSUPPORTED), eps > 0 and finite, scales finite.  With rows = 0 nothing is written but gradients of weights
 * (zeros, unless accumulated).  Returns CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef FUSED_NORM_H_
#define FUSED_NORM_H_

#include "chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FUSED_NORM_MAX_COLS 16384

enum { FUSED_NORM_GATE_PLAIN = 0, FUSED_NORM_GATE_SIGMOID = 1, FUSED_NORM_GATE_SILU = 2 };

/* What both directions share.  residual: r of the forward; unused by the backward. */
typedef struct {
  int64_t rows;
  int32_t cols;
  int32_t gate_kind;       /* FUSED_NORM_GATE_*; looked at where there is a gate */
  int32_t residual_is_f32; /* type of residual, residual_out and their gradients */
  int32_t weight_is_f32;
  float eps, residual_scale, block_scale;
  const void *y, *gate, *residual;
  int64_t y_stride, gate_stride, residual_stride;
  const void *post_weight, *pre_weight;
} fused_norm_desc;

int fused_norm_fwd(const fused_norm_desc* desc, void* residual_out, int64_t residual_out_stride, void* h, int64_t h_stride, void* hip_stream);

int fused_norm_bwd_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes);

/* residual_out: as the forward left it (read where pre_weight is set).  accumulate_weights: add to the gradients of the weights instead of writing them. */
int fused_norm_bwd(const fused_norm_desc* desc, const void* residual_out, int64_t residual_out_stride, const void* d_residual_out,
                   int64_t d_residual_out_stride, const void* d_h, int64_t d_h_stride, void* dy, int64_t dy_stride, void* d_gate,
                   int64_t d_gate_stride, void* d_residual, int64_t d_residual_stride, float* d_post_weight, float* d_pre_weight,
                   int32_t accumulate_weights, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FUSED_NORM_H_ */
