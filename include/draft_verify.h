/*
 * draft_verify.h -- C ABI of the verification of drafted tokens: how many of the tokens that a draft proposes for each request the target keeps, and the token that follows them, such that
 * the tokens are distributed as if the target had drawn them one by one.  All random numbers are inputs.
 *
 * Request r has count[r] drafted tokens d_j, drawn from the draft's probabilities q_j; the target's probabilities p_j are given for each of these places and for the one behind the last.
 * Token j is kept if all before it are and u_j * q_j(d_j) < p_j(d_j), in exact arithmetic.  At the first place a that is not, the token is drawn from the weights
 * max(0, p_a(x) - q_a(x)), or, if all are kept (a = count), from p_a(x): it is the lowest x of positive weight whose sum of weights up to and with it exceeds last_uniform * (sum of all), in float64; the
 * highest x of positive weight if none does.  Where no weight is positive it is drawn from p_a, and if nothing in p_a is positive either, it is -1.  Without draft
 * probabilities q_j is 1 at d_j and 0 elsewhere (a draft that does not draw).
 * A probability that is not finite (or a difference of two that float32 does not hold) weighs nothing, and keeps no token.  A drafted token outside [0, vocab) is not kept.
 *
 * Tensors (DEVICE; the caller owns them):
 *   target       : row j of request r at (r * (max_drafts + 1) + j) * target_stride, vocab contiguous elements; float32 or bf16, aligned to their type
 *   draft        : row j of request r at (r * max_drafts + j) * draft_stride, of the same type; or null
 *   tokens       : [batch][max_drafts] int32;  count: [batch] int32, counted as 0 .. max_drafts at most, or null: max_drafts each, where that many drafted tokens of every request are in the cache
 *   uniforms     : [batch][max_drafts] float32;  last_uniform: [batch] float32; both in [0, 1)
 *   accepted     : [batch] int32, tokens kept;  rejected: [batch] int32, count - accepted, or null: what paged_cache_truncate takes off again.  Of a request with nothing new,
 *                  or that paged_cache_extend did not serve (`granted` 0), no drafted token is in the cache: its count has to be 0, so that nothing is taken off it, and its row of `out` means nothing
 *   out          : [batch][max_drafts + 1] int32: the tokens kept, the one that follows them, then -1
 * Rows of probabilities that the result does not depend on are not read, but for one number of each drafted token.
 *
 * The call is asynchronous on `hip_stream`, keeps nothing, allocates nothing and may be captured into a graph.  Results do not depend on timing.  Scratch space is the caller's `workspace` (DEVICE memory,
 * 256-byte aligned, of draft_verify_workspace_bytes; its contents need not survive, and calls that may run at the same time need one each).  Outputs may overlap nothing else.
 * Return CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef DRAFT_VERIFY_H_
#define DRAFT_VERIFY_H_

#include "chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DRAFT_VERIFY_MAX_DRAFTS 64
#define DRAFT_VERIFY_MAX_VOCAB (1 << 24)

/* batch 0 .. 2^23 - 1, max_drafts 0 .. DRAFT_VERIFY_MAX_DRAFTS and vocab 1 .. DRAFT_VERIFY_MAX_VOCAB (above: CHUNK_ATTN_UNSUPPORTED), batch * vocab < 2^36. */
int draft_verify_workspace_bytes(int32_t batch, int32_t max_drafts, int32_t vocab, size_t* bytes);

int draft_verify(int32_t batch, int32_t max_drafts, int32_t vocab, int32_t probabilities_are_f32, const void* target, int64_t target_stride, const void* draft,
                 int64_t draft_stride, const int32_t* tokens, const int32_t* count, const float* uniforms, const float* last_uniform, int32_t* accepted, int32_t* rejected,
                 int32_t* out, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DRAFT_VERIFY_H_ */
