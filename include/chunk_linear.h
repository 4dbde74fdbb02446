/*
 * chunk_linear.h -- C ABI of linear attention with a decay for each head over the sequences of a chunk.
 *
 * A token's output is a sum over the tokens up to it, without softmax, in which a token further back counts for less:
 *
 *   S_t = l S_(t-1) + k_t^T v_t        o_t = scale * q_t S_t        l = exp(log_decay[h]),  S: head_dim x head_dim, of key/value head h
 *
 * that is o_t = scale * sum over s <= t of l^(t-s) (q_t . k_s) v_s.  Query head i uses key/value head i / (num_q_heads / num_kv_heads),
 * its state and its decay.  Sequences packed into a chunk do not see each other.  Where softmax attention needs the keys and values of a split sequence's earlier
 * slices, this needs the state they leave: a segment may start from a given state and may leave its own, and in the backward gradients of states travel
 * from slice to slice the other way.
 *
 * Tensors (DEVICE pointers, contiguous, bf16, 16-byte aligned; the caller owns them):
 *   q, o, d_o, dq : [total][num_q_heads][head_dim]
 *   k, v, dk, dv  : [total][num_kv_heads][head_dim]
 *   log_decay     : [num_kv_heads] float32, natural logarithm of the decay, normally <= 0 (0: nothing decays, -inf: only the token itself counts; a
 *                   larger one is taken as it is, as long as float32 has the powers of l up to the sequence's length, rounded up to a multiple of 8: past that
 *                   results may be infinite or NaN; a NaN makes all results of its head NaN).  A constant: it has no gradient here.
 *   states        : [num_states][num_kv_heads][head_dim of k][head_dim of v] float32, 16-byte aligned
 * Rows of no segment stay as they are.  States (and their gradients) that a call leaves are summed up in float32, from products that are as good as float32's; products
 * that form outputs, and sums inside the call that go into no state that it leaves, are good to 2^-16 and summed up in float32.  A result is rounded once.  A value that is not finite
 * in a token may make what its sequence has in the same 64 rows (counted from the sequence's start) not finite, and all that follows it (in gradients: that
 * comes before it).
 *
 * The calls are asynchronous on `hip_stream`, keep nothing, allocate nothing and may be captured into a graph.  The segment table is HOST memory, read during the call; it
 * travels as kernel arguments.  Scratch space is the caller's `workspace` (DEVICE memory, 256-byte aligned, of chunk_linear_workspace_bytes; its contents
 * need not survive, and calls that may run at the same time need one each).
 * Return CHUNK_ATTN_OK or a negative code of chunk_attn.h; errors are found on the host before any launch.
 */
#ifndef CHUNK_LINEAR_H_
#define CHUNK_LINEAR_H_

#include "chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CHUNK_LINEAR_MAX_HEADS 16384

/* One sequence, or a slice of one: rows start .. start + len - 1; state_in: slot of the state before its first token (-1: zeros); state_out: slot that
 * takes the state behind its last token (-1: not wanted). */
typedef struct {
  int32_t start, len, state_in, state_out;
} chunk_linear_seg;

typedef struct {
  int32_t num_q_heads;  /* 1 .. CHUNK_LINEAR_MAX_HEADS, else CHUNK_ATTN_UNSUPPORTED */
  int32_t num_kv_heads; /* > 0, divides num_q_heads */
  int32_t head_dim;     /* 64, 96, 128 or 256 */
  int32_t total;        /* rows of the tensors */
  int32_t num_states;   /* slots of the state tensors, >= 0 */
  int32_t num_segments; /* >= 1 */
  /* HOST array, borrowed for the call.  Requirements (else CHUNK_ATTN_BAD_SEGMENT): len >= 1, rows inside [0, total), in increasing order without overlap
   * (gaps are allowed); slots -1 or inside [0, num_states); no two segments with the same state_out. */
  const chunk_linear_seg* segments;
  float scale; /* finite, > 0 */
} chunk_linear_desc;

int chunk_linear_validate(const chunk_linear_desc* desc);

/* Scratch sizes in bytes: float32 states of the pieces that long sequences are cut into. */
int chunk_linear_workspace_bytes(const chunk_linear_desc* desc, size_t* fwd_bytes, size_t* bwd_bytes);

/*
 * states_in: may be null if no segment has a state_in; states_out likewise.  They may be the same tensor (slots are then updated in place) as long as no
 * segment's state_out is another one's state_in, else CHUNK_ATTN_BAD_SEGMENT; apart from that outputs must overlap nothing.
 */
int chunk_linear_fwd(const chunk_linear_desc* desc, const void* q, const void* k, const void* v, const float* log_decay, const float* states_in, void* o,
                     float* states_out, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradients, for the gradients d_o of the outputs and d_states_out (or null: zeros) of the states left, slot by slot as states_out.  Writes dq, dk, dv and, if
 * d_states_in is not null, the gradient of each state_in to its slot (two segments then must not share one, else CHUNK_ATTN_BAD_SEGMENT); slots
 * that no segment starts from stay as they are.  d_states_in may be d_states_out, with the same condition as in the forward.
 */
int chunk_linear_bwd(const chunk_linear_desc* desc, const void* q, const void* k, const void* v, const float* log_decay, const float* states_in,
                     const void* d_o, const float* d_states_out, void* dq, void* dk, void* dv, float* d_states_in, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

/*
 * One token for each of `batch` sequences whose states lie in slots: q, o [batch][num_q_heads][head_dim], k, v [batch][num_kv_heads][head_dim]; slots
 * [batch] int32, DEVICE.  Reads state slots[i] from states_in, adds token i, writes the state to the same slot of states_out (which may be states_in) and the
 * output to row i of o.  Several rows with the same slot are consecutive tokens of that sequence, in the order of the rows.  A row whose slot is negative or >= num_states
 * is skipped: its row of o stays as it is.  Slots that no row names are not touched.  batch >= 0, batch * num_kv_heads < 2^24.  Each row looks for its slot in all of `slots`: with some 10^4 rows
 * of few heads that takes longer than the states do.
 */
int chunk_linear_step(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, const void* q, const void* k, const void* v,
                      const float* log_decay, const float* states_in, float* states_out, int32_t num_states, const int32_t* slots, void* o, float scale,
                      void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CHUNK_LINEAR_H_ */
