// Rotary positions of a chunk (include/chunk_rope.h): queries and keys rotated by the positions that the segment table gives their rows, forward
// and backward, between the projection's rows and the attention's buffers.
//
// Bound by memory: every element is read once and written once.  A wave takes one token at a time.  Its lanes stand for (head, slot): a slot is
// eight pairs (16 bytes of either half of the pairs; interleaved: 16 bytes, four pairs) or eight elements to copy, and keeps its place in the head
// from one head to the next, so that a lane forms the sines and cosines of its pairs once per token and keeps them in registers.  No tables are read, and no position is too far: the angle is reduced to a fraction of
// a turn in 64 bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/chunk_rope.h"
#include "kernels.hpp"
#include "operators.hpp"

namespace chunk_attn {
namespace {

constexpr int kRopeSegs = 192;  // segments that travel with one launch (kernel arguments are limited to 4 KB)
constexpr int kMaxPairs = 128;

struct RopeTensor {
  const void* in;
  void* out;
  int64_t in_stride, out_stride;  // elements
  int heads;
};
struct RopeArgs {
  RopeTensor q, k;
  int first_row, rows;  // rows of this launch
  int num_segs;
  int dim, pairs;          // pairs = rotary_dim / 2
  int pair_slots, slots;   // slots of a head that rotate; all
  int heads_per_wave;      // 64 / slots
  int waves_per_row;
  int keys_from_buffer;    // backward: keys come from the key buffer's rows and go to the tokens'
  float magnitude;
  double turns[kMaxPairs]; // frequencies in turns per position
  int start[kRopeSegs], to_position[kRopeSegs], to_key[kRopeSegs];  // first row of a segment; what a row's position and key row are ahead of it
};
static_assert(sizeof(RopeArgs) <= 3900, "fits the kernel arguments");

// One token's heads of one tensor.  c, s: cosines and (signed) sines of the lane's pairs, times the magnitude.
template <bool INTERLEAVED, class T>
__device__ __forceinline__ void rotate_heads(const T* in, __bf16* out, int heads, int dim, int first_head, int head_step, bool rotates, int at, int n,
                                             int pairs, const float* c, const float* s) {
  for (int h = first_head; h < heads; h += head_step) {
    const T* const x = in + (int64_t)h * dim + at;
    __bf16* const y = out + (int64_t)h * dim + at;
    float a[8];
    load_up_to_8(x, n, a);
    if (rotates) {
      if constexpr (INTERLEAVED) {
        float r[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r[2 * j] = a[2 * j] * c[j] - a[2 * j + 1] * s[j];
          r[2 * j + 1] = a[2 * j + 1] * c[j] + a[2 * j] * s[j];
        }
        store_up_to_8(y, n, r);
      } else {
        float b[8], r[8];
        load_up_to_8(x + pairs, n, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = a[j] * c[j] - b[j] * s[j];
        store_up_to_8(y, n, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = b[j] * c[j] + a[j] * s[j];
        store_up_to_8(y + pairs, n, r);
      }
    } else {
      store_up_to_8(y, n, a);
    }
  }
}

template <bool INTERLEAVED, class TK>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + ((int)threadIdx.x >> 6);
  const int index = __builtin_amdgcn_readfirstlane(unit / a.waves_per_row), part = __builtin_amdgcn_readfirstlane(unit % a.waves_per_row);
  if (index >= a.rows) return;
  const int row = a.first_row + index;
  int seg = -1;  // the last segment that starts at or before the row
  for (int i = 0; i < a.num_segs; i += 64) seg += __popcll(__ballot(i + lane < a.num_segs && a.start[i + lane < a.num_segs ? i + lane : 0] <= row));
  seg = __builtin_amdgcn_readfirstlane(seg);
  const double position = (double)(row + a.to_position[seg]);
  const int key_row = row + a.to_key[seg];

  const int sub = lane / a.slots, slot = lane - sub * a.slots;
  if (sub >= a.heads_per_wave) return;
  const bool rotates = slot < a.pair_slots;
  constexpr int kPairs = INTERLEAVED ? 4 : 8;
  float c[kPairs], s[kPairs];
  int at, n;  // the lane's first element of a head, and how many from there on
  if (rotates) {
    at = 8 * slot;
    n = min(8, (INTERLEAVED ? 2 * a.pairs : a.pairs) - at);
    const int first = kPairs * slot;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      double t = position * a.turns[first + j < a.pairs ? first + j : 0];
      t -= rint(t);
      sincospif((float)(2.0 * t), &s[j], &c[j]);
      c[j] *= a.magnitude;
      s[j] *= a.keys_from_buffer ? -a.magnitude : a.magnitude;
    }
  } else {
    at = 2 * a.pairs + 8 * (slot - a.pair_slots);
    n = min(8, a.dim - at);
  }
  const int first_head = part * a.heads_per_wave + sub, step = a.waves_per_row * a.heads_per_wave;
  if (a.q.in)
    rotate_heads<INTERLEAVED>((const __bf16*)a.q.in + row * a.q.in_stride, (__bf16*)a.q.out + row * a.q.out_stride, a.q.heads, a.dim, first_head, step, rotates, at, n,
                              a.pairs, c, s);
  if (a.k.in) {
    const int64_t from = a.keys_from_buffer ? key_row : row, to = a.keys_from_buffer ? row : key_row;
    rotate_heads<INTERLEAVED>((const TK*)a.k.in + from * a.k.in_stride, (__bf16*)a.k.out + to * a.k.out_stride, a.k.heads, a.dim, first_head, step, rotates, at, n, a.pairs, c, s);
  }
}

int rope(const chunk_attn_desc* d, const chunk_rope_desc* r, RopeTensor q, RopeTensor k, bool backward, bool k_f32, hipStream_t stream) {
  const int rc = chunk_attn_validate(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!r || !r->frequencies || r->rotary_dim < 2 || r->rotary_dim % 2 != 0 || r->rotary_dim > d->head_dim || !finite_number(r->magnitude)) return CHUNK_ATTN_INVALID_ARG;
  const int pairs = r->rotary_dim / 2;
  for (int j = 0; j < pairs; ++j)
    if (!finite_number(r->frequencies[j])) return CHUNK_ATTN_INVALID_ARG;
  q.heads = d->num_q_heads;
  k.heads = d->num_kv_heads;
  bool copies = false;  // whether the elements behind the pairs have to be moved
  for (const RopeTensor* t : {&q, &k}) {
    if (!t->in != !t->out) return CHUNK_ATTN_INVALID_ARG;
    if (!t->in) continue;
    const bool f32 = t == &k && k_f32;
    const int64_t least = (int64_t)t->heads * d->head_dim;
    if (t->in_stride < least || t->out_stride < least || ((uintptr_t)t->in & (f32 ? 3 : 1)) != 0 || ((uintptr_t)t->out & 1) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (t->in != t->out) copies = true;
    else if (f32 || t->in_stride != t->out_stride) return CHUNK_ATTN_INVALID_ARG;
  }
  if (k.in && k.in == k.out)
    for (int i = 0; i < d->num_segments; ++i)
      if (d->segments[i].kv_start + d->segments[i].kv_len - d->segments[i].q_len != d->segments[i].q_start) return CHUNK_ATTN_INVALID_ARG;
  if (!q.in && !k.in) return CHUNK_ATTN_OK;

  RopeArgs a{};
  a.q = q;
  a.k = k;
  a.dim = d->head_dim;
  a.pairs = pairs;
  a.pair_slots = ((r->interleaved ? 2 * pairs : pairs) + 7) / 8;
  a.slots = a.pair_slots + (copies ? (d->head_dim - 2 * pairs + 7) / 8 : 0);
  a.heads_per_wave = 64 / a.slots;
  a.keys_from_buffer = backward;
  a.magnitude = r->magnitude;
  for (int j = 0; j < pairs; ++j) a.turns[j] = r->frequencies[j] * 0.15915494309189533577;  // 1 / 2 pi
  for (int s0 = 0; s0 < d->num_segments; s0 += kRopeSegs) {
    a.num_segs = std::min(kRopeSegs, d->num_segments - s0);
    const chunk_attn_seg* const segs = d->segments + s0;
    for (int i = 0; i < a.num_segs; ++i) {
      const int context = segs[i].kv_len - segs[i].q_len;
      a.start[i] = segs[i].q_start;
      a.to_position[i] = context - segs[i].q_start;
      a.to_key[i] = segs[i].kv_start + context - segs[i].q_start;
    }
    a.first_row = segs[0].q_start;
    a.rows = segs[a.num_segs - 1].q_start + segs[a.num_segs - 1].q_len - a.first_row;
    a.waves_per_row = a.rows < 4 * kCus ? 4 : 1;  // few tokens: a token's heads go to four waves
    const dim3 grid((unsigned)(((int64_t)a.rows * a.waves_per_row + 3) / 4));
    if (r->interleaved) {
      if (k_f32) hipLaunchKernelGGL((rope_kernel<true, float>), grid, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((rope_kernel<true, __bf16>), grid, dim3(256), 0, stream, a);
    } else {
      if (k_f32) hipLaunchKernelGGL((rope_kernel<false, float>), grid, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((rope_kernel<false, __bf16>), grid, dim3(256), 0, stream, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report_hip(e, "rotary positions");
  }
  return CHUNK_ATTN_OK;
}

}  // namespace
}  // namespace chunk_attn

extern "C" int chunk_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double low_rotations,
                                      double high_rotations, double* frequencies) {
  using chunk_attn::finite_number;
  if (!frequencies || rotary_dim < 2 || rotary_dim % 2 != 0 || !finite_number(base) || base <= 1.0 || !finite_number(factor) || factor < 1.0)
    return CHUNK_ATTN_INVALID_ARG;
  if (scaling < CHUNK_ROPE_PLAIN || scaling > CHUNK_ROPE_RAMP || (scaling == CHUNK_ROPE_BASE && rotary_dim == 2)) return CHUNK_ATTN_INVALID_ARG;
  if (scaling == CHUNK_ROPE_RAMP &&
      !(finite_number(original_length) && original_length > 0.0 && finite_number(low_rotations) && low_rotations >= 0.0 && finite_number(high_rotations) &&
        high_rotations > low_rotations))
    return CHUNK_ATTN_INVALID_ARG;
  const double R = rotary_dim, two_pi = 6.283185307179586477;
  if (scaling == CHUNK_ROPE_BASE) base *= std::pow(factor, R / (R - 2.0));
  for (int j = 0; j < rotary_dim / 2; ++j) {
    double f = std::pow(base, -2.0 * j / R);
    if (scaling == CHUNK_ROPE_LINEAR) f /= factor;
    if (scaling == CHUNK_ROPE_RAMP) {
      const double g = std::min(1.0, std::max(0.0, (original_length * f / two_pi - low_rotations) / (high_rotations - low_rotations)));
      f = g * f + (1.0 - g) * f / factor;
    }
    frequencies[j] = f;
  }
  return CHUNK_ATTN_OK;
}

extern "C" int chunk_rope_fwd(const chunk_attn_desc* desc, const chunk_rope_desc* rope, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                              int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* hip_stream) {
  return chunk_attn::rope(desc, rope, {q, q_out, q_stride, q_out_stride, 0}, {k, k_out, k_stride, k_out_stride, 0}, false, false, (hipStream_t)hip_stream);
}

extern "C" int chunk_rope_bwd(const chunk_attn_desc* desc, const chunk_rope_desc* rope, const void* dq, int64_t dq_stride, const void* dk, int64_t dk_stride,
                              int32_t dk_is_f32, void* dq_out, int64_t dq_out_stride, void* dk_out, int64_t dk_out_stride, void* hip_stream) {
  return chunk_attn::rope(desc, rope, {dq, dq_out, dq_stride, dq_out_stride, 0}, {dk, dk_out, dk_stride, dk_out_stride, 0}, true, dk_is_f32 != 0, (hipStream_t)hip_stream);
}
