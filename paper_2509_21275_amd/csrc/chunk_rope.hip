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
#include <type_traits>

#include "../../include/chunk_rope.h"
#include "kernels.hpp"
#include "operators.hpp"

namespace chunk_attn {
namespace {

constexpr int kRopeSegs = 192;  // segments that travel with one launch (kernel arguments are limited to 4 KB)
constexpr int kRopeRows = 1 << 25;  // rows of a launch (its threads are limited to 2^32)
constexpr int kMaxPairs = 128;
// Calls that move more than the last-level cache (256 MiB) holds pass their rows by the caches.  us, kept / streamed, 32/8 heads of 128: 4096 tokens (84 MB) 16.2 / 17.6; 16384 (336 MB) 65 / 62, 5.4 TB/s;
// 65536 (1.34 GB) 246 / 221, 6.1 TB/s; backward of 65536 with float32 dk (1.48 GB) 267 / 253.  Loose pieces are kept: 65536 tokens with rotary_dim 126 397, 3.4 TB/s, 38 of 96 192, 5.2.
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

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

// Eight elements of 16-byte aligned bf16 or float32 rows, by the caches or past them.
template <bool STREAM, class T>
__device__ __forceinline__ void load_8(const T* p, float* x) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8* const q = reinterpret_cast<const bf16x8*>(p);
    const bf16x8 v = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {  // (two pieces that leave half a line to each other: kept)
    const f32x4 v0 = reinterpret_cast<const f32x4*>(p)[0], v1 = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = v0[e];
      x[4 + e] = v1[e];
    }
  }
}
template <bool STREAM>
__device__ __forceinline__ void store_8(__bf16* p, const float* x) {
  bf16x8* const q = reinterpret_cast<bf16x8*>(p);
  const bf16x8 v = pack8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
  if constexpr (STREAM) __builtin_nontemporal_store(v, q);
  else *q = v;
}

// How a lane's pieces of eight elements are accessed.  kLoose: some rows or halves of pairs are not 16-byte aligned, or the last piece is shorter.
enum Access { kLoose, kKeep, kStream };
template <Access A, class T>
__device__ __forceinline__ void load_piece(const T* p, int n, float* x) {
  if constexpr (A == kLoose) load_up_to_8(p, n, x);
  else load_8<A == kStream>(p, x);
}
template <Access A>
__device__ __forceinline__ void store_piece(__bf16* p, int n, const float* x) {
  if constexpr (A == kLoose) store_up_to_8(p, n, x);
  else store_8<A == kStream>(p, x);
}

// x c + y s, rounded in the same places however the pieces are accessed.
__device__ __forceinline__ float turned(float x, float y, float c, float s) { return __builtin_fmaf(y, s, x * c); }

// One token's heads of one tensor, as many at a time as are in flight together.  c, s: cosines and (signed) sines of the lane's pairs, times the magnitude.
template <bool INTERLEAVED, Access A, class T>
__device__ __forceinline__ void rotate_heads(const T* in, __bf16* out, int heads, int dim, int first_head, int head_step, bool rotates, int at, int n,
                                             int pairs, const float* c, const float* s) {
  constexpr int kTogether = 2;
  const int second = !INTERLEAVED && rotates ? pairs : 0;  // how far the other half of the lane's pairs is; what it copies, it reads once
  for (int h0 = first_head; h0 < heads; h0 += kTogether * head_step) {
    float a[kTogether][8], b[kTogether][8];
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const int h = h0 + k * head_step;
      if (h < heads) {
        const T* const x = in + (int64_t)h * dim + at;
        load_piece<A>(x, n, a[k]);
        if (second) load_piece<A>(x + second, n, b[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const int h = h0 + k * head_step;
      if (h >= heads) continue;
      __bf16* const y = out + (int64_t)h * dim + at;
      if (!rotates) {
        store_piece<A>(y, n, a[k]);
        continue;
      }
      float r[8];
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r[2 * j] = turned(a[k][2 * j], a[k][2 * j + 1], c[j], -s[j]);
          r[2 * j + 1] = turned(a[k][2 * j + 1], a[k][2 * j], c[j], s[j]);
        }
        store_piece<A>(y, n, r);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = turned(a[k][j], b[k][j], c[j], -s[j]);
        store_piece<A>(y, n, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = turned(b[k][j], a[k][j], c[j], s[j]);
        store_piece<A>(y + pairs, n, r);
      }
    }
  }
}

template <bool INTERLEAVED, Access A, class TK>
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
  // The last piece of several begins eight elements before the end: what it shares with the one before, both lanes form alike (from the same loads, also in place, as one wave has the whole head).
  if (rotates) {
    const int end = INTERLEAVED ? 2 * a.pairs : a.pairs;
    at = max(0, min(8 * slot, end - 8));
    n = min(8, end);
    const int first = INTERLEAVED ? at / 2 : at;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      double t = position * a.turns[first + j < a.pairs ? first + j : 0];
      t -= rint(t);
      sincospif((float)(2.0 * t), &s[j], &c[j]);
      c[j] *= a.magnitude;
      s[j] *= a.keys_from_buffer ? -a.magnitude : a.magnitude;
    }
  } else {
    const int end = a.dim - 2 * a.pairs;
    at = 2 * a.pairs + max(0, min(8 * (slot - a.pair_slots), end - 8));
    n = min(8, end);
  }
  const int first_head = part * a.heads_per_wave + sub, step = a.waves_per_row * a.heads_per_wave;
  if (a.q.in)
    rotate_heads<INTERLEAVED, A>((const __bf16*)a.q.in + row * a.q.in_stride, (__bf16*)a.q.out + row * a.q.out_stride, a.q.heads, a.dim, first_head, step, rotates, at, n,
                                 a.pairs, c, s);
  if (a.k.in) {
    const int64_t from = a.keys_from_buffer ? key_row : row, to = a.keys_from_buffer ? row : key_row;
    rotate_heads<INTERLEAVED, A>((const TK*)a.k.in + from * a.k.in_stride, (__bf16*)a.k.out + to * a.k.out_stride, a.k.heads, a.dim, first_head, step, rotates, at, n, a.pairs, c, s);
  }
}

template <bool INTERLEAVED, Access A>
void launch_rope(const RopeArgs& a, bool k_f32, hipStream_t stream) {
  const dim3 grid((unsigned)(((int64_t)a.rows * a.waves_per_row + 3) / 4));
  if (k_f32) hipLaunchKernelGGL((rope_kernel<INTERLEAVED, A, float>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((rope_kernel<INTERLEAVED, A, __bf16>), grid, dim3(256), 0, stream, a);
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
  bool loose = (r->interleaved ? r->rotary_dim : pairs) % 8 != 0;
  int64_t bytes = 0;
  for (const RopeTensor* t : {&q, &k}) {
    if (!t->in != !t->out) return CHUNK_ATTN_INVALID_ARG;
    if (!t->in) continue;
    const bool f32 = t == &k && k_f32;
    const int64_t least = (int64_t)t->heads * d->head_dim;
    if (t->in_stride < least || t->out_stride < least || ((uintptr_t)t->in & (f32 ? 3 : 1)) != 0 || ((uintptr_t)t->out & 1) != 0) return CHUNK_ATTN_INVALID_ARG;
    bytes += least * d->total_q * (f32 ? 6 : 4);
    loose |= (((uintptr_t)t->in | (uintptr_t)t->out) & 15) != 0 || t->in_stride % (f32 ? 4 : 8) != 0 || t->out_stride % 8 != 0;
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
    const int64_t end = (int64_t)segs[a.num_segs - 1].q_start + segs[a.num_segs - 1].q_len;
    for (int64_t row = segs[0].q_start; row < end; row += kRopeRows) {
      a.first_row = (int)row;
      a.rows = (int)std::min<int64_t>(kRopeRows, end - row);
      a.waves_per_row = a.rows < 4 * kCus ? 4 : 1;  // few tokens: a token's heads go to four waves
      auto launch = [&](auto access) {
        constexpr Access A = decltype(access)::value;
        if (r->interleaved) launch_rope<true, A>(a, k_f32, stream);
        else launch_rope<false, A>(a, k_f32, stream);
      };
      if (loose) launch(std::integral_constant<Access, kLoose>{});
      else if (bytes > kStreamBytes) launch(std::integral_constant<Access, kStream>{});
      else launch(std::integral_constant<Access, kKeep>{});
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return report_hip(e, "rotary positions");
    }
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
