// Norms around a block with its gate and residual scale (include/fused_norm.h), forward and backward.
//
// Bound by memory: every given tensor is read or written once.  A group of TPR lanes holds a row in registers, eight neighbouring elements to a lane
// and chunk (16 bytes of bf16), NCH chunks, so that the statistics cost no second read: the forward forms the mean square of y, then that of r'; the backward forms in one
// sum over the row all that t needs, and in a second one what dy needs.  Groups walk the rows with a grid stride and keep their weights and the sums of the
// weights' gradients in registers (long rows: the sums in LDS, see NormBack); the latter go to the workspace, one row of sums for each workgroup, and a second kernel adds those in a fixed order.
//
// Measured: 16384 rows of 4096, forward with a gate (671 MB) 130 us, 5.2 TB/s; 8191 of 8192, backward with float32 residuals (1.21 GB) 233 us, 5.2; 524288 of 128, backward (671 MB) 126 us, 5.3;
// 64 rows 9 us, which is the host's part.  Loose rows take an access for each element: 1.7 - 2.9 TB/s (16384 of 4095, backward, 231 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "../../include/fused_norm.h"
#include "kernels.hpp"
#include "operators.hpp"
#include "tiles.hpp"

namespace chunk_attn {
namespace {

struct NormArgs {
  int64_t rows;
  int cols, gate_kind, weight_is_f32;
  float eps, residual_scale, block_scale;
  const __bf16 *y, *gate;
  const void *residual, *post_weight, *pre_weight;
  int64_t y_stride, gate_stride, residual_stride;
  // forward: residual_out, h; backward: the stored residual_out is `residual`
  void* residual_out;
  __bf16* h;
  int64_t residual_out_stride, h_stride;
  const void* d_residual_out;
  const __bf16* d_h;
  int64_t d_residual_out_stride, d_h_stride;
  __bf16 *dy, *d_gate;
  void* d_residual;
  int64_t dy_stride, d_gate_stride, d_residual_stride;
  float *post_parts, *pre_parts;  // [workgroups][cols], or null
};

__device__ __forceinline__ float sigmoid_of(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
__device__ __forceinline__ float gate_of(float g, int kind) {
  if (kind == FUSED_NORM_GATE_PLAIN) return g;
  const float p = sigmoid_of(g);
  return kind == FUSED_NORM_GATE_SIGMOID ? p : g * p;
}
__device__ __forceinline__ void gate_and_slope(float g, int kind, float& act, float& slope) {
  if (kind == FUSED_NORM_GATE_PLAIN) {
    act = g;
    slope = 1.f;
    return;
  }
  // p = sigmoid(g) and q = sigmoid(-g), both from exp(-|g|): 1 - p has no digits left where the gate is wide open (none at all from g = 17 on)
  const float e = __expf(-fabsf(g)), larger = __builtin_amdgcn_rcpf(1.f + e), smaller = e * larger;
  const float p = g < 0.f ? smaller : larger, q = g < 0.f ? larger : smaller;
  act = kind == FUSED_NORM_GATE_SIGMOID ? p : g * p;
  slope = kind == FUSED_NORM_GATE_SIGMOID ? p * q : p * (1.f + g * q);
}

template <int TPR>
constexpr int norm_threads() { return TPR > 256 ? TPR : 256; }

// Rows as buffers: elements past a row's end, rows past the last and tensors that are not there read as zeros and are not written, by the hardware, so that no access is behind a branch.
//
// A thread's eight elements of a chunk are pieces of PIECE neighbours, which the threads of a row fetch next to each other: 8 (16 bytes of bf16), or 4 beside a float32 residual (16 bytes of that: with eight, a
// thread's two accesses would each leave half of a line to the other), of rows that consist of such pieces; a buffer then covers the rows that a workgroup has at a time.  1 (loose rows: of other lengths, strides or
// alignments): each element is fetched by itself, and a buffer covers one row.
//
// Calls whose tensors are larger than the last-level cache (256 MiB) pass their rows by the caches (STREAM); what fits is kept for who wrote it and who reads it next.  us, kept / streamed: 16384 rows of 4096,
// forward with a gate (671 MB) 137 / 129, backward with a gate (1.07 GB) 216 / 192; 524288 rows of 128, backward (671 MB) 137 / 124.  Loose rows are kept: streamed, a line would be fetched for each
// sixteen-bit access (16384 of 4095, backward, 231 / 281).
constexpr int64_t kStreamBytes = (int64_t)256 << 20;
constexpr int kNonTemporal = 2;             // the buffer instructions' nt bit
constexpr unsigned kNowhere = 0x7fffff00u;  // an offset past the end of every buffer
template <class T, int TPR, int PIECE>
struct Rows {
  static constexpr int kSize = sizeof(T), kTogether = PIECE == 1 ? 1 : norm_threads<TPR>() / TPR;
  const char* base;
  int64_t stride;  // bytes
  int row_bytes;
  unsigned at;     // the thread's first byte, from the first of a buffer's rows on
  __device__ __forceinline__ Rows(const void* p, int64_t elements, int cols)
      : base((const char*)p), stride(elements * kSize), row_bytes(cols * kSize),
        at((PIECE == 1 ? 0u : (unsigned)((int)threadIdx.x / TPR * (int)stride)) + (int)threadIdx.x % TPR * PIECE * kSize) {}
  // rows from `row0` on, the first that a workgroup has at a time
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(int64_t row0, int64_t rows) const {
    if constexpr (PIECE == 1) row0 += __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int n = (int)min(rows - row0, (int64_t)kTogether);
    const int bytes = base && n > 0 ? (n - 1) * (int)stride + row_bytes : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base) + (bytes ? row0 * stride : 0), 0, bytes, 0x00027000);
  }
  // the thread's piece i
  __device__ __forceinline__ unsigned piece(int i, int cols) const {
    return PIECE == 1 || (i * TPR + (int)threadIdx.x % TPR) * PIECE < cols ? at + i * TPR * PIECE * kSize : kNowhere;
  }
};
// Column of a thread's element e of chunk c.
template <int TPR, int PIECE>
__device__ __forceinline__ int column(int c, int e) {
  return (c * (8 / PIECE) + e / PIECE) * TPR * PIECE + (int)threadIdx.x % TPR * PIECE + e % PIECE;
}
template <class T, int TPR, int PIECE>
struct Chunk {
  static constexpr int kPieces = 8 / PIECE, kBytes = PIECE * sizeof(T);  // of a piece
  static_assert(kBytes == 16 || kBytes == 8 || kBytes == 4 || kBytes == 2);
  static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
  unsigned raw[kPieces * kWords];
  template <int AUX = 0>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, const Rows<T, TPR, PIECE>& r, int c, int cols) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const unsigned at = r.piece(c * kPieces + i, cols);
      unsigned* const x = raw + i * kWords;
      if constexpr (kBytes == 16) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, AUX);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = v[k];
      } else if constexpr (kBytes == 8) {
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, AUX);
        x[0] = v[0];
        x[1] = v[1];
      } else if constexpr (kBytes == 4) {
        x[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, AUX);
      } else {
        x[0] = (unsigned)__builtin_amdgcn_raw_buffer_load_b16(from, at, 0, AUX) << 16;
      }
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(T) == 4 || PIECE == 1) x[e] = __uint_as_float(raw[e]);
      else x[e] = __uint_as_float(e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
    }
  }
  template <int AUX>
  static __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t to, const Rows<T, TPR, PIECE>& r, int c, int cols, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const unsigned at = r.piece(c * kPieces + i, cols);
      const float* const y = x + i * PIECE;
      if constexpr (sizeof(T) == 4 && PIECE == 4) {
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])}, to, at, 0, AUX);
      } else if constexpr (sizeof(T) == 4) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y[0]), to, at, 0, AUX);
      } else if constexpr (PIECE == 8) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, pack8(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7])), to, at, 0, AUX);
      } else if constexpr (PIECE == 4) {
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, pack4(y[0], y[1], y[2], y[3])), to, at, 0, AUX);
      } else {
        __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (__bf16)y[0]), to, at, 0, AUX);
      }
    }
  }
};

// A weight's elements, zeros past the end and where there is none.
template <int TPR, int PIECE>
struct Weight {
  __amdgpu_buffer_rsrc_t buffer;
  bool f32;
  __device__ __forceinline__ Weight(const void* w, bool f32, int cols)
      : buffer(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(w), 0, w ? cols * (f32 ? 4 : 2) : 0, 0x00027000)), f32(f32) {}
  __device__ __forceinline__ void load(int c, float (&x)[8]) const {
    if constexpr (PIECE == 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = column<TPR, PIECE>(c, e);
        x[e] = __uint_as_float(f32 ? __builtin_amdgcn_raw_buffer_load_b32(buffer, at * 4, 0, 0) : (unsigned)__builtin_amdgcn_raw_buffer_load_b16(buffer, at * 2, 0, 0) << 16);
      }
    } else if (f32) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(buffer, column<TPR, PIECE>(c, e) * 4, 0, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[e + k] = __uint_as_float(v[k]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(buffer, column<TPR, PIECE>(c, e) * 2, 0, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[e + k] = __uint_as_float(k % 2 ? v[k / 2] & 0xffff0000u : v[k / 2] << 16);
      }
    }
  }
};

// Sums over the threads of each row; rows of several waves meet in LDS, in two places by turns.
template <int TPR, int N>
struct RowSums {
  float (*place)[N][norm_threads<TPR>() / 64];
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum<TPR < 64 ? TPR : 64>(x[i]);
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6, first = wave / (TPR / 64) * (TPR / 64);
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) place[turn][i][wave] = x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) x[i] += place[turn][i][first + w];
      }
      turn ^= 1;
    }
  }
};

template <int TPR, int NCH, class TR, int PIECE, bool STREAM>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_fwd_kernel(const NormArgs a) {
  __shared__ float sums[2][1][norm_threads<TPR>() / 64];
  constexpr int kGroups = norm_threads<TPR>() / TPR;
  constexpr int kAux = STREAM ? kNonTemporal : 0;
  using Bf = Chunk<__bf16, TPR, PIECE>;
  using Re = Chunk<TR, TPR, PIECE>;
  RowSums<TPR, 1> row_sums{sums};
  const float inv_cols = 1.f / (float)a.cols;
  const Rows<__bf16, TPR, PIECE> y(a.y, a.y_stride, a.cols), gate(a.gate, a.gate_stride, a.cols), h(a.h, a.h_stride, a.cols);
  const Rows<TR, TPR, PIECE> res(a.residual, a.residual_stride, a.cols), out(a.residual_out, a.residual_out_stride, a.cols);
  const Weight<TPR, PIECE> post_weight(a.post_weight, a.weight_is_f32, a.cols), pre_weight(a.pre_weight, a.weight_is_f32, a.cols);
  float post[NCH][8], pre[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    post_weight.load(c, post[c]);
    pre_weight.load(c, pre[c]);
  }
  Bf ny[NCH], ng[NCH];
  Re nr[NCH];
  auto load = [&](int64_t row0) {
    const auto by = y.buffer(row0, a.rows), bg = gate.buffer(row0, a.rows), br = res.buffer(row0, a.rows);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      ny[c].template load<kAux>(by, y, c, a.cols);
      ng[c].template load<kAux>(bg, gate, c, a.cols);
      nr[c].template load<kAux>(br, res, c, a.cols);
    }
  };
  const int64_t step = (int64_t)gridDim.x * kGroups;
  wait_all_but<0>();
  load((int64_t)blockIdx.x * kGroups);
  for (int64_t row0 = (int64_t)blockIdx.x * kGroups; row0 < a.rows; row0 += step) {
    float x[NCH][8];
    Bf g[NCH];
    Re r[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      ny[c].get(x[c]);
      g[c] = ng[c];
      r[c] = nr[c];
    }
    load(row0 + step);
    if (a.post_weight) {
      float s[1] = {0.f};
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += x[c][e] * x[c][e];
      row_sums(s);
      const float inv = rsqrtf(s[0] * inv_cols + a.eps);
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] *= inv * post[c][e];
    }
    float s[1] = {0.f};
    const auto bo = out.buffer(row0, a.rows);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float q[8];
      if (a.gate) {
        g[c].get(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] *= gate_of(q[e], a.gate_kind);
      }
      r[c].get(q);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[c][e] = a.block_scale * x[c][e] + a.residual_scale * q[e];
        s[0] += x[c][e] * x[c][e];
      }
      Re::template store<kAux>(bo, out, c, a.cols, x[c]);
    }
    if (a.pre_weight) {
      row_sums(s);
      const float inv = rsqrtf(s[0] * inv_cols + a.eps);
      const auto bh = h.buffer(row0, a.rows);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] *= inv * pre[c][e];
        Bf::template store<kAux>(bh, h, c, a.cols, x[c]);
      }
    }
  }
}

// How the backward of such rows runs, in 128 registers: four waves to a SIMD hide the loads of one row behind another's sums (next row's loads ahead of time took the registers of one of them: 524288 rows
// of 128, 136 / 139 us, 8191 of 8192 254 / 311).  Long rows keep the sums of the weights' gradients in LDS and read the weights again for every row (from the cache).
template <int TPR, int NCH>
struct NormBack {
  static constexpr bool kInLds = TPR * NCH >= 1024, kHeld = !kInLds;
  static constexpr int kGroups = norm_threads<TPR>() / TPR;
  // sums in LDS: of both weights while the rows run, or of one of them from each of the groups at the end
  static constexpr size_t smem = sizeof(float) * TPR * NCH * 8 * (kInLds ? 2 : kGroups > 1 ? kGroups : 0);
};
template <int TPR, int NCH, class TR, int PIECE, bool STREAM>
__global__ __launch_bounds__(norm_threads<TPR>(), 4) void norm_bwd_kernel(const NormArgs a) {
  constexpr int kAux = STREAM ? kNonTemporal : 0;
  using Bf = Chunk<__bf16, TPR, PIECE>;
  using Re = Chunk<TR, TPR, PIECE>;
  using How = NormBack<TPR, NCH>;
  constexpr int kGroups = How::kGroups, kRow = TPR * NCH * 8;
  extern __shared__ __attribute__((aligned(16))) float lds_sums[];
  __shared__ float sums3[2][3][norm_threads<TPR>() / 64], sums1[2][1][norm_threads<TPR>() / 64];
  RowSums<TPR, 3> row_sums3{sums3};
  RowSums<TPR, 1> row_sums1{sums1};
  const float inv_cols = 1.f / (float)a.cols;
  const bool has_post = a.post_weight != nullptr, has_pre = a.pre_weight != nullptr, has_gate = a.gate != nullptr;
  const Rows<__bf16, TPR, PIECE> y(a.y, a.y_stride, a.cols), gate(a.gate, a.gate_stride, a.cols), dh(a.d_h, a.d_h_stride, a.cols), dy(a.dy, a.dy_stride, a.cols),
      dg(a.d_gate, a.d_gate_stride, a.cols);
  const Rows<TR, TPR, PIECE> res(a.residual, a.residual_stride, a.cols), dout(a.d_residual_out, a.d_residual_out_stride, a.cols),
      dres(a.d_residual, a.d_residual_stride, a.cols);
  const Weight<TPR, PIECE> post_weight(a.post_weight, a.weight_is_f32, a.cols), pre_weight(a.pre_weight, a.weight_is_f32, a.cols);
  float post_held[NCH][8], pre_held[NCH][8], d_post[NCH][8], d_pre[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if (How::kHeld) {
      post_weight.load(c, post_held[c]);
      pre_weight.load(c, pre_held[c]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      d_post[c][e] = d_pre[c][e] = 0.f;
      if (How::kInLds) lds_sums[column<TPR, PIECE>(c, e)] = lds_sums[kRow + column<TPR, PIECE>(c, e)] = 0.f;
    }
  }
  Bf cy[NCH], cg[NCH], ch[NCH];
  Re cr[NCH], co[NCH];
  auto load = [&](int64_t row0) {
    const auto by = y.buffer(row0, a.rows), bg = gate.buffer(row0, a.rows), bh = dh.buffer(row0, a.rows), br = res.buffer(row0, a.rows), bo = dout.buffer(row0, a.rows);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      cr[c].template load<kAux>(br, res, c, a.cols);
      ch[c].template load<kAux>(bh, dh, c, a.cols);
      cy[c].template load<kAux>(by, y, c, a.cols);
      co[c].template load<kAux>(bo, dout, c, a.cols);
      cg[c].template load<kAux>(bg, gate, c, a.cols);
    }
  };
  const int64_t step = (int64_t)gridDim.x * kGroups;
  wait_all_but<0>();
  for (int64_t row0 = (int64_t)blockIdx.x * kGroups; row0 < a.rows; row0 += step) {
    load(row0);
    float s[3] = {0.f, 0.f, 0.f};  // y^2, r'^2, d_h w r'
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float p[8], q[8];
      if (has_post) {
        cy[c].get(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += p[e] * p[e];
      }
      if (has_pre) {
        if (!How::kHeld) pre_weight.load(c, pre_held[c]);
        cr[c].get(p);
        ch[c].get(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[1] += p[e] * p[e];
          s[2] += q[e] * pre_held[c][e] * p[e];
        }
      }
    }
    row_sums3(s);
    const float inv_r = rsqrtf(s[1] * inv_cols + a.eps), mean_r = s[2] * inv_cols * inv_r;  // the mean is that of d_h w x^
    const float inv_y = has_post ? rsqrtf(s[0] * inv_cols + a.eps) : 1.f;
    const auto bdr = dres.buffer(row0, a.rows), bdg = dg.buffer(row0, a.rows), bdy = dy.buffer(row0, a.rows);
    float u[NCH][8], s1[1] = {0.f};
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float p[8], q[8];
      co[c].get(u[c]);
      if (has_pre) {
        if (!How::kHeld) pre_weight.load(c, pre_held[c]);
        cr[c].get(p);
        ch[c].get(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = p[e] * inv_r;
          if (How::kInLds) lds_sums[kRow + column<TPR, PIECE>(c, e)] += q[e] * x;
          else d_pre[c][e] += q[e] * x;
          u[c][e] += inv_r * (q[e] * pre_held[c][e] - x * mean_r);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = a.residual_scale * u[c][e];
      Re::template store<kAux>(bdr, dres, c, a.cols, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[c][e] *= a.block_scale;
      cy[c].get(p);
      if (has_gate) {
        cg[c].get(q);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float act, slope;
          gate_and_slope(q[e], a.gate_kind, act, slope);
          o[e] = u[c][e] * slope * (p[e] * inv_y);
          u[c][e] *= act;
        }
        if (has_post) {
          if (!How::kHeld) post_weight.load(c, post_held[c]);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] *= post_held[c][e];
        }
        Bf::template store<kAux>(bdg, dg, c, a.cols, o);
      }
      if (has_post) {
        if (!How::kHeld) post_weight.load(c, post_held[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = p[e] * inv_y;
          if (How::kInLds) lds_sums[column<TPR, PIECE>(c, e)] += u[c][e] * x;
          else d_post[c][e] += u[c][e] * x;
          u[c][e] *= post_held[c][e];
          s1[0] += u[c][e] * x;
        }
      }
    }
    if (has_post) {
      row_sums1(s1);
      const float mean = s1[0] * inv_cols;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float p[8];
        cy[c].get(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[c][e] = inv_y * (u[c][e] - p[e] * inv_y * mean);
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) Bf::template store<kAux>(bdy, dy, c, a.cols, u[c]);
  }
  // the workgroup's row of sums; several groups add theirs up in LDS, in order
  for (int k = 0; k < 2; ++k) {
    float* const to = k ? a.pre_parts : a.post_parts;
    if (!to) continue;
    if constexpr (kGroups > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) lds_sums[threadIdx.x / TPR * kRow + column<TPR, PIECE>(c, e)] = k ? d_pre[c][e] : d_post[c][e];
      __syncthreads();
      for (int i = threadIdx.x; i < a.cols; i += norm_threads<TPR>()) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) sum += lds_sums[j * kRow + i];
        to[(int64_t)blockIdx.x * a.cols + i] = sum;
      }
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = column<TPR, PIECE>(c, e);
          if (i < a.cols) to[(int64_t)blockIdx.x * a.cols + i] = How::kInLds ? lds_sums[k * kRow + i] : k ? d_pre[c][e] : d_post[c][e];
        }
    }
  }
}

// Adds up the workgroups' sums of one weight's gradient: 64 columns to a workgroup, whose sixteen waves take every sixteenth row, eight rows at a time.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* post_parts, const float* pre_parts, int parts, int cols, float* d_post, float* d_pre,
                                                            int accumulate) {
  const float* const from = blockIdx.y ? pre_parts : post_parts;
  float* const to = blockIdx.y ? d_pre : d_post;
  if (!to) return;
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (col < cols) {
    int p = wave;
    for (; p + 7 * 16 < parts; p += 8 * 16) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = from[(int64_t)(p + 16 * i) * cols + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    for (; p < parts; p += 16) sum += from[(int64_t)p * cols + col];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < cols) {
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += sums[w][lane];
    to[col] = accumulate ? to[col] + sum : sum;
  }
}

// Threads and chunks of a row by its length: eight elements to a thread while a row fits a workgroup.  A loose row takes a wave at least.
template <bool BACK, class F>
auto by_cols(int cols, bool loose, bool f32, bool stream, F&& f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  auto with_piece = [&](auto tpr, auto nch, auto piece) {
    return !stream ? f(tpr, nch, piece, std::false_type{}) : f(tpr, nch, piece, std::true_type{});
  };
  auto whole = [&](auto tpr, auto nch) { return f32 ? with_piece(tpr, nch, integral_constant<int, 4>{}) : with_piece(tpr, nch, integral_constant<int, 8>{}); };
  auto either = [&](auto tpr, auto nch) { return loose ? f(tpr, nch, one, std::false_type{}) : whole(tpr, nch); };
  if (cols <= 256 && !loose) return cols <= 128 ? whole(integral_constant<int, 16>{}, one) : whole(integral_constant<int, 32>{}, one);
  if (cols <= 512) return either(integral_constant<int, 64>{}, one);
  if (cols <= 1024) return either(integral_constant<int, 128>{}, one);
  if (cols <= 2048) return either(integral_constant<int, 256>{}, one);
  if (cols <= 4096) return either(integral_constant<int, 512>{}, one);
  const integral_constant<int, 2> two;
  if constexpr (BACK) {  // (two workgroups to a compute unit: 8191 rows of 8192 with float32 residuals 247 -> 236 us)
    if (cols <= 8192) return either(integral_constant<int, 512>{}, two);
  } else {
    if (cols <= 8192) return either(integral_constant<int, 1024>{}, one);
  }
  return either(integral_constant<int, 1024>{}, two);
}
// Workgroups of the backward, each of which leaves a row of sums.
int64_t norm_workgroups(int64_t rows, int cols, bool loose) {
  return by_cols<true>(cols, loose, false, false, [&](auto tpr, auto, auto, auto) -> int64_t {
    constexpr int kTpr = decltype(tpr)::value, kGroups = norm_threads<kTpr>() / kTpr;
    return std::min<int64_t>((rows + kGroups - 1) / kGroups, kTpr > 512 ? kCus : kTpr > 256 ? 2 * kCus : 4 * kCus);
  });
}
int64_t most_workgroups(int64_t rows, int cols) { return std::max(norm_workgroups(rows, cols, false), norm_workgroups(rows, cols, true)); }

struct RowTensor {
  const void* p;
  int64_t stride;
  bool f32;
};
// Whether rows of some tensor do not consist of whole 16-byte pieces, or are too far apart for a buffer of several.
bool any_loose(int cols, std::initializer_list<RowTensor> tensors) {
  if (cols % 8 != 0) return true;
  for (const RowTensor& t : tensors)
    if (t.p && (((uintptr_t)t.p & 15) != 0 || t.stride % (t.f32 ? 4 : 8) != 0 || t.stride >= (1 << 24))) return true;
  return false;
}

bool row_tensor_ok(const void* p, int64_t stride, int cols, bool f32) { return !p || (stride >= cols && ((uintptr_t)p & (f32 ? 3 : 1)) == 0); }

// Bytes of one row of the tensors that are there.
int64_t row_bytes(std::initializer_list<const void*> bf16s, std::initializer_list<const void*> residuals, bool f32, int cols) {
  int64_t n = 0;
  for (const void* p : bf16s) n += p ? 2 : 0;
  for (const void* p : residuals) n += p ? (f32 ? 4 : 2) : 0;
  return n * cols;
}

int check(const fused_norm_desc* d) {
  if (!d || d->rows < 0 || d->cols < 1) return CHUNK_ATTN_INVALID_ARG;
  if (d->cols > FUSED_NORM_MAX_COLS) return CHUNK_ATTN_UNSUPPORTED;
  if (!finite_number(d->eps) || d->eps <= 0.f || !finite_number(d->residual_scale) || !finite_number(d->block_scale)) return CHUNK_ATTN_INVALID_ARG;
  if (d->gate && (d->gate_kind < FUSED_NORM_GATE_PLAIN || d->gate_kind > FUSED_NORM_GATE_SILU)) return CHUNK_ATTN_INVALID_ARG;
  if ((d->gate || d->post_weight) && !d->y && d->rows > 0) return CHUNK_ATTN_INVALID_ARG;  // (nothing to gate or to norm)
  const uintptr_t w = d->weight_is_f32 ? 3 : 1;
  if (((uintptr_t)d->post_weight & w) != 0 || ((uintptr_t)d->pre_weight & w) != 0) return CHUNK_ATTN_INVALID_ARG;
  if (!row_tensor_ok(d->y, d->y_stride, d->cols, false) || !row_tensor_ok(d->gate, d->gate_stride, d->cols, false) ||
      !row_tensor_ok(d->residual, d->residual_stride, d->cols, d->residual_is_f32))
    return CHUNK_ATTN_INVALID_ARG;
  return CHUNK_ATTN_OK;
}

template <int TPR, int NCH, class TR, int PIECE, bool STREAM>
hipError_t launch_norm_bwd(const NormArgs& a, int64_t workgroups, hipStream_t stream) {
  constexpr size_t smem = NormBack<TPR, NCH>::smem;
  if constexpr (smem > (48 << 10)) {
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&norm_bwd_kernel<TPR, NCH, TR, PIECE, STREAM>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (attr != hipSuccess) return attr;
  }
  hipLaunchKernelGGL((norm_bwd_kernel<TPR, NCH, TR, PIECE, STREAM>), dim3((unsigned)workgroups), dim3(norm_threads<TPR>()), smem, stream, a);
  return hipGetLastError();
}

NormArgs common_args(const fused_norm_desc* d) {
  NormArgs a{};
  a.rows = d->rows;
  a.cols = d->cols;
  a.gate_kind = d->gate_kind;
  a.weight_is_f32 = d->weight_is_f32 != 0;
  a.eps = d->eps;
  a.residual_scale = d->residual_scale;
  a.block_scale = d->block_scale;
  a.y = (const __bf16*)d->y;
  a.gate = (const __bf16*)d->gate;
  a.y_stride = d->y_stride;
  a.gate_stride = d->gate_stride;
  a.post_weight = d->post_weight;
  a.pre_weight = d->pre_weight;
  return a;
}

}  // namespace
}  // namespace chunk_attn

extern "C" int fused_norm_fwd(const fused_norm_desc* d, void* residual_out, int64_t residual_out_stride, void* h, int64_t h_stride, void* hip_stream) {
  using namespace chunk_attn;
  const int rc = check(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (d->rows == 0) return CHUNK_ATTN_OK;  // (the pointers of empty buffers may be null)
  if ((!d->y && !d->residual) || !h != !d->pre_weight || (!h && !residual_out)) return CHUNK_ATTN_INVALID_ARG;
  if (!row_tensor_ok(residual_out, residual_out_stride, d->cols, d->residual_is_f32) || !row_tensor_ok(h, h_stride, d->cols, false)) return CHUNK_ATTN_INVALID_ARG;
  NormArgs a = common_args(d);
  a.residual = d->residual;
  a.residual_stride = d->residual_stride;
  a.residual_out = residual_out;
  a.residual_out_stride = residual_out_stride;
  a.h = (__bf16*)h;
  a.h_stride = h_stride;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool f32 = d->residual_is_f32;
  const bool loose = any_loose(d->cols, {{d->y, d->y_stride, false}, {d->gate, d->gate_stride, false}, {h, h_stride, false}, {d->residual, d->residual_stride, f32}, {residual_out, residual_out_stride, f32}});
  const bool stream_by = row_bytes({d->y, d->gate, h}, {d->residual, residual_out}, f32, d->cols) * d->rows > kStreamBytes;
  by_cols<false>(d->cols, loose, f32, stream_by, [&](auto tpr, auto nch, auto piece, auto stream_c) {
    constexpr int kTpr = decltype(tpr)::value, kNch = decltype(nch)::value, kGroups = norm_threads<kTpr>() / kTpr;
    constexpr int kPiece = decltype(piece)::value;
    constexpr bool kStream = decltype(stream_c)::value;
    const dim3 grid((unsigned)std::min<int64_t>((d->rows + kGroups - 1) / kGroups, kTpr > 512 ? 2 * kCus : kTpr > 256 ? 4 * kCus : 8 * kCus)), block(norm_threads<kTpr>());
    auto launch = [&](auto type) { hipLaunchKernelGGL((norm_fwd_kernel<kTpr, kNch, decltype(type), kPiece, kStream>), grid, block, 0, stream, a); };
    if constexpr (kPiece == 4) launch(0.f);
    else if constexpr (kPiece == 8) launch((__bf16)0.f);
    else if (f32) launch(0.f);
    else launch((__bf16)0.f);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "norm forward");
}

extern "C" int fused_norm_bwd_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes) {
  using namespace chunk_attn;
  if (!bytes || rows < 0 || cols < 1) return CHUNK_ATTN_INVALID_ARG;
  if (cols > FUSED_NORM_MAX_COLS) return CHUNK_ATTN_UNSUPPORTED;
  *bytes = (size_t)(2 * most_workgroups(rows, cols) * cols) * sizeof(float);
  return CHUNK_ATTN_OK;
}

extern "C" int fused_norm_bwd(const fused_norm_desc* d, const void* residual_out, int64_t residual_out_stride, const void* d_residual_out,
                              int64_t d_residual_out_stride, const void* d_h, int64_t d_h_stride, void* dy, int64_t dy_stride, void* d_gate, int64_t d_gate_stride,
                              void* d_residual, int64_t d_residual_stride, float* d_post_weight, float* d_pre_weight, int32_t accumulate_weights, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  using namespace chunk_attn;
  const int rc = check(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if ((d_post_weight && !d->post_weight) || (d_pre_weight && !d->pre_weight) || ((uintptr_t)d_post_weight & 3) != 0 || ((uintptr_t)d_pre_weight & 3) != 0)
    return CHUNK_ATTN_INVALID_ARG;
  const bool f32 = d->residual_is_f32;
  if (d->rows > 0) {
    if (!d_h != !d->pre_weight || (d->pre_weight && !residual_out) || (!d_h && !d_residual_out)) return CHUNK_ATTN_INVALID_ARG;
    if ((dy && !d->y) || (d_gate && !d->gate)) return CHUNK_ATTN_INVALID_ARG;
    if (!row_tensor_ok(residual_out, residual_out_stride, d->cols, f32) || !row_tensor_ok(d_residual_out, d_residual_out_stride, d->cols, f32) ||
        !row_tensor_ok(d_h, d_h_stride, d->cols, false) || !row_tensor_ok(dy, dy_stride, d->cols, false) || !row_tensor_ok(d_gate, d_gate_stride, d->cols, false) ||
        !row_tensor_ok(d_residual, d_residual_stride, d->cols, f32))
      return CHUNK_ATTN_INVALID_ARG;
  }
  const bool loose = any_loose(d->cols, {{d->y, d->y_stride, false}, {d->gate, d->gate_stride, false}, {d_h, d_h_stride, false}, {dy, dy_stride, false}, {d_gate, d_gate_stride, false},
                                         {residual_out, residual_out_stride, f32}, {d_residual_out, d_residual_out_stride, f32}, {d_residual, d_residual_stride, f32}});
  const int64_t groups = norm_workgroups(d->rows, d->cols, loose);
  if ((d_post_weight || d_pre_weight) && d->rows > 0) {
    if (!workspace || ((uintptr_t)workspace & 15) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < (size_t)(2 * most_workgroups(d->rows, d->cols) * d->cols) * sizeof(float)) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  const hipStream_t stream = (hipStream_t)hip_stream;
  NormArgs a = common_args(d);
  hipError_t e = hipSuccess;
  if (d_post_weight) a.post_parts = (float*)workspace;
  if (d_pre_weight) a.pre_parts = (float*)workspace + groups * d->cols;
  if (d->rows > 0) {
    a.residual = d->pre_weight ? residual_out : nullptr;  // (else not wanted)
    a.residual_stride = residual_out_stride;
    a.d_residual_out = d_residual_out;
    a.d_residual_out_stride = d_residual_out_stride;
    a.d_h = (const __bf16*)d_h;
    a.d_h_stride = d_h_stride;
    a.dy = (__bf16*)dy;
    a.dy_stride = dy_stride;
    a.d_gate = (__bf16*)d_gate;
    a.d_gate_stride = d_gate_stride;
    a.d_residual = d_residual;
    a.d_residual_stride = d_residual_stride;
    const bool stream_by = row_bytes({d->y, d->gate, d_h, dy, d_gate}, {d->pre_weight ? residual_out : nullptr, d_residual_out, d_residual}, f32, d->cols) * d->rows > kStreamBytes;
    e = by_cols<true>(d->cols, loose, f32, stream_by, [&](auto tpr, auto nch, auto piece, auto stream_c) {
      constexpr int kTpr = decltype(tpr)::value, kNch = decltype(nch)::value;
      constexpr int kPiece = decltype(piece)::value;
      constexpr bool kStream = decltype(stream_c)::value;
      if constexpr (kPiece == 4) return launch_norm_bwd<kTpr, kNch, float, 4, kStream>(a, groups, stream);
      else if constexpr (kPiece == 8) return launch_norm_bwd<kTpr, kNch, __bf16, 8, kStream>(a, groups, stream);
      else return f32 ? launch_norm_bwd<kTpr, kNch, float, 1, false>(a, groups, stream) : launch_norm_bwd<kTpr, kNch, __bf16, 1, false>(a, groups, stream);
    });
    if (e != hipSuccess) return report_hip(e, "norm backward");
  }
  if (d_post_weight || d_pre_weight) {
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((d->cols + 63) / 64), 2), dim3(1024), 0, stream, a.post_parts, a.pre_parts, (int)groups, d->cols,
                       d_post_weight, d_pre_weight, accumulate_weights != 0);
    if ((e = hipGetLastError()) != hipSuccess) return report_hip(e, "norm backward, weights");
  }
  return CHUNK_ATTN_OK;
}
