// Norms around a block with its gate and residual scale (include/fused_norm.h), forward and backward.
//
// Bound by memory: every given tensor is read or written once.  A group of TPR lanes holds a row in registers, eight neighbouring elements to a lane
// and chunk (16 bytes of bf16), NCH chunks, so that the statistics cost no second read: the forward forms the mean square of y, then that of r'; the backward forms in one
// sum over the row all that t needs, and in a second one what dy needs.  Groups walk the rows with a grid stride and keep their weights and the sums of the
// weights' gradients in registers; the latter go to the workspace, one row of sums for each workgroup, and a second kernel adds those in a fixed order.
#include <hip/hip_runtime.h>

#include "../../include/fused_norm.h"
#include "kernels.hpp"
#include "operators.hpp"

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
  const float p = sigmoid_of(g);
  act = kind == FUSED_NORM_GATE_SIGMOID ? p : g * p;
  slope = kind == FUSED_NORM_GATE_SIGMOID ? p * (1.f - p) : p * (1.f + g * (1.f - p));
}

// Sum over the TPR threads of a row.  A group of several waves goes through LDS, by turns in two places: a place is written again only after the
// barrier of the sum between, when everyone has read it.
template <int TPR, int N>
struct RowSum {
  float (*place)[N][TPR / 64 > 0 ? TPR / 64 : 1];
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum<TPR < 64 ? TPR : 64>(x[i]);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) place[turn][i][threadIdx.x >> 6] = x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) x[i] += place[turn][i][w];
      }
      turn ^= 1;
    }
  }
};

__device__ __forceinline__ void load_weight(const void* w, int is_f32, int at, int n, float* x) {
  if (is_f32) load_up_to_8((const float*)w + at, n, x);
  else load_up_to_8((const __bf16*)w + at, n, x);
}

template <int TPR>
constexpr int norm_threads() { return TPR > 256 ? TPR : 256; }

template <int TPR, int NCH, class TR>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_fwd_kernel(const NormArgs a) {
  __shared__ float sums[2][1][TPR / 64 > 0 ? TPR / 64 : 1];
  constexpr int kGroups = norm_threads<TPR>() / TPR;
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  RowSum<TPR, 1> row_sum{sums};
  const float inv_cols = 1.f / (float)a.cols;
  float post[NCH][8], pre[NCH][8];
  int count[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int at = (c * TPR + t) * 8;
    count[c] = max(0, min(8, a.cols - at));
    if (a.post_weight) load_weight(a.post_weight, a.weight_is_f32, at, count[c], post[c]);
    if (a.pre_weight) load_weight(a.pre_weight, a.weight_is_f32, at, count[c], pre[c]);
  }
  for (int64_t row0 = (int64_t)blockIdx.x * kGroups; row0 < a.rows; row0 += (int64_t)gridDim.x * kGroups) {
    const int64_t row = row0 + group;
    if (kGroups > 1 && row >= a.rows) return;  // (no barrier among groups)
    float x[NCH][8], r[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * TPR + t) * 8;
      if (a.y) load_up_to_8(a.y + row * a.y_stride + at, count[c], x[c]);
      if (a.residual) load_up_to_8((const TR*)a.residual + row * a.residual_stride + at, count[c], r[c]);
    }
    if (a.y) {
      float g[NCH][8];
      if (a.gate) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) load_up_to_8(a.gate + row * a.gate_stride + (c * TPR + t) * 8, count[c], g[c]);
      }
      if (a.post_weight) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[0] += x[c][e] * x[c][e];
        row_sum(s);
        const float inv = rsqrtf(s[0] * inv_cols + a.eps);
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[c][e] *= inv * post[c][e];
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[c][e] *= a.gate ? a.block_scale * gate_of(g[c][e], a.gate_kind) : a.block_scale;
          if (a.residual) x[c][e] += a.residual_scale * r[c][e];
        }
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = a.residual_scale * r[c][e];
    }
    if (a.residual_out) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
        store_up_to_8((TR*)a.residual_out + row * a.residual_out_stride + (c * TPR + t) * 8, count[c], x[c]);
    }
    if (a.pre_weight) {
      float s[1] = {0.f};
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += x[c][e] * x[c][e];
      row_sum(s);
      const float inv = rsqrtf(s[0] * inv_cols + a.eps);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] *= inv * pre[c][e];
        store_up_to_8(a.h + row * a.h_stride + (c * TPR + t) * 8, count[c], x[c]);
      }
    }
  }
}

template <int TPR, int NCH, class TR>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_bwd_kernel(const NormArgs a) {
  constexpr int kGroups = norm_threads<TPR>() / TPR;
  __shared__ float sums3[2][3][TPR / 64 > 0 ? TPR / 64 : 1];
  __shared__ float sums1[2][1][TPR / 64 > 0 ? TPR / 64 : 1];
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  RowSum<TPR, 3> row_sum3{sums3};
  RowSum<TPR, 1> row_sum1{sums1};
  const float inv_cols = 1.f / (float)a.cols;
  float post[NCH][8], pre[NCH][8], d_post[NCH][8], d_pre[NCH][8];
  int count[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int at = (c * TPR + t) * 8;
    count[c] = max(0, min(8, a.cols - at));
    if (a.post_weight) load_weight(a.post_weight, a.weight_is_f32, at, count[c], post[c]);
    if (a.pre_weight) load_weight(a.pre_weight, a.weight_is_f32, at, count[c], pre[c]);
#pragma unroll
    for (int e = 0; e < 8; ++e) d_post[c][e] = d_pre[c][e] = 0.f;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * kGroups; row0 < a.rows; row0 += (int64_t)gridDim.x * kGroups) {
    const int64_t row = row0 + group;
    if (kGroups > 1 && row >= a.rows) break;
    float y[NCH][8], r[NCH][8], dh[NCH][8], u[NCH][8], g[NCH][8];
    float s[3] = {0.f, 0.f, 0.f};  // y^2, r'^2, d_h w r'
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * TPR + t) * 8, n = count[c];
      if (a.y) load_up_to_8(a.y + row * a.y_stride + at, n, y[c]);
      if (a.gate) load_up_to_8(a.gate + row * a.gate_stride + at, n, g[c]);
      if (a.pre_weight) {
        load_up_to_8((const TR*)a.residual + row * a.residual_stride + at, n, r[c]);
        load_up_to_8(a.d_h + row * a.d_h_stride + at, n, dh[c]);
      }
      if (a.d_residual_out) load_up_to_8((const TR*)a.d_residual_out + row * a.d_residual_out_stride + at, n, u[c]);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[c][e] = 0.f;
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (a.post_weight) s[0] += y[c][e] * y[c][e];
        if (a.pre_weight) {
          s[1] += r[c][e] * r[c][e];
          s[2] += dh[c][e] * pre[c][e] * r[c][e];
        }
      }
    row_sum3(s);
    if (a.pre_weight) {
      const float inv = rsqrtf(s[1] * inv_cols + a.eps), mean = s[2] * inv_cols * inv;  // mean of d_h w x^
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = r[c][e] * inv;
          d_pre[c][e] += dh[c][e] * x;
          u[c][e] += inv * (dh[c][e] * pre[c][e] - x * mean);
        }
    }
    if (a.d_residual) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = a.residual_scale * u[c][e];
        store_up_to_8((TR*)a.d_residual + row * a.d_residual_stride + (c * TPR + t) * 8, count[c], o);
      }
    }
    if (!a.y) continue;
    const float inv = a.post_weight ? rsqrtf(s[0] * inv_cols + a.eps) : 1.f;
    float s1[1] = {0.f};
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[c][e] *= inv;
        u[c][e] *= a.block_scale;
        if (a.gate) {
          float act, slope;
          gate_and_slope(g[c][e], a.gate_kind, act, slope);
          o[e] = u[c][e] * slope * (a.post_weight ? y[c][e] * post[c][e] : y[c][e]);
          u[c][e] *= act;
        }
        if (a.post_weight) {
          d_post[c][e] += u[c][e] * y[c][e];
          u[c][e] *= post[c][e];
          s1[0] += u[c][e] * y[c][e];
        }
      }
      if (a.d_gate) store_up_to_8(a.d_gate + row * a.d_gate_stride + (c * TPR + t) * 8, count[c], o);
    }
    if (a.post_weight) {
      row_sum1(s1);
      const float mean = s1[0] * inv_cols;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) u[c][e] = inv * (u[c][e] - y[c][e] * mean);
    }
    if (a.dy) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) store_up_to_8(a.dy + row * a.dy_stride + (c * TPR + t) * 8, count[c], u[c]);
    }
  }
  // the workgroup's row of sums; several groups add theirs up in LDS, in order
  __shared__ float all[kGroups > 1 ? kGroups : 1][kGroups > 1 ? TPR * NCH * 8 : 1];
  for (int k = 0; k < 2; ++k) {
    float* const to = k ? a.pre_parts : a.post_parts;
    if (!to) continue;
    if constexpr (kGroups > 1) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) all[group][(c * TPR + t) * 8 + e] = k ? d_pre[c][e] : d_post[c][e];
      __syncthreads();
      for (int i = threadIdx.x; i < a.cols; i += norm_threads<TPR>()) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) sum += all[j][i];
        to[(int64_t)blockIdx.x * a.cols + i] = sum;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c) store_up_to_8(to + (int64_t)blockIdx.x * a.cols + (c * TPR + t) * 8, count[c], k ? d_pre[c] : d_post[c]);
    }
  }
}

// Adds up the workgroups' sums of one weight's gradient: 64 columns to a workgroup, four waves take every fourth row.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* post_parts, const float* pre_parts, int parts, int cols, float* d_post, float* d_pre,
                                                           int accumulate) {
  const float* const from = blockIdx.y ? pre_parts : post_parts;
  float* const to = blockIdx.y ? d_pre : d_post;
  if (!to) return;
  __shared__ float quarter[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (col < cols)
    for (int p = wave; p < parts; p += 4) sum += from[(int64_t)p * cols + col];
  quarter[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < cols) {
    sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
    to[col] = accumulate ? to[col] + sum : sum;
  }
}

// Threads and chunks of a row by its length.
template <class F>
auto by_cols(int cols, F&& f) {
  using std::integral_constant;
  if (cols <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (cols <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (cols <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (cols <= 1024) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (cols <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (cols <= 4096) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (cols <= 8192) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

int64_t norm_workgroups(int64_t rows, int cols) {
  return by_cols(cols, [&](auto tpr, auto) -> int64_t {
    constexpr int kTpr = decltype(tpr)::value, kGroups = norm_threads<kTpr>() / kTpr;
    return std::min<int64_t>((rows + kGroups - 1) / kGroups, kTpr > 256 ? 2 * kCus : 4 * kCus);
  });
}

bool row_tensor_ok(const void* p, int64_t stride, int cols, bool f32) { return !p || (stride >= cols && ((uintptr_t)p & (f32 ? 3 : 1)) == 0); }

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
  by_cols(d->cols, [&](auto tpr, auto nch) {
    constexpr int kTpr = decltype(tpr)::value, kNch = decltype(nch)::value, kGroups = norm_threads<kTpr>() / kTpr;
    const dim3 grid((unsigned)std::min<int64_t>((d->rows + kGroups - 1) / kGroups, 8 * kCus)), block(norm_threads<kTpr>());
    if (d->residual_is_f32) hipLaunchKernelGGL((norm_fwd_kernel<kTpr, kNch, float>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((norm_fwd_kernel<kTpr, kNch, __bf16>), grid, block, 0, stream, a);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "norm forward");
}

extern "C" int fused_norm_bwd_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes) {
  using namespace chunk_attn;
  if (!bytes || rows < 0 || cols < 1) return CHUNK_ATTN_INVALID_ARG;
  if (cols > FUSED_NORM_MAX_COLS) return CHUNK_ATTN_UNSUPPORTED;
  *bytes = (size_t)(2 * norm_workgroups(rows, cols) * cols) * sizeof(float);
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
  const int64_t groups = norm_workgroups(d->rows, d->cols);
  if ((d_post_weight || d_pre_weight) && d->rows > 0) {
    if (!workspace || ((uintptr_t)workspace & 15) != 0) return CHUNK_ATTN_INVALID_ARG;
    if (workspace_bytes < (size_t)(2 * groups * d->cols) * sizeof(float)) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  }
  const hipStream_t stream = (hipStream_t)hip_stream;
  NormArgs a = common_args(d);
  hipError_t e = hipSuccess;
  if (d_post_weight) a.post_parts = (float*)workspace;
  if (d_pre_weight) a.pre_parts = (float*)workspace + groups * d->cols;
  if (d->rows > 0) {
    a.residual = residual_out;
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
    by_cols(d->cols, [&](auto tpr, auto nch) {
      constexpr int kTpr = decltype(tpr)::value, kNch = decltype(nch)::value;
      const dim3 grid((unsigned)groups), block(norm_threads<kTpr>());
      if (f32) hipLaunchKernelGGL((norm_bwd_kernel<kTpr, kNch, float>), grid, block, 0, stream, a);
      else hipLaunchKernelGGL((norm_bwd_kernel<kTpr, kNch, __bf16>), grid, block, 0, stream, a);
    });
    if ((e = hipGetLastError()) != hipSuccess) return report_hip(e, "norm backward");
  }
  if (d_post_weight || d_pre_weight) {
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((d->cols + 63) / 64), 2), dim3(256), 0, stream, a.post_parts, a.pre_parts, (int)groups, d->cols,
                       d_post_weight, d_pre_weight, accumulate_weights != 0);
    if ((e = hipGetLastError()) != hipSuccess) return report_hip(e, "norm backward, weights");
  }
  return CHUNK_ATTN_OK;
}
