// Verification of drafted tokens (include/draft_verify.h).
//
// Bound by memory: one row of the target's probabilities, and one of the draft's where a token is rejected, of each request.  The sum of weights has to be known before the place
// can be found where the running sum passes a share of it, so: sums_kernel finds the row and leaves the sum of every kGranule weights, taken by one wave; choose_kernel sums these up, finds the granule
// and reads it again.  float64 throughout: products of two float32 and differences that matter are exact, and sums of 10^5 weights are off by 10^-15 of them or so.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/draft_verify.h"
#include "kernels.hpp"
#include "operators.hpp"

namespace chunk_attn {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRun = 64 * 8, kGranule = 2 * kRun;  // a wave takes eight neighbouring weights to a lane

template <class T>
struct VerifyArgs {
  const T *target, *draft;
  int64_t target_stride, draft_stride;
  const int32_t *tokens, *count;
  const float *uniforms, *last_uniform;
  int32_t *accepted, *rejected, *out;
  double* sums;  // [batch][granules]
  int32_t max_drafts, vocab, granules, each, groups;  // granules to a wave; workgroups to a request
};

__device__ __forceinline__ double weight_of(double x) { return x > 0.0 && x <= 1.7976931348623157e308 ? x : 0.0; }

// The row that the last token is drawn from.
template <class T>
struct Weights {
  const T *p, *q;  // q: null if all is drawn from p
  int without;     // a token that weighs nothing, or -1
  int vocab;
  // Weights first .. first + 7 (behind the vocabulary: zeros).
  __device__ void load(int first, double* w) const {
    float x[8], y[8];
    const int n = vocab - first;
    load_up_to_8(p + first, n, x);
    if (q) load_up_to_8(q + first, n, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = weight_of(q ? (double)x[e] - (double)y[e] : (double)x[e]);
      if (q && !(fabsf(x[e]) <= 3.402823466e38f && fabsf(y[e]) <= 3.402823466e38f)) w[e] = 0.0;
      if (first + e == without) w[e] = 0.0;
    }
  }
};
template <class T>
__device__ __forceinline__ int count_of(const VerifyArgs<T>& a, int r) {
  return a.count ? min(max(a.count[r], 0), a.max_drafts) : a.max_drafts;
}
// `kept`: tokens kept; residual: drawn from what the draft leaves.
template <class T>
__device__ __forceinline__ Weights<T> weights_of(const VerifyArgs<T>& a, int r, int kept, bool residual) {
  Weights<T> w{a.target + ((int64_t)r * (a.max_drafts + 1) + kept) * a.target_stride, nullptr, -1, a.vocab};
  if (residual) {
    if (a.draft) w.q = a.draft + ((int64_t)r * a.max_drafts + kept) * a.draft_stride;
    else w.without = a.tokens[(int64_t)r * a.max_drafts + kept];
  }
  return w;
}

__device__ __forceinline__ double wave_total(double x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ double wave_up_to(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

template <class T>
__global__ __launch_bounds__(kThreads) void sums_kernel(const VerifyArgs<T> a) {
  __shared__ int kept_by_all;
  const int r = blockIdx.x / a.groups, group = blockIdx.x % a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = count_of(a, r);
  if (wave == 0) {
    bool stands = false;
    if (lane < count) {
      const int64_t at = (int64_t)r * a.max_drafts + lane;
      const int d = a.tokens[at];
      if (d >= 0 && d < a.vocab) {
        const float p = (float)a.target[((int64_t)r * (a.max_drafts + 1) + lane) * a.target_stride + d], q = a.draft ? (float)a.draft[at * a.draft_stride + d] : 1.f;
        stands = fabsf(p) <= 3.402823466e38f && fabsf(q) <= 3.402823466e38f && (double)a.uniforms[at] * (double)q < (double)p;
      }
    }
    const unsigned long long falls = ~__ballot(stands);
    if (lane == 0) {
      const int kept = falls == 0 ? 64 : __ffsll((long long)falls) - 1;
      kept_by_all = kept;
      if (group == 0) {
        a.accepted[r] = kept;
        if (a.rejected) a.rejected[r] = count - kept;
      }
    }
  }
  __syncthreads();
  const int kept = kept_by_all;
  const Weights<T> weights = weights_of(a, r, kept, kept < count);
  const int first = (group * kWaves + wave) * a.each;
  for (int g = first; g < min(first + a.each, a.granules); ++g) {
    double sum = 0.0;
#pragma unroll
    for (int n = 0; n < kGranule / kRun; ++n) {
      double w[8];
      weights.load(g * kGranule + n * kRun + lane * 8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += w[e];
    }
    sum = wave_total(sum);
    if (lane == 0) a.sums[(int64_t)r * a.granules + g] = sum;
  }
}

// One workgroup to a request.
template <class T>
__global__ __launch_bounds__(kThreads) void choose_kernel(const VerifyArgs<T> a) {
  __shared__ double room[kWaves];
  __shared__ int chosen, highest;
  __shared__ double before_chosen;
  const int r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = count_of(a, r), kept = a.accepted[r];
  double* const sums = a.sums + (int64_t)r * a.granules;
  const int each = (a.granules + kThreads - 1) / kThreads, first = min((int)threadIdx.x * each, a.granules), last = min(first + each, a.granules);
  Weights<T> weights = weights_of(a, r, kept, kept < count);
  double total = 0.0, before = 0.0;
  for (int again = 0;; ++again) {
    double mine = 0.0;
    for (int g = first; g < last; ++g) mine += sums[g];
    const double up_to = wave_up_to(mine);
    if (lane == 63) room[wave] = up_to;
    __syncthreads();
    before = up_to - mine;
    total = 0.0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += room[w];
      total += room[w];
    }
    __syncthreads();
    if (total > 0.0 || again || kept >= count) break;
    // the draft leaves nothing: from the target's row itself
    weights = weights_of(a, r, kept, false);
    for (int g = wave; g < a.granules; g += kWaves) {
      double sum = 0.0;
      for (int n = 0; n < kGranule / kRun; ++n) {
        double w[8];
        weights.load(g * kGranule + n * kRun + lane * 8, w);
        for (int e = 0; e < 8; ++e) sum += w[e];
      }
      sum = wave_total(sum);
      if (lane == 0) sums[g] = sum;
    }
    __syncthreads();
  }
  // the first granule whose sum with those before it passes the share, and the highest with a weight
  const double share = (double)a.last_uniform[r] * total;
  if (threadIdx.x == 0) {
    chosen = INT32_MAX;
    highest = -1;
  }
  __syncthreads();
  int mine = INT32_MAX, top = -1;
  double at_mine = 0.0, at_top = 0.0;
  {
    double at = before;
    for (int g = first; g < last; ++g) {
      const double s = sums[g];
      if (s > 0.0) {
        top = g;
        at_top = at;
        if (mine == INT32_MAX && at + s > share) {
          mine = g;
          at_mine = at;
        }
      }
      at += s;
    }
  }
  if (mine != INT32_MAX) atomicMin(&chosen, mine);
  if (top >= 0) atomicMax(&highest, top);
  __syncthreads();
  const bool passes = chosen != INT32_MAX;
  const int granule = passes ? chosen : highest;
  if (passes ? mine == granule : top == granule && top >= 0) before_chosen = passes ? at_mine : at_top;
  __syncthreads();
  if (wave == 0) {
    int token = -1;
    if (granule >= 0) {
      double at = before_chosen;
      int top_token = -1;
      for (int n = 0; n < kGranule / kRun; ++n) {
        double w[8], sum = 0.0;
        const int x = granule * kGranule + n * kRun + lane * 8;
        weights.load(x, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += w[e];
        const double up_to = wave_up_to(sum);
        double running = at + (up_to - sum);
        int found = INT32_MAX;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          running += w[e];
          if (w[e] > 0.0) {
            top_token = x + e;
            if (found == INT32_MAX && running > share) found = x + e;
          }
        }
        at += __shfl(up_to, 63);
        const unsigned long long who = __ballot(found != INT32_MAX);
        if (who != 0) {
          token = __shfl(found, __ffsll((long long)who) - 1);
          break;
        }
      }
      if (token < 0) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) top_token = max(top_token, __shfl_xor(top_token, o));
        token = top_token;
      }
    }
    for (int j = lane; j <= a.max_drafts; j += 64)
      a.out[(int64_t)r * (a.max_drafts + 1) + j] = j < kept ? a.tokens[(int64_t)r * a.max_drafts + j] : j == kept ? token : -1;
  }
}

int check_sizes(int32_t batch, int32_t max_drafts, int32_t vocab) {
  if (batch < 0 || max_drafts < 0 || vocab < 1 || (int64_t)batch * vocab >= (int64_t)1 << 38) return CHUNK_ATTN_INVALID_ARG;
  return max_drafts > DRAFT_VERIFY_MAX_DRAFTS || vocab > DRAFT_VERIFY_MAX_VOCAB ? CHUNK_ATTN_UNSUPPORTED : CHUNK_ATTN_OK;
}
int count_granules(int32_t vocab) { return (vocab + kGranule - 1) / kGranule; }
bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }

template <class T>
hipError_t launch(VerifyArgs<T> a, int batch, hipStream_t stream) {
  a.granules = count_granules(a.vocab);
  // granules to a wave: one, or more (eight at most) where the chip is full with that
  a.each = (int)std::max<int64_t>(1, std::min<int64_t>(8, (int64_t)batch * a.granules / (kCus * 32)));
  a.groups = (a.granules + a.each * kWaves - 1) / (a.each * kWaves);
  hipLaunchKernelGGL((sums_kernel<T>), dim3((unsigned)((int64_t)batch * a.groups)), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((choose_kernel<T>), dim3((unsigned)batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace chunk_attn

extern "C" int draft_verify_workspace_bytes(int32_t batch, int32_t max_drafts, int32_t vocab, size_t* bytes) {
  const int rc = chunk_attn::check_sizes(batch, max_drafts, vocab);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!bytes) return CHUNK_ATTN_INVALID_ARG;
  *bytes = (size_t)batch * chunk_attn::count_granules(vocab) * sizeof(double);
  return CHUNK_ATTN_OK;
}

extern "C" int draft_verify(int32_t batch, int32_t max_drafts, int32_t vocab, int32_t probabilities_are_f32, const void* target, int64_t target_stride, const void* draft,
                            int64_t draft_stride, const int32_t* tokens, const int32_t* count, const float* uniforms, const float* last_uniform, int32_t* accepted,
                            int32_t* rejected, int32_t* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace chunk_attn;
  size_t need = 0;
  const int rc = draft_verify_workspace_bytes(batch, max_drafts, vocab, &need);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (batch == 0) return CHUNK_ATTN_OK;
  const uintptr_t size = probabilities_are_f32 ? 4 : 2;
  if (!aligned(target, size) || target_stride < vocab || ((uintptr_t)draft & (size - 1)) != 0 || (draft && draft_stride < vocab) ||
      (max_drafts > 0 && (!aligned(tokens, 4) || !aligned(uniforms, 4))) || ((uintptr_t)count & 3) != 0 || !aligned(last_uniform, 4) || !aligned(accepted, 4) ||
      ((uintptr_t)rejected & 3) != 0 || !aligned(out, 4) || !aligned(workspace, 256))
    return CHUNK_ATTN_INVALID_ARG;
  if (workspace_bytes < need) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  auto run = [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    VerifyArgs<T> a{(const T*)target, (const T*)draft, target_stride, draft_stride, tokens, count, uniforms, last_uniform, accepted, rejected, out, (double*)workspace, max_drafts, vocab};
    return launch(a, batch, (hipStream_t)hip_stream);
  };
  const hipError_t e = probabilities_are_f32 ? run((float*)nullptr) : run((__bf16*)nullptr);
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "verification of drafted tokens");
}
