// Verification of drafted tokens (include/draft_verify.h).
//
// Bound by memory: one row of the target's probabilities, and one of the draft's where a token is rejected, of each request.  The sum of weights has to be known before the place
// can be found where the running sum passes a share of it, so: sums_kernel finds the row and leaves the sum of every kGranule weights, taken by one wave; choose_kernel sums these up, finds the granule
// and reads it again.  A weight is there or not by a comparison in float32, which is exact; sums are float64: differences that matter are exact, and sums of 10^5 weights are off by 10^-15 of them or so.
// Measured: 256 requests, 131072 bf16 probabilities (134 MB) 29.3 us, of which the choice 6; 8 of 32000 4.4 + 5.6.  With both in one kernel, a workgroup of 16
// waves to a request: 27.6 us there, and 10.5 against 11.4 for one request of 32000, but 36 against 28 for 128 requests of 131072 float32, 66 against 49 for 300, 21 against 12 for one.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/draft_verify.h"
#include "kernels.hpp"
#include "operators.hpp"

namespace chunk_attn {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRun = 64 * 8, kGranule = 2 * kRun;  // a wave takes eight neighbouring weights to a lane, twice

template <class T>
struct VerifyArgs {
  const T *target, *draft;
  int64_t target_stride, draft_stride;
  const int32_t *tokens, *count;
  const float *uniforms, *last_uniform;
  int32_t *accepted, *rejected, *out;
  double* sums;  // [batch][granules]
  int32_t max_drafts, vocab, granules, groups;  // workgroups to a request
};

// The row that the last token is drawn from.
template <class T>
struct Weights {
  const T *p, *q;  // q: null if all is drawn from p
  int without;     // a token that weighs nothing, or -1
  int vocab;
  // Probabilities first .. first + 7 (behind the vocabulary: zeros), such that x - y is their weight: both zero where that is not positive, or not finite.
  // INSIDE: all of them are in the vocabulary (no branch stands between loads then).
  template <bool INSIDE>
  __device__ void load(int first, float* x, float* y) const {
    const int n = INSIDE ? 8 : vocab - first;
    load_up_to_8(p + first, n, x);
    load_up_to_8((q ? q : p) + first, n, y);
  }
  __device__ void clear(int first, float* x, float* y) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = q ? y[e] : 0.f;
      const float d = x[e] - y[e];  // (rounded, but of the right sign)
      const bool some = d > 0.f && d <= 3.402823466e38f && first + e != without;
      x[e] = some ? x[e] : 0.f;
      y[e] = some ? y[e] : 0.f;
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

// Sum of a granule, by one wave.
template <class T, bool INSIDE>
__device__ __forceinline__ void leave_sum(const VerifyArgs<T>& a, const Weights<T>& weights, int r, int granule) {
  const int lane = threadIdx.x & 63;
  float x[2][8], y[2][8];
#pragma unroll
  for (int n = 0; n < 2; ++n) weights.template load<INSIDE>(INSIDE ? granule * kGranule + n * kRun + lane * 8 : min(granule * kGranule + n * kRun + lane * 8, a.vocab), x[n], y[n]);
  double sum = 0.0;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    weights.clear(granule * kGranule + n * kRun + lane * 8, x[n], y[n]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += (double)x[n][e] - (double)y[n][e];
  }
  sum = wave_total(sum);
  if (lane == 0) a.sums[(int64_t)r * a.granules + granule] = sum;
}

// A wave takes one granule (more only where a launch would have too many threads).  Four at once, so that more loads are under way, was slower but for large batches of bf16 rows that are a multiple of them: one / four, us, 512 requests of 32000 27.2 / 29.6 (float32)
// and 20.1 / 25.2 (bf16), 900 of 50257 bf16 45 / 53, 256 of 131072 45.0 / 46.5 (float32) and 29.3 / 30.2 (bf16), 100 of 262144 bf16 24.9 / 25.6; 512 and 1000 of 131072 bf16 52.4 / 50.5 and 89.6 / 82.9.
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
  for (int granule = group * kWaves + wave; granule < a.granules; granule += a.groups * kWaves) {
    if ((granule + 1) * kGranule <= a.vocab) leave_sum<T, true>(a, weights, r, granule);
    else leave_sum<T, false>(a, weights, r, granule);
  }
}

// One workgroup to a request.
template <class T>
__global__ __launch_bounds__(kThreads) void choose_kernel(const VerifyArgs<T> a) {
  __shared__ double room[kWaves], before_first[kWaves], before_last[kWaves];
  __shared__ int first_past[kWaves], last_some[kWaves];
  const int r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double* const sums = a.sums + (int64_t)r * a.granules;
  const int each = (a.granules + kThreads - 1) / kThreads, first = min((int)threadIdx.x * each, a.granules), last = min(first + each, a.granules);
  // loads that depend on nothing, together
  const int kept = a.accepted[r], count = count_of(a, r), drafted = lane < a.max_drafts ? a.tokens[(int64_t)r * a.max_drafts + lane] : -1;
  const float uniform = a.last_uniform[r];
  double mine = first < last ? sums[first] : 0.0;
  for (int g = first + 1; g < last; ++g) mine += sums[g];
  Weights<T> weights = weights_of(a, r, kept, kept < count);
  double total = 0.0, before = 0.0;
  for (int again = 0;; ++again) {
    const double up_to = wave_up_to(mine);
    if (lane == 63) room[wave] = up_to;
    __syncthreads();
    before = up_to - mine;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += room[w];
      total += room[w];
    }
    if (total > 0.0 || again || kept >= count) break;
    // the draft leaves nothing: from the target's row itself
    weights = weights_of(a, r, kept, false);
    for (int g = wave; g < a.granules; g += kWaves) {
      double sum = 0.0;
      for (int n = 0; n < kGranule / kRun; ++n) {
        float x[8], y[8];
        const int at = g * kGranule + n * kRun + lane * 8;
        weights.template load<false>(min(at, a.vocab), x, y);
        weights.clear(at, x, y);
        for (int e = 0; e < 8; ++e) sum += (double)x[e];
      }
      sum = wave_total(sum);
      if (lane == 0) sums[g] = sum;
    }
    __syncthreads();
    mine = 0.0;
    for (int g = first; g < last; ++g) mine += sums[g];
  }
  // the first granule whose sum with those before it passes the share, and the highest with a weight
  const double share = (double)uniform * total;
  int past = INT32_MAX, some = -1;
  double at_past = 0.0, at_some = 0.0, at = before;
  for (int g = first; g < last; ++g) {
    const double s = each == 1 ? mine : sums[g];
    if (s > 0.0) {
      some = g;
      at_some = at;
      if (past == INT32_MAX && at + s > share) {
        past = g;
        at_past = at;
      }
    }
    at += s;
  }
  const unsigned long long who_past = __ballot(past != INT32_MAX), who_some = __ballot(some >= 0);
  if (lane == (who_past ? __ffsll((long long)who_past) - 1 : 0)) {
    first_past[wave] = past;
    before_first[wave] = at_past;
  }
  if (lane == (who_some ? 63 - __clzll((long long)who_some) : 0)) {
    last_some[wave] = some;
    before_last[wave] = at_some;
  }
  __syncthreads();
  if (wave != 0) return;
  int granule = -1;
  at = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    if (last_some[w] >= 0) {
      granule = last_some[w];
      at = before_last[w];
    }
#pragma unroll
  for (int w = kWaves - 1; w >= 0; --w)
    if (first_past[w] != INT32_MAX) {
      granule = first_past[w];
      at = before_first[w];
    }
  int token = -1, highest = -1;
  if (granule >= 0) {
    float x[2][8], y[2][8];
#pragma unroll
    for (int n = 0; n < 2; ++n) weights.template load<false>(min(granule * kGranule + n * kRun + lane * 8, a.vocab), x[n], y[n]);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int base = granule * kGranule + n * kRun + lane * 8;
      weights.clear(base, x[n], y[n]);
      double sum = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)x[n][e] - (double)y[n][e];
      const double up_to = wave_up_to(sum);
      double running = at + (up_to - sum);
      int found = INT32_MAX;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        running += (double)x[n][e] - (double)y[n][e];
        if (x[n][e] > y[n][e]) {
          highest = base + e;
          if (found == INT32_MAX && running > share) found = base + e;
        }
      }
      at += __shfl(up_to, 63);
      const unsigned long long who = __ballot(found != INT32_MAX);
      if (who != 0 && token < 0) token = __shfl(found, __ffsll((long long)who) - 1);
    }
    if (token < 0) {
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) highest = max(highest, __shfl_xor(highest, o));
      token = highest;
    }
  }
  // (64 drafts at most: a place for each lane, and one behind them)
  int32_t* const out = a.out + (int64_t)r * (a.max_drafts + 1);
  if (lane <= a.max_drafts) out[lane] = lane < kept ? drafted : lane == kept ? token : -1;
  if (lane == 0 && a.max_drafts == 64) out[64] = kept == 64 ? token : -1;
}

int check_sizes(int32_t batch, int32_t max_drafts, int32_t vocab) {
  if (batch < 0 || max_drafts < 0 || vocab < 1 || batch >= 1 << 23 || (int64_t)batch * vocab >= (int64_t)1 << 36) return CHUNK_ATTN_INVALID_ARG;
  return max_drafts > DRAFT_VERIFY_MAX_DRAFTS || vocab > DRAFT_VERIFY_MAX_VOCAB ? CHUNK_ATTN_UNSUPPORTED : CHUNK_ATTN_OK;
}
int count_granules(int32_t vocab) { return (vocab + kGranule - 1) / kGranule; }
bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }

template <class T>
hipError_t launch(VerifyArgs<T> a, int batch, hipStream_t stream) {
  a.granules = count_granules(a.vocab);
  a.groups = std::min((a.granules + kWaves - 1) / kWaves, ((1 << 24) - 1) / batch);  // (threads of a launch: below 2^32)
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
