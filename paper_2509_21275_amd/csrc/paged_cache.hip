// Pages of a cache for the tokens of many requests, and keys and values on their way into them (include/paged_cache.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/paged_cache.h"
#include "kernels.hpp"
#include "operators.hpp"
#include "paged.hpp"

namespace chunk_attn {
namespace {

// ---- tables ----
// Requests in order, pages in order: two running sums, of rows and of pages.  One workgroup of 1024 threads takes them, each thread over neighbouring requests; what follows
// from the sums (slots of rows, entries of the table, entries of the stack) goes row by row and page by page.  Few requests with few rows: the same workgroup does that too, with the sums in LDS, in which
// each row finds its request by halving (one launch, 3.7 us).  Else the sums go to the workspace and a second launch fills the chip.
// Bound by latency: 4096 requests with 48000 rows, 0.4 MB, take 6 and 5 us, each a chain of four or five loads that depend on each other; with the requests read again for each sum, 64-bit sums, a store for
// each number, and rows that looked for their request among all in memory, it was 16 and 8.
constexpr int kScanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kInOne = 4096;  // rows that the one workgroup goes through itself

struct TableArgs {
  int32_t n, max_pages, page_size, num_pages;
  const int32_t* change;  // new tokens, or tokens to drop
  const int32_t *kv_len, *held;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* num_free;
  int32_t *kv_len_out, *held_out, *num_free_out, *q_start, *granted;
  int64_t* slots;
  int32_t max_rows;
  // workspace: what the second launch goes by
  int32_t* sums;  // [kSums][n] and the totals behind them
  Divide by_page{1};
};
// Of each request: pages before it, tokens before the call (extend: -1 if it is not served), pages that it had (truncate: that it keeps).
enum { kPagesBefore, kOldLen, kHeld, kSums };
// Behind them: pages that change hands, pages on the stack before the call.
enum { kMoved, kOnStack, kTotals };

// Sum over the threads before the own one; `room`: one number for each wave, used by no other sum.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* room) {
  const uint32_t up_to = wave_sum_up_to(x);
  uint32_t before = (uint32_t)__shfl_up((int)up_to, 1);
  if ((threadIdx.x & 63) == 0) before = 0;
  if ((threadIdx.x & 63) == 63) room[threadIdx.x >> 6] = up_to;
  __syncthreads();
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) before = sum_at_most(before, w < wave ? room[w] : 0);
  return before;
}
__device__ __forceinline__ int at_most(uint32_t x, int most) { return (int)min(x, (uint32_t)most); }

// A request, its numbers brought into their ranges.
struct Request {
  int old_len, held, change, len, need;  // need: pages that it takes (extend, if it is served) or gives (truncate)
  bool fits;
};
__device__ __forceinline__ int pages_of(const TableArgs& a, int len) { return len > 0 ? a.by_page(len - 1) + 1 : 0; }
template <bool EXTEND>
__device__ __forceinline__ Request request_of(const TableArgs& a, int change, int kv_len, int held) {
  const int most = a.max_pages * a.page_size;  // < 2^31
  Request r;
  r.old_len = min(max(kv_len, 0), most);
  r.held = min(max(held, 0), a.max_pages);
  r.change = max(change, 0);
  if (EXTEND) {
    r.fits = r.change <= most - r.old_len;
    r.len = r.fits ? r.old_len + r.change : r.old_len;
    r.need = r.fits ? max(0, pages_of(a, r.len) - r.held) : 0;
  } else {
    r.fits = true;
    r.len = max(r.old_len - r.change, 0);
    r.need = r.held - min(r.held, pages_of(a, r.len));
  }
  return r;
}
template <bool EXTEND>
__device__ __forceinline__ Request request_at(const TableArgs& a, int i) {
  return request_of<EXTEND>(a, a.change[i], a.kv_len[i], a.held[i]);
}

// Last i < n with sums[i] <= x, for sums[0] = 0 <= x.
__device__ __forceinline__ int find(const int32_t* sums, int n, int x) {
  int lo = 0;
  for (int hi = n; hi - lo > 1;) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Slot of a row of request i, from the sums.
__device__ __forceinline__ int64_t slot_of_row(const TableArgs& a, const int32_t* q_start, const int32_t* pages_before, const int32_t* old_lens, const int32_t* helds, int on_stack, int row, int i) {
  if (old_lens[i] < 0) return -1;
  const int at = old_lens[i] + row - q_start[i], b = a.by_page(at);
  const int page = b < helds[i] ? a.table[(int64_t)i * a.max_pages + b] : a.free_pages[on_stack - 1 - (pages_before[i] + b - helds[i])];
  return page >= 0 && page < a.num_pages ? (int64_t)page * a.page_size + at - b * a.page_size : -1;
}
// One page that changes hands, of request i (truncate: one for which the stack has room).
template <bool EXTEND>
__device__ __forceinline__ void move_page(const TableArgs& a, const int32_t* pages_before, const int32_t* helds, int on_stack, int p, int i) {
  int32_t* const entry = a.table + (int64_t)i * a.max_pages + helds[i] + p - pages_before[i];
  if (EXTEND) *entry = a.free_pages[on_stack - 1 - p];
  else a.free_pages[on_stack + p] = *entry;
}

// What becomes of a request (members as in the arrays they go to).
struct Outcome {
  int start, end, pages_before, old_len, held, granted, len_out, held_out;
};
// Four neighbouring numbers, from any address that suits one.
struct __attribute__((packed, aligned(4))) LooseInts {
  int x[4];
};

// IN_ONE: at most kScanThreads requests and kInOne rows; everything is done here.  EACH: requests of a thread (0: any number, read again wherever they are used).
template <bool EXTEND, bool IN_ONE, int EACH>
__global__ __launch_bounds__(kScanThreads) void tables_kernel(const TableArgs a) {
  __shared__ uint32_t room[2][kScanThreads / 64];
  __shared__ int32_t in_lds[IN_ONE ? kSums + 1 : 1][IN_ONE ? kScanThreads + 1 : 1];
  __shared__ int moved;
  static_assert(!IN_ONE || EACH == 1);
  const int each = EACH ? EACH : (a.n + kScanThreads - 1) / kScanThreads;
  const int first = min((int)threadIdx.x * each, a.n), last = min(first + each, a.n);
  Request held_back[EACH ? EACH : 1];
  if constexpr (EACH == 4) {
    if (last == first + EACH) {
      const LooseInts change = *reinterpret_cast<const LooseInts*>(a.change + first), kv_len = *reinterpret_cast<const LooseInts*>(a.kv_len + first), held = *reinterpret_cast<const LooseInts*>(a.held + first);
#pragma unroll
      for (int i = 0; i < EACH; ++i) held_back[i] = request_of<EXTEND>(a, change.x[i], kv_len.x[i], held.x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) held_back[i] = first + i < last ? request_at<EXTEND>(a, first + i) : Request{};
    }
  } else if constexpr (EACH == 1) {
    held_back[0] = first < last ? request_at<EXTEND>(a, first) : Request{};
  }
  auto each_request = [&](auto&& f) {
    if constexpr (EACH > 0) {
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (first + i < last) f(first + i, held_back[i]);
    } else {
      for (int i = first; i < last; ++i) f(i, request_at<EXTEND>(a, i));
    }
  };
  const int on_stack = min(max(*a.num_free, 0), a.num_pages);
  int32_t* const pages_before = IN_ONE ? in_lds[kPagesBefore] : a.sums + (int64_t)kPagesBefore * a.n;
  int32_t* const old_lens = IN_ONE ? in_lds[kOldLen] : a.sums + (int64_t)kOldLen * a.n;
  int32_t* const helds = IN_ONE ? in_lds[kHeld] : a.sums + (int64_t)kHeld * a.n;
  int32_t* const starts = IN_ONE ? in_lds[kSums] : a.q_start;
  auto leave = [&](int i, const Outcome& o) {
    pages_before[i] = o.pages_before;
    old_lens[i] = o.old_len;
    helds[i] = o.held;
    a.kv_len_out[i] = o.len_out;
    a.held_out[i] = o.held_out;
    if (EXTEND) {
      starts[i] = o.start;
      if (IN_ONE) a.q_start[i] = o.start;
      if (i == a.n - 1) {
        starts[a.n] = o.end;
        if (IN_ONE) a.q_start[a.n] = o.end;
      }
      if (a.granted) a.granted[i] = o.granted;
    }
  };
  if (threadIdx.x == 0) moved = 0;  // (before the sums' barrier)
  // rows first: who does not fit in them has no claim on pages
  uint32_t rows = 0, pages = 0;
  if (EXTEND) {
    each_request([&](int, const Request& r) { rows = sum_at_most(rows, r.change); });
    rows = sum_before(rows, room[0]);
  }
  uint32_t row = rows;
  each_request([&](int, const Request& r) {
    row = sum_at_most(row, r.change);
    if (!EXTEND || r.change == 0 || row <= (uint32_t)a.max_rows) pages = sum_at_most(pages, r.need);
  });
  pages = sum_before(pages, room[1]);
  row = rows;
  int mine = 0;
  Outcome outcome[EACH ? EACH : 1];
  each_request([&](int i, const Request& r) {
    const uint32_t end = sum_at_most(row, r.change);
    const bool in_rows = !EXTEND || r.change == 0 || end <= (uint32_t)a.max_rows;
    const int need = in_rows ? r.need : 0;
    const bool served = r.fits && in_rows && (!EXTEND || need == 0 || sum_at_most(pages, need) <= (uint32_t)on_stack);
    Outcome o;
    o.start = at_most(row, a.max_rows);
    o.end = at_most(end, a.max_rows);
    o.pages_before = at_most(pages, INT32_MAX);
    pages = sum_at_most(pages, need);
    if (served && need > 0) mine = at_most(pages, INT32_MAX);  // (the sums grow: those that are served are the first of those that need pages)
    row = end;
    o.old_len = served ? r.old_len : -1;
    o.held = EXTEND ? r.held : r.held - need;
    o.granted = served;
    o.len_out = served ? r.len : r.old_len;
    o.held_out = EXTEND ? r.held + (served ? need : 0) : r.held - need;
    if constexpr (EACH > 0) outcome[i - first] = o;
    else leave(i, o);
  });
  if constexpr (EACH == 4) {
    if (last == first + EACH) {
      // four neighbouring numbers to a store
      auto four = [&](int32_t* p, auto member) {
        *reinterpret_cast<LooseInts*>(p + first) = LooseInts{{outcome[0].*member, outcome[1].*member, outcome[2].*member, outcome[3].*member}};
      };
      four(pages_before, &Outcome::pages_before);
      four(old_lens, &Outcome::old_len);
      four(helds, &Outcome::held);
      four(a.kv_len_out, &Outcome::len_out);
      four(a.held_out, &Outcome::held_out);
      if (EXTEND) {
        four(a.q_start, &Outcome::start);
        if (a.granted) four(a.granted, &Outcome::granted);
        if (last == a.n) a.q_start[a.n] = outcome[3].end;
      }
    } else {
      each_request([&](int i, const Request&) { leave(i, outcome[i - first]); });
    }
  } else if constexpr (EACH == 1) {
    each_request([&](int i, const Request&) { leave(i, outcome[0]); });
  }
  if constexpr (EXTEND && !IN_ONE) {
    // fill_kernel's workgroups begin to look for their rows' requests where the first row's slot will be
    row = rows;
    each_request([&](int i, const Request& r) {
      const int64_t end = min(sum_at_most(row, r.change), (uint32_t)a.max_rows);
      for (int64_t at = ((int64_t)row + kFillThreads - 1) / kFillThreads * kFillThreads; at < end; at += kFillThreads) a.slots[at] = i;
      row = sum_at_most(row, r.change);
    });
  }
  if (mine > 0) atomicMax(&moved, mine);
  __syncthreads();
  if (threadIdx.x == 0) {
    *a.num_free_out = EXTEND ? on_stack - moved : at_most((uint32_t)on_stack + (uint32_t)moved, a.num_pages);
    if (!IN_ONE) {
      a.sums[(int64_t)kSums * a.n + kMoved] = moved;
      a.sums[(int64_t)kSums * a.n + kOnStack] = on_stack;
    }
  }
  if constexpr (IN_ONE) {
    if (EXTEND)
      for (int r = threadIdx.x; r < a.max_rows; r += kScanThreads) a.slots[r] = r < starts[a.n] ? slot_of_row(a, starts, pages_before, old_lens, helds, on_stack, r, find(starts, a.n, r)) : -1;
    // (unsigned: `moved` may be the largest int, and the next p past it)
    const uint32_t moves = (uint32_t)(EXTEND ? moved : min(moved, a.num_pages - on_stack));
    for (uint32_t p = threadIdx.x; p < moves; p += kScanThreads) move_page<EXTEND>(a, pages_before, helds, on_stack, (int)p, find(pages_before, a.n, (int)p));
  }
}

// The first `page_groups` workgroups: pages that change hands, a wave to a request.  The others: slots, kFillThreads neighbouring rows to a workgroup, whose requests are looked for among the sums from the
// first row's request on, in LDS (rows of requests that have none may lie between, so that kWindow of them need not reach the last row).
constexpr int kWindow = 1024;
template <bool EXTEND>
__global__ __launch_bounds__(kFillThreads) void fill_kernel(const TableArgs a, const int page_groups) {
  const int32_t *const pages_before = a.sums + (int64_t)kPagesBefore * a.n, *const old_lens = a.sums + (int64_t)kOldLen * a.n, *const helds = a.sums + (int64_t)kHeld * a.n;
  const int moved = a.sums[(int64_t)kSums * a.n + kMoved], on_stack = a.sums[(int64_t)kSums * a.n + kOnStack];
  if ((int)blockIdx.x < page_groups) {
    const int i = __builtin_amdgcn_readfirstlane(blockIdx.x * (kFillThreads / 64) + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
    if (i >= a.n) return;
    const int first = pages_before[i], held = helds[i], end = i + 1 < a.n ? pages_before[i + 1] : INT32_MAX;
    // (extend: none of a request that is not served)
    const int last = EXTEND ? first + (a.held_out[i] - held) : min(end, moved);
    constexpr int kAtOnce = 4;
    int32_t* const entries = a.table + (int64_t)i * a.max_pages + held;
    for (int64_t p0 = first; p0 < last; p0 += 64 * kAtOnce) {
      int32_t page[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int64_t p = p0 + k * 64 + lane;
        page[k] = p >= last ? 0 : EXTEND ? a.free_pages[on_stack - 1 - p] : entries[p - first];
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int64_t p = p0 + k * 64 + lane;
        if (p >= last) continue;
        if (EXTEND) entries[p - first] = page[k];
        else if (on_stack + p < a.num_pages) a.free_pages[on_stack + p] = page[k];
      }
    }
    return;
  }
  if constexpr (EXTEND) {
    __shared__ int32_t window[kWindow];
    const int rows = a.q_start[a.n];
    for (int64_t r0 = (int64_t)(blockIdx.x - page_groups) * kFillThreads; r0 < a.max_rows; r0 += (int64_t)(gridDim.x - page_groups) * kFillThreads) {
      const int64_t r = r0 + threadIdx.x;
      const int first = r0 < rows ? (int)a.slots[r0] : 0, count = min(kWindow, a.n - first);
      for (int i = threadIdx.x; i < count; i += kFillThreads) window[i] = a.q_start[first + i];
      __syncthreads();  // (and the first row's slot has been read)
      if (r < a.max_rows) {
        int64_t slot = -1;
        if (r < rows) {
          const bool behind = first + count < a.n && r >= window[count - 1];
          slot = slot_of_row(a, a.q_start, pages_before, old_lens, helds, on_stack, (int)r, behind ? find(a.q_start, a.n, (int)r) : first + find(window, count, (int)r));
        }
        a.slots[r] = slot;
      }
      __syncthreads();
    }
  }
}

int check_desc(const paged_cache_desc* d) {
  if (!d || d->num_requests < 1 || d->max_pages < 1 || d->num_pages < 1 || d->page_size < 1) return CHUNK_ATTN_INVALID_ARG;
  if (d->num_requests > PAGED_CACHE_MAX_REQUESTS || d->page_size > PAGED_CACHE_MAX_PAGE_SIZE) return CHUNK_ATTN_UNSUPPORTED;
  return (int64_t)d->max_pages * d->page_size > INT32_MAX ? CHUNK_ATTN_INVALID_ARG : CHUNK_ATTN_OK;
}
size_t table_bytes(const paged_cache_desc* d) { return ((size_t)d->num_requests * kSums + kTotals) * sizeof(int32_t); }
bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }

template <bool EXTEND>
int run_tables(const paged_cache_desc* d, TableArgs a, void* workspace, size_t workspace_bytes, hipStream_t stream, const char* what) {
  for (const void* p : {(const void*)a.change, (const void*)a.kv_len, (const void*)a.held, (const void*)a.table, (const void*)a.free_pages, (const void*)a.num_free,
                        (const void*)a.kv_len_out, (const void*)a.held_out, (const void*)a.num_free_out})
    if (!aligned(p, 4)) return CHUNK_ATTN_INVALID_ARG;
  if (!aligned(workspace, 256)) return CHUNK_ATTN_INVALID_ARG;
  if (workspace_bytes < table_bytes(d)) return CHUNK_ATTN_WORKSPACE_TOO_SMALL;
  a.n = d->num_requests;
  a.max_pages = d->max_pages;
  a.page_size = d->page_size;
  a.num_pages = d->num_pages;
  a.sums = (int32_t*)workspace;
  a.by_page = Divide(d->page_size);
  // One launch / two, us, in a graph.  Extensions: 64 requests with 64 rows 3.2 / 5.9, 1024 with 1024 4.3 / 8.2, 256 with 4096 8.9 / 9.9, 1024 with 4096 7.2 / 8.0; 64 with 4096 8.1 / 7.8, 64 with 16384
  // 18.6 / 8.4.  Truncations, of which the host does not know how many pages they give back: rejected drafts and some requests' ends, 64 requests with 64 pages 4.5 / 5.2, 256 with 256 4.7 / 6.5, 1024 with 1024
  // 6.3 / 6.7; everything at once, 256 with 4096 6.9 / 6.5, 1024 with 65536 61 / 6.7, with 2^20 1012 / 9.1, which is seldom, and is left to cost that.
  if (a.n <= kScanThreads && a.max_rows <= kInOne) {
    hipLaunchKernelGGL((tables_kernel<EXTEND, true, 1>), dim3(1), dim3(kScanThreads), 0, stream, a);
  } else {
    if (a.n <= 4 * kScanThreads) hipLaunchKernelGGL((tables_kernel<EXTEND, false, 4>), dim3(1), dim3(kScanThreads), 0, stream, a);
    else hipLaunchKernelGGL((tables_kernel<EXTEND, false, 0>), dim3(1), dim3(kScanThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report_hip(e, what);
    const int page_groups = (a.n + kFillThreads / 64 - 1) / (kFillThreads / 64);
    const int row_groups = EXTEND ? (int)std::min<int64_t>(((int64_t)a.max_rows + kFillThreads - 1) / kFillThreads, 4 * kCus) : 0;
    hipLaunchKernelGGL((fill_kernel<EXTEND>), dim3((unsigned)(page_groups + row_groups)), dim3(kFillThreads), 0, stream, a, page_groups);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, what);
}

// ---- keys and values into the pages ----
// Bound by memory, as long as the vector work is kept small: with true divisions, and what belongs to a head found anew for each row, the vector units were busy for 97 % of the time.  A thread takes eight
// elements of one place in a row, of both tensors, of ROWS rows that are `apart` rows from each other: one; two to e4m3 where the chip is full with that.  65536 rows of 8 heads of 128 out of wider rows, us,
// one / two / four: e4m3 108 / 77 (5.2 TB/s) / 79, bf16 103 / 104 / 105; 16384 rows 30 / 20 / 21 and 27.6 / 29 / 31.
constexpr int kWriteThreads = 256, kManyRows = 2;
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

struct WriteArgs {
  const __bf16 *k, *v;
  int64_t k_stride, v_stride;
  const int64_t* slots;
  const float *k_scale, *v_scale;
  void *k_cache, *v_cache;
  int64_t num_slots, pieces;  // pieces of eight elements in `apart` rows
  int32_t rows, apart, heads, head_pieces, row_pieces, page_size;
  Divide by_row, by_head, by_page;
};

// Division by a head's scale.  x / s as q + r y with y the nearest to 1 / s, q = x y and r = x - q s, which a fused multiply and add gives exactly: the nearest to the quotient, where nothing
// leaves float32's normal range (equal to the division for 4 * 10^8 drawn pairs), but for -0, which comes out as 0 (the remainder is 0, and -0 + 0 = 0): to_e4m3 puts the sign back.
// Quotients past 1024 only have to stay past 448: q is kept to 1024, so that nothing becomes infinite less infinite.
struct Scale {
  float s, y;
  bool usual;  // the quotient of anything by s that 8 bits hold is far from the ends of float32's range
  explicit __device__ Scale(float scale) : s(scale), y(1.f / scale), usual(scale > 0x1p-80f && scale < 0x1p80f) {}
  __device__ float divides(float x) const {
    const float q = __builtin_amdgcn_fmed3f(x * y, -1024.f, 1024.f);
    return __builtin_fmaf(__builtin_fmaf(-s, q, x), y, q);
  }
};
__device__ __forceinline__ float element(const u32x4& x, int e) { return __uint_as_float(e & 1 ? x[e >> 1] & 0xffff0000u : x[e >> 1] << 16); }
// Eight bf16 numbers over the scale as e4m3.
__device__ __forceinline__ u32x2 to_e4m3(const u32x4& x, const Scale& scale) {
  unsigned special = 0;  // infinities and NaN: their exponents are ones, which overflow into the bit above
#pragma unroll
  for (int w = 0; w < 4; ++w) special |= ((x[w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  float c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = __builtin_amdgcn_fmed3f(scale.divides(element(x, e)), -448.f, 448.f);
  // set in a byte of the result: its sign, which is the number's (a scale is positive); where quotients are divided truly, NaN
  unsigned bits[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) bits[w] = __builtin_amdgcn_perm(x[2 * w + 1], x[2 * w], 0x07050301) & 0x80808080u;
  if (special != 0 || !scale.usual) {
    bits[0] = bits[1] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = element(x, e) / scale.s;
      c[e] = f > 448.f ? 448.f : f < -448.f ? -448.f : f;
      bits[e >> 2] |= f != f ? 0x7fu << (8 * (e & 3)) : 0u;
    }
  }
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * w], c[4 * w + 1], 0, false);
    word = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * w + 2], c[4 * w + 3], word, true);
    r[w] = (unsigned)word | bits[w];
  }
  return r;
}

typedef u32x4 __attribute__((aligned(2))) LooseWords;
template <bool STREAM, class T>
__device__ __forceinline__ void store_words(T* p, T x) {
  if (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

// STREAM: past the caches, for calls of more bytes than the last-level cache holds (87 -> 84 us before the vector work was cut); what fits is kept for who reads it next.
template <bool E4M3, bool STREAM, int ROWS>
__global__ __launch_bounds__(kWriteThreads) void write_kernel(const WriteArgs a) {
  // (the workgroup's first row and piece: scalar work)
  const int64_t piece0 = (int64_t)blockIdx.x * kWriteThreads, row0 = a.by_row.wide(piece0);
  if (piece0 + threadIdx.x >= a.pieces) return;
  const int ahead = (int)(piece0 - row0 * a.row_pieces) + threadIdx.x, rows_ahead = a.by_row(ahead), in_row = ahead - rows_ahead * a.row_pieces;
  const int row = (int)row0 + rows_ahead, head = a.by_head(in_row);
  u32x4 k[ROWS], v[ROWS];
  int64_t slot[ROWS];
#pragma unroll
  for (int n = 0; n < ROWS; ++n) {
    const int64_t at = row + (int64_t)n * a.apart;
    slot[n] = ROWS == 1 || at < a.rows ? a.slots[at] : -1;
  }
#pragma unroll
  for (int n = 0; n < ROWS; ++n) {
    const int64_t at = row + (int64_t)n * a.apart;
    if (ROWS > 1 && at >= a.rows) continue;
    const LooseWords *const pk = reinterpret_cast<const LooseWords*>(a.k + at * a.k_stride + in_row * 8), *const pv = reinterpret_cast<const LooseWords*>(a.v + at * a.v_stride + in_row * 8);
    k[n] = STREAM ? __builtin_nontemporal_load(pk) : *pk;
    v[n] = STREAM ? __builtin_nontemporal_load(pv) : *pv;
  }
  const Scale k_scale(E4M3 ? a.k_scale[head] : 1.f), v_scale(E4M3 ? a.v_scale[head] : 1.f);
#pragma unroll
  for (int n = 0; n < ROWS; ++n) {
    if (slot[n] < 0 || slot[n] >= a.num_slots) continue;
    const int64_t page = a.by_page.wide(slot[n]);
    const int64_t to = ((page * a.heads + head) * a.page_size + (slot[n] - page * a.page_size)) * a.head_pieces + (in_row - head * a.head_pieces);
    if constexpr (E4M3) {
      store_words<STREAM>(reinterpret_cast<u32x2*>(a.k_cache) + to, to_e4m3(k[n], k_scale));
      store_words<STREAM>(reinterpret_cast<u32x2*>(a.v_cache) + to, to_e4m3(v[n], v_scale));
    } else {
      store_words<STREAM>(reinterpret_cast<u32x4*>(a.k_cache) + to, k[n]);
      store_words<STREAM>(reinterpret_cast<u32x4*>(a.v_cache) + to, v[n]);
    }
  }
}

}  // namespace
}  // namespace chunk_attn

extern "C" int paged_cache_validate(const paged_cache_desc* d) { return chunk_attn::check_desc(d); }

extern "C" int paged_cache_workspace_bytes(const paged_cache_desc* d, size_t* bytes) {
  const int rc = chunk_attn::check_desc(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (!bytes) return CHUNK_ATTN_INVALID_ARG;
  *bytes = chunk_attn::table_bytes(d);
  return CHUNK_ATTN_OK;
}

extern "C" int paged_cache_extend(const paged_cache_desc* d, const int32_t* new_tokens, const int32_t* kv_len, const int32_t* held, int32_t* table, const int32_t* free_pages,
                                  const int32_t* num_free, int32_t* kv_len_out, int32_t* held_out, int32_t* num_free_out, int32_t* q_start, int64_t* slots, int32_t max_rows,
                                  int32_t* granted, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace chunk_attn;
  const int rc = check_desc(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  if (max_rows < 0 || !aligned(q_start, 4) || (max_rows > 0 && !aligned(slots, 8)) || ((uintptr_t)granted & 3) != 0) return CHUNK_ATTN_INVALID_ARG;
  TableArgs a{};
  a.change = new_tokens;
  a.kv_len = kv_len;
  a.held = held;
  a.table = table;
  a.free_pages = const_cast<int32_t*>(free_pages);  // (read only where tokens come in)
  a.num_free = num_free;
  a.kv_len_out = kv_len_out;
  a.held_out = held_out;
  a.num_free_out = num_free_out;
  a.q_start = q_start;
  a.slots = slots;
  a.max_rows = max_rows;
  a.granted = granted;
  return run_tables<true>(d, a, workspace, workspace_bytes, (hipStream_t)hip_stream, "pages for new tokens");
}

extern "C" int paged_cache_truncate(const paged_cache_desc* d, const int32_t* drop, const int32_t* kv_len, const int32_t* held, const int32_t* table, int32_t* free_pages,
                                    const int32_t* num_free, int32_t* kv_len_out, int32_t* held_out, int32_t* num_free_out, void* workspace, size_t workspace_bytes,
                                    void* hip_stream) {
  using namespace chunk_attn;
  const int rc = check_desc(d);
  if (rc != CHUNK_ATTN_OK) return rc;
  TableArgs a{};
  a.change = drop;
  a.kv_len = kv_len;
  a.held = held;
  a.table = const_cast<int32_t*>(table);  // (read only where tokens go)
  a.free_pages = free_pages;
  a.num_free = num_free;
  a.kv_len_out = kv_len_out;
  a.held_out = held_out;
  a.num_free_out = num_free_out;
  return run_tables<false>(d, a, workspace, workspace_bytes, (hipStream_t)hip_stream, "pages given back");
}

extern "C" int paged_cache_write(int32_t rows, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages, int32_t cache_type, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, const int64_t* slots, const float* k_scale, const float* v_scale, void* k_cache, void* v_cache,
                                 void* hip_stream) {
  using namespace chunk_attn;
  if (rows < 0 || num_kv_heads < 1 || page_size < 1 || num_pages < 1 || (cache_type != PAGED_CACHE_BF16 && cache_type != PAGED_CACHE_E4M3)) return CHUNK_ATTN_INVALID_ARG;
  if (!paged_head_dim(head_dim) || num_kv_heads > PAGED_MAX_HEADS || page_size > PAGED_CACHE_MAX_PAGE_SIZE) return CHUNK_ATTN_UNSUPPORTED;
  const int64_t row_elements = (int64_t)num_kv_heads * head_dim;
  if ((int64_t)rows * row_elements >= (int64_t)1 << 40) return CHUNK_ATTN_INVALID_ARG;
  if (rows == 0) return CHUNK_ATTN_OK;
  if (!aligned(k, 2) || !aligned(v, 2) || k_stride < row_elements || v_stride < row_elements || !aligned(slots, 8) || !aligned(k_cache, 16) || !aligned(v_cache, 16) ||
      (cache_type == PAGED_CACHE_E4M3 && (!aligned(k_scale, 4) || !aligned(v_scale, 4))))
    return CHUNK_ATTN_INVALID_ARG;
  const int row_pieces = (int)(row_elements / 8), head_pieces = head_dim / 8;
  const bool e4m3 = cache_type == PAGED_CACHE_E4M3, stream = (int64_t)rows * row_pieces * (e4m3 ? 48 : 64) > kStreamBytes;
  const bool many = e4m3 && (int64_t)rows * row_pieces >= (int64_t)kManyRows * kCus * 2048;
  const int apart = many ? (rows + kManyRows - 1) / kManyRows : rows;
  const int64_t pieces = (int64_t)apart * row_pieces, groups = (pieces + kWriteThreads - 1) / kWriteThreads;
  if (groups * kWriteThreads >= (int64_t)1 << 32) return CHUNK_ATTN_INVALID_ARG;
  const WriteArgs a{(const __bf16*)k, (const __bf16*)v, k_stride, v_stride, slots, k_scale, v_scale, k_cache, v_cache, (int64_t)num_pages * page_size, pieces, rows, apart, num_kv_heads,
                    head_pieces, row_pieces, page_size, Divide(row_pieces), Divide(head_pieces), Divide(page_size)};
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kWriteThreads), 0, (hipStream_t)hip_stream, a); };
  if (many) stream ? launch(write_kernel<true, true, kManyRows>) : launch(write_kernel<true, false, kManyRows>);
  else if (e4m3) launch(write_kernel<true, false, 1>);
  else stream ? launch(write_kernel<false, true, 1>) : launch(write_kernel<false, false, 1>);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CHUNK_ATTN_OK : report_hip(e, "keys and values into pages");
}
