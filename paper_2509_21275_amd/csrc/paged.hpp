// What the operators of the paged cache share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace chunk_attn {

constexpr int PAGED_MAX_HEADS = 16384;
inline bool paged_head_dim(int d) { return d == 64 || d == 96 || d == 128 || d == 256; }

// Division by a number d (1 .. 2^30) that a launch does not know when it is compiled: x / d = x * M / 2^(31 + l) rounded down, with l = ceil(log2 d) and M = floor(2^(31 + l) / d) + 1 < 2^32 + 1.
// M d exceeds 2^(31 + l) by e <= d <= 2^l, so that x M / 2^(31 + l) exceeds x / d by x e / (2^(31 + l) d) < 1 / d for x < 2^31: never to the next whole number.
struct Divide {
  uint64_t m;
  int32_t shift, by;
  explicit Divide(int d) : by(d) {
    int l = 0;
    while (((int64_t)1 << l) < d) ++l;
    shift = 31 + l;
    m = ((uint64_t)1 << shift) / (uint64_t)d + 1;
  }
  // 0 <= x < 2^31
  __host__ __device__ int operator()(int x) const { return (int)((uint64_t)(uint32_t)x * m >> shift); }
  // x >= 0
  __host__ __device__ int64_t wide(int64_t x) const { return x <= INT32_MAX ? (*this)((int)x) : x / by; }
};

// Sums that stay at the largest number once they are there: whatever the inputs are, what is below 2^32 - 1 is right.
__device__ __forceinline__ uint32_t sum_at_most(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
// The same over the lanes up to the own one: within rows of 16 lanes, then from row to row.
__device__ __forceinline__ uint32_t wave_sum_up_to(uint32_t x) {
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));  // from 1, 2, 4 and 8 lanes before
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));  // the last lane of the row before, to rows 1 and 3
  x = sum_at_most(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));  // lane 31 to rows 2 and 3
  return x;
}

}  // namespace chunk_attn
