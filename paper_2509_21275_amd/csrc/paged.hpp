// What the operators of the paged cache share.
#pragma once
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

}  // namespace chunk_attn
