// Whole numbers of the attention over a paged cache that are formed of what the host does not know: constexpr, so that the kernels and host programs have the same.
#pragma once
#include <stdint.h>

namespace chunk_attn {

// Rows of q from `start` up to `end`, which may be any numbers: those of them that lie in [0, total).  (Brought into that range before they are subtracted: 32 bits do not hold the difference of any two.)
struct Rows {
  int32_t first, count;
};
constexpr Rows rows_between(int32_t start, int32_t end, int32_t total) {
  const int32_t first = start < 0 ? 0 : start < total ? start : total, last = end < first ? first : end < total ? end : total;
  return Rows{first, last - first};
}

// In how many shares of `size` units each, of `total` units in all, a block's units lie, from the share that its first unit is in.  (Sums of units stay at a largest number, which a block may reach
// past where starts of rows do not increase: what lies behind it is in no share.)
constexpr int32_t shares_of_block(int32_t first, int32_t units, int32_t size, int32_t total) {
  const int32_t last = units < total - first ? first + units - 1 : total - 1;
  return (int32_t)((uint32_t)last / (uint32_t)size - (uint32_t)first / (uint32_t)size) + 1;
}

}  // namespace chunk_attn
