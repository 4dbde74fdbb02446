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

}  // namespace chunk_attn
