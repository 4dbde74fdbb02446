// The attention's division of its work (csrc/paged_shares.hpp) against the same in 64 bits, one by one: any starts of rows, blocks at and past the end of all units.
#include <algorithm>
#include <cstdio>
#include <random>

#include "../../paper_2509_21275_amd/csrc/paged_shares.hpp"

#define REQUIRE(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
using namespace chunk_attn;

static int rows() {
  const int32_t ends[] = {INT32_MIN, INT32_MIN + 1, -5, -1, 0, 1, 2, 7, 100, 101, INT32_MAX - 1, INT32_MAX};
  for (int32_t total : {0, 1, 7, 100, INT32_MAX})
    for (int32_t start : ends)
      for (int32_t end : ends) {
        const Rows r = rows_between(start, end, total);
        // what lies in both ranges
        const int64_t lo = start > 0 ? start : 0, hi = end < total ? end : total, count = hi > lo ? hi - lo : 0;
        REQUIRE(r.count == count && r.first >= 0 && r.first <= total && r.count >= 0 && r.count <= total - r.first);
        REQUIRE(count == 0 || r.first == lo);
      }
  return 0;
}

// `shares` shares of a total, as the kernel cuts them; blocks of `units` units from `first` on, of which those up to the total are dealt.
static int block(int64_t total, int64_t shares, int64_t first, int64_t units) {
  const int64_t size = std::max<int64_t>(1, (total + shares - 1) / shares), end = std::min(first + units, total);
  const int64_t got = shares_of_block((int32_t)first, (int32_t)units, (int32_t)size, (int32_t)total);
  REQUIRE(got == (end - 1) / size - first / size + 1 && got >= 1 && first / size + got <= shares);
  if (end - first <= 4096) {  // unit by unit
    int64_t count = 0;
    for (int64_t u = first; u < end; ++u) count += u == first || u / size != (u - 1) / size;
    REQUIRE(got == count);
  }
  return 0;
}

static int blocks() {
  std::mt19937_64 rng(5);
  for (int64_t total : {(int64_t)1, (int64_t)2, (int64_t)511, (int64_t)512, (int64_t)513, (int64_t)100000, (int64_t)1 << 30})
    for (int64_t shares : {1, 2, 3, 63, 64, 512})
      for (int i = 0; i < 2000; ++i) {
        const int64_t units = 1 + (int64_t)(rng() % (i % 2 ? 40 : 1 << 23)), back = 1 + (int64_t)(rng() % (i % 3 ? 64 : total));
        if (block(total, shares, std::max<int64_t>(0, total - back), units)) return 1;
      }
  // 65536 sequences of 2176 tokens and 65536 rows, starts 0, 65536, 0, ..: 2^31 units and more in blocks of 17 are cut at 2^30, within a block
  for (int64_t shares : {64, 512})
    if (block((int64_t)1 << 30, shares, ((int64_t)1 << 30) / 17 * 17, 17)) return 1;
  return 0;
}

int main() {
  if (rows() || blocks()) return 1;
  std::puts("ok");
}
