// The attention's division of its work (csrc/paged_shares.hpp) against the same in 64 bits, one by one: any starts of rows.
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

int main() {
  if (rows()) return 1;
  std::puts("ok");
}
