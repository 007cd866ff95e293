// edge_steps.hpp built for the CPU (hip_cpu/): every edge of a row once, in
// order, also in rows of nearly 2^31 edges, and nothing after the last.
// Prints "ok".
#include <cstdio>
#include <cstdlib>

#include "edge_steps.hpp"

#define CHECK(c)                                                            \
  do {                                                                      \
    if (!(c)) {                                                             \
      std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
      std::exit(1);                                                         \
    }                                                                       \
  } while (0)

template <int U>
static void walk(int32_t beg, int32_t end) {
  const int64_t want = end > beg ? static_cast<int64_t>(end) - beg : 0;
  int64_t seen = 0;
  gmb::edge_steps<U>(beg, end, [&](int32_t e, int32_t k, auto&& at) {
    CHECK(k == want && e == seen && e < k);
    const int64_t first = beg + seen;
    for (int u = 0; u < U; ++u) {
      CHECK(at(u) == first + (u < k - e ? u : 0));
      seen += u < k - e;
    }
  });
  CHECK(seen == want);
}

int main() {
  constexpr int32_t kMost = 0x7FFFFFFF;
  for (int32_t k = 0; k < 40; ++k) walk<8>(5, 5 + k);
  walk<8>(9, 3);               // not rising: nothing
  walk<8>(kMost, kMost);
  for (int32_t k = 0; k < 20; ++k) walk<8>(kMost - k, kMost);
  walk<8>(0, kMost - 7);       // the last step is whole
  walk<8>(0, kMost);           // the step after the last is past an int32
  std::printf("ok\n");
}
