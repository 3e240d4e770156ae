// Reads lines "units blocks threads" and prints, for each, the slices that over_slices launches as "first:count",
// or "stopped" for a launch that fails at its third slice.
#include <cstdio>

#include "slices.hpp"

int main() {
  long long units, blocks;
  int threads;
  while (std::scanf("%lld %lld %d", &units, &blocks, &threads) == 3) {
    const int rc = hmoe::over_slices(units, blocks, threads, [](int64_t first, int64_t count) {
      std::printf(" %lld:%lld", (long long)first, (long long)count);
      return 0;
    });
    int calls = 0;
    const int third = hmoe::over_slices(units, blocks, threads, [&](int64_t, int64_t) { return ++calls == 3 ? -7 : 0; });
    std::printf(" %d %d %d\n", rc, calls, third);
  }
}
