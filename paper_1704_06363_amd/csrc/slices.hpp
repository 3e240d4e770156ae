// slices.hpp -- problems of more workgroups than a launch holds: fewer than 2^32 threads.
#pragma once
#include <stdint.h>

namespace hmoe {

// launch(first, count) over slices of `units`, each of them `blocks` workgroups of `threads` (fewer than 2^32 threads
// together); stops at the first code that is not 0 and returns it.
template <typename F>
int over_slices(int64_t units, int64_t blocks, int threads, F launch) {
  const int64_t most = ((int64_t(1) << 32) - 1) / (blocks * threads);
  for (int64_t u = 0; u < units; u += most) {
    const int rc = launch(u, units - u < most ? units - u : most);
    if (rc != 0) return rc;
  }
  return 0;
}

}  // namespace hmoe
