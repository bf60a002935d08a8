// A grid in as many launches as it takes (host code).
#pragma once

#include <stdint.h>

namespace lmz {

// HIP launches fewer than 2^32 threads at once: 2^24 - 1 workgroups of 256. launch(first, n)
// sends out the workgroups from number `first` on, n of them, and returns LM_OK or an error,
// which ends the calls.
template <typename F>
static inline int launch_parts(int64_t blocks, int threads, F launch) {
  const int64_t most = ((int64_t(1) << 32) - 1) / threads;
  for (int64_t first = 0; first < blocks; first += most) {
    const int64_t left = blocks - first;
    if (const int rc = launch(static_cast<uint32_t>(first),
                              static_cast<uint32_t>(left < most ? left : most)))
      return rc;
  }
  return 0;
}

}  // namespace lmz
