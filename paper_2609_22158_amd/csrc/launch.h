// What a launch takes.
#pragma once

#include <stdint.h>

namespace stepkv {

// A launch has fewer than 2^32 threads: of more, it runs the first modulo 2^32 and
// reports no error.
inline bool grid_fits(int64_t workgroups, int threads) {
  return workgroups <= (int64_t)UINT32_MAX / threads;
}

}  // namespace stepkv
