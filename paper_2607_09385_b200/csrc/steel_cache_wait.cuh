// What the cache's attention does when a bounded wait has expired.  tests/cache_wait.cpp runs the code on the host.
#pragma once

namespace steel {

// A warp's wait for step i of its ring has expired.  Copies go into the ring for steps i ... i + kStages - 1, as far as there are any: each is
// awaited once more, step i's with the others, before anything else uses its place.
template <int kStages, class Wait>
__device__ __forceinline__ void await_copies(int i, int steps, Wait &&wait) {
  for (int j = i; j < i + kStages && j < steps; ++j) wait(j);
}

}  // namespace steel
