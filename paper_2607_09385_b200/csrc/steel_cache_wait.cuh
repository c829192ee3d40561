// The bounded waits of the cache's attention: how a part is handed from one CTA to another, and what happens when a wait has expired.
// (load_acquire, exchange_release, compare_and_swap and clock64 are those of sm100_ptx.cuh, or what tests/cache_wait.cpp
// declares, which runs the code on the host.)
#pragma once

namespace steel {

// A warp's wait for step i of its ring has expired.  Copies go into the ring for steps i ... i + kStages - 1, as far as there are any: each is
// awaited once more, step i's with the others, before anything else uses its place.
template <int kStages, class Wait>
__device__ __forceinline__ void await_copies(int i, int steps, Wait &&wait) {
  for (int j = i; j < i + kStages && j < steps; ++j) wait(j);
}

// A part of a segment is handed over once in a launch, by one thread, and taken once, by another: its flag becomes the launch's token, which is
// odd and which memory does not hold by chance.  Nobody clears flags, and a launch in a graph has the same token each time, so whoever
// comes second leaves a flag that means nothing: the taker clears what it has seen, and one whose wait has expired says so, for the other to clear.
// Without that a part that came too late was taken at once by the next replay, while it was being written.
__device__ __forceinline__ uint64_t given_up(uint64_t token) { return token - 1; }

__device__ __forceinline__ void hand_over(uint64_t *flag, uint64_t token) {
  if (exchange_release(flag, token) == given_up(token)) *flag = 0;
}

// Waits for `limit` cycles at most, looking at least once; whether the part is there.
__device__ __forceinline__ bool take_over(uint64_t *flag, uint64_t token, long long limit) {
  const long long since = clock64();
  for (;;) {
    const uint64_t seen = load_acquire(flag);
    if (seen == token) break;
    // the part may come between the look and the word that nobody waits for it: then it is taken
    if (clock64() - since >= limit && compare_and_swap(flag, seen, given_up(token)) == seen) return false;
  }
  *flag = 0;
  return true;
}

}  // namespace steel
