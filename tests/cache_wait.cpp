// Runs the code of steel_cache_wait.cuh on the host, for tests/test_cache_wait.py.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#define __device__
#define __forceinline__ inline

#include "../paper_2607_09385_b200/csrc/steel_cache_wait.cuh"

[[noreturn]] void fail(const char *what) {
  std::printf("%s\n", what);
  std::fflush(stdout);
  std::_Exit(1);
}

// A warp that goes through `steps` steps as the kernel does, and whose wait for step `expires` runs out: which copies are in flight then?
template <int S>
void ring(int steps, int expires) {
  std::vector<bool> flying(steps, false);
  for (int i = -S; i < steps; ++i) {
    if (i >= 0) {
      if (i == expires) {
        steel::await_copies<S>(i, steps, [&](int j) {
          if (j < 0 || j >= steps || !flying[j]) fail("a wait for a copy that nobody has asked for");
          flying[j] = false;
        });
        break;
      }
      flying[i] = false;
    }
    if (i + S < steps) flying[i + S] = true;
  }
  for (bool f : flying)
    if (f) fail("the warp goes on while a copy is in flight");
}

int main(int argc, char **argv) {
  const char *what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "ring")) {
    for (int steps = 1; steps < 20; ++steps)
      for (int expires = 0; expires < steps; ++expires) {
        ring<2>(steps, expires);
        ring<4>(steps, expires);
      }
  } else {
    return 2;
  }
  return 0;
}
