// Runs the code of steel_cache_wait.cuh on the host, for tests/test_cache_wait.py.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <thread>
#include <vector>

#define __device__
#define __forceinline__ inline

std::function<void()> g_before_swap;  // run once, between a look and the swap behind it
uint64_t load_acquire(const uint64_t *p) { return __atomic_load_n(p, __ATOMIC_ACQUIRE); }
uint64_t exchange_release(uint64_t *p, uint64_t value) { return __atomic_exchange_n(p, value, __ATOMIC_ACQ_REL); }
uint64_t compare_and_swap(uint64_t *p, uint64_t expected, uint64_t value) {
  if (g_before_swap) {
    const auto f = g_before_swap;
    g_before_swap = nullptr;
    f();
  }
  __atomic_compare_exchange_n(p, &expected, value, false, __ATOMIC_ACQ_REL, __ATOMIC_ACQUIRE);
  return expected;
}
thread_local long long g_clock;
long long clock64() { return ++g_clock; }

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

// Executions of one captured launch, whose token is the same each time.
void replays(uint64_t flag) {
  constexpr uint64_t token = 0x123456789abcdef1ull;
  for (int run = 0; run < 3; ++run) {
    if (steel::take_over(&flag, token, 0)) fail("a part is taken that has not been handed over in this execution");
    steel::hand_over(&flag, token);  // too late
  }
  for (int run = 0; run < 3; ++run) {
    steel::hand_over(&flag, token);
    if (!steel::take_over(&flag, token, 0)) fail("a part that is there is not taken");
  }
  for (int run = 0; run < 3; ++run) {  // it comes between the last look and the taker's word
    g_before_swap = [&] { steel::hand_over(&flag, token); };
    if (!steel::take_over(&flag, token, 0)) fail("a part that came in the last moment is lost");
  }
  long long before = g_clock;
  if (steel::take_over(&flag, token, 1000)) fail("a part is taken that has not been handed over in this execution");
  if (g_clock - before < 1000 || g_clock - before > 1010) fail("the wait does not keep its bound");
  steel::hand_over(&flag, token);
  if (steel::take_over(&flag, token, 0)) fail("a part is taken that has not been handed over in this execution");
}

// Two threads, many executions; the part is a plain number.
void threads() {
  constexpr uint64_t token = 0xfedcba9876543211ull;
  uint64_t flag = 77, part = 0;
  int taken = 0, late = 0;
  for (uint64_t run = 1; run <= 20000; ++run) {
    const auto write = [&] {
      __atomic_store_n(&part, run, __ATOMIC_RELAXED);
      steel::hand_over(&flag, token);
    };
    // too late for certain, in time for certain, or as it comes
    std::thread writer;
    if (run % 8 != 0) writer = std::thread(write);
    g_clock = 0;
    const bool got = steel::take_over(&flag, token, run % 8 == 1 ? 1ll << 60 : run % 8 * 500);
    if (got && __atomic_load_n(&part, __ATOMIC_RELAXED) != run) fail("an earlier execution's part is taken");
    ++(got ? taken : late);
    if (run % 8 == 0) write();
    else writer.join();
    if (flag == token) fail("a flag is left behind");
  }
  if (taken < 2500 || late < 2500) fail("one of the two outcomes is missing");
}

int main(int argc, char **argv) {
  const char *what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "ring")) {
    for (int steps = 1; steps < 20; ++steps)
      for (int expires = 0; expires < steps; ++expires) {
        ring<2>(steps, expires);
        ring<4>(steps, expires);
      }
  } else if (!std::strcmp(what, "replays")) {
    for (uint64_t flag : {uint64_t(0), uint64_t(1), ~uint64_t(0), uint64_t(0x7f7f7f7f7f7f7f7f)}) replays(flag);
  } else if (!std::strcmp(what, "threads")) {
    threads();
  } else {
    return 2;
  }
  return 0;
}
