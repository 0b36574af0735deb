// What has to be done once per device before a kernel's first launch there (function attributes are per device, not per
// process).  It counts as done when it has succeeded, not when somebody has begun it: a second host thread does it again
// rather than launch too early, and what failed is tried again.
#pragma once
#include <atomic>

namespace rpo {

struct OncePerDevice {
  static constexpr int DEVICES = 64;       // on devices behind them it is done every time
  std::atomic<bool> done[DEVICES] = {};

  // set() returns an error code, 0 for success.
  template <typename F>
  auto run(int device, F set) -> decltype(set()) {
    const bool known = device >= 0 && device < DEVICES;
    if (known && done[device].load(std::memory_order_acquire)) return decltype(set())(0);
    const auto rc = set();
    if (known && rc == decltype(set())(0)) done[device].store(true, std::memory_order_release);
    return rc;
  }
};

}  // namespace rpo
