// A number above 0 that the driver is asked for once per device.
#pragma once

#include <atomic>

namespace mtf {

class KnownPerDevice {
  static constexpr int kDevices = 64;
  std::atomic<int> known_[kDevices] = {};

 public:
  // ask(): the number, or 0 where the question failed.  That is not kept: this call has 0, the next one asks again.
  template <typename Ask>
  int get(int device, Ask ask) {
    if (device < 0 || device >= kDevices) return ask();
    int n = known_[device].load(std::memory_order_relaxed);
    if (n <= 0) {
      n = ask();
      if (n > 0) known_[device].store(n, std::memory_order_relaxed);
    }
    return n;
  }
};

}  // namespace mtf
