// Settings of the host runtime that a device needs once (a kernel's shared-memory limit belongs to the
// device that was current when it was set). Plain C++, so that it can be tested without a GPU.
#pragma once
#include <atomic>

namespace fd {

class OncePerDevice {
 public:
  // set() unless it has succeeded (returned zero) for this device before. A failure is returned
  // and not kept: the next call tries again. Two threads may both set: the setting is the same.
  template <class Set>
  auto run(int device, Set set) -> decltype(set()) {
    const bool known = device >= 0 && device < kDevices;
    if (known && done_[device].load(std::memory_order_acquire)) return {};
    const auto e = set();
    if (known && e == decltype(set()){}) done_[device].store(true, std::memory_order_release);
    return e;
  }

 private:
  static constexpr int kDevices = 64;
  std::atomic<bool> done_[kDevices] = {};
};

}  // namespace fd
