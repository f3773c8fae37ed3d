// What a device needs once before a launch (host code alone).
#pragma once
#include <stdint.h>

#include <atomic>

namespace adwin {

// `prepare` runs until it has succeeded once for a device, and a call returns only when it has: a thread that comes while another one
// prepares the device prepares it as well, which has to be harmless.  Devices beyond 63 are prepared every time.
class DeviceOnce {
 public:
  template <typename Prepare>
  auto run(int device, Prepare prepare) -> decltype(prepare()) {
    const uint64_t bit = device >= 0 && device < 64 ? (uint64_t)1 << device : 0;
    if (done_.load(std::memory_order_acquire) & bit) return {};
    const auto error = prepare();
    if (error == decltype(prepare()){}) done_.fetch_or(bit, std::memory_order_release);
    return error;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

}  // namespace adwin
