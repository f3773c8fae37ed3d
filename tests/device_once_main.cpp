// What a device needs once: tried again until it has succeeded, for every device by itself, and no thread is told that it is done
// before it is.
#include <atomic>
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>

#include "device_once.h"

static int bad = 0;
static void expect(bool fine, const char* what) {
  if (!fine) std::printf("bad: %s\n", what), ++bad;
}

int main() {
  enum Error { kFine, kFailed };
  {
    adwin::DeviceOnce once;
    int runs = 0;
    auto fails_twice = [&] { return ++runs <= 2 ? kFailed : kFine; };
    expect(once.run(3, fails_twice) == kFailed && once.run(3, fails_twice) == kFailed, "a failure is reported each time");
    expect(once.run(3, fails_twice) == kFine && runs == 3, "tried again after a failure");
    expect(once.run(3, fails_twice) == kFine && runs == 3, "not again after a success");
    expect(once.run(4, fails_twice) == kFine && runs == 4, "another device");
    for (int device : {63, 64, -1}) {
      runs = 2;
      expect(once.run(device, fails_twice) == kFine && once.run(device, fails_twice) == kFine, "success");
      expect(runs == (device == 63 ? 3 : 4), "devices that no bit stands for are prepared every time");
    }
  }
  {
    adwin::DeviceOnce once;
    std::mutex m;
    std::condition_variable changed;
    bool inside = false, go_on = false;
    std::atomic<int> prepared{0};
    std::thread first([&] {
      once.run(0, [&] {
        std::unique_lock<std::mutex> lock(m);
        inside = true;
        changed.notify_all();
        changed.wait(lock, [&] { return go_on; });
        ++prepared;
        return kFine;
      });
    });
    {
      std::unique_lock<std::mutex> lock(m);
      changed.wait(lock, [&] { return inside; });
    }
    // the first thread is preparing the device and has not done so
    expect(once.run(0, [&] { ++prepared; return kFine; }) == kFine && prepared == 1, "the device is prepared when a call returns");
    {
      std::lock_guard<std::mutex> lock(m);
      go_on = true;
    }
    changed.notify_all();
    first.join();
    expect(once.run(0, [&] { ++prepared; return kFine; }) == kFine && prepared == 2, "and stays so");
  }
  std::printf(bad ? "bad\n" : "ok\n");
  return bad != 0;
}
