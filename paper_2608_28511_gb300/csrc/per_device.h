// What a launch sets up once on every device (opting a kernel in to its shared
// memory, counting how many clusters fit): function attributes belong to a
// device, and several host threads may launch at once.  No CUDA in here.
#pragma once

#include <atomic>

namespace moe {

constexpr int kMaxDevices = 64;

// A value of at least 0 for each device.  Threads that come first together may
// each set up the device; the set-up has to give all of them the same.
class PerDevice {
 public:
  // The value of device `dev` (0 .. kMaxDevices - 1).  Unless it is known, setup(&value)
  // finds it and returns a status; any but `ok` is returned, and the next call tries again.
  template <typename Status, typename F>
  Status get(int dev, Status ok, int* value, F setup) {
    const int known = plus1_[dev].load(std::memory_order_acquire);
    if (known) {
      *value = known - 1;
      return ok;
    }
    const Status st = setup(value);
    if (st == ok) plus1_[dev].store(*value + 1, std::memory_order_release);
    return st;
  }

 private:
  std::atomic<int> plus1_[kMaxDevices] = {};
};

}  // namespace moe
