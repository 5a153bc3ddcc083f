// What is done once on every device of the process before a kernel's first launch there: a kernel's attributes belong to a
// device, and calls without a context run on whichever device is current.  Host code only.
#pragma once

#include <mutex>

namespace ist {

template <typename T>
class OncePerDevice {
 public:
  // f()'s value, from the first call for this device on.
  template <typename F>
  T get(int device, F f) {
    if (device < 0 || device >= kDevices) return f();
    std::call_once(once_[device], [&] { value_[device] = f(); });
    return value_[device];
  }

 private:
  static constexpr int kDevices = 64;
  std::once_flag once_[kDevices];
  T value_[kDevices] = {};
};

}  // namespace ist
