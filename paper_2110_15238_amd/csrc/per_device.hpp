// What differs from one GPU to the next (a device variable's address), looked up once for each.
#pragma once
#include <mutex>

namespace bolt {

struct PerDevice {
  static constexpr int kMaxDevices = 64;
  std::once_flag once[kMaxDevices];
  void* at[kMaxDevices] = {};
  // lookup(): the address on `device`, which is the current one; null where there is none.
  template <typename F>
  void* get(int device, F&& lookup) {
    if (device < 0 || device >= kMaxDevices) return nullptr;
    std::call_once(once[device], [&] { at[device] = lookup(); });
    return at[device];
  }
};

}  // namespace bolt
