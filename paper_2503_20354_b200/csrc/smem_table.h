// Which kernels have been allowed how much dynamic shared memory on which device.  Host code without CUDA, so that it can be
// tested by itself.
#pragma once

#include <atomic>
#include <mutex>

namespace surgeon {

class SmemTable {
 public:
  static constexpr int kDevices = 64, kKernels = 512;            // (the library has some 200 kernels that ask for it)
  static constexpr int kNoRoom = -1;

  // Sees to it that `kernel` may use `bytes` on device `dev`: set(bytes) is called where it may not yet, and its result returned if
  // it is not 0.  Attribute and entry change together under the lock and only grow: what was allowed once stays allowed, in
  // whichever order threads ask for larger and smaller sizes.
  template <typename Set>
  int allow(const void* kernel, int dev, int bytes, Set&& set) {
    if (dev < 0 || dev >= kDevices) return kNoRoom;
    Device& d = devices_[dev];
    if (allowed(d, d.n.load(std::memory_order_acquire), kernel, bytes)) return 0;
    const std::lock_guard<std::mutex> hold(lock_);
    const int n = d.n.load(std::memory_order_relaxed);
    if (allowed(d, n, kernel, bytes)) return 0;
    Entry* e = find(d, n, kernel);
    if (!e && n == kKernels) return kNoRoom;
    if (const int failed = set(bytes)) return failed;
    if (e) {
      e->bytes.store(bytes, std::memory_order_release);
    } else {
      d.entries[n].kernel = kernel;
      d.entries[n].bytes.store(bytes, std::memory_order_relaxed);
      d.n.store(n + 1, std::memory_order_release);
    }
    return 0;
  }

 private:
  struct Entry {
    const void* kernel;
    std::atomic<int> bytes;
  };
  struct Device {
    Entry entries[kKernels];
    std::atomic<int> n;
  };
  static Entry* find(Device& d, int n, const void* kernel) {
    for (int i = 0; i < n; ++i)
      if (d.entries[i].kernel == kernel) return &d.entries[i];
    return nullptr;
  }
  static bool allowed(Device& d, int n, const void* kernel, int bytes) {
    const Entry* e = find(d, n, kernel);
    return e && e->bytes.load(std::memory_order_acquire) >= bytes;
  }
  Device devices_[kDevices] = {};
  std::mutex lock_;
};

}  // namespace surgeon
