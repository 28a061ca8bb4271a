// What launchers keep between calls, for each device by itself and whatever threads call (no CUDA in here: the tests
// compile it for the host).
#pragma once
#include <atomic>
#include <stdint.h>

namespace jab {

constexpr int kDevices = 64;  // (a device past these is set up by every call)

// Whether a device has been set up. Two threads may set it up at once: they do the same.
class SetUp {
  std::atomic<bool> done_[kDevices];

 public:
  SetUp() {
    for (auto& d : done_) d.store(false, std::memory_order_relaxed);
  }
  // f() sets the current device, `dev`, up and returns its status, 0 if it could; the next call tries again what failed.
  template <class F>
  auto once(int dev, F f) -> decltype(f()) {
    const bool known = dev >= 0 && dev < kDevices;
    if (known && done_[dev].load(std::memory_order_acquire)) return decltype(f())(0);
    const auto status = f();
    if (known && status == 0) done_[dev].store(true, std::memory_order_release);
    return status;
  }
};

// Numbers found out for a device and a key, the latest of each eight keys: key and number are one word.
class Found {
  static constexpr int kSlots = 8;
  std::atomic<uint64_t> word_[kDevices][kSlots];  // (key + 1) << 32 | number; 0: empty

 public:
  Found() {
    for (auto& d : word_)
      for (auto& w : d) w.store(0, std::memory_order_relaxed);
  }
  // f() finds the number of `key` (0 .. 2^31) on the current device, `dev`; one that is not positive is not kept.
  template <class F>
  int get(int dev, uint32_t key, F f) {
    const bool known = dev >= 0 && dev < kDevices;
    if (known) {
      const uint64_t w = word_[dev][key % kSlots].load(std::memory_order_relaxed);
      if (w >> 32 == (uint64_t)key + 1) return (int)(uint32_t)w;
    }
    const int n = f();
    if (known && n > 0) word_[dev][key % kSlots].store(((uint64_t)key + 1) << 32 | (uint32_t)n, std::memory_order_relaxed);
    return n;
  }
};

}  // namespace jab
