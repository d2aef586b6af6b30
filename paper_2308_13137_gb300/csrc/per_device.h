// Work that is done once for each device of the process: a function's attribute, a device's properties.  Both
// belong to the current device, and a process may run on several.
#pragma once
#include <atomic>
#include <cstdint>

// Calls set() unless it has already returned true for device dev under this flag; false when it fails.  Devices
// beyond the 64 of the flag are set at every call.  (Two threads may both set: it is idempotent.)
template <class F>
inline bool omq_once_per_device(std::atomic<uint64_t>& done, int dev, F set) {
  const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (bit && (done.load(std::memory_order_acquire) & bit)) return true;
  if (!set()) return false;
  done.fetch_or(bit, std::memory_order_release);
  return true;
}

// The value of get() for device dev, asked once; get() must not return 0.
template <class F>
inline int omq_value_per_device(std::atomic<int> (&known)[64], int dev, F get) {
  if (dev < 0 || dev >= 64) return get();
  int v = known[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    v = get();
    known[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}
