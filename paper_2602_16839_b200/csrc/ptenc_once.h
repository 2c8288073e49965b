// What a launcher has to do once per device, ahead of its first launch there.
#pragma once

#include <atomic>

constexpr int PTENC_MAX_DEVICES = 64;

// One per kernel (or group of kernels), in static storage: all false at the start.
struct PtencOnce {
  std::atomic<bool> done[PTENC_MAX_DEVICES];
};

// Runs `set` unless it has succeeded on the device before; `set` returns an error code, zero for success.  Two handles may be
// used from two host threads, so the mark is made behind `set`, not in front of it: a thread that finds no mark calls `set`
// itself (setting a kernel attribute twice does no harm) and none launches ahead of the attributes.  A failure leaves no mark, and
// the next launch tries again.
template <typename Set>
inline auto ptenc_first_use(PtencOnce& once, int device, Set set) -> decltype(set()) {
  const bool known = device >= 0 && device < PTENC_MAX_DEVICES;   // an ordinal out of the table: every time
  if (known && once.done[device].load(std::memory_order_acquire)) return static_cast<decltype(set())>(0);
  const auto e = set();
  if (known && e == 0) once.done[device].store(true, std::memory_order_release);
  return e;
}
