// once_per_device.h -- what a process asks for once for each of its devices.  Host code without
// HIP: the tests compile it by itself.
#pragma once

#include <stdint.h>

#include <atomic>

namespace sieve {

// ask() where it has not yet succeeded for the device (0 is success); done: a bit a device, 64 of
// them, devices past these are asked every time.
template <typename F>
auto once_per_device(std::atomic<uint64_t>& done, int device, F ask) -> decltype(ask()) {
  const uint64_t bit = device >= 0 && device < 64 ? uint64_t(1) << device : 0;
  if (done.load(std::memory_order_acquire) & bit) return decltype(ask())(0);
  const auto status = ask();
  if (status == decltype(ask())(0)) done.fetch_or(bit, std::memory_order_release);
  return status;
}

}  // namespace sieve
