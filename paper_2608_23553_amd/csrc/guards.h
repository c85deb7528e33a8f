// guards.h - what the C entry points share: the caller's device kept, a handle
// marked busy, exceptions turned into status codes.
#pragma once

#include <new>

#include "internal.h"

namespace chimera {

// Restores the caller's current device on scope exit.
struct DeviceGuard {
  int prev = -1;
  bool ok = false;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) {
      prev = -1;
    } else if (prev == dev) {
      prev = -1;  // nothing to restore
      ok = true;
    } else {
      ok = hipSetDevice(dev) == hipSuccess;
    }
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

// Marks a handle busy for the duration of a host call (none: nothing to mark).
template <class H>
struct BusyGuard {
  H *h;
  bool ok;
  explicit BusyGuard(H *handle) : h(handle), ok(!handle || handle->busy.exchange(1) == 0) {}
  ~BusyGuard() {
    if (ok && h) h->busy.store(0);
  }
};

// No C++ exception leaves the C ABI: host allocations inside a call that fail
// report E_NOMEM.
template <class F>
static int guarded(F &&f) {
  try {
    return f();
  } catch (const std::bad_alloc &) {
    return fail(CHIMERA_E_NOMEM, "host allocation failed");
  } catch (...) {
    return fail(CHIMERA_E_INVAL, "internal error");
  }
}

}  // namespace chimera
