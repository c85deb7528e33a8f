// pages_handle.h - the handle of the paged MXFP4 token store.
#pragma once

#include <atomic>

#include "internal.h"

namespace chimera {
constexpr int64_t kPagesMaxItems = (1 << 24) - 1;  // work items of a launch (256 threads each, counted in 32 bits)

// Pinned host memory that calls' plans lie in, taken from the front to the back
// of two halves in turn.  Behind the last call of a half an event is recorded;
// the half is used again once that has passed.  Small plans are read by the
// kernels from there, larger ones from a copy at the same place of `dev`.
struct PlanRing {
  char *host = nullptr, *dev = nullptr;
  size_t half = 0;  // bytes of each half
  size_t used = 0;  // of the current half
  int cur = 0;
  hipEvent_t left[2] = {nullptr, nullptr};
  bool pending[2] = {false, false};
};
}  // namespace chimera

struct chimera_pages {
  int device = 0;
  int64_t device_bytes = 0;
  chimera::PageBook book;
  chimera::PagesView view;
  chimera::PlanRing ring;
  // The last call's work, which a call on another stream waits for: an event on
  // its stream or, where that was the null stream, none yet.  Work on the null
  // stream is in order by itself and that stream cannot be destroyed, so the
  // event (5.7 us of host time, twice a launch) is left until it is needed.
  hipEvent_t done = nullptr;
  bool pending = false, on_null = false;
  std::atomic<int> busy{0};
};
