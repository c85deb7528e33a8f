// pages_handle.h - the handle of the paged MXFP4 token store.
#pragma once

#include <atomic>

#include "internal.h"

namespace chimera {
constexpr int kPagesRing = 16;                    // calls whose plans may be under way
constexpr int64_t kPagesMaxItems = (1 << 24) - 1;  // work items of a launch (256 threads each, counted in 32 bits)

struct PagesSlot {
  char *host = nullptr;  // pinned
  size_t bytes = 0;
  hipEvent_t done = nullptr;
  bool pending = false;
};
}  // namespace chimera

struct chimera_pages {
  int device = 0;
  int64_t device_bytes = 0;
  chimera::PageBook book;
  chimera::PagesView view;
  chimera::PagesSlot ring[chimera::kPagesRing];
  int next_slot = 0;
  // the last call's work, which the next call's stream waits for
  hipEvent_t done = nullptr;
  bool pending = false;
  std::atomic<int> busy{0};
};
