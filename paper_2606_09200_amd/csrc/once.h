// What a call sets up once and later calls of any host thread rely on.
#pragma once

#include <atomic>
#include <mutex>

namespace occ {

inline std::mutex once_lock;

// run(f): f until it has once returned true, by one host thread at a time.  Who gets true sees all that f did: a
// kernel's attribute before a launch that needs it, a structure filled in.
class Once {
 public:
  template <class F>
  bool run(F f) {
    if (done_.load(std::memory_order_acquire)) return true;
    std::lock_guard<std::mutex> hold(once_lock);
    if (done_.load(std::memory_order_relaxed)) return true;
    if (!f()) return false;
    done_.store(true, std::memory_order_release);
    return true;
  }

 private:
  std::atomic<bool> done_{false};
};

}  // namespace occ
