// What is asked of a device once for each kernel and kept (plain C++, no CUDA).
#pragma once

#include <map>
#include <mutex>
#include <utility>

namespace unif {

// Attributes of a kernel belong to a device: an answer is kept per kernel and device.
template <typename V>
class PerDevice {
 public:
  // The answer kept for (kernel, device), or else the one that ask(&answer) gives, kept
  // where it returns true; false where it does not. May throw std::bad_alloc.
  template <typename F>
  bool get(const void* kernel, int device, V* answer, F ask) {
    std::lock_guard<std::mutex> hold(lock_);
    const auto at = kept_.find({kernel, device});
    if (at != kept_.end()) {
      *answer = at->second;
      return true;
    }
    if (!ask(answer)) return false;
    kept_[{kernel, device}] = *answer;
    return true;
  }

 private:
  std::mutex lock_;
  std::map<std::pair<const void*, int>, V> kept_;
};

}  // namespace unif
