// Where the kernels of routed calls report that they gave up a wait: page-locked words, which the host reads without waiting.
//
// A route may be gone before the kernels launched on it are done (a function that plans, launches and returns), or before a graph
// that holds them is replayed.  So the memory of a word is never given back, and a word that the next route has got by then still tells whose
// report it holds: its owners are numbered, a kernel writes its owner's number and leaves a later owner's alone.
#pragma once
#include <cstdint>
#include <mutex>
#include <vector>

#ifdef __CUDACC__
#define GM_HOST_DEVICE __host__ __device__
#else
#define GM_HOST_DEVICE
#endif

namespace gm {

struct RouteWord {
  volatile uint32_t* at = nullptr;
  uint32_t owner = 0;
};

// By a kernel.  (Of two kernels of different owners that give up at the same moment the later owner's report could be lost; nothing on a sound
// device gives up.)
GM_HOST_DEVICE inline void route_word_report(const RouteWord& w) {
  if (static_cast<int32_t>(w.owner - *w.at) > 0) *w.at = w.owner;  // (numbers may wrap around)
}
GM_HOST_DEVICE inline bool route_word_reported(const RouteWord& w) { return *w.at == w.owner; }

class RouteWords {
 public:
  // more(bytes): memory that is never given back, or nullptr.  The result's `at` is nullptr where there is none.
  template <typename More>
  RouteWord take(const More& more) {
    std::lock_guard<std::mutex> lock(mutex_);
    if (free_.empty()) {
      constexpr int kWords = 1024;
      free_.reserve(total_ + kWords);  // (so that give() never has to grow it)
      uint32_t* slab = static_cast<uint32_t*>(more(kWords * sizeof(uint32_t)));
      if (!slab) return RouteWord{};
      total_ += kWords;
      for (int i = kWords - 1; i >= 0; --i) {
        slab[i] = 0;
        free_.push_back(RouteWord{slab + i, 0});
      }
    }
    RouteWord w = free_.back();
    free_.pop_back();
    *w.at = w.owner++;  // a report of the last owner is over
    return w;
  }
  void give(const RouteWord& w) {
    if (!w.at) return;
    std::lock_guard<std::mutex> lock(mutex_);
    free_.push_back(w);
  }

 private:
  std::mutex mutex_;
  std::vector<RouteWord> free_;  // with their last owner's number
  size_t total_ = 0;
};

}  // namespace gm
