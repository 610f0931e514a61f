// What is asked of a device once and then known, by calls that may come from several threads.  Plain C++.
#pragma once
#include <atomic>

template <int DEVICES>
class KnownNumbers {
  std::atomic<int> known[DEVICES] = {};

 public:
  // The number of device `dev`, positive, from `ask` the first time (threads that come at once ask each for themselves and get
  // the same); what is not positive is not kept.
  template <typename Ask> int of(int dev, Ask ask) {
    const int have = known[dev].load(std::memory_order_relaxed);
    if (have > 0) return have;
    const int n = ask();
    if (n > 0) known[dev].store(n, std::memory_order_relaxed);
    return n;
  }
};
