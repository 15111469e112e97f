// An answer that the device gives the same every time, asked for until it has come once.
#pragma once

#include <atomic>

namespace adaption {

// The answer kept in `slot` (0: none yet), else what ask() returns.  0 from ask() says that the question failed: then the answer is
// `guess`, which is not kept, so that one failure does not decide for the rest of the process.
template <typename Ask>
int remembered(std::atomic<int>& slot, int guess, const Ask& ask) {
  const int known = slot.load(std::memory_order_relaxed);
  if (known > 0) return known;
  const int n = ask();
  if (n <= 0) return guess;
  slot.store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace adaption
