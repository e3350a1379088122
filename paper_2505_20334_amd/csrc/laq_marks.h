// The numbers that launches mark their finished work with in a workspace that comes as the allocator left it.  Plain C++: tested on the host.
#pragma once

#include <atomic>
#include <chrono>
#include <cstdint>

namespace laq {

// One to one on 64 bits: the finalizer of SplitMix64 (Steele, Lea, Flood: Fast splittable pseudorandom number generators, 2014).
constexpr uint64_t mixed(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

// A process's launches count through all 64 bits from a start of their own, and a mark is the mixed count: no two launches have the same one, and a word that
// something else left in the workspace is a given launch's mark with a probability of 2^-64.  Words whose upper half is 0, which small integers and numbers beside a zero
// have (and marks that were cleared), are none at all.
class MarkNumbers {
 public:
  explicit MarkNumbers(uint64_t start) : count(start) {}
  MarkNumbers()
      : MarkNumbers(mixed((uint64_t)std::chrono::steady_clock::now().time_since_epoch().count()) ^
                    mixed((uint64_t)std::chrono::system_clock::now().time_since_epoch().count() + reinterpret_cast<uintptr_t>(this))) {}
  uint64_t next() {
    uint64_t x;
    do x = mixed(count.fetch_add(1)); while (x >> 32 == 0);
    return x;
  }

 private:
  std::atomic<uint64_t> count;
};

}  // namespace laq
