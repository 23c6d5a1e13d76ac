// keysearch.hpp -- the search for a threshold among distinct 64-bit keys that
// at least k and not many more of them reach, by counting alone: whatever the
// keys and their order, 64 counts at most.
#pragma once
#include <stdint.h>

#ifdef __HIP__
#define BART_BOTH __host__ __device__ __forceinline__
#else
#define BART_BOTH inline
#endif

namespace bart {

// At least k keys reach lo and fewer than k reach hi.  A count halves what lies
// between the two; where they are neighbours, exactly k keys reach lo.
struct KeySearch {
  uint64_t lo, hi;

  BART_BOTH uint64_t probe() const { return lo + (hi - lo) / 2; }

  // Takes the number of keys that reach `at`, the probe.
  BART_BOTH void take(uint64_t at, uint32_t count, uint32_t k) { (count < k ? hi : lo) = at; }
};

}  // namespace bart
