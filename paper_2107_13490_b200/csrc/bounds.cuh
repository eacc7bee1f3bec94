// Index checks of the bounds-checking build (-DADAPT_CHECK_BOUNDS; the stand-in for a memory
// checker): every table index that is formed from the data - a cell position from a float's
// bit pattern, a bin, a sub-cell, a queue slot, a candidate's place, a token - goes through ADAPT_IN_BOUNDS,
// which in that build skips an access outside [0, limit) and records the first such event in a device
// word of its translation unit; adapt_bounds_check_status returns them; nothing traps.  In the normal build the macro is
// `true` and the checks cost nothing.
#pragma once

#include <cuda_runtime.h>

namespace adapt {

#ifdef ADAPT_CHECK_BOUNDS
static __device__ unsigned g_bounds_error[4];   // {events, site of the first, its index, its limit}
__device__ __forceinline__ bool index_in_bounds(long long idx, long long limit, int site) {
  if (idx >= 0 && idx < limit) return true;
  if (atomicAdd(&g_bounds_error[0], 1u) == 0u) {
    g_bounds_error[1] = static_cast<unsigned>(site);
    g_bounds_error[2] = static_cast<unsigned>(idx);
    g_bounds_error[3] = static_cast<unsigned>(limit);
  }
  return false;
}
#define ADAPT_IN_BOUNDS(idx, limit, site) \
  ::adapt::index_in_bounds(static_cast<long long>(idx), static_cast<long long>(limit), (site))

// The words of all translation units, entered when the library is loaded.
constexpr int kMaxBoundsWords = 16;
inline const void* g_bounds_words[kMaxBoundsWords];
inline int g_bounds_word_count = 0;
inline bool enter_bounds_word(const void* word) {
  g_bounds_words[g_bounds_word_count++] = word;
  return true;
}
static const bool g_bounds_word_entered = enter_bounds_word(g_bounds_error);
#else
#define ADAPT_IN_BOUNDS(idx, limit, site) true
#endif

}  // namespace adapt
