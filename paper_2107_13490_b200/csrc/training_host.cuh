// Host side that the training-step operators' entry points share.
#pragma once

#include <cstdint>

#include "../../include/adapt.h"
#include "host.cuh"
#include "k_elem.cuh"

namespace adapt {

// Bytes of an element, 0 for an unknown type.
inline int elem_bytes(int dtype) {
  return dtype == ADAPT_DTYPE_F32 ? 4 : (dtype == ADAPT_DTYPE_F16 || dtype == ADAPT_DTYPE_BF16) ? 2 : 0;
}

inline bool misaligned(const void* p, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(bytes - 1)) != 0;
}

// Calls f(T{}) with the element type.
template <typename F>
inline void with_type(int dtype, F f) {
  if (dtype == ADAPT_DTYPE_F32) f(float{});
  else if (dtype == ADAPT_DTYPE_F16) f(__half{});
  else f(__nv_bfloat16{});
}

}  // namespace adapt
