// Host side that the entry points of the training-step operators and of those around the layers share.
#pragma once

#include <cstdint>

#include "../../include/adapt.h"
#include "host.cuh"
#include "k_elem.cuh"

namespace adapt {

// SMs of a B200.  A constant: workspaces are sized without a device, and grids and cuts go by the same number.
constexpr int kSms = 148;

// Whether a size is in a kernel's reach (with room for what is added to it before it is compared).
inline bool in_int(int64_t v, int64_t least) { return v >= least && v <= (1 << 30); }

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
