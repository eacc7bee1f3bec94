// Dropout whose mask is never stored: y = r + [u(e) >= p 2^32] x / (1 - p), with u(e) 32 bits of a
// counter hash of (seed, layer, element number).  The backward pass is the same call on dy.
#pragma once

#include "k_elem.cuh"

namespace adapt {

struct DropoutParams {
  const void* x;
  const void* r;          // may be null
  void* y;
  long long rows, cols, ldx, ldr, ldy;
  unsigned long long base;        // hash state of pair 0: seed, domain and layer
  unsigned long long index_base;  // element number of x[0][0]
  unsigned long long threshold;   // round(p 2^32), 0..2^32
  float scale;                    // 1 / (1 - p)
};

// The 64-bit hash of pair j (elements 2j and 2j + 1): the scheme of the stochastic-rounding hash,
// with the whole final state used - the high word for the even element, the low one for the odd.
__device__ __forceinline__ unsigned long long dropout_hash(unsigned long long z) {
  z ^= z >> 32;
  z *= 0x9E3779B97F4A7C15ull;
  z ^= z >> 29;
  z *= 0xBB67AE8584CAA73Bull;
  z ^= z >> 32;
  return z;
}
constexpr unsigned long long kPairStep = 0x6A09E667F3BCC909ull;

template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutParams p) {
  const long long n = p.rows * p.cols;
  const long long stride = static_cast<long long>(gridDim.x) * blockDim.x;
  for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += stride) {
    const long long row = i / p.cols, col = i - row * p.cols;
    const unsigned long long e = p.index_base + static_cast<unsigned long long>(i);
    const unsigned long long z = dropout_hash(p.base + (e >> 1) * kPairStep);
    const unsigned u = static_cast<unsigned>((e & 1ull) ? z : z >> 32);
    const float x = to_float(static_cast<const T*>(p.x)[row * p.ldx + col]);
    float y = u >= p.threshold ? x * p.scale : 0.0f;
    if (p.r) y += to_float(static_cast<const T*>(p.r)[row * p.ldr + col]);
    static_cast<T*>(p.y)[row * p.ldy + col] = from_float<T>(y);
  }
}

}  // namespace adapt
