// Dropout whose mask is never stored: y = r + [u(e) >= p 2^32] x / (1 - p), with u(e) 32 bits of a
// counter hash of (seed, layer, element number).  The backward pass is the same call on dy.
//
// What bounds it: HBM (x and r read, y written once); the hash costs about 16 lane instructions for two
// elements, half of what the memory rate leaves room for with 16-bit elements.
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kDropoutThreads = 256;
constexpr int kDropoutUnroll = 2;   // chunks of 16 bytes of a thread

struct DropoutParams {
  const void* x;
  const void* r;          // may be null
  void* y;
  long long cols, ldx, ldr, ldy;
  unsigned chunks;        // of 16 bytes of x, over all rows
  unsigned per_row;       // chunks of a row (the most that any alignment needs)
  unsigned magic, shift;  // i / per_row = (i * magic >> 32) >> shift, magic 0: one row
  unsigned long long base;        // hash state of pair 0: seed, domain and layer
  long long index_base;           // element number of x[0][0]
  unsigned threshold;             // round(p 2^32), held below 2^32
  bool none;                      // p = 1: nothing is kept
  float scale;                    // 1 / (1 - p)
};

// The 64-bit hash of pair j (elements 2j and 2j + 1): the scheme of the stochastic-rounding hash,
// with the whole final state used - the high word for the even element, the low one for the odd.
__device__ __forceinline__ uint2 dropout_hash(unsigned long long z) {
  z ^= z >> 32;
  z *= 0x9E3779B97F4A7C15ull;
  z ^= z >> 29;
  z *= 0xBB67AE8584CAA73Bull;
  const unsigned high = static_cast<unsigned>(z >> 32);
  return make_uint2(high, static_cast<unsigned>(z) ^ high);
}
constexpr unsigned long long kPairStep = 0x6A09E667F3BCC909ull;

// The words of kCount elements from number e on (which may lie before element 0: those are not used).
template <int kCount>
__device__ __forceinline__ void dropout_words(unsigned long long base, long long e, unsigned (&u)[kCount]) {
  const unsigned long long z = base + static_cast<unsigned long long>(e >> 1) * kPairStep;
  if ((e & 1) == 0) {
#pragma unroll
    for (int k = 0; k < kCount; k += 2) {
      const uint2 w = dropout_hash(z + (k / 2) * kPairStep);
      u[k] = w.x; u[k + 1] = w.y;
    }
  } else {
    u[0] = dropout_hash(z).y;
#pragma unroll
    for (int k = 1; k < kCount; k += 2) {
      const uint2 w = dropout_hash(z + ((k + 1) / 2) * kPairStep);
      u[k] = w.x;
      if (k + 1 < kCount) u[k + 1] = w.y;
    }
  }
}

// kVec: rows of x, r and y lie alike to the 16-byte boundary, so a chunk moves as a whole; chunks over a
// row's ends, and all of them otherwise, go element by element.
template <typename T, bool kVec, bool kResidual>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const DropoutParams p) {
  constexpr int kCount = 16 / sizeof(T);
  const unsigned first = blockIdx.x * (kDropoutThreads * kDropoutUnroll) + threadIdx.x;
  const T *x[kDropoutUnroll], *r[kDropoutUnroll];
  T* y[kDropoutUnroll];
  long long col[kDropoutUnroll];
  long long e[kDropoutUnroll];
  bool whole[kDropoutUnroll];
  uint4 vx[kDropoutUnroll], vr[kDropoutUnroll];
#pragma unroll
  for (int i = 0; i < kDropoutUnroll; ++i) {
    const unsigned c = first + i * kDropoutThreads;
    const unsigned row = p.magic ? __umulhi(c, p.magic) >> p.shift : 0u;
    const unsigned q = c - row * p.per_row;
    const T* start = static_cast<const T*>(p.x) + row * p.ldx;
    const int mis = kVec ? static_cast<int>((reinterpret_cast<uintptr_t>(start) & 15u) / sizeof(T)) : 0;
    col[i] = static_cast<long long>(q) * kCount - mis;
    x[i] = start + col[i];
    y[i] = static_cast<T*>(p.y) + row * p.ldy + col[i];
    r[i] = kResidual ? static_cast<const T*>(p.r) + row * p.ldr + col[i] : nullptr;
    e[i] = p.index_base + static_cast<long long>(row) * p.cols + col[i];
    const bool on = c < p.chunks;
    whole[i] = kVec && on && col[i] >= 0 && col[i] + kCount <= p.cols;
    if (!on) col[i] = p.cols;   // no element of it exists
    if (whole[i]) {
      vx[i] = *reinterpret_cast<const uint4*>(x[i]);
      if (kResidual) vr[i] = *reinterpret_cast<const uint4*>(r[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kDropoutUnroll; ++i) {
    if (col[i] >= p.cols) continue;
    unsigned u[kCount];
    dropout_words<kCount>(p.base, e[i], u);
    if (p.none) {
#pragma unroll
      for (int k = 0; k < kCount; ++k) u[k] = 0;
    }
    const unsigned least = p.none ? 1u : p.threshold;
    if (whole[i]) {
      float f[kCount], g[kCount];
      unpack16<T>(vx[i], f);
      if (kResidual) unpack16<T>(vr[i], g);
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        f[k] = u[k] >= least ? f[k] * p.scale : 0.0f;
        if (kResidual) f[k] += g[k];
      }
      *reinterpret_cast<uint4*>(y[i]) = pack16<T>(f);
    } else {
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        if (col[i] + k < 0 || col[i] + k >= p.cols) continue;
        float f = u[k] >= least ? to_float(x[i][k]) * p.scale : 0.0f;
        if (kResidual) f += to_float(r[i][k]);
        y[i][k] = from_float<T>(f);
      }
    }
  }
}

}  // namespace adapt
