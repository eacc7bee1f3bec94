// Dropout whose mask is never stored: y = r + [u(e) >= p 2^32] x / (1 - p), with u(e) 32 bits of a
// counter hash of (seed, layer, element number).  The backward pass is the same call on dy.
//
// What bounds it: HBM (x and r read, y written once); the hash costs about 16 lane instructions for two
// elements, half of what the memory rate leaves room for with 16-bit elements.
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kDropoutThreads = 256;

struct DropoutParams {
  const void* x;
  const void* r;          // may be null
  void* y;
  long long cols, ldx, ldr, ldy;
  unsigned chunks;        // of 16 bytes of x, or of two elements, over all rows
  unsigned per_row;       // chunks of a row (the most that any alignment needs)
  unsigned magic, shift;  // i / per_row = (i * magic >> 32) >> shift
  unsigned from, to;      // one row: its whole chunks
  int mis;                // one row: elements of chunk 0 that lie before it
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

// A chunk is 16 bytes where the rows of x, r and y lie alike to the 16-byte boundary (kCount = 16 /
// sizeof(T)), a hash's pair of elements otherwise (kCount = 2; then neighbouring threads read and write
// neighbouring pairs: 4099 x 1001 fp16 into rows of another alignment takes 7 us, 17 with 8 elements a
// thread).  Chunks over a row's ends go element by element.  kRows: several rows.
template <typename T, int kCount, bool kResidual, bool kRows>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const DropoutParams p) {
  constexpr bool kVec = kCount * sizeof(T) == 16;
  constexpr int kUnroll = kVec ? 2 : 4;
  const unsigned first = blockIdx.x * (kDropoutThreads * kUnroll) + threadIdx.x;
  const T *x[kUnroll], *r[kUnroll];
  T* y[kUnroll];
  long long e[kUnroll];        // number of the chunk's first element (kRows)
  int from[kUnroll], to[kUnroll];   // its elements that exist
  uint4 vx[kUnroll], vr[kUnroll];
  T sx[kUnroll][2], sr[kUnroll][2];
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    const unsigned c = first + i * kDropoutThreads;
    from[i] = 0;
    to[i] = kCount;
    if (kRows) {
      const unsigned row = __umulhi(c, p.magic) >> p.shift;
      const unsigned q = c - row * p.per_row;
      const T* start = static_cast<const T*>(p.x) + row * p.ldx;
      const long long number = p.index_base + row * p.cols;
      const int mis = kVec ? static_cast<int>((reinterpret_cast<uintptr_t>(start) & 15u) / sizeof(T)) : static_cast<int>(number & 1);
      const int col = static_cast<int>(q) * kCount - mis, cols = static_cast<int>(p.cols);
      x[i] = start + col;
      y[i] = static_cast<T*>(p.y) + row * p.ldy + col;
      if (kResidual) r[i] = static_cast<const T*>(p.r) + row * p.ldr + col;
      e[i] = number + col;
      from[i] = max(0, -col);
      to[i] = min(kCount, cols - col);
    } else {
      const long long col = static_cast<long long>(c) * kCount - p.mis;
      x[i] = static_cast<const T*>(p.x) + col;
      y[i] = static_cast<T*>(p.y) + col;
      if (kResidual) r[i] = static_cast<const T*>(p.r) + col;
      if (c < p.from || c >= p.to) {
        from[i] = c == 0 ? p.mis : 0;
        to[i] = static_cast<int>(min(static_cast<long long>(kCount), p.cols - col));
      }
    }
    if (c >= p.chunks) to[i] = 0;
    if (kVec) {
      if (to[i] - from[i] == kCount) {
        vx[i] = *reinterpret_cast<const uint4*>(x[i]);
        if (kResidual) vr[i] = *reinterpret_cast<const uint4*>(r[i]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool on = k >= from[i] && k < to[i];
        sx[i][k] = on ? x[i][k] : from_float<T>(0.0f);
        if (kResidual) sr[i][k] = on ? r[i][k] : from_float<T>(0.0f);
      }
    }
  }
  const unsigned least = p.none ? 1u : p.threshold;
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    if (to[i] <= from[i]) continue;
    const unsigned c = first + i * kDropoutThreads;
    unsigned u[kCount];
    const long long number = kRows ? e[i] : p.index_base - p.mis + static_cast<long long>(c) * kCount;
    dropout_words<kCount>(p.base, number, u);
    if (p.none) {
#pragma unroll
      for (int k = 0; k < kCount; ++k) u[k] = 0;
    }
    if (kVec && to[i] - from[i] == kCount) {
      float f[kCount], g[kCount];
      unpack16<T>(vx[i], *reinterpret_cast<float(*)[16 / sizeof(T)]>(&f));
      if (kResidual) unpack16<T>(vr[i], *reinterpret_cast<float(*)[16 / sizeof(T)]>(&g));
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        f[k] = u[k] >= least ? f[k] * p.scale : 0.0f;
        if (kResidual) f[k] += g[k];
      }
      *reinterpret_cast<uint4*>(y[i]) = pack16<T>(*reinterpret_cast<float(*)[16 / sizeof(T)]>(&f));
    } else {
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        if (k < from[i] || k >= to[i]) continue;
        float f = u[k] >= least ? to_float(kVec ? x[i][k] : sx[i][k & 1]) * p.scale : 0.0f;
        if (kResidual) f += to_float(kVec ? r[i][k] : sr[i][k & 1]);
        y[i][k] = from_float<T>(f);
      }
    }
  }
}

}  // namespace adapt
