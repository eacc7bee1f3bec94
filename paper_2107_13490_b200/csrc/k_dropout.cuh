// Dropout whose mask is never stored: y = r + [u(e) >= p 2^32] x / (1 - p), with u(e) 32 bits of a
// counter hash of (seed, layer, element number).  The backward pass is the same call on dy.
//
// What bounds it: HBM (x and r read, y written once); the hash costs about 16 lane instructions for two
// elements, half of what the memory rate leaves room for with 16-bit elements.
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kDropoutThreads = 256;
constexpr int kDropoutUnroll = 2, kShiftUnroll = 1;   // chunks of a thread (kShift with 2 is within 2 % of 1)
constexpr int kPairsUnroll = 4;                       // pairs of a thread
constexpr int kPairsBelow = 16;                       // shorter rows of other alignments go in pairs

struct DropoutParams {
  const void* x;
  const void* r;          // may be null
  void* y;
  const void *x_end, *r_end;
  long long cols, ldx, ldr, ldy;
  unsigned chunks;        // of 16 bytes of y, over all rows
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

// 16 bytes from any address: the aligned blocks that hold them (the second only where it is needed, so that
// an operand that lies like y - the one y may be - is read by the thread that writes it).  False, and nothing
// read, where a block reaches beyond the operand.
__device__ __forceinline__ bool fetch_blocks(const void* from, const void* begin, const void* end, uint4& low, uint4& high) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(from), block = a & ~static_cast<uintptr_t>(15);
  const bool two = (a & 15u) != 0;
  if (block < reinterpret_cast<uintptr_t>(begin) || block + (two ? 32 : 16) > reinterpret_cast<uintptr_t>(end)) return false;
  low = *reinterpret_cast<const uint4*>(block);
  high = two ? *reinterpret_cast<const uint4*>(block + 16) : make_uint4(0u, 0u, 0u, 0u);
  return true;
}
__device__ __forceinline__ uint4 join_blocks(const uint4& low, const uint4& high, const void* from) {
  const unsigned off = static_cast<unsigned>(reinterpret_cast<uintptr_t>(from) & 15u);
  unsigned a[8] = {low.x, low.y, low.z, low.w, high.x, high.y, high.z, high.w};
  if (off & 8) {
#pragma unroll
    for (int k = 0; k < 6; ++k) a[k] = a[k + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int k = 0; k < 5; ++k) a[k] = a[k + 1];
  }
  const unsigned bits = (off & 3) * 8;
  return make_uint4(__funnelshift_r(a[0], a[1], bits), __funnelshift_r(a[1], a[2], bits),
                    __funnelshift_r(a[2], a[3], bits), __funnelshift_r(a[3], a[4], bits));
}

// A chunk is 16 bytes of y.  Where the rows of x, r and y lie alike to the 16-byte boundary, so is its part of
// x and r, and chunks over a row's ends go element by element (whole blocks there too: 16384 x 4096 bf16 51 us,
// 49 without).  Otherwise (kShift) x and r are shifted out of the aligned blocks around them, over a row's ends
// too: 16384 x 4095 bf16 into rows of another alignment 64 us (device time), 96 with pairs of elements; 4099 x 1001
// fp16 5.3 and 7.3; rows of fewer than kPairsBelow elements go in pairs (below).  kRows: several rows.
template <typename T, bool kShift, bool kResidual, bool kRows>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const DropoutParams p) {
  constexpr int kCount = 16 / sizeof(T);
  constexpr int kUnroll = kShift ? kShiftUnroll : kDropoutUnroll;
  const unsigned first = blockIdx.x * (kDropoutThreads * kUnroll) + threadIdx.x;
  const T *x[kUnroll], *r[kUnroll];
  T* y[kUnroll];
  long long e[kUnroll];        // number of the chunk's first element (kRows)
  int from[kUnroll], to[kUnroll];   // its elements that exist
  bool blocks[kUnroll];             // its operands are in vx and vr
  uint4 vx[kUnroll], vr[kUnroll], hx[kUnroll], hr[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    const unsigned c = first + i * kDropoutThreads;
    from[i] = 0;
    to[i] = kCount;
    if (kRows) {
      const unsigned row = __umulhi(c, p.magic) >> p.shift;
      const unsigned q = c - row * p.per_row;
      T* start = static_cast<T*>(p.y) + row * p.ldy;
      const int mis = static_cast<int>((reinterpret_cast<uintptr_t>(start) & 15u) / sizeof(T));
      const int col = static_cast<int>(q) * kCount - mis, cols = static_cast<int>(p.cols);
      x[i] = static_cast<const T*>(p.x) + row * p.ldx + col;
      y[i] = start + col;
      if (kResidual) r[i] = static_cast<const T*>(p.r) + row * p.ldr + col;
      e[i] = p.index_base + row * p.cols + col;
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
    if (kShift) {
      blocks[i] = to[i] > from[i] && fetch_blocks(x[i], p.x, p.x_end, vx[i], hx[i]);
      if (kResidual) blocks[i] = blocks[i] && fetch_blocks(r[i], p.r, p.r_end, vr[i], hr[i]);
    } else {
      blocks[i] = to[i] - from[i] == kCount;
      if (blocks[i]) {
        vx[i] = *reinterpret_cast<const uint4*>(x[i]);
        if (kResidual) vr[i] = *reinterpret_cast<const uint4*>(r[i]);
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
    if (blocks[i]) {
      float f[kCount], g[kCount];
      unpack16<T>(kShift ? join_blocks(vx[i], hx[i], x[i]) : vx[i], f);
      if (kResidual) unpack16<T>(kShift ? join_blocks(vr[i], hr[i], r[i]) : vr[i], g);
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        f[k] = u[k] >= least ? f[k] * p.scale : 0.0f;
        if (kResidual) f[k] += g[k];
      }
      if (!kShift || to[i] - from[i] == kCount) {
        *reinterpret_cast<uint4*>(y[i]) = pack16<T>(f);
      } else {
#pragma unroll
        for (int k = 0; k < kCount; ++k)
          if (k >= from[i] && k < to[i]) y[i][k] = from_float<T>(f[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kCount; ++k) {
        if (k < from[i] || k >= to[i]) continue;
        float f = u[k] >= least ? to_float(x[i][k]) * p.scale : 0.0f;
        if (kResidual) f += to_float(r[i][k]);
        y[i][k] = from_float<T>(f);
      }
    }
  }
}

// Short rows of other alignments: a chunk is a hash's pair of elements, so a row of 10 takes five or six threads of
// one hash, not two or three of four.  Always several rows.  Measured on 10^7 elements, us, pairs against shifted
// chunks: bf16 rows of 3 33 / 60, of 10 21 / 31, of 15 21 / 23, of 16 21 / 18, of 64 19 / 14; fp32 of 3 31 / 43, of
// 10 21 / 27, of 15 21 / 23, of 16 21 / 21, of 64 20 / 19.
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kDropoutThreads) dropout_pairs_kernel(const DropoutParams p) {
  const unsigned first = blockIdx.x * (kDropoutThreads * kPairsUnroll) + threadIdx.x;
  T x[kPairsUnroll][2], r[kPairsUnroll][2], *y[kPairsUnroll];
  bool on[kPairsUnroll][2];
  long long e[kPairsUnroll];   // number of the pair's first element, an even one
#pragma unroll
  for (int i = 0; i < kPairsUnroll; ++i) {
    const unsigned c = first + i * kDropoutThreads;
    const unsigned row = __umulhi(c, p.magic) >> p.shift;
    const long long number = p.index_base + row * p.cols;
    const int col = static_cast<int>(c - row * p.per_row) * 2 - static_cast<int>(number & 1);
    e[i] = number + col;
    y[i] = static_cast<T*>(p.y) + row * p.ldy + col;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      on[i][k] = c < p.chunks && col + k >= 0 && col + k < static_cast<int>(p.cols);
      if (on[i][k]) x[i][k] = static_cast<const T*>(p.x)[row * p.ldx + col + k];
      if (kResidual && on[i][k]) r[i][k] = static_cast<const T*>(p.r)[row * p.ldr + col + k];
    }
  }
  const unsigned least = p.none ? 1u : p.threshold;
#pragma unroll
  for (int i = 0; i < kPairsUnroll; ++i) {
    const uint2 w = dropout_hash(p.base + static_cast<unsigned long long>(e[i] >> 1) * kPairStep);
    const unsigned u[2] = {p.none ? 0u : w.x, p.none ? 0u : w.y};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!on[i][k]) continue;
      float f = u[k] >= least ? to_float(x[i][k]) * p.scale : 0.0f;
      if (kResidual) f += to_float(r[i][k]);
      y[i][k] = from_float<T>(f);
    }
  }
}

}  // namespace adapt
