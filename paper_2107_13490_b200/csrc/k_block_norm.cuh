// Norms after a block and before the next one, with the block's gate and the residual sum, and their gradient.
//
//   y = beta residual + alpha g(gate) norm_a(block) w_a,   normed = norm_b(y) w_b
//
// With hat = (v - mean) / deviation of a norm's input v and d the gradient of hat, the gradient of v is
//   (d - hat mean(d hat) [- mean(d)]) / deviation          (the last mean with ADAPT_NORM_LAYER only).
// A row is read once and held in fp32; what the backward pass needs of the forward one is two numbers a norm
// and row.  HBM bounds both.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "k_elem.cuh"
#include "norm_shape.h"
#include "tensor_core.cuh"

namespace adapt {

constexpr int kNormNone = 0, kNormRms = 1, kNormLayer = 2;

struct NormParams {
  const void *block, *residual, *gate, *d_y, *d_normed;
  const float *weight_after, *weight_before;
  void *y, *normed, *d_block, *d_residual, *d_gate;
  float *d_weight_after, *d_weight_before;
  const float* stats_in;
  float* stats;
  float* partial;        // [3][ctas][dim] sums over a CTA's rows: of a shared gate, of the weights after and before
  long long ld_block, ld_residual, ld_gate, ld_y, ld_normed, ld_d_y, ld_d_normed, ld_d_block, ld_d_residual, ld_d_gate;
  int rows, dim;
  int after, before;
  bool sigmoid, shared;
  float scale, residual_scale, eps;
};

// The gate's value and its derivative by the gate.  With t = e^-|v|: t / (1 + t)^2 loses nothing where the gate
// is far open or closed, as g (1 - g) would.
struct Gate { float open, slope; };
__device__ __forceinline__ Gate norm_gate(float v, bool sigmoid) {
  if (!sigmoid) return {v, 1.0f};
  const float t = __expf(-fabsf(v)), s = __fdividef(1.0f, 1.0f + t);
  return {v >= 0.0f ? s : v < 0.0f ? t * s : v, t * s * s};
}

// Sums of `a` and `b` over a CTA of kThreads; every thread gets them.
template <int kThreads>
__device__ __forceinline__ float2 cta_sum(float a, float b, float2* shared) {
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    a += __shfl_xor_sync(~0u, a, d);
    b += __shfl_xor_sync(~0u, b, d);
  }
  __syncthreads();   // (what was there has been read)
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  float2 s = shared[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) { s.x += shared[w].x; s.y += shared[w].y; }
  return s;
}

constexpr int kNormThreads = 256;

// Rows of any length and alignment: a CTA a row, which it holds in shared memory.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_any_kernel(NormParams q) {
  extern __shared__ float row[];
  __shared__ float2 sums[kNormThreads / 32];
  const long long r = blockIdx.x;
  const T* block = static_cast<const T*>(q.block) + r * q.ld_block;
  const T* residual = q.residual ? static_cast<const T*>(q.residual) + r * q.ld_residual : nullptr;
  const T* gate = q.gate && !q.shared ? static_cast<const T*>(q.gate) + r * q.ld_gate : nullptr;
  const float* gate_shared = q.gate && q.shared ? static_cast<const float*>(q.gate) : nullptr;
  const float inv = 1.0f / static_cast<float>(q.dim);
  // mean and 1 / deviation of what is in `row`
  auto statistics = [&](int kind) -> float2 {
    float mean = 0.0f, s = 0.0f;
    if (kind == kNormLayer) {
      for (int c = threadIdx.x; c < q.dim; c += kNormThreads) s += row[c];
      mean = cta_sum<kNormThreads>(s, 0.0f, sums).x * inv;
      s = 0.0f;
    }
    for (int c = threadIdx.x; c < q.dim; c += kNormThreads) { const float d = row[c] - mean; s = fmaf(d, d, s); }
    return make_float2(mean, rsqrtf(fmaf(cta_sum<kNormThreads>(s, 0.0f, sums).x, inv, q.eps)));
  };
  for (int c = threadIdx.x; c < q.dim; c += kNormThreads) row[c] = to_float(block[c]);
  const float2 a = q.after != kNormNone ? statistics(q.after) : make_float2(0.0f, 1.0f);
  for (int c = threadIdx.x; c < q.dim; c += kNormThreads) {
    float v = row[c];
    if (q.after != kNormNone) {
      v = (v - a.x) * a.y;
      if (q.weight_after) v *= q.weight_after[c];
    }
    if (q.gate) {
      const float g = gate ? to_float(gate[c]) : gate_shared[c];
      v *= norm_gate(g, q.sigmoid).open;
    }
    v *= q.scale;
    if (residual) v = fmaf(to_float(residual[c]), q.residual_scale, v);
    row[c] = v;
  }
  const float2 b = q.before != kNormNone ? statistics(q.before) : make_float2(0.0f, 1.0f);
  for (int c = threadIdx.x; c < q.dim; c += kNormThreads) {
    const float v = row[c];
    if (q.y) static_cast<T*>(q.y)[r * q.ld_y + c] = from_float<T>(v);
    if (q.normed) {
      float o = (v - b.x) * b.y;
      if (q.weight_before) o *= q.weight_before[c];
      static_cast<T*>(q.normed)[r * q.ld_normed + c] = from_float<T>(o);
    }
  }
  if (q.stats && threadIdx.x == 0) reinterpret_cast<float4*>(q.stats)[r] = make_float4(a.x, a.y, b.x, b.y);
}

// Their gradient: a CTA takes every gridDim-th row; its sums over rows are in its part of `partial`, where
// every thread finds its own columns again.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_any_backward_kernel(NormParams q) {
  extern __shared__ float row[];
  __shared__ float2 sums[kNormThreads / 32];
  const float inv = 1.0f / static_cast<float>(q.dim);
  const long long plane = static_cast<long long>(gridDim.x) * q.dim;
  float* mine = q.partial ? q.partial + static_cast<long long>(blockIdx.x) * q.dim : nullptr;
  const bool sum_gate = q.d_gate && q.shared;
  for (long long r = blockIdx.x; r < q.rows; r += gridDim.x) {
    const bool fresh = r == blockIdx.x;
    auto add = [&](int plane_no, int c, float v) {
      float* p = mine + plane_no * plane + c;
      *p = fresh ? v : *p + v;
    };
    const T* block = static_cast<const T*>(q.block) + r * q.ld_block;
    const T* residual = q.residual ? static_cast<const T*>(q.residual) + r * q.ld_residual : nullptr;
    const T* gate = q.gate && !q.shared ? static_cast<const T*>(q.gate) + r * q.ld_gate : nullptr;
    const float* gate_shared = q.gate && q.shared ? static_cast<const float*>(q.gate) : nullptr;
    const T* d_y = q.d_y ? static_cast<const T*>(q.d_y) + r * q.ld_d_y : nullptr;
    const T* d_normed = q.d_normed ? static_cast<const T*>(q.d_normed) + r * q.ld_d_normed : nullptr;
    const float4 st = reinterpret_cast<const float4*>(q.stats_in)[r];
    struct Forward { float hat, value; Gate gate; };   // norm_a(block), times its weight, the gate
    auto forward = [&](int c) {
      Forward f;
      f.hat = to_float(block[c]);
      if (q.after != kNormNone) f.hat = (f.hat - st.x) * st.y;
      f.value = q.after != kNormNone && q.weight_after ? f.hat * q.weight_after[c] : f.hat;
      f.gate = norm_gate(gate ? to_float(gate[c]) : gate_shared ? gate_shared[c] : 1.0f, q.sigmoid);
      return f;
    };
    auto before_hat = [&](int c, const Forward& f) {
      float y = f.value * f.gate.open * q.scale;
      if (residual) y = fmaf(to_float(residual[c]), q.residual_scale, y);
      return (y - st.z) * st.w;
    };
    float2 m = make_float2(0.0f, 0.0f);
    if (d_normed) {
      float sh = 0.0f, s = 0.0f;
      for (int c = threadIdx.x; c < q.dim; c += kNormThreads) {
        const float hat = before_hat(c, forward(c)), dn = to_float(d_normed[c]);
        const float d = q.weight_before ? dn * q.weight_before[c] : dn;
        if (q.d_weight_before) add(2, c, dn * hat);
        sh = fmaf(d, hat, sh);
        s += d;
      }
      m = cta_sum<kNormThreads>(sh, s, sums);
      m.x *= inv;
      m.y = q.before == kNormLayer ? m.y * inv : 0.0f;
    }
    float sh = 0.0f, s = 0.0f;
    for (int c = threadIdx.x; c < q.dim; c += kNormThreads) {
      const Forward f = forward(c);
      float d = d_y ? to_float(d_y[c]) : 0.0f;
      if (d_normed) {
        const float dn = to_float(d_normed[c]);
        d += (fmaf(-before_hat(c, f), m.x, q.weight_before ? dn * q.weight_before[c] : dn) - m.y) * st.w;
      }
      if (q.d_residual) static_cast<T*>(q.d_residual)[r * q.ld_d_residual + c] = from_float<T>(d * q.residual_scale);
      d *= q.scale;
      if (q.d_gate) {
        const float g = d * f.value * f.gate.slope;
        if (sum_gate) add(0, c, g); else static_cast<T*>(q.d_gate)[r * q.ld_d_gate + c] = from_float<T>(g);
      }
      d *= f.gate.open;
      if (q.after != kNormNone) {
        if (q.d_weight_after) add(1, c, d * f.hat);
        if (q.weight_after) d *= q.weight_after[c];
        sh = fmaf(d, f.hat, sh);
        s += d;
      }
      row[c] = d;
    }
    if (!q.d_block) { __syncthreads(); continue; }
    if (q.after != kNormNone) {
      m = cta_sum<kNormThreads>(sh, s, sums);
      m.x *= inv;
      m.y = q.after == kNormLayer ? m.y * inv : 0.0f;
    }
    for (int c = threadIdx.x; c < q.dim; c += kNormThreads) {
      float d = row[c];
      if (q.after != kNormNone) d = (fmaf(-(to_float(block[c]) - st.x) * st.y, m.x, d) - m.y) * st.y;
      static_cast<T*>(q.d_block)[r * q.ld_d_block + c] = from_float<T>(d);
    }
  }
}

// ---- rows held in registers ------------------------------------------------------------------------------
//
// A CTA walks over rows, a row at a time; a thread holds kElems elements of it, in chunks of 16 bytes.  The rows come
// through a ring of stages in shared memory that bulk copies fill rows ahead, so that loads are under way while the
// sums of a row meet.
//
// Rows that do not begin on 16-byte boundaries (an odd dim) are copied with the aligned blocks around them.  All tensors
// have to lie alike (kEdges): then chunks are cut at those boundaries, the first and the last hold fewer
// elements, and a CTA takes rows that lie alike too, so that a thread keeps its columns.
//
// Rows that one CTA cannot hold are shared by the CTAs of a cluster, which add up their sums through shared memory.

constexpr int kNormMaxStages = 4;

struct NormRing {
  int streams, stages;       // rows of a stage, stages
  int stage_row;             // bytes of a row in a stage
  int parts;                 // CTAs of a cluster that share a row
  int place[5];              // bytes into a stage of block, residual, gate, d_y, d_normed, -1: none
  int weights[3];            // (kEdges) bytes into shared memory of the copies of weight_after, weight_before and a shared gate
};

// Two elements.  What multiplies or adds elements with elements takes both in one packed instruction; a factor for all
// would have to be held in a pair of registers, so that is done one by one.
typedef float2 Two;
__device__ __forceinline__ Two both(float v) { return make_float2(v, v); }
__device__ __forceinline__ f32x2 packed(Two a) { return pack2(a.x, a.y); }
__device__ __forceinline__ Two sum(Two a, Two b) { return unpack2(add2(packed(a), packed(b))); }
__device__ __forceinline__ Two times(Two a, Two b) { return unpack2(mul2(packed(a), packed(b))); }
__device__ __forceinline__ Two times_plus(Two a, Two b, Two c) { return unpack2(fma2(packed(a), packed(b), packed(c))); }
__device__ __forceinline__ Two times(Two a, float b) { return make_float2(a.x * b, a.y * b); }
__device__ __forceinline__ Two times_plus(Two a, float b, float c) { return make_float2(fmaf(a.x, b, c), fmaf(a.y, b, c)); }
__device__ __forceinline__ Two times_plus(Two a, float b, Two c) { return make_float2(fmaf(a.x, b, c.x), fmaf(a.y, b, c.y)); }
__device__ __forceinline__ Two times_plus(Two a, Two b, float c) { return make_float2(fmaf(a.x, b.x, c), fmaf(a.y, b.y, c)); }
__device__ __forceinline__ float fast_exp2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float fast_inverse(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
constexpr float kLog2E = 1.4426950408889634f;

// g(gate) of a pair: 1 / (1 + e^-v), to 2^-22 and |v| steps of the exponent's argument; 0 below 2^-126.
__device__ __forceinline__ Two gate_open(Two v) {
  const Two e = times(v, -kLog2E);
  return make_float2(fast_inverse(1.0f + fast_exp2(e.x)), fast_inverse(1.0f + fast_exp2(e.y)));
}

// The gate of the backward pass's first phase, kept in one number for the second: the smaller of g and 1 - g (the
// other is 1 minus it, to a rounding), with the sign that says which.  So g (1 - g) keeps its relative precision
// where the gate is far open or closed.
__device__ __forceinline__ float gate_kept(float v) {
  const float t = fast_exp2(fabsf(v) * -kLog2E);
  return copysignf(t * fast_inverse(1.0f + t), v);
}
__device__ __forceinline__ Two gate_kept(Two v) { return make_float2(gate_kept(v.x), gate_kept(v.y)); }
__device__ __forceinline__ Two kept_open(Two k) {
  const Two most = make_float2(1.0f - fabsf(k.x), 1.0f - fabsf(k.y));
  return make_float2(signbit(k.x) ? fabsf(k.x) : most.x, signbit(k.y) ? fabsf(k.y) : most.y);
}
__device__ __forceinline__ Two kept_slope(Two k) { return make_float2(fmaf(-fabsf(k.x), fabsf(k.x), fabsf(k.x)), fmaf(-fabsf(k.y), fabsf(k.y), fabsf(k.y))); }

// Sums over a CTA, up to kMost at a time, in one of two sets of places in turn, so that one barrier each is enough.
template <int kThreads, int kMost>
struct CtaSums {
  float (*places)[kMost][kThreads / 32];
  float (*parts)[kNormMaxParts][kMost];   // sums of each CTA of the cluster
  int turn, part, count;
  template <int N>
  __device__ __forceinline__ static void over_warp(float (&v)[N]) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] += __shfl_xor_sync(~0u, v[j], d);
  }
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
    over_warp(v);
    if (blockDim.x == 32) { __syncwarp(); return; }   // (rows so short are not shared)
    const int lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
      for (int j = 0; j < N; ++j) places[turn][j][threadIdx.x >> 5] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = lane < static_cast<int>(blockDim.x >> 5) ? places[turn][j][lane] : 0.0f;
    over_warp(v);
    if (count > 1) {
      if (threadIdx.x < static_cast<unsigned>(count)) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(peer_address(shared_address(&parts[turn][part][j]), threadIdx.x)), "f"(v[j]) : "memory");
      }
      meet_cluster();
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = 0.0f;
      for (int p = 0; p < count; ++p)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += parts[turn][p][j];
    }
    turn ^= 1;
  }
  __device__ __forceinline__ float one(float a) {
    float v[1] = {a};
    (*this)(v);
    return v[0];
  }
};

// The rows of a CTA in order, read ahead into the ring by its first thread, and the columns of a thread.
template <typename T, int kElems, bool kEdges>
struct NormRows {
  static constexpr int V = 16 / sizeof(T), P = V / 2, kChunks = kElems / V;
  const NormParams& q;
  const NormRing& ring;
  unsigned char* stages;
  unsigned bars;             // an address
  unsigned stage, parity;    // the stage of the row at hand, its barrier's phase
  const unsigned char* at;   // this thread's place in the stage
  int part;                  // of the row, for this CTA
  unsigned group, groups;    // clusters take the rows in turn
  int offset;                // column of the CTA's first element: below 0 where rows begin behind a 16-byte boundary
  unsigned in;               // which of the thread's elements are elements of the row (kEdges)
  __device__ __forceinline__ NormRows(const NormParams& q_, const NormRing& r, unsigned char* smem, unsigned long long* b)
      : q(q_), ring(r), stages(smem), bars(shared_address(b)), stage(0), parity(0), at(smem + threadIdx.x * 16), part(0),
        group(blockIdx.x), groups(gridDim.x), offset(0), in(~0u) {
    if (ring.parts > 1) {
      part = cta_in_cluster();
      group = blockIdx.x / ring.parts;
      groups = gridDim.x / ring.parts;
      offset = part * kElems * static_cast<int>(blockDim.x);
    }
    if constexpr (kEdges) {
      offset -= static_cast<int>((reinterpret_cast<uintptr_t>(static_cast<const T*>(q.block) + group * q.ld_block) & 15u) / sizeof(T));
      in = 0;
#pragma unroll
      for (int j = 0; j < kElems; ++j) {
        const int c = column(j / V) + j % V;
        in |= (c >= 0 && c < q.dim ? 1u : 0u) << j;
      }
    }
    if constexpr (kEdges) {   // weights beside their columns, so that they are read in 16 bytes too
      const float* from[3] = {q.weight_after, q.weight_before, q.shared ? static_cast<const float*>(q.gate) : nullptr};
      const int width = kChunks * static_cast<int>(blockDim.x) * V;
#pragma unroll
      for (int w = 0; w < 3; ++w)
        if (ring.weights[w] >= 0)
          for (int c = threadIdx.x; c < width; c += blockDim.x)
            reinterpret_cast<float*>(smem + ring.weights[w])[c] =
                offset + c < 0 || offset + c >= q.dim ? 0.0f : from[w] ? __ldg(from[w] + offset + c) : 1.0f;
    }
    if (threadIdx.x == 0) {
      for (int s = 0; s < ring.stages; ++s) barrier_init(bars + 8 * s, 1);
      barrier_init_fence();
      for (int s = 0; s < ring.stages; ++s) fill(s, group + s * groups);
    }
    if (ring.parts > 1) meet_cluster(); else __syncthreads();
  }
  __device__ __forceinline__ int column(int i) const { return offset + (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * V; }
  // Whether chunk i has an element of the row, and whether all of its elements are.
  __device__ __forceinline__ bool any(int i) const { return column(i) < q.dim; }
  __device__ __forceinline__ bool whole(int i) const { return !kEdges || ((in >> (i * V)) & ((1u << V) - 1)) == (1u << V) - 1; }
  __device__ __forceinline__ bool inside(int j) const { return kEdges ? (in >> j & 1) : any(j / V); }
  // Sets chunk i of a thread's elements, or a chunk by itself, to 0 beyond the row.
  template <int N>
  __device__ __forceinline__ void blank(int i, Two (&v)[N]) const {
    if (whole(i)) return;
    const int first = N == P ? 0 : i * P;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      if (!has(i * V + 2 * k)) v[first + k].x = 0.0f;
      if (!has(i * V + 2 * k + 1)) v[first + k].y = 0.0f;
    }
  }
  __device__ __forceinline__ bool has(int j) const { return !kEdges || (in >> j & 1); }

  __device__ __forceinline__ void fill(int s, unsigned r) const {
    if (r >= static_cast<unsigned>(q.rows)) return;
    const int from_column = offset, columns = min(q.dim - from_column, kElems * static_cast<int>(blockDim.x));
    if (columns <= 0) { barrier_expect_bytes(bars + 8 * s, 0); return; }
    const unsigned bytes = (columns * static_cast<int>(sizeof(T)) + 15) & ~15;
    barrier_expect_bytes(bars + 8 * s, ring.streams * bytes);
    const void* from[5] = {q.block, q.residual, q.gate, q.d_y, q.d_normed};
    const long long ld[5] = {q.ld_block, q.ld_residual, q.ld_gate, q.ld_d_y, q.ld_d_normed};
#pragma unroll
    for (int i = 0; i < 5; ++i)
      if (ring.place[i] >= 0)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     :: "r"(shared_address(stages) + s * ring.streams * ring.stage_row + ring.place[i]), "l"(static_cast<const T*>(from[i]) + r * ld[i] + from_column),
                        "r"(bytes), "r"(bars + 8 * s) : "memory");
  }
  // Waits for the row's data (or the next row's); 0, or NaN where they never came.
  __device__ __forceinline__ float ready(int behind = 0) const {
    return barrier_wait(bars + 8 * (stage + behind), parity) ? 0.0f : __int_as_float(0x7FC00000);
  }
  // Called when every thread has read what it needs of the row `r`.
  __device__ __forceinline__ void release(unsigned r) {
    if (threadIdx.x == 0) fill(stage, r + ring.stages * groups);
    at += ring.streams * ring.stage_row;
    if (++stage == static_cast<unsigned>(ring.stages)) { stage = 0; parity ^= 1; at = stages + threadIdx.x * 16; }
  }
  // Chunk i of stream kStream; 0 for what is not in the row.
  template <int kStream>
  __device__ __forceinline__ void read(int i, Two (&f)[P], int behind = 0) const {   // (1: of the next row, in the next stage)
    const uint4 raw = *reinterpret_cast<const uint4*>(at + behind * ring.streams * ring.stage_row + ring.place[kStream] + i * blockDim.x * 16);
    float v[V];
    unpack16<T>(raw, v);
    if (kEdges && !whole(i)) {
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = has(i * V + k) ? v[k] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < P; ++k) f[k] = make_float2(v[2 * k], v[2 * k + 1]);
  }
  // Weights kWhich: after, before, a shared gate (none: 1).
  template <int kWhich>
  __device__ __forceinline__ void weights(int i, Two (&f)[P]) const {
    const float* w = kWhich == 0 ? q.weight_after : kWhich == 1 ? q.weight_before : static_cast<const float*>(q.gate);
    const float4* from;
    if constexpr (kEdges) {
      from = reinterpret_cast<const float4*>(stages + ring.weights[kWhich]) + (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * (V / 4);
    } else if (!w) {
#pragma unroll
      for (int k = 0; k < P; ++k) f[k] = both(1.0f);
      return;
    } else {
      from = reinterpret_cast<const float4*>(w + column(i));
    }
#pragma unroll
    for (int k = 0; k < V / 4; ++k) {
      const float4 t = kEdges ? from[k] : __ldg(from + k);
      f[2 * k] = make_float2(t.x, t.y);
      f[2 * k + 1] = make_float2(t.z, t.w);
    }
  }
  __device__ __forceinline__ void write(void* to, long long at, int i, const Two (&f)[P]) const {
    float v[V];
#pragma unroll
    for (int k = 0; k < P; ++k) { const float2 t = f[k]; v[2 * k] = t.x; v[2 * k + 1] = t.y; }
    T* p = static_cast<T*>(to) + at + column(i);
    if (whole(i)) {
      __stcs(reinterpret_cast<uint4*>(p), pack16<T>(v));
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (has(i * V + k)) p[k] = from_float<T>(v[k]);
    }
  }
  // A column's sum over the rows.
  __device__ __forceinline__ void write_sums(float* to, int i, const Two* f) const {
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const float2 t = f[k];
      float* p = to + column(i) + 2 * k;
      if (has(i * V + 2 * k)) p[0] = t.x;
      if (has(i * V + 2 * k + 1)) p[1] = t.y;
    }
  }
};

// What a kernel is made for, so that nothing is decided element by element.
constexpr int kGateNone = 0, kGateEach = 1, kGateEachSigmoid = 2, kGateForAll = 3;

template <typename T, bool kEdges, bool kAfter, bool kBefore, int kGate>
__global__ __launch_bounds__(kNormMaxThreads, 1) void norm_row_kernel(const NormParams q, const NormRing ring) {
  typedef NormRows<T, kNormElems, kEdges> Rows;
  constexpr int P = Rows::P, kChunks = Rows::kChunks, kPairs = kNormElems / 2;
  extern __shared__ __align__(128) unsigned char norm_smem[];
  __shared__ __align__(8) unsigned long long bars[kNormMaxStages];
  __shared__ float places[2][1][kNormMaxThreads / 32], parts[2][kNormMaxParts][1];
  Rows rows(q, ring, norm_smem, bars);
  CtaSums<kNormMaxThreads, 1> sums{places, parts, 0, rows.part, ring.parts};
  const float inv = 1.0f / static_cast<float>(q.dim);
  // mean and 1 / deviation; the deviation around the mean, in a second sum
  auto statistics = [&](const Two (&v)[kPairs], int kind) {
    float mean = 0.0f, s = 0.0f;
    if (kind == kNormLayer) {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) s += v[k].x + v[k].y;   // (0 beyond the row)
      mean = sums.one(s) * inv;
      s = 0.0f;
#pragma unroll
      for (int j = 0; j < kNormElems; ++j) {
        const float d = (j & 1 ? v[j / 2].y : v[j / 2].x) - mean;
        if (rows.inside(j)) s = fmaf(d, d, s);
      }
    } else {
      Two t = both(0.0f);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) t = times_plus(v[k], v[k], t);
      s = t.x + t.y;
    }
    return make_float2(mean, rsqrtf(fmaf(sums.one(s), inv, q.eps)));
  };
  for (unsigned r = rows.group; r < static_cast<unsigned>(q.rows); r += rows.groups) {
    const float poison = rows.ready();
    Two v[kPairs];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      Two f[P];
#pragma unroll
      for (int k = 0; k < P; ++k) f[k] = both(0.0f);
      if (rows.any(i)) rows.template read<0>(i, f);
#pragma unroll
      for (int k = 0; k < P; ++k) v[i * P + k] = f[k];
    }
    v[0].x += poison;
    float2 a = make_float2(0.0f, 1.0f), b = a;
    if (kAfter) a = statistics(v, q.after);
    // (where there is a norm, its factor takes the scale along)
    const float r_a = a.y * q.scale, mean_a = -a.x * r_a;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!rows.any(i)) break;
      Two g[P];
      if (kAfter) rows.template weights<0>(i, g);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        if (kAfter) v[i * P + k] = times(times_plus(v[i * P + k], r_a, mean_a), g[k]);
        else v[i * P + k] = times(v[i * P + k], q.scale);
      }
      if (kGate == kGateForAll) rows.template weights<2>(i, g);
      else if (kGate != kGateNone) rows.template read<2>(i, g);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        if (kGate == kGateEachSigmoid || (kGate == kGateForAll && q.sigmoid)) g[k] = gate_open(g[k]);
        if (kGate != kGateNone) v[i * P + k] = times(v[i * P + k], g[k]);
      }
      if (q.residual) {
        rows.template read<1>(i, g);
#pragma unroll
        for (int k = 0; k < P; ++k) v[i * P + k] = times_plus(g[k], q.residual_scale, v[i * P + k]);
      }
      if (kEdges) rows.blank(i, v);
      if (q.y) {
#pragma unroll
        for (int k = 0; k < P; ++k) g[k] = v[i * P + k];
        rows.write(q.y, r * q.ld_y, i, g);
      }
    }
    if (kBefore) b = statistics(v, q.before); else __syncthreads();
    rows.release(r);
    if (kBefore) {
      const float mean_b = -b.x * b.y;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        if (!rows.any(i)) break;
        Two f[P], w[P];
        rows.template weights<1>(i, w);
#pragma unroll
        for (int k = 0; k < P; ++k) f[k] = times(times_plus(v[i * P + k], b.y, mean_b), w[k]);
        rows.write(q.normed, r * q.ld_normed, i, f);
      }
    }
    if (q.stats && threadIdx.x == 0 && rows.part == 0) reinterpret_cast<float4*>(q.stats)[r] = make_float4(a.x, a.y, b.x, b.y);
  }
}

template <typename T, bool kEdges, bool kAfter, bool kBefore, int kGate>
__global__ __launch_bounds__(kNormBackwardThreads, 1) void norm_row_backward_kernel(const NormParams q, const NormRing ring) {
  typedef NormRows<T, kNormElems, kEdges> Rows;
  constexpr int P = Rows::P, kChunks = Rows::kChunks, kPairs = kNormElems / 2;
  constexpr bool kForAll = kGate == kGateForAll;
  extern __shared__ __align__(128) unsigned char norm_smem[];
  __shared__ __align__(8) unsigned long long bars[kNormMaxStages];
  __shared__ float places[2][2][kNormBackwardThreads / 32], parts[2][kNormMaxParts][2];
  Rows rows(q, ring, norm_smem, bars);
  CtaSums<kNormBackwardThreads, 2> sums{places, parts, 0, rows.part, ring.parts};
  const float inv = 1.0f / static_cast<float>(q.dim);
  Two of_after[kAfter ? kPairs : 1], of_before[kBefore ? kPairs : 1], of_gate[kForAll ? kPairs : 1];   // sums over rows
#pragma unroll
  for (int k = 0; k < kPairs; ++k) of_after[kAfter ? k : 0] = of_before[kBefore ? k : 0] = of_gate[kForAll ? k : 0] = both(0.0f);
  const float4* statistics = reinterpret_cast<const float4*>(q.stats_in);
  float4 next = rows.group < static_cast<unsigned>(q.rows) ? __ldg(statistics + rows.group) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (unsigned r = rows.group; r < static_cast<unsigned>(q.rows); r += rows.groups) {
    const float4 st = next;
    if (r + rows.groups < static_cast<unsigned>(q.rows)) next = __ldg(statistics + r + rows.groups);
    const float poison = rows.ready();
    const float mean_a = -st.x * st.y, mean_b = -st.z * st.w, scale_b = q.scale * st.w, residual_b = q.residual_scale * st.w;
    // norm_before(y) and the gate; then the gradient of norm_after's output, and that output
    Two one[kPairs], two[kPairs];
    auto block_hat = [&](int i, Two (&hat)[P], Two (&value)[P]) {
      rows.template read<0>(i, hat);
      if (kAfter) {
        Two w[P];
        rows.template weights<0>(i, w);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          hat[k] = times_plus(hat[k], st.y, mean_a);
          value[k] = times(hat[k], w[k]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < P; ++k) value[k] = hat[k];
      }
    };
    auto keep_gate = [&](int i) {
      if (kGate == kGateNone) return;
      Two g[P];
      if (kForAll) rows.template weights<2>(i, g); else rows.template read<2>(i, g);
#pragma unroll
      for (int k = 0; k < P; ++k) two[i * P + k] = kGate == kGateEachSigmoid || (kForAll && q.sigmoid) ? gate_kept(g[k]) : g[k];
    };
    auto opened = [&](Two kept) { return kGate == kGateEachSigmoid || (kForAll && q.sigmoid) ? kept_open(kept) : kept; };
    float2 m = make_float2(0.0f, 0.0f);
    if (kBefore) {
      Two sh = both(0.0f), s = sh;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        if (!rows.any(i)) break;
        Two hat[P], y[P], f[P], w[P], base[P];
        block_hat(i, hat, y);
        keep_gate(i);
        if (q.residual) {
          rows.template read<1>(i, f);
#pragma unroll
          for (int k = 0; k < P; ++k) base[k] = times_plus(f[k], residual_b, mean_b);
        } else {
#pragma unroll
          for (int k = 0; k < P; ++k) base[k] = both(mean_b);
        }
        rows.template read<4>(i, f);   // (0 beyond the row, so that nothing there counts)
        rows.template weights<1>(i, w);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          if (kGate != kGateNone) y[k] = times(y[k], opened(two[i * P + k]));
          const Two y_hat = times_plus(y[k], scale_b, base[k]);
          one[i * P + k] = y_hat;
          of_before[kBefore ? i * P + k : 0] = times_plus(f[k], y_hat, of_before[kBefore ? i * P + k : 0]);
          const Two d = times(f[k], w[k]);
          sh = times_plus(d, y_hat, sh);
          s = sum(s, d);
        }
      }
      float t[2] = {sh.x + sh.y, s.x + s.y + poison};
      sums(t);
      m = make_float2(t[0] * inv, t[1]);
      m.y = q.before == kNormLayer ? m.y * inv : poison;
    }
    Two sh = both(0.0f), s = sh;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!rows.any(i)) break;
      Two hat[P], value[P], d[P], f[P], w[P];
      block_hat(i, hat, value);
      if (!kBefore) keep_gate(i);
      if (q.d_y) {
        rows.template read<3>(i, d);
      } else {
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = both(0.0f);
      }
      if (kBefore) {
        rows.template read<4>(i, f);
        rows.template weights<1>(i, w);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = times_plus(times_plus(one[i * P + k], -m.x, times_plus(f[k], w[k], -m.y)), st.w, d[k]);
      }
      if (kEdges) rows.blank(i, d);
      if (q.d_residual) {
#pragma unroll
        for (int k = 0; k < P; ++k) f[k] = times(d[k], q.residual_scale);
        rows.write(q.d_residual, r * q.ld_d_residual, i, f);
      }
#pragma unroll
      for (int k = 0; k < P; ++k) d[k] = times(d[k], q.scale);
      if (kGate != kGateNone) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
          f[k] = times(d[k], value[k]);
          if (kGate == kGateEachSigmoid || (kForAll && q.sigmoid)) f[k] = times(f[k], kept_slope(two[i * P + k]));
          d[k] = times(d[k], opened(two[i * P + k]));
          if (kForAll) of_gate[kForAll ? i * P + k : 0] = sum(of_gate[kForAll ? i * P + k : 0], f[k]);
        }
        if (!kForAll && q.d_gate) rows.write(q.d_gate, r * q.ld_d_gate, i, f);
      }
      if (kAfter) {
        rows.template weights<0>(i, w);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          of_after[kAfter ? i * P + k : 0] = times_plus(d[k], hat[k], of_after[kAfter ? i * P + k : 0]);
          d[k] = times(d[k], w[k]);
          sh = times_plus(d[k], hat[k], sh);
          s = sum(s, d[k]);
          two[i * P + k] = hat[k];
        }
      }
#pragma unroll
      for (int k = 0; k < P; ++k) one[i * P + k] = d[k];
    }
    if (kAfter) {
      float t[2] = {sh.x + sh.y, s.x + s.y + poison};
      sums(t);
      m = make_float2(t[0] * inv, t[1]);
      m.y = q.after == kNormLayer ? m.y * inv : poison;
    } else {
      __syncthreads();
    }
    rows.release(r);
    if (!q.d_block) continue;
    const float by_x = -m.x * st.y, by_y = -m.y * st.y;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!rows.any(i)) break;
      Two f[P];
#pragma unroll
      for (int k = 0; k < P; ++k)
        f[k] = kAfter ? times_plus(two[i * P + k], by_x, times_plus(one[i * P + k], st.y, by_y)) : one[i * P + k];
      rows.write(q.d_block, r * q.ld_d_block, i, f);
    }
  }
  if (!q.partial) return;
  const long long plane = static_cast<long long>(rows.groups) * q.dim;
  float* mine = q.partial + static_cast<long long>(rows.group) * q.dim;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (!rows.any(i)) break;
    if (kForAll) rows.write_sums(mine, i, of_gate + (kForAll ? i * P : 0));
    if (kAfter) rows.write_sums(mine + plane, i, of_after + (kAfter ? i * P : 0));
    if (kBefore) rows.write_sums(mine + 2 * plane, i, of_before + (kBefore ? i * P : 0));
  }
}

// The same for shorter rows, two at a time: they share the reading of the weights and the rounds of sums, and each one's
// latencies hide behind the other's.  A thread holds eight elements of both; the ring has an even number of stages.
template <typename T, bool kEdges, bool kAfter, bool kBefore, int kGate>
__global__ __launch_bounds__(kNormPairThreads, 2) void norm_pair_backward_kernel(const NormParams q, const NormRing ring) {
  typedef NormRows<T, kNormPairElems, kEdges> Rows;
  constexpr int P = Rows::P, kChunks = Rows::kChunks, kPairs = kNormPairElems / 2;
  constexpr bool kForAll = kGate == kGateForAll;
  extern __shared__ __align__(128) unsigned char norm_smem[];
  __shared__ __align__(8) unsigned long long bars[kNormMaxStages];
  __shared__ float places[2][4][kNormPairThreads / 32], parts[2][kNormMaxParts][4];
  Rows rows(q, ring, norm_smem, bars);
  CtaSums<kNormPairThreads, 4> sums{places, parts, 0, rows.part, ring.parts};
  const float inv = 1.0f / static_cast<float>(q.dim);
  const unsigned total = static_cast<unsigned>(q.rows);
  const bool sigmoid = kGate == kGateEachSigmoid || (kForAll && q.sigmoid);
  Two of_after[kAfter ? kPairs : 1], of_before[kBefore ? kPairs : 1], of_gate[kForAll ? kPairs : 1];   // sums over rows
#pragma unroll
  for (int k = 0; k < kPairs; ++k) of_after[kAfter ? k : 0] = of_before[kBefore ? k : 0] = of_gate[kForAll ? k : 0] = both(0.0f);
  const float4* statistics = reinterpret_cast<const float4*>(q.stats_in);
  auto statistic = [&](unsigned r) { return r < total ? __ldg(statistics + r) : make_float4(0.0f, 0.0f, 0.0f, 0.0f); };
  float4 next[2] = {statistic(rows.group), statistic(rows.group + rows.groups)};
  for (unsigned r = rows.group; r < total; r += 2 * rows.groups) {
    const bool second = r + rows.groups < total;
    const float4 st[2] = {next[0], next[1]};
    next[0] = statistic(r + 2 * rows.groups);
    next[1] = statistic(r + 3 * rows.groups);
    const float poison[2] = {rows.ready(), second ? rows.ready(1) : 0.0f};
    // of both rows: norm_before(y) and the gate; then the gradient of norm_after's output, and that output
    Two one[2][kPairs], two[2][kPairs];
    auto block_hat = [&](int j, int i, const Two (&w)[P], Two (&hat)[P], Two (&value)[P]) {
      rows.template read<0>(i, hat, j);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        if (kAfter) hat[k] = times_plus(hat[k], st[j].y, -st[j].x * st[j].y);
        value[k] = kAfter ? times(hat[k], w[k]) : hat[k];
      }
    };
    auto keep_gate = [&](int j, int i, const Two (&for_all)[P]) {
      if (kGate == kGateNone) return;
      Two g[P];
      if (!kForAll) rows.template read<2>(i, g, j);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const Two v = kForAll ? for_all[k] : g[k];
        two[j][i * P + k] = sigmoid ? gate_kept(v) : v;
      }
    };
    auto opened = [&](Two kept) { return sigmoid ? kept_open(kept) : kept; };
    float2 m[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
    if (kBefore) {
      Two sh[2] = {both(0.0f), both(0.0f)}, s[2] = {both(0.0f), both(0.0f)};
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        if (!rows.any(i)) break;
        Two wa[P], wb[P], wg[P];
        if (kAfter) rows.template weights<0>(i, wa);
        rows.template weights<1>(i, wb);
        if (kForAll) rows.template weights<2>(i, wg);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (j && !second) continue;
          const float mean_b = -st[j].z * st[j].w;
          Two hat[P], y[P], f[P], base[P];
          block_hat(j, i, wa, hat, y);
          keep_gate(j, i, wg);
          if (q.residual) {
            rows.template read<1>(i, f, j);
#pragma unroll
            for (int k = 0; k < P; ++k) base[k] = times_plus(f[k], q.residual_scale * st[j].w, mean_b);
          } else {
#pragma unroll
            for (int k = 0; k < P; ++k) base[k] = both(mean_b);
          }
          rows.template read<4>(i, f, j);   // (0 beyond the row, so that nothing there counts)
#pragma unroll
          for (int k = 0; k < P; ++k) {
            if (kGate != kGateNone) y[k] = times(y[k], opened(two[j][i * P + k]));
            const Two y_hat = times_plus(y[k], q.scale * st[j].w, base[k]);
            one[j][i * P + k] = y_hat;
            of_before[kBefore ? i * P + k : 0] = times_plus(f[k], y_hat, of_before[kBefore ? i * P + k : 0]);
            const Two d = times(f[k], wb[k]);
            sh[j] = times_plus(d, y_hat, sh[j]);
            s[j] = sum(s[j], d);
          }
        }
      }
      float t[4] = {sh[0].x + sh[0].y, s[0].x + s[0].y, sh[1].x + sh[1].y, s[1].x + s[1].y};
      sums(t);
#pragma unroll
      for (int j = 0; j < 2; ++j) m[j] = make_float2(t[2 * j] * inv, q.before == kNormLayer ? t[2 * j + 1] * inv : 0.0f);
    }
    Two sh[2] = {both(0.0f), both(0.0f)}, s[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!rows.any(i)) break;
      Two wa[P], wb[P], wg[P];
      if (kAfter) rows.template weights<0>(i, wa);
      if (kBefore) rows.template weights<1>(i, wb);
      if (kForAll && !kBefore) rows.template weights<2>(i, wg);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (j && !second) continue;
        const unsigned row = r + j * rows.groups;
        Two hat[P], value[P], d[P], f[P];
        block_hat(j, i, wa, hat, value);
        if (!kBefore) keep_gate(j, i, wg);
        if (q.d_y) {
          rows.template read<3>(i, d, j);
        } else {
#pragma unroll
          for (int k = 0; k < P; ++k) d[k] = both(0.0f);
        }
        if (kBefore) {
          rows.template read<4>(i, f, j);
#pragma unroll
          for (int k = 0; k < P; ++k)
            d[k] = times_plus(times_plus(one[j][i * P + k], -m[j].x, times_plus(f[k], wb[k], -m[j].y)), st[j].w, d[k]);
        }
        if (kEdges) rows.blank(i, d);
        if (q.d_residual) {
#pragma unroll
          for (int k = 0; k < P; ++k) f[k] = times(d[k], q.residual_scale);
          rows.write(q.d_residual, row * q.ld_d_residual, i, f);
        }
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = times(d[k], q.scale);
        if (kGate != kGateNone) {
#pragma unroll
          for (int k = 0; k < P; ++k) {
            f[k] = times(d[k], value[k]);
            if (sigmoid) f[k] = times(f[k], kept_slope(two[j][i * P + k]));
            d[k] = times(d[k], opened(two[j][i * P + k]));
            if (kForAll) of_gate[kForAll ? i * P + k : 0] = sum(of_gate[kForAll ? i * P + k : 0], f[k]);
          }
          if (!kForAll && q.d_gate) rows.write(q.d_gate, row * q.ld_d_gate, i, f);
        }
        if (kAfter) {
#pragma unroll
          for (int k = 0; k < P; ++k) {
            of_after[kAfter ? i * P + k : 0] = times_plus(d[k], hat[k], of_after[kAfter ? i * P + k : 0]);
            d[k] = times(d[k], wa[k]);
            sh[j] = times_plus(d[k], hat[k], sh[j]);
            s[j] = sum(s[j], d[k]);
            two[j][i * P + k] = hat[k];
          }
        }
#pragma unroll
        for (int k = 0; k < P; ++k) one[j][i * P + k] = d[k];
      }
    }
    if (kAfter) {
      float t[4] = {sh[0].x + sh[0].y, s[0].x + s[0].y, sh[1].x + sh[1].y, s[1].x + s[1].y};
      sums(t);
#pragma unroll
      for (int j = 0; j < 2; ++j) m[j] = make_float2(t[2 * j] * inv, q.after == kNormLayer ? t[2 * j + 1] * inv : 0.0f);
    } else {
      __syncthreads();
    }
    rows.release(r);
    rows.release(r + rows.groups);
    if (!q.d_block) continue;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!rows.any(i)) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (j && !second) continue;
        Two f[P];
#pragma unroll
        for (int k = 0; k < P; ++k) {
          f[k] = one[j][i * P + k];
          if (kAfter) f[k] = times_plus(two[j][i * P + k], -m[j].x * st[j].y, times_plus(f[k], st[j].y, -m[j].y * st[j].y));
          f[k].x += poison[j];
        }
        rows.write(q.d_block, (r + j * rows.groups) * q.ld_d_block, i, f);
      }
    }
  }
  if (!q.partial) return;
  const long long plane = static_cast<long long>(rows.groups) * q.dim;
  float* mine = q.partial + static_cast<long long>(rows.group) * q.dim;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (!rows.any(i)) break;
    if (kForAll) rows.write_sums(mine, i, of_gate + (kForAll ? i * P : 0));
    if (kAfter) rows.write_sums(mine + plane, i, of_after + (kAfter ? i * P : 0));
    if (kBefore) rows.write_sums(mine + 2 * plane, i, of_before + (kBefore ? i * P : 0));
  }
}

// Adds up the CTAs' sums: 32 columns a CTA, the CTAs dealt to its warps.
struct NormColumns { const float* partial; float* out[3]; int ctas, dim; };
constexpr int kNormColumnWarps = 32;

__global__ __launch_bounds__(32 * kNormColumnWarps) void norm_columns_kernel(NormColumns q) {
  __shared__ float part[kNormColumnWarps][33];
  const int plane = blockIdx.y, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane, warp = threadIdx.x >> 5;
  float* out = q.out[plane];
  if (!out) return;
  wait_for_previous_kernel();
  float s = 0.0f;
  if (c < q.dim) {
    const float* from = q.partial + static_cast<long long>(plane) * q.ctas * q.dim + c;
#pragma unroll 8
    for (int i = warp; i < q.ctas; i += kNormColumnWarps) s += __ldcg(from + static_cast<long long>(i) * q.dim);
  }
  part[warp][lane] = s;
  __syncthreads();
  s = part[lane][warp];   // warp w: column w of the 32
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
  if (lane == 0 && blockIdx.x * 32 + warp < q.dim) out[blockIdx.x * 32 + warp] = s;
}

}  // namespace adapt
