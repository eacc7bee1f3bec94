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

// Adds up the CTAs' sums: 32 columns a CTA, which its warps take in turn.
struct NormColumns { const float* partial; float* out[3]; int ctas, dim; };
constexpr int kNormColumnWarps = 8;

__global__ __launch_bounds__(32 * kNormColumnWarps) void norm_columns_kernel(NormColumns q) {
  __shared__ float part[kNormColumnWarps][32];
  const int plane = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
  float* out = q.out[plane];
  if (!out) return;
  float s = 0.0f;
  if (c < q.dim) {
    const float* from = q.partial + static_cast<long long>(plane) * q.ctas * q.dim + c;
    for (int i = warp; i < q.ctas; i += kNormColumnWarps) s += from[static_cast<long long>(i) * q.dim];
  }
  part[warp][threadIdx.x & 31] = s;
  __syncthreads();
  if (warp == 0 && c < q.dim) {
#pragma unroll
    for (int w = 1; w < kNormColumnWarps; ++w) s += part[w][threadIdx.x & 31];
    out[c] = s;
  }
}

}  // namespace adapt
