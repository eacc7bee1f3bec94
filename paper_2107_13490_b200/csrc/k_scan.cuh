// Gated linear recurrence: h_t = a_t h_{t-1} + b_t per channel.
//   sigmoid form: a = s(g), b = (1 - a) x;   value form: a = g, b = x.
// At a reset h_{t-1} counts as 0; steps at or beyond a sequence's length leave the state alone.
// States are fp32.  The state before every kScanTile-th step can be kept (carry) for the backward
// pass, which recomputes the states in between in fp32:
//   dh_t = dy_t + a_{t+1} dh_{t+1},  dx = dh db/dx,  dg = dh (h_{t-1} da/dg + db/dg).
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kScanTile = 128;
constexpr int kGateSigmoid = 0, kGateValue = 1;

struct ScanParams {
  const void *x, *gate, *dy;
  void *y, *dx, *dgate;
  const float *h0, *dh_last;
  float *h_last, *dh0, *carry;        // carry is read by the backward pass
  const int* lengths;
  const unsigned char* reset;
  float* partial;                      // per-channel gate gradients, summed by a second kernel
  long long batch, steps, channels;
  long long xb, xt, gb, gt, yb, yt;    // strides (elements) of x, gate, y / dy
  long long dxb, dxt, dgb, dgt;        // strides of dx, dgate
  int group;
};

// a and the factor of x (1 - a, or 1).  e^-g is held below 2^125 so that 1 - a = e^-g a stays a
// number; NaN passes through.
template <int kMode>
__device__ __forceinline__ void gate_coefs(float g, float& a, float& c) {
  if (kMode == kGateValue) { a = g; c = 1.0f; return; }
  float e;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(e) : "f"(-g), "f"(86.0f));
  e = expf(e);
  a = 1.0f / (1.0f + e);
  c = e * a;
}

template <typename T, int kMode>
__global__ void __launch_bounds__(128) scan_serial_kernel(const ScanParams p) {
  const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.batch * p.channels) return;
  const long long b = i / p.channels, d = i - b * p.channels;
  const long long len = p.lengths ? min(max(static_cast<long long>(p.lengths[b]), 0ll), p.steps) : p.steps;
  const T* x = static_cast<const T*>(p.x) + b * p.xb + d;
  const T* g = static_cast<const T*>(p.gate) + b * p.gb + d / p.group;
  T* y = static_cast<T*>(p.y) + b * p.yb + d;
  float h = p.h0 ? p.h0[i] : 0.0f;
  const long long tiles = (p.steps + kScanTile - 1) / kScanTile;
  for (long long t = 0; t < p.steps; ++t) {
    if (p.carry && t % kScanTile == 0) p.carry[(b * tiles + t / kScanTile) * p.channels + d] = h;
    if (t >= len) { y[t * p.yt] = from_float<T>(0.0f); continue; }
    float a, c;
    gate_coefs<kMode>(to_float(g[t * p.gt]), a, c);
    const bool cut = p.reset && p.reset[b * p.steps + t];
    const float u = kMode == kGateValue ? to_float(x[t * p.xt]) : c * to_float(x[t * p.xt]);
    h = cut ? u : fmaf(a, h, u);
    y[t * p.yt] = from_float<T>(h);
  }
  if (p.h_last) p.h_last[i] = h;
}

template <typename T, int kMode>
__global__ void __launch_bounds__(128) scan_serial_backward_kernel(const ScanParams p) {
  const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.batch * p.channels) return;
  const long long b = i / p.channels, d = i - b * p.channels;
  const long long len = p.lengths ? min(max(static_cast<long long>(p.lengths[b]), 0ll), p.steps) : p.steps;
  const T* x = static_cast<const T*>(p.x) + b * p.xb + d;
  const T* g = static_cast<const T*>(p.gate) + b * p.gb + d / p.group;
  const T* dy = static_cast<const T*>(p.dy) + b * p.yb + d;
  T* dx = static_cast<T*>(p.dx) + b * p.dxb + d;
  const long long tiles = (p.steps + kScanTile - 1) / kScanTile;
  float before[kScanTile];
  float flow = p.dh_last ? p.dh_last[i] : 0.0f;
  for (long long tile = tiles - 1; tile >= 0; --tile) {
    const long long t0 = tile * kScanTile;
    const int n = static_cast<int>(min(static_cast<long long>(kScanTile), p.steps - t0));
    float h = p.carry[(b * tiles + tile) * p.channels + d];
    for (int k = 0; k < n; ++k) {
      const long long t = t0 + k;
      before[k] = h;
      if (t >= len) continue;
      float a, c;
      gate_coefs<kMode>(to_float(g[t * p.gt]), a, c);
      const float u = kMode == kGateValue ? to_float(x[t * p.xt]) : c * to_float(x[t * p.xt]);
      if (p.reset && p.reset[b * p.steps + t]) { before[k] = 0.0f; h = u; }
      else h = fmaf(a, h, u);
    }
    for (int k = n - 1; k >= 0; --k) {
      const long long t = t0 + k;
      float gx = 0.0f, gg = 0.0f;
      if (t < len) {
        float a, c;
        gate_coefs<kMode>(to_float(g[t * p.gt]), a, c);
        const float dh = to_float(dy[t * p.yt]) + flow;
        gx = kMode == kGateValue ? dh : dh * c;
        gg = kMode == kGateValue ? dh * before[k] : dh * (before[k] - to_float(x[t * p.xt])) * a * c;
        flow = p.reset && p.reset[b * p.steps + t] ? 0.0f : a * dh;
      }
      dx[t * p.dxt] = from_float<T>(gx);
      if (p.partial) p.partial[(b * p.steps + t) * p.channels + d] = gg;
      else static_cast<T*>(p.dgate)[b * p.dgb + t * p.dgt + d] = from_float<T>(gg);
    }
  }
  if (p.dh0) p.dh0[i] = flow;
}

// dgate of a shared gate: the sum over its channels, in a fixed order.
template <typename T>
__global__ void __launch_bounds__(256) scan_gate_sum_kernel(const ScanParams p) {
  const long long gates = p.channels / p.group;
  const long long n = p.batch * p.steps * gates;
  for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n;
       i += static_cast<long long>(gridDim.x) * blockDim.x) {
    const long long bt = i / gates, k = i - bt * gates, b = bt / p.steps, t = bt - b * p.steps;
    const float* v = p.partial + bt * p.channels + k * p.group;
    float s = 0.0f;
    for (int j = 0; j < p.group; ++j) s += v[j];
    static_cast<T*>(p.dgate)[b * p.dgb + t * p.dgt + k] = from_float<T>(s);
  }
}

}  // namespace adapt
