// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient of the log probability and the entropy.
//   z = scale x,  lse = m + ln sum e^(z - m),  logprob = z_t - lse,
//   H = ln s - (sum e^(z - m) (z - m)) / s,
//   dx_j = scale (dlp ([j = t] - p_j) - dH p_j (ln p_j + H)).
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kMaxTop = 32;

struct LogprobParams {
  const void* logits;
  long long rows, ld, ld_grad;
  int vocab, n_top;
  float scale;
  const long long* targets;  // may be null
  float *logprob, *entropy, *lse;   // each may be null
  int* top_ids;
  float* top_logprobs;
  const float *d_logprob, *d_entropy;   // each may be null
  void* dlogits;                        // may be null
  const float *lse_in, *entropy_in;     // backward alone
};

// Order of the alternatives: larger logit first, equal ones (and +-0) by the lower index, NaN before
// everything.  One 64-bit key, all keys of a row distinct.
__device__ __forceinline__ unsigned long long top_key(float v, int j) {
  unsigned b = __float_as_uint(__fadd_rn(v, 0.0f));
  b = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
  if (v != v) b = 0xFFFFFFFFu;
  return (static_cast<unsigned long long>(b) << 32) | (0xFFFFFFFFu - static_cast<unsigned>(j));
}

// One element's gradient from its log probability.
__device__ __forceinline__ float logprob_grad(float logp, bool hot, float dlp, float dh, float h) {
  const float p = expf(logp);
  float g = (hot ? dlp : 0.0f) - dlp * p;
  if (dh != 0.0f && p > 0.0f) g -= dh * p * (logp + h);
  return g;
}

constexpr int kRowThreads = 256;

template <typename F>
__device__ __forceinline__ float row_reduce(float v, float* sh, F f) {
  __syncthreads();
  sh[threadIdx.x] = v;
  __syncthreads();
  for (int w = kRowThreads / 2; w > 0; w >>= 1) {
    if (threadIdx.x < w) sh[threadIdx.x] = f(sh[threadIdx.x], sh[threadIdx.x + w]);
    __syncthreads();
  }
  return sh[0];
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) logprob_kernel(const LogprobParams p) {
  __shared__ float sh[kRowThreads];
  __shared__ unsigned long long best[kRowThreads];
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  T* dx = p.dlogits ? static_cast<T*>(p.dlogits) + row * p.ld_grad : nullptr;
  const long long target = p.targets ? p.targets[row] : 0;
  const bool backward_only = p.lse_in != nullptr;
  if (target < 0) {   // a row without a target: not read, all zero
    if (!backward_only && threadIdx.x == 0) {
      if (p.logprob) p.logprob[row] = 0.0f;
      if (p.entropy) p.entropy[row] = 0.0f;
      if (p.lse) p.lse[row] = 0.0f;
      for (int k = 0; k < p.n_top; ++k) { p.top_ids[row * p.n_top + k] = -1; p.top_logprobs[row * p.n_top + k] = 0.0f; }
    }
    if (dx) for (int j = threadIdx.x; j < p.vocab; j += kRowThreads) dx[j] = from_float<T>(0.0f);
    return;
  }
  float lse, h;
  if (!backward_only) {
    float m = -INFINITY;
    bool nan = false;
    for (int j = threadIdx.x; j < p.vocab; j += kRowThreads) {
      const float v = to_float(x[j]) * p.scale;
      nan |= v != v;
      m = fmaxf(m, v);
    }
    m = row_reduce(m, sh, [](float a, float b) { return fmaxf(a, b); });
    const bool bad = row_reduce(nan ? 1.0f : 0.0f, sh, [](float a, float b) { return fmaxf(a, b); }) != 0.0f || m == INFINITY;
    float s = 0.0f, w = 0.0f;
    for (int j = threadIdx.x; j < p.vocab; j += kRowThreads) {
      const float t = to_float(x[j]) * p.scale - m;
      const float e = expf(t);
      s += e;
      if (e > 0.0f) w += e * t;
    }
    s = row_reduce(s, sh, [](float a, float b) { return a + b; });
    w = row_reduce(w, sh, [](float a, float b) { return a + b; });
    lse = m + logf(s);
    h = logf(s) - w / s;
    if (m == -INFINITY) { lse = -INFINITY; h = 0.0f; }
    if (bad) lse = h = NAN;
    if (threadIdx.x == 0) {
      if (p.logprob) {
        float lp = target < p.vocab ? to_float(x[target]) * p.scale - lse : NAN;
        if (lse == -INFINITY && target < p.vocab) lp = -INFINITY;
        p.logprob[row] = lp;
      }
      if (p.entropy) p.entropy[row] = h;
      if (p.lse) p.lse[row] = lse;
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < p.n_top; ++k) {
      unsigned long long b = 0;
      for (int j = threadIdx.x; j < p.vocab; j += kRowThreads) {
        const unsigned long long key = top_key(to_float(x[j]), j);
        if (key < last && key > b) b = key;
      }
      __syncthreads();
      best[threadIdx.x] = b;
      __syncthreads();
      for (int w2 = kRowThreads / 2; w2 > 0; w2 >>= 1) {
        if (threadIdx.x < w2) best[threadIdx.x] = max(best[threadIdx.x], best[threadIdx.x + w2]);
        __syncthreads();
      }
      last = best[0];
      if (threadIdx.x == 0) {
        const int j = static_cast<int>(0xFFFFFFFFu - static_cast<unsigned>(last));
        p.top_ids[row * p.n_top + k] = j;
        p.top_logprobs[row * p.n_top + k] = lse == -INFINITY ? -INFINITY : to_float(x[j]) * p.scale - lse;
      }
    }
  } else {
    lse = p.lse_in[row];
    h = p.entropy_in ? p.entropy_in[row] : 0.0f;
  }
  if (dx) {
    __syncthreads();
    const float dlp = p.d_logprob ? p.d_logprob[row] : 0.0f, dh = p.d_entropy ? p.d_entropy[row] : 0.0f;
    for (int j = threadIdx.x; j < p.vocab; j += kRowThreads) {
      float g = 0.0f;
      if (lse != -INFINITY) g = p.scale * logprob_grad(to_float(x[j]) * p.scale - lse, j == target, dlp, dh, h);
      if (p.d_logprob && target >= p.vocab) g = NAN;
      dx[j] = from_float<T>(g);
    }
  }
}

}  // namespace adapt
