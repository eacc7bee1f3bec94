// Rows to 8-bit codes, and the product of codes with scales for each token and channel.
//
//   m = max |x_k|,  code_k = rne(x_k fl(127 / m)),  scale = m / 127
//   y_ij = (x_scale_i weight_scale_j) sum_k x_ik w_jk (+ bias_j),   the sum in int32: exact
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "k_elem.cuh"

namespace adapt {

constexpr float kInt8Least = 7.8886090522101181e-31f;   // 2^-100: 127 / m stays in fp32's range

// ---- rows to codes -------------------------------------------------------------------------------

struct RowsParams {
  const void* x;
  signed char* codes;
  float* scales;
  long long ldx, ld_codes;
  int rows, cols;
};

// The largest magnitude as a bit pattern: those of NaN and Inf are above all others.
struct RowScale { float inverse, scale; };
__device__ __forceinline__ RowScale row_scale(unsigned largest) {
  if (largest >= 0x7F800000u) return {0.0f, __int_as_float(0x7FC00000)};
  const float m = fmaxf(__uint_as_float(largest), kInt8Least);
  return {127.0f / m, m / 127.0f};
}

// rne(x r) of the unrounded product: it is rounded once, in the addition, to a multiple of 1.
__device__ __forceinline__ int to_code(float x, float r) {
  return __float_as_int(fmaf(x, r, 12582912.0f)) - 0x4B400000;
}

constexpr int kRowsThreads = 256;

template <typename T>
__global__ __launch_bounds__(kRowsThreads) void int8_rows_kernel(RowsParams q) {
  __shared__ unsigned largest_of[kRowsThreads / 32];
  const T* x = static_cast<const T*>(q.x) + blockIdx.x * q.ldx;
  signed char* codes = q.codes + blockIdx.x * q.ld_codes;
  unsigned largest = 0;
  for (int c = threadIdx.x; c < q.cols; c += kRowsThreads) largest = max(largest, __float_as_uint(fabsf(to_float(x[c]))));
  largest = __reduce_max_sync(~0u, largest);
  if ((threadIdx.x & 31) == 0) largest_of[threadIdx.x >> 5] = largest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowsThreads / 32; ++w) largest = max(largest, largest_of[w]);
  const RowScale s = row_scale(largest);
  for (int c = threadIdx.x; c < q.cols; c += kRowsThreads)
    codes[c] = static_cast<signed char>(s.inverse != 0.0f ? to_code(to_float(x[c]), s.inverse) : 0);
  if (threadIdx.x == 0) q.scales[blockIdx.x] = s.scale;
}

// ---- product -------------------------------------------------------------------------------------

struct LinearParams {
  const signed char *x, *w;
  const float *x_scales, *w_scales, *bias;
  void* y;
  long long ldx, ldw, ldy;
  int rows, n, k;
  bool x_one, w_one;   // one scale for all
};

template <typename T>
__device__ __forceinline__ T linear_out(const LinearParams& q, int sum, int i, int j) {
  float v = static_cast<float>(sum) * q.x_scales[q.x_one ? 0 : i] * q.w_scales[q.w_one ? 0 : j];
  if (q.bias) v += q.bias[j];
  return from_float<T>(v);
}

constexpr int kTile = 64;

// Tiles of 64 x 64, codes of any alignment.
template <typename T>
__global__ __launch_bounds__(256) void int8_any_kernel(LinearParams q) {
  __shared__ signed char xs[kTile][kTile + 4], ws[kTile][kTile + 4];
  const int row0 = blockIdx.y * kTile, col0 = blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int sum[4][4] = {};
  for (int k0 = 0; k0 < q.k; k0 += kTile) {
    for (int i = threadIdx.x; i < kTile * kTile; i += 256) {
      const int r = i / kTile, c = i % kTile;
      xs[r][c] = row0 + r < q.rows && k0 + c < q.k ? q.x[(row0 + r) * q.ldx + k0 + c] : 0;
      ws[r][c] = col0 + r < q.n && k0 + c < q.k ? q.w[(col0 + r) * q.ldw + k0 + c] : 0;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kTile; c += 4) {
      int a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        a[u] = *reinterpret_cast<const int*>(&xs[ty + 16 * u][c]);
        b[u] = *reinterpret_cast<const int*>(&ws[tx + 16 * u][c]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[u][v] = __dp4a(a[u], b[v], sum[u][v]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = row0 + ty + 16 * u, j = col0 + tx + 16 * v;
      if (i < q.rows && j < q.n) static_cast<T*>(q.y)[i * q.ldy + j] = linear_out<T>(q, sum[u][v], i, j);
    }
}

}  // namespace adapt
