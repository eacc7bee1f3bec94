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
// A CTA walks over rows, a row at a time; a thread holds kElems elements of it.  Where all rows are 16-byte
// aligned (kStaged) they come through a ring of stages in shared memory that bulk copies fill rows ahead, so that
// loads are under way while the sums of a row meet; others are read where they lie, element by element.
//
// dim 4096, bf16: 256 threads of 16 elements, two CTAs of two stages an SM for the backward pass.

constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxStages = 4;

struct NormRing {
  int streams, stages;       // rows of a stage, stages
  int slot[5];               // place of block, residual, gate, d_y, d_normed in a stage, -1: none
};

// Sums over a CTA, in one of two sets of places in turn, so that one barrier each is enough.
struct CtaSums {
  float2 (*places)[kNormMaxThreads / 32];
  int turn;
  __device__ __forceinline__ float2 operator()(float a, float b) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      a += __shfl_xor_sync(~0u, a, d);
      b += __shfl_xor_sync(~0u, b, d);
    }
    if (blockDim.x == 32) { __syncwarp(); return make_float2(a, b); }
    if ((threadIdx.x & 31) == 0) places[turn][threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = places[turn][0];
    for (unsigned w = 1; w < blockDim.x / 32; ++w) { const float2 p = places[turn][w]; s.x += p.x; s.y += p.y; }
    turn ^= 1;
    return s;
  }
};

// The rows of a CTA in order, read ahead into the ring by its first thread.
template <typename T, bool kStaged>
struct NormRows {
  const NormParams& q;
  const NormRing& ring;
  unsigned stages, bars;     // addresses
  int row_bytes;
  unsigned use;
  __device__ __forceinline__ NormRows(const NormParams& q_, const NormRing& r, unsigned char* smem, unsigned long long* b)
      : q(q_), ring(r), stages(shared_address(smem)), bars(shared_address(b)), row_bytes(q_.dim * static_cast<int>(sizeof(T))), use(0) {
    if constexpr (kStaged) {
      if (threadIdx.x == 0) {
        for (int s = 0; s < ring.stages; ++s) barrier_init(bars + 8 * s, 1);
        barrier_init_fence();
        for (int s = 0; s < ring.stages; ++s) fill(s, static_cast<long long>(blockIdx.x) + static_cast<long long>(s) * gridDim.x);
      }
      __syncthreads();
    }
  }
  __device__ __forceinline__ void fill(int s, long long r) const {
    if (r >= q.rows) return;
    barrier_expect_bytes(bars + 8 * s, ring.streams * row_bytes);
    const void* from[5] = {q.block, q.residual, q.gate, q.d_y, q.d_normed};
    const long long ld[5] = {q.ld_block, q.ld_residual, q.ld_gate, q.ld_d_y, q.ld_d_normed};
#pragma unroll
    for (int i = 0; i < 5; ++i)
      if (ring.slot[i] >= 0)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     :: "r"(stages + (s * ring.streams + ring.slot[i]) * row_bytes), "l"(static_cast<const T*>(from[i]) + r * ld[i]), "r"(row_bytes),
                        "r"(bars + 8 * s) : "memory");
  }
  // Waits for the row's data; 0, or NaN where they never came.
  __device__ __forceinline__ float ready() const {
    if constexpr (kStaged)
      if (!barrier_wait(bars + 8 * (use % ring.stages), (use / ring.stages) & 1)) return __int_as_float(0x7FC00000);
    return 0.0f;
  }
  // Called when every thread has read what it needs of the row `r`.
  __device__ __forceinline__ void release(long long r) {
    if constexpr (kStaged) {
      if (threadIdx.x == 0) fill(use % ring.stages, r + static_cast<long long>(ring.stages) * gridDim.x);
      ++use;
    }
  }
  // Elements c .. c + V - 1 of stream kStream of row r, which has to be there.
  template <int kStream, int V>
  __device__ __forceinline__ void read(long long r, int c, float (&f)[V]) const {
    if constexpr (kStaged) {
      uint4 raw;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w)
                   : "r"(stages + ((use % ring.stages) * ring.streams + ring.slot[kStream]) * row_bytes + c * static_cast<int>(sizeof(T))));
      unpack16<T>(raw, f);
    } else {
      const void* from = kStream == 0 ? q.block : kStream == 1 ? q.residual : kStream == 2 ? q.gate : kStream == 3 ? q.d_y : q.d_normed;
      const long long ld = kStream == 0 ? q.ld_block : kStream == 1 ? q.ld_residual : kStream == 2 ? q.ld_gate : kStream == 3 ? q.ld_d_y : q.ld_d_normed;
      f[0] = to_float(static_cast<const T*>(from)[r * ld + c]);
    }
  }
};

template <int V>
__device__ __forceinline__ void read_weights(const float* w, int c, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = __ldg(w + c);
  } else {
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(w + c + k));
      f[k] = t.x; f[k + 1] = t.y; f[k + 2] = t.z; f[k + 3] = t.w;
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void write_part(T* p, const float (&f)[V]) {
  if constexpr (V == 1) *p = from_float<T>(f[0]);
  else __stcs(reinterpret_cast<uint4*>(p), pack16<T>(f));
}

template <typename T, bool kStaged>
__host__ __device__ constexpr int norm_unit() { return kStaged ? 16 / static_cast<int>(sizeof(T)) : 1; }

template <typename T, int kElems, bool kStaged>
__global__ __launch_bounds__(kNormMaxThreads, kElems <= 16 ? 2 : 1) void norm_row_kernel(const NormParams q, const NormRing ring) {
  constexpr int V = norm_unit<T, kStaged>(), kChunks = kElems / V;
  extern __shared__ __align__(128) unsigned char norm_smem[];
  __shared__ __align__(8) unsigned long long bars[kNormMaxStages];
  __shared__ float2 places[2][kNormMaxThreads / 32];
  NormRows<T, kStaged> rows(q, ring, norm_smem, bars);
  CtaSums sums{places, 0};
  const float inv = 1.0f / static_cast<float>(q.dim);
  auto column = [&](int i) { return (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * V; };
  // mean and 1 / deviation; the deviation around the mean, in a second sum
  auto statistics = [&](const float (&v)[kElems], int kind) {
    float mean = 0.0f, s = 0.0f;
    if (kind == kNormLayer) {
#pragma unroll
      for (int j = 0; j < kElems; ++j) s += v[j];   // (0 beyond the row)
      mean = sums(s, 0.0f).x * inv;
      s = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (column(i) >= q.dim) break;
#pragma unroll
      for (int k = 0; k < V; ++k) { const float d = v[i * V + k] - mean; s = fmaf(d, d, s); }
    }
    return make_float2(mean, rsqrtf(fmaf(sums(s, 0.0f).x, inv, q.eps)));
  };
  for (long long r = blockIdx.x; r < q.rows; r += gridDim.x) {
    const float poison = rows.ready();
    float v[kElems];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      float f[V] = {};
      const int c = column(i);
      if (c < q.dim) rows.template read<0>(r, c, f);
#pragma unroll
      for (int k = 0; k < V; ++k) v[i * V + k] = f[k];
    }
    v[0] += poison;
    float2 a = make_float2(0.0f, 1.0f), b = a;
    if (q.after != kNormNone) a = statistics(v, q.after);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = column(i);
      if (c >= q.dim) break;
      float g[V], w[V];
      if (q.after != kNormNone) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[i * V + k] = (v[i * V + k] - a.x) * a.y;
        if (q.weight_after) {
          read_weights<V>(q.weight_after, c, w);
#pragma unroll
          for (int k = 0; k < V; ++k) v[i * V + k] *= w[k];
        }
      }
      if (q.gate) {
        if (q.shared) read_weights<V>(static_cast<const float*>(q.gate), c, g); else rows.template read<2>(r, c, g);
#pragma unroll
        for (int k = 0; k < V; ++k) v[i * V + k] *= norm_gate(g[k], q.sigmoid).open;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) v[i * V + k] *= q.scale;
      if (q.residual) {
        rows.template read<1>(r, c, g);
#pragma unroll
        for (int k = 0; k < V; ++k) v[i * V + k] = fmaf(g[k], q.residual_scale, v[i * V + k]);
      }
    }
    if (q.before != kNormNone) b = statistics(v, q.before); else __syncthreads();
    rows.release(r);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = column(i);
      if (c >= q.dim) break;
      float f[V], w[V];
      if (q.y) {
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = v[i * V + k];
        write_part<T, V>(static_cast<T*>(q.y) + r * q.ld_y + c, f);
      }
      if (q.normed) {
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = (v[i * V + k] - b.x) * b.y;
        if (q.weight_before) {
          read_weights<V>(q.weight_before, c, w);
#pragma unroll
          for (int k = 0; k < V; ++k) f[k] *= w[k];
        }
        write_part<T, V>(static_cast<T*>(q.normed) + r * q.ld_normed + c, f);
      }
    }
    if (q.stats && threadIdx.x == 0) reinterpret_cast<float4*>(q.stats)[r] = make_float4(a.x, a.y, b.x, b.y);
  }
}

// The gate of the first phase kept in one number for the second: the smaller of g and 1 - g (the other is 1 minus it,
// to a rounding), with the sign that says which.
__device__ __forceinline__ float gate_kept(float v, bool sigmoid) {
  if (!sigmoid) return v;
  const float t = __expf(-fabsf(v));
  return copysignf(__fdividef(t, 1.0f + t), v);
}
__device__ __forceinline__ Gate gate_again(float kept, bool sigmoid) {
  if (!sigmoid) return {kept, 1.0f};
  const float least = fabsf(kept), most = 1.0f - least;
  return {signbit(kept) ? least : most, least * most};
}

template <typename T, int kElems, bool kStaged, bool kSharedGate>
__global__ __launch_bounds__(kNormMaxThreads, 1) void norm_row_backward_kernel(const NormParams q, const NormRing ring) {
  constexpr int V = norm_unit<T, kStaged>(), kChunks = kElems / V;
  extern __shared__ __align__(128) unsigned char norm_smem[];
  __shared__ __align__(8) unsigned long long bars[kNormMaxStages];
  __shared__ float2 places[2][kNormMaxThreads / 32];
  NormRows<T, kStaged> rows(q, ring, norm_smem, bars);
  CtaSums sums{places, 0};
  const float inv = 1.0f / static_cast<float>(q.dim);
  auto column = [&](int i) { return (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * V; };
  float of_after[kElems] = {}, of_before[kElems] = {}, of_gate[kSharedGate ? kElems : 1] = {};   // sums over rows
  for (long long r = blockIdx.x; r < q.rows; r += gridDim.x) {
    const float4 st = __ldg(reinterpret_cast<const float4*>(q.stats_in) + r);
    const float poison = rows.ready();
    float one[kElems], two[kElems];   // norm_before(y) and the gate; then the gradient of norm_after's output and the output
    auto block_hat = [&](int c, float (&hat)[V], float (&value)[V]) {
      rows.template read<0>(r, c, hat);
      if (q.after != kNormNone) {
#pragma unroll
        for (int k = 0; k < V; ++k) hat[k] = (hat[k] - st.x) * st.y;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) value[k] = hat[k];
      if (q.weight_after) {
        float w[V];
        read_weights<V>(q.weight_after, c, w);
#pragma unroll
        for (int k = 0; k < V; ++k) value[k] *= w[k];
      }
    };
    auto keep_gate = [&](int i, int c) {
      float g[V];
      if (kSharedGate) read_weights<V>(static_cast<const float*>(q.gate), c, g);
      else if (q.gate) rows.template read<2>(r, c, g);
#pragma unroll
      for (int k = 0; k < V; ++k) two[i * V + k] = q.gate ? gate_kept(g[k], q.sigmoid) : 1.0f;
    };
    float2 m = make_float2(0.0f, 0.0f);
    if (q.d_normed) {
      float sh = 0.0f, s = poison;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int c = column(i);
        if (c >= q.dim) break;
        float hat[V], value[V], f[V];
        block_hat(c, hat, value);
        keep_gate(i, c);
#pragma unroll
        for (int k = 0; k < V; ++k) value[k] *= gate_again(two[i * V + k], q.sigmoid).open * q.scale;
        if (q.residual) {
          rows.template read<1>(r, c, f);
#pragma unroll
          for (int k = 0; k < V; ++k) value[k] = fmaf(f[k], q.residual_scale, value[k]);
        }
        rows.template read<4>(r, c, f);
        float w[V];
        if (q.weight_before) read_weights<V>(q.weight_before, c, w);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float y_hat = (value[k] - st.z) * st.w, d = q.weight_before ? f[k] * w[k] : f[k];
          one[i * V + k] = y_hat;
          of_before[i * V + k] = fmaf(f[k], y_hat, of_before[i * V + k]);
          sh = fmaf(d, y_hat, sh);
          s += d;
        }
      }
      m = sums(sh, s);
      m.x *= inv;
      m.y = q.before == kNormLayer ? m.y * inv : poison;
    }
    float sh = 0.0f, s = poison;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = column(i);
      if (c >= q.dim) break;
      float hat[V], value[V], d[V] = {}, f[V];
      block_hat(c, hat, value);
      if (!q.d_normed) keep_gate(i, c);
      if (q.d_y) rows.template read<3>(r, c, d);
      if (q.d_normed) {
        float w[V];
        rows.template read<4>(r, c, f);
        if (q.weight_before) read_weights<V>(q.weight_before, c, w);
#pragma unroll
        for (int k = 0; k < V; ++k)
          d[k] = fmaf(fmaf(-one[i * V + k], m.x, q.weight_before ? f[k] * w[k] : f[k]) - m.y, st.w, d[k]);
      }
      if (q.d_residual) {
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = d[k] * q.residual_scale;
        write_part<T, V>(static_cast<T*>(q.d_residual) + r * q.ld_d_residual + c, f);
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const Gate gate = gate_again(two[i * V + k], q.sigmoid);
        d[k] *= q.scale;
        f[k] = d[k] * value[k] * gate.slope;
        d[k] *= gate.open;
        if (kSharedGate) of_gate[kSharedGate ? i * V + k : 0] += f[k];
      }
      if (!kSharedGate && q.d_gate) write_part<T, V>(static_cast<T*>(q.d_gate) + r * q.ld_d_gate + c, f);
      if (q.after != kNormNone) {
        float w[V];
        if (q.weight_after) read_weights<V>(q.weight_after, c, w);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          of_after[i * V + k] = fmaf(d[k], hat[k], of_after[i * V + k]);
          if (q.weight_after) d[k] *= w[k];
          sh = fmaf(d[k], hat[k], sh);
          s += d[k];
        }
      }
#pragma unroll
      for (int k = 0; k < V; ++k) { one[i * V + k] = d[k]; two[i * V + k] = hat[k]; }
    }
    if (q.after != kNormNone) {
      m = sums(sh, s);
      m.x *= inv;
      m.y = q.after == kNormLayer ? m.y * inv : poison;
    } else {
      __syncthreads();
    }
    rows.release(r);
    if (!q.d_block) continue;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = column(i);
      if (c >= q.dim) break;
      float f[V];
#pragma unroll
      for (int k = 0; k < V; ++k)
        f[k] = q.after != kNormNone ? (fmaf(-two[i * V + k], m.x, one[i * V + k]) - m.y) * st.y : one[i * V + k];
      write_part<T, V>(static_cast<T*>(q.d_block) + r * q.ld_d_block + c, f);
    }
  }
  if (!q.partial) return;
  const long long plane = static_cast<long long>(gridDim.x) * q.dim;
  float* mine = q.partial + static_cast<long long>(blockIdx.x) * q.dim;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = column(i);
    if (c >= q.dim) break;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (kSharedGate) mine[c + k] = of_gate[kSharedGate ? i * V + k : 0];
      mine[plane + c + k] = of_after[i * V + k];
      mine[2 * plane + c + k] = of_before[i * V + k];
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
