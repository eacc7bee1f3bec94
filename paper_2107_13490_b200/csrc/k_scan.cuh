// Gated linear recurrence: h_t = a_t h_{t-1} + b_t per channel.
//   sigmoid form: a = s(g), b = (1 - a) x;   value form: a = g, b = x.
// At a reset h_{t-1} counts as 0; steps at or beyond a sequence's length leave the state alone.
// States are fp32.  The state before every kScanTile-th step can be kept (carry) for the backward
// pass, which recomputes the states in between in fp32:
//   dh_t = dy_t + a_{t+1} dh_{t+1},  dx = dh db/dx,  dg = dh (h_{t-1} da/dg + db/dg).
#pragma once

#include "k_elem.cuh"

namespace adapt {

constexpr int kScanTile = 64;        // steps of a tile
constexpr int kScanChannels = 64;    // channels of a CTA: two for each lane
constexpr int kScanSteps = 8;        // steps of a thread
constexpr int kScanWarps = kScanTile / kScanSteps;
constexpr int kScanThreads = 32 * kScanWarps;
constexpr int kScanStages = 2;       // tiles in shared memory: the one worked on and the next
constexpr int kScanMaxCluster = 16;
constexpr int kGateSigmoid = 0, kGateValue = 1;

struct ScanParams {
  const void *x, *gate, *dy;
  void *y, *dx, *dgate;
  const float *h0, *dh_last;
  float *h_last, *dh0, *carry;        // carry is read by the backward pass
  const int* lengths;
  const unsigned char* reset;
  float* partial;                      // gate gradients summed over 64 channels, where a gate has more
  long long batch, steps, channels;
  long long xb, xt, gb, gt, yb, yt;    // strides (elements) of x, gate, y / dy
  long long dxb, dxt, dgb, dgt;        // strides of dx, dgate
  int group;
};

// a and the factor of x (1 - a, or 1).  e^-g is held below 2^125 so that 1 - a = e^-g a stays a
// number; NaN passes through.  ex2 and rcp are good to a few units of 2^-23.
template <int kMode>
__device__ __forceinline__ void gate_coefs(float g, float& a, float& c) {
  if (kMode == kGateValue) { a = g; c = 1.0f; return; }
  float e;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(e) : "f"(g * -1.4426950408889634f), "f"(125.0f));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.0f + e));
  c = e * a;
}

// ---- short sequences: one thread a channel, step after step ------------------------------------

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

// ---- tiles -------------------------------------------------------------------------------------
//
// A chain is 64 channels of one sequence.  The CTAs of a cluster take its tiles of 64 steps in
// turn (tile s K + rank in round s), a thread two channels and 8 steps of a tile.  Threads reduce
// their steps to h -> A h + B, the 8 warps of a tile join through shared memory, the tiles of a round
// through the cluster's: every CTA sends its tile's (A, B) to all others, one cluster barrier a round.
// So the data is read once, whatever the number of chains, and nothing is kept in global memory.
// A reset's cut is carried as a flag (it is the same for all channels), not as a factor of 0: what the
// state holds before it, Inf and NaN included, must not come through.

__device__ __forceinline__ float through(bool cut, float a, float b, float h) {
  return cut || h == 0.0f ? b : fmaf(a, h, b);
}

__device__ __forceinline__ unsigned scan_smem(const void* p) {
  return static_cast<unsigned>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_size() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_address(unsigned addr, unsigned rank) {
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_store(unsigned addr, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(addr), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void cluster_store(unsigned addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Two neighbouring channels as they lie in memory.
template <typename T> struct ScanPair { T v[2]; };
template <> struct __align__(8) ScanPair<float> { float v[2]; };
template <> struct __align__(4) ScanPair<__half> { __half v[2]; };
template <> struct __align__(4) ScanPair<__nv_bfloat16> { __nv_bfloat16 v[2]; };

template <typename T>
__device__ __forceinline__ float2 widen(const ScanPair<T>& p) { return make_float2(to_float(p.v[0]), to_float(p.v[1])); }

// Copies (asynchronously, where alignment allows) a thread's pairs of `kScanSteps` rows into its own
// slots of a stage; rows at or beyond `rows` and channels beyond the last are filled with zeros.
template <typename T, bool kAsync>
__device__ __forceinline__ void fetch_rows(ScanPair<T>* slot, const T* src, long long stride, int rows, int channels) {
#pragma unroll
  for (int k = 0; k < kScanSteps; ++k) {
    const T* q = src + k * stride;
    if (kAsync) {
      const int n = k < rows && channels > 0 ? static_cast<int>(sizeof(ScanPair<T>)) : 0;
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::
                   "r"(scan_smem(slot + k * kScanThreads)), "l"(n ? q : src), "n"(sizeof(ScanPair<T>)), "r"(n) : "memory");
    } else {
      ScanPair<T> v;
      v.v[0] = k < rows && channels > 0 ? q[0] : from_float<T>(0.0f);
      v.v[1] = k < rows && channels > 1 ? q[1] : from_float<T>(0.0f);
      slot[k * kScanThreads] = v;
    }
  }
}
// The same for a gate that serves both channels.
template <typename T>
__device__ __forceinline__ void fetch_shared_gate(ScanPair<T>* slot, const T* src, long long stride, int rows, int channels) {
#pragma unroll
  for (int k = 0; k < kScanSteps; ++k) {
    ScanPair<T> v;
    v.v[0] = v.v[1] = k < rows && channels > 0 ? src[k * stride] : from_float<T>(0.0f);
    slot[k * kScanThreads] = v;
  }
}

template <typename T, bool kAsync>
__device__ __forceinline__ void store_pair(T* dst, float a, float b, int channels) {
  if (kAsync) {
    if (channels > 0) {
      ScanPair<T> v;
      v.v[0] = from_float<T>(a); v.v[1] = from_float<T>(b);
      *reinterpret_cast<ScanPair<T>*>(dst) = v;
    }
  } else {
    if (channels > 0) dst[0] = from_float<T>(a);
    if (channels > 1) dst[1] = from_float<T>(b);
  }
}

__host__ __device__ constexpr size_t scan_stage_bytes(int tensors, size_t elem) {
  return static_cast<size_t>(kScanThreads) * kScanSteps * 2 * elem * tensors;
}
__host__ __device__ constexpr size_t scan_totals_bytes(int cluster) {
  return cluster > 1 ? 2 * static_cast<size_t>(cluster) * (kScanChannels * sizeof(float2) + sizeof(unsigned)) : 0;
}

// What forward and backward share: where a thread stands.
struct ScanPlace {
  long long b, len;
  int rank, cluster, warp, lane, tiles, rounds;
  int c0, channels;   // first of the thread's two channels, how many of them exist
  __device__ __forceinline__ ScanPlace(const ScanParams& p) {
    rank = cluster_rank(); cluster = cluster_size();
    warp = threadIdx.x >> 5; lane = threadIdx.x & 31;
    const unsigned blocks = static_cast<unsigned>((p.channels + kScanChannels - 1) / kScanChannels);
    const unsigned chain = blockIdx.x / cluster;
    b = chain / blocks;
    c0 = static_cast<int>(chain % blocks) * kScanChannels + 2 * lane;
    channels = max(0, min(2, static_cast<int>(p.channels) - c0));
    len = p.lengths ? min(max(static_cast<long long>(p.lengths[b]), 0ll), p.steps) : p.steps;
    tiles = static_cast<int>((p.steps + kScanTile - 1) / kScanTile);
    rounds = (tiles + cluster - 1) / cluster;
  }
  // first step of this warp in its tile of round s
  __device__ __forceinline__ long long first(int s) const {
    return (static_cast<long long>(s) * cluster + rank) * kScanTile + warp * kScanSteps;
  }
  __device__ __forceinline__ int live(int s) const {   // how many of the warp's steps are before the length
    return static_cast<int>(max(0ll, min(static_cast<long long>(kScanSteps), len - first(s))));
  }
  __device__ __forceinline__ unsigned reset_byte(const ScanParams& p, int s) const {   // lane k: step k's byte
    return p.reset && lane < live(s) ? p.reset[b * p.steps + first(s) + lane] : 0u;
  }
};

// A tile's map for 64 channels, sent to every CTA of the cluster (buffer of this round): the threads
// take a channel each and share the receivers out.
__device__ __forceinline__ void send_totals(float2* totals, unsigned* cuts, const ScanPlace& w, int buffer, float a, float b, bool cut) {
  const int ch = threadIdx.x & 63;
  const unsigned at = scan_smem(totals + (buffer * w.cluster + w.rank) * kScanChannels + ch);
  const unsigned flag = scan_smem(cuts + buffer * w.cluster + w.rank);
  for (int q = threadIdx.x >> 6; q < w.cluster; q += kScanThreads / kScanChannels) {
    cluster_store(cluster_address(at, q), make_float2(a, b));
    if (ch == 0) cluster_store(cluster_address(flag, q), cut ? 1u : 0u);
  }
  __syncwarp();
  cluster_sync();
}

// What bounds it: HBM (2 reads and a write an element); the arithmetic is about 20 lane instructions
// an element.
template <typename T, int kMode, bool kAsync>
__global__ void __launch_bounds__(kScanThreads) scan_kernel(const ScanParams p) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ float4 maps[2][kScanWarps][32];    // {A, B} of the lane's two channels
  __shared__ unsigned warp_cut[2][kScanWarps];
  const ScanPlace w(p);
  ScanPair<T>* stage = reinterpret_cast<ScanPair<T>*>(dynamic) + threadIdx.x;
  float2* totals = reinterpret_cast<float2*>(dynamic + kScanStages * scan_stage_bytes(2, sizeof(T)));
  unsigned* cuts = reinterpret_cast<unsigned*>(totals + 2 * w.cluster * kScanChannels);
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.c0;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + w.c0 / p.group;
  T* y = static_cast<T*>(p.y) + w.b * p.yb + w.c0;

  auto fetch = [&](int s) {
    if (s < w.rounds) {
      ScanPair<T>* slot = stage + (s & 1) * (2 * kScanSteps * kScanThreads);
      const long long t = w.first(s);
      const int n = w.live(s);
      fetch_rows<T, kAsync>(slot, n ? x + t * p.xt : x, p.xt, n, w.channels);
      slot += kScanSteps * kScanThreads;
      if (p.group > 1) fetch_shared_gate<T>(slot, gate + (n ? t * p.gt : 0), p.gt, n, w.channels);
      else fetch_rows<T, kAsync>(slot, n ? gate + t * p.gt : gate, p.gt, n, w.channels);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  float2 state = make_float2(0.0f, 0.0f);
  if (p.h0) {
    const float* h0 = p.h0 + w.b * p.channels + w.c0;
    if (w.channels > 0) state.x = h0[0];
    if (w.channels > 1) state.y = h0[1];
  }
  if (w.cluster > 1) cluster_sync();   // every CTA of the cluster is there, and has read h0
  fetch(0);
  unsigned next_reset = w.rounds ? w.reset_byte(p, 0) : 0u;
  for (int s = 0; s < w.rounds; ++s) {
    fetch(s + 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    const int live = w.live(s);
    const unsigned resets = __ballot_sync(~0u, next_reset != 0);
    next_reset = s + 1 < w.rounds ? w.reset_byte(p, s + 1) : 0u;

    float2 a[kScanSteps], u[kScanSteps];
    float2 A = make_float2(1.0f, 1.0f), Bv = make_float2(0.0f, 0.0f);
    const ScanPair<T>* slot = stage + (s & 1) * (2 * kScanSteps * kScanThreads);
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) {
      const float2 xv = widen(slot[k * kScanThreads]), gv = widen(slot[(kScanSteps + k) * kScanThreads]);
      float2 c;
      gate_coefs<kMode>(gv.x, a[k].x, c.x);
      gate_coefs<kMode>(gv.y, a[k].y, c.y);
      u[k] = kMode == kGateValue ? xv : make_float2(c.x * xv.x, c.y * xv.y);
      if (k >= live) { a[k] = make_float2(1.0f, 1.0f); u[k] = make_float2(0.0f, 0.0f); }
      if (resets >> k & 1) {
        Bv = u[k];
      } else {
        Bv.x = fmaf(a[k].x, Bv.x, u[k].x); Bv.y = fmaf(a[k].y, Bv.y, u[k].y);
      }
      A.x *= a[k].x; A.y *= a[k].y;
    }
    const int buffer = s & 1;
    maps[buffer][w.warp][w.lane] = make_float4(A.x, Bv.x, A.y, Bv.y);
    if (w.lane == 0) warp_cut[buffer][w.warp] = resets;
    __syncthreads();

    float2 in = state;      // the state before this tile
    if (w.cluster > 1) {
      const float2* map = reinterpret_cast<const float2*>(maps[buffer]) + (threadIdx.x & 63);
      float ta = 1.0f, tb = 0.0f;
      bool cut = false;
#pragma unroll
      for (int v = 0; v < kScanWarps; ++v) {
        const float2 m = map[v * kScanChannels];
        const bool cv = warp_cut[buffer][v] != 0;
        tb = through(cv, m.x, m.y, tb);
        ta *= m.x;
        cut |= cv;
      }
      send_totals(totals, cuts, w, buffer, ta, tb, cut);
      const float4* all = reinterpret_cast<const float4*>(totals + buffer * w.cluster * kScanChannels) + w.lane;
      for (int q = 0; q < w.cluster; ++q) {
        if (q == w.rank) in = state;
        const float4 m = all[q * (kScanChannels / 2)];
        const bool cv = cuts[buffer * w.cluster + q] != 0;
        state.x = through(cv, m.x, m.y, state.x);
        state.y = through(cv, m.z, m.w, state.y);
      }
    }
    float2 h = in, mine = in;
#pragma unroll
    for (int v = 0; v < kScanWarps; ++v) {
      if (v == w.warp) mine = h;
      if (w.cluster > 1 && v >= w.warp) break;
      const float4 m = maps[buffer][v][w.lane];
      const bool cv = warp_cut[buffer][v] != 0;
      h.x = through(cv, m.x, m.y, h.x);
      h.y = through(cv, m.z, m.w, h.y);
    }
    if (w.cluster == 1) state = h;

    const long long t = w.first(s);
    const int tile = s * w.cluster + w.rank;
    if (p.carry && w.warp == 0 && tile < w.tiles) {
      float* at = p.carry + (w.b * w.tiles + tile) * p.channels + w.c0;
      if (w.channels > 0) at[0] = in.x;
      if (w.channels > 1) at[1] = in.y;
    }
    const int rows = static_cast<int>(max(0ll, min(static_cast<long long>(kScanSteps), p.steps - t)));
    h = mine;
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) {
      if (resets >> k & 1) {
        h = u[k];
      } else {
        h.x = fmaf(a[k].x, h.x, u[k].x); h.y = fmaf(a[k].y, h.y, u[k].y);
      }
      if (k < rows) {
        const bool on = k < live;
        store_pair<T, kAsync>(y + (t + k) * p.yt, on ? h.x : 0.0f, on ? h.y : 0.0f, w.channels);
      }
    }
  }
  if (p.h_last && w.rank == 0 && w.warp == 0) {
    float* at = p.h_last + w.b * p.channels + w.c0;
    if (w.channels > 0) at[0] = state.x;
    if (w.channels > 1) at[1] = state.y;
  }
}

// The reverse: the flow R of the gradient through the state, tiles from the last to the first.  Each
// tile starts its states from carry, so only R is handed from tile to tile.
template <typename T, int kMode, bool kAsync>
__global__ void __launch_bounds__(kScanThreads) scan_backward_kernel(const ScanParams p) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ float4 maps[2][kScanWarps][32];      // {A, B} of the states
  __shared__ float2 flows[2][kScanWarps][32];     // B of the gradient flow (A is the same)
  __shared__ unsigned warp_cut[2][kScanWarps];
  const ScanPlace w(p);
  ScanPair<T>* stage = reinterpret_cast<ScanPair<T>*>(dynamic) + threadIdx.x;
  float2* totals = reinterpret_cast<float2*>(dynamic + kScanStages * scan_stage_bytes(3, sizeof(T)));
  unsigned* cuts = reinterpret_cast<unsigned*>(totals + 2 * w.cluster * kScanChannels);
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.c0;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + w.c0 / p.group;
  const T* dy = static_cast<const T*>(p.dy) + w.b * p.yb + w.c0;
  T* dx = static_cast<T*>(p.dx) + w.b * p.dxb + w.c0;
  T* dgate = static_cast<T*>(p.dgate) + w.b * p.dgb + w.c0 / p.group;

  auto fetch = [&](int s) {
    if (s >= 0) {
      ScanPair<T>* slot = stage + (s & 1) * (3 * kScanSteps * kScanThreads);
      const long long t = w.first(s);
      const int n = w.live(s);
      fetch_rows<T, kAsync>(slot, n ? x + t * p.xt : x, p.xt, n, w.channels);
      slot += kScanSteps * kScanThreads;
      if (p.group > 1) fetch_shared_gate<T>(slot, gate + (n ? t * p.gt : 0), p.gt, n, w.channels);
      else fetch_rows<T, kAsync>(slot, n ? gate + t * p.gt : gate, p.gt, n, w.channels);
      slot += kScanSteps * kScanThreads;
      fetch_rows<T, kAsync>(slot, n ? dy + t * p.yt : dy, p.yt, n, w.channels);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto kept_state = [&](int s) {
    float2 h = make_float2(0.0f, 0.0f);
    const int tile = s * w.cluster + w.rank;
    if (s >= 0 && tile < w.tiles) {
      const float* at = p.carry + (w.b * w.tiles + tile) * p.channels + w.c0;
      if (w.channels > 0) h.x = at[0];
      if (w.channels > 1) h.y = at[1];
    }
    return h;
  };

  float2 flow = make_float2(0.0f, 0.0f);
  if (p.dh_last) {
    const float* at = p.dh_last + w.b * p.channels + w.c0;
    if (w.channels > 0) flow.x = at[0];
    if (w.channels > 1) flow.y = at[1];
  }
  if (w.cluster > 1) cluster_sync();
  fetch(w.rounds - 1);
  unsigned next_reset = w.rounds ? w.reset_byte(p, w.rounds - 1) : 0u;
  float2 next_state = kept_state(w.rounds - 1);
  for (int s = w.rounds - 1; s >= 0; --s) {
    fetch(s - 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    const int live = w.live(s);
    const unsigned resets = __ballot_sync(~0u, next_reset != 0);
    next_reset = s > 0 ? w.reset_byte(p, s - 1) : 0u;
    const float2 start = next_state;
    next_state = kept_state(s - 1);

    float2 a[kScanSteps], c[kScanSteps];
    float2 A = make_float2(1.0f, 1.0f), Bv = make_float2(0.0f, 0.0f);
    const ScanPair<T>* slot = stage + (s & 1) * (3 * kScanSteps * kScanThreads);
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) {
      const float2 xv = widen(slot[k * kScanThreads]), gv = widen(slot[(kScanSteps + k) * kScanThreads]);
      gate_coefs<kMode>(gv.x, a[k].x, c[k].x);
      gate_coefs<kMode>(gv.y, a[k].y, c[k].y);
      if (k >= live) { a[k] = make_float2(1.0f, 1.0f); c[k] = make_float2(0.0f, 0.0f); }
      const float2 u = make_float2(c[k].x * xv.x, c[k].y * xv.y);
      if (resets >> k & 1) {
        Bv = u;
      } else {
        Bv.x = fmaf(a[k].x, Bv.x, u.x); Bv.y = fmaf(a[k].y, Bv.y, u.y);
      }
      A.x *= a[k].x; A.y *= a[k].y;
    }
    float2 Q = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = kScanSteps - 1; k >= 0; --k) {
      const float2 g = widen(slot[(2 * kScanSteps + k) * kScanThreads]);
      Q.x = a[k].x * (g.x + Q.x); Q.y = a[k].y * (g.y + Q.y);
      if (resets >> k & 1) Q = make_float2(0.0f, 0.0f);
    }
    const int buffer = s & 1;
    maps[buffer][w.warp][w.lane] = make_float4(A.x, Bv.x, A.y, Bv.y);
    flows[buffer][w.warp][w.lane] = Q;
    if (w.lane == 0) warp_cut[buffer][w.warp] = resets;
    __syncthreads();

    float2 in = flow;       // the flow that comes from behind this tile
    if (w.cluster > 1) {
      const float2* map = reinterpret_cast<const float2*>(maps[buffer]) + (threadIdx.x & 63);
      const float* fl = reinterpret_cast<const float*>(flows[buffer]) + (threadIdx.x & 63);
      float ta = 1.0f, tb = 0.0f;
      bool cut = false;
#pragma unroll
      for (int v = kScanWarps - 1; v >= 0; --v) {
        const float m = map[v * kScanChannels].x;
        const bool cv = warp_cut[buffer][v] != 0;
        tb = through(cv, m, fl[v * kScanChannels], tb);
        ta *= m;
        cut |= cv;
      }
      send_totals(totals, cuts, w, buffer, ta, tb, cut);
      const float4* all = reinterpret_cast<const float4*>(totals + buffer * w.cluster * kScanChannels) + w.lane;
      for (int q = w.cluster - 1; q >= 0; --q) {
        if (q == w.rank) in = flow;
        const float4 m = all[q * (kScanChannels / 2)];
        const bool cv = cuts[buffer * w.cluster + q] != 0;
        flow.x = through(cv, m.x, m.y, flow.x);
        flow.y = through(cv, m.z, m.w, flow.y);
      }
    }
    float2 r = in, mine = in;
#pragma unroll
    for (int v = kScanWarps - 1; v >= 0; --v) {
      if (v == w.warp) mine = r;
      if (w.cluster > 1 && v <= w.warp) break;
      const float4 m = maps[buffer][v][w.lane];
      const float2 f = flows[buffer][v][w.lane];
      const bool cv = warp_cut[buffer][v] != 0;
      r.x = through(cv, m.x, f.x, r.x);
      r.y = through(cv, m.z, f.y, r.y);
    }
    if (w.cluster == 1) flow = r;
    float2 h = start;
#pragma unroll
    for (int v = 0; v < kScanWarps - 1; ++v) {
      if (v >= w.warp) break;
      const float4 m = maps[buffer][v][w.lane];
      const bool cv = warp_cut[buffer][v] != 0;
      h.x = through(cv, m.x, m.y, h.x);
      h.y = through(cv, m.z, m.w, h.y);
    }

    float2 before[kScanSteps];
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) {
      const float2 xv = widen(slot[k * kScanThreads]);
      const bool cut = resets >> k & 1;
      before[k] = cut ? make_float2(0.0f, 0.0f) : h;
      const float2 u = make_float2(c[k].x * xv.x, c[k].y * xv.y);
      h.x = cut ? u.x : fmaf(a[k].x, h.x, u.x);
      h.y = cut ? u.y : fmaf(a[k].y, h.y, u.y);
    }
    const long long t = w.first(s);
    const int rows = static_cast<int>(max(0ll, min(static_cast<long long>(kScanSteps), p.steps - t)));
    r = mine;
#pragma unroll
    for (int k = kScanSteps - 1; k >= 0; --k) {
      const float2 xv = widen(slot[k * kScanThreads]), g = widen(slot[(2 * kScanSteps + k) * kScanThreads]);
      const float2 dh = make_float2(g.x + r.x, g.y + r.y);
      const bool on = k < live;
      float2 gx, gg;
      if (kMode == kGateValue) {
        gx = dh;
        gg = make_float2(dh.x * before[k].x, dh.y * before[k].y);
      } else {
        gx = make_float2(dh.x * c[k].x, dh.y * c[k].y);
        gg = make_float2(gx.x * a[k].x * (before[k].x - xv.x), gx.y * a[k].y * (before[k].y - xv.y));
      }
      if (!on) { gx = make_float2(0.0f, 0.0f); gg = gx; }
      r.x = a[k].x * dh.x; r.y = a[k].y * dh.y;
      if (resets >> k & 1) r = make_float2(0.0f, 0.0f);
      if (k < rows) store_pair<T, kAsync>(dx + (t + k) * p.dxt, gx.x, gx.y, w.channels);
      if (p.group == 1) {
        if (k < rows) store_pair<T, kAsync>(dgate + (t + k) * p.dgt, gg.x, gg.y, w.channels);
      } else {
        // sum over the gate's channels: the lanes that share it, by halving distances
        float sum = w.channels > 0 ? gg.x + (w.channels > 1 ? gg.y : 0.0f) : 0.0f;
        const int lanes = min(p.group, kScanChannels) / 2;
        for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (k < rows && w.channels > 0 && (w.lane & (lanes - 1)) == 0) {
          if (p.partial)
            p.partial[(w.b * p.steps + t + k) * (p.channels / kScanChannels) + w.c0 / kScanChannels] = sum;
          else
            dgate[(t + k) * p.dgt] = from_float<T>(sum);
        }
      }
    }
  }
  if (p.dh0 && w.rank == 0 && w.warp == 0) {
    float* at = p.dh0 + w.b * p.channels + w.c0;
    if (w.channels > 0) at[0] = flow.x;
    if (w.channels > 1) at[1] = flow.y;
  }
}

// dgate of a gate with more than 64 channels: the sum of its blocks' partial sums, in order.
template <typename T>
__global__ void __launch_bounds__(256) scan_gate_sum_kernel(const ScanParams p) {
  const long long gates = p.channels / p.group;
  const int parts = p.group / kScanChannels;
  const long long n = p.batch * p.steps * gates;
  for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n;
       i += static_cast<long long>(gridDim.x) * blockDim.x) {
    const long long bt = i / gates, k = i - bt * gates, b = bt / p.steps, t = bt - b * p.steps;
    const float* v = p.partial + i * parts;
    float s = 0.0f;
    for (int j = 0; j < parts; ++j) s += v[j];
    static_cast<T*>(p.dgate)[b * p.dgb + t * p.dgt + k] = from_float<T>(s);
  }
}

}  // namespace adapt
