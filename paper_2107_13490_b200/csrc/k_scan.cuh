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

constexpr f32x2 kOnes2 = 0x3F8000003F800000ull, kMinusOnes2 = 0xBF800000BF800000ull;

// a and the factor of x (1 - a, or 1).  e^-g is held at 2^125 so that 1 - a = e^-g a stays a
// number; NaN passes through.  ex2 and rcp are good to a few units of 2^-23.
__device__ __forceinline__ float held_exp2(float v) {
  float e;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(e) : "f"(v), "f"(125.0f));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e));
  return e;
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
template <int kMode>
__device__ __forceinline__ void gate_coefs(float g, float& a, float& c) {
  if (kMode == kGateValue) { a = g; c = 1.0f; return; }
  const float e = held_exp2(g * -1.4426950408889634f);
  a = reciprocal(1.0f + e);
  c = e * a;
}
template <int kMode>
__device__ __forceinline__ void gate_coefs2(f32x2 g, f32x2& a, f32x2& c) {
  if (kMode == kGateValue) { a = g; c = kOnes2; return; }
  const float2 v = unpack2(mul2(g, pack2(-1.4426950408889634f, -1.4426950408889634f)));
  const f32x2 e = pack2(held_exp2(v.x), held_exp2(v.y));
  const float2 d = unpack2(add2(e, kOnes2));
  a = pack2(reciprocal(d.x), reciprocal(d.y));
  c = mul2(e, a);
}

// ---- short sequences: a thread runs through the steps of one or four channels -------------------------

constexpr int kSerialAhead = 4;   // steps whose inputs are under way

template <typename T, int kWide> struct __align__(kWide * sizeof(T)) ScanWide { T v[kWide]; };

template <typename T, int kMode, int kWide>
__global__ void __launch_bounds__(128) scan_serial_kernel(const ScanParams p) {
  typedef ScanWide<T, kWide> Wide;
  const int threads = static_cast<int>(p.channels / kWide);   // of a sequence
  const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.batch * threads) return;
  const long long b = i / threads;
  const int d = static_cast<int>(i - b * threads) * kWide, steps = static_cast<int>(p.steps);
  const int len = p.lengths ? min(max(p.lengths[b], 0), steps) : steps;
  const T* x = static_cast<const T*>(p.x) + b * p.xb + d;
  const bool shared_gate = p.group > 1;   // (then one gate serves all of the thread's channels)
  const T* g = static_cast<const T*>(p.gate) + b * p.gb + (shared_gate ? d / p.group : d);
  T* y = static_cast<T*>(p.y) + b * p.yb + d;
  const unsigned char* reset = p.reset ? p.reset + b * p.steps : nullptr;
  float h[kWide];
#pragma unroll
  for (int j = 0; j < kWide; ++j) h[j] = p.h0 ? p.h0[b * p.channels + d + j] : 0.0f;
  const int tiles = (steps + kScanTile - 1) / kScanTile;
  for (int t0 = 0; t0 < steps; t0 += kSerialAhead) {
    Wide xv[kSerialAhead], gv[kSerialAhead];
    bool cut[kSerialAhead];
#pragma unroll
    for (int k = 0; k < kSerialAhead; ++k) {
      const int t = t0 + k;
      if (t >= len) continue;
      xv[k] = *reinterpret_cast<const Wide*>(x + t * p.xt);
      if (shared_gate) gv[k].v[0] = g[t * p.gt];
      else gv[k] = *reinterpret_cast<const Wide*>(g + t * p.gt);
      cut[k] = reset && reset[t];
    }
#pragma unroll
    for (int k = 0; k < kSerialAhead; ++k) {
      const int t = t0 + k;
      if (t >= steps) break;
      if (p.carry && t % kScanTile == 0) {
        float* at = p.carry + (b * tiles + t / kScanTile) * p.channels + d;
#pragma unroll
        for (int j = 0; j < kWide; ++j) at[j] = h[j];
      }
      Wide out;
#pragma unroll
      for (int j = 0; j < kWide; ++j) {
        out.v[j] = from_float<T>(0.0f);
        if (t >= len) continue;
        float a, c;
        gate_coefs<kMode>(to_float(gv[k].v[shared_gate ? 0 : j]), a, c);
        const float u = kMode == kGateValue ? to_float(xv[k].v[j]) : c * to_float(xv[k].v[j]);
        h[j] = cut[k] ? u : fmaf(a, h[j], u);
        out.v[j] = from_float<T>(h[j]);
      }
      *reinterpret_cast<Wide*>(y + t * p.yt) = out;
    }
  }
  if (p.h_last) {
#pragma unroll
    for (int j = 0; j < kWide; ++j) p.h_last[b * p.channels + d + j] = h[j];
  }
}

// ---- tiles -------------------------------------------------------------------------------------
//
// A chain is a block of 64, 32 or 16 channels of one sequence (kLanes lanes of two channels); a tile is
// 4096 of its elements, 64, 128 or 256 steps.  A thread has two channels and 8 steps of a tile - a piece -
// and reduces them to h -> A h + B; the pieces of a tile join through shared memory.  The CTAs of a
// cluster take a chain's tiles in turn (tile s K + rank in round s) and send each other their tiles'
// (A, B), so the data is read once whatever the number of chains, and nothing goes through global memory.
// A reset's cut is carried as a flag (it is the same for all channels), not as a factor of 0: what the
// state holds before it, Inf and NaN included, must not come through.

template <bool kCut>
__device__ __forceinline__ float through(bool cut, float a, float b, float h) {
  return kCut && cut ? b : fmaf(a, h, b);
}
template <bool kCut>
__device__ __forceinline__ f32x2 through2(bool cut, f32x2 a, f32x2 b, f32x2 h) {
  return kCut && cut ? b : fma2(a, h, b);
}
// A product of decays, held finite so that a state of 0 stays 0 under it; NaN passes.
__device__ __forceinline__ float held(float a) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(3.0e38f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(r) : "f"(-3.0e38f));
  return r;
}
__device__ __forceinline__ f32x2 held2(f32x2 a) {
  const float2 v = unpack2(a);
  return pack2(held(v.x), held(v.y));
}
// f(true) or f(false), the argument a constant.
template <bool kValue> struct Flag { static constexpr bool value = kValue; };
template <typename F>
__device__ __forceinline__ void with_flag(bool v, F f) {
  if (v) f(Flag<true>{});
  else f(Flag<false>{});
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
// Remote stores that count themselves off at a barrier beside the data they write: no fence, so an
// exchange does not wait for the output rows on their way to memory.
__device__ __forceinline__ void cluster_store(unsigned addr, unsigned barrier, float2 v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
               :: "r"(addr), "f"(v.x), "f"(v.y), "r"(barrier) : "memory");
}
__device__ __forceinline__ void cluster_store(unsigned addr, unsigned barrier, unsigned v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];"
               :: "r"(addr), "r"(v), "r"(barrier) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned barrier, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(barrier), "r"(bytes) : "memory");
}
// Waits for a phase of a barrier, a bounded number of times; false if it never came.
__device__ __forceinline__ bool barrier_wait(unsigned barrier, unsigned parity) {
  for (int i = 0; i < (1 << 20); ++i) {
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(barrier), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Two neighbouring channels as they lie in memory.
template <typename T> struct Pair { typedef unsigned raw; };
template <> struct Pair<float> { typedef f32x2 raw; };

__device__ __forceinline__ f32x2 widen(f32x2 raw, float) { return raw; }
__device__ __forceinline__ f32x2 widen(unsigned raw, __nv_bfloat16) {
  return pack2(__uint_as_float(raw << 16), __uint_as_float(raw & 0xFFFF0000u));
}
__device__ __forceinline__ f32x2 widen(unsigned raw, __half) {
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&raw));
  return pack2(v.x, v.y);
}
__device__ __forceinline__ f32x2 narrow(f32x2 v, float) { return v; }
__device__ __forceinline__ unsigned narrow(f32x2 v, __nv_bfloat16) {
  const float2 f = unpack2(v);
  const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const unsigned*>(&r);
}
__device__ __forceinline__ unsigned narrow(f32x2 v, __half) {
  const float2 f = unpack2(v);
  const __half2 r = __floats2half2_rn(f.x, f.y);
  return *reinterpret_cast<const unsigned*>(&r);
}
// A pair from single elements.
__device__ __forceinline__ f32x2 join(float a, float b) { return pack2(a, b); }
template <typename T>
__device__ __forceinline__ unsigned join(T a, T b) {
  return static_cast<unsigned>(*reinterpret_cast<const unsigned short*>(&a)) |
         static_cast<unsigned>(*reinterpret_cast<const unsigned short*>(&b)) << 16;
}

// How a tile moves: 16 bytes at a time, two channels, or one.
constexpr int kMoveOne = 0, kMovePair = 1, kMoveVec = 2;

// Where a CTA and a thread stand.
template <int kLanes>
struct ScanPlace {
  static constexpr int kParts = 32 / kLanes;             // pieces side by side in a warp
  static constexpr int kPieces = kScanWarps * kParts;    // of a tile
  static constexpr int kTileSteps = kPieces * kScanSteps;
  static constexpr int kChannels = 2 * kLanes;
  long long b;
  int steps, len;     // of the call, of this sequence
  int rank, cluster, warp, lane, pair, piece, rounds;
  int block, left;    // first channel of the CTA's, how many there are
  int channels;       // how many of the thread's two exist
  __device__ __forceinline__ ScanPlace(const ScanParams& p) {
    rank = cluster_rank(); cluster = cluster_size();
    warp = threadIdx.x >> 5; lane = threadIdx.x & 31;
    pair = lane % kLanes; piece = warp * kParts + lane / kLanes;
    const unsigned blocks = static_cast<unsigned>((p.channels + kChannels - 1) / kChannels);
    const unsigned chain = blockIdx.x / cluster;
    b = chain / blocks;
    block = static_cast<int>(chain % blocks) * kChannels;
    left = min(kChannels, static_cast<int>(p.channels) - block);
    channels = max(0, min(2, left - 2 * pair));
    steps = static_cast<int>(p.steps);
    len = p.lengths ? min(max(p.lengths[b], 0), steps) : steps;
    const int tiles = (steps + kTileSteps - 1) / kTileSteps;
    rounds = (tiles + cluster - 1) / cluster;
  }
  // first step of this warp, of this thread, in its tile of round s; steps from round to round
  __device__ __forceinline__ int warp_first(int s) const { return (s * cluster + rank) * kTileSteps + warp * (kParts * kScanSteps); }
  __device__ __forceinline__ int first(int s) const { return (s * cluster + rank) * kTileSteps + piece * kScanSteps; }
  __device__ __forceinline__ int stride() const { return cluster * kTileSteps; }
  __device__ __forceinline__ static int clamp_steps(int n, int most) { return max(0, min(most, n)); }
  __device__ __forceinline__ int live(int s) const { return clamp_steps(len - first(s), kScanSteps); }   // before the length
  // lanes 0..7 of a piece: the reset bytes of its steps
  __device__ __forceinline__ unsigned reset_byte(const ScanParams& p, int s) const {
    return p.reset && pair < live(s) ? p.reset[b * p.steps + first(s) + pair] : 0u;
  }
  __device__ __forceinline__ unsigned reset_bits(unsigned byte) const {   // of this thread's piece
    return __ballot_sync(~0u, byte != 0) >> (lane - pair) & (kLanes < 32 ? (1u << (kLanes & 31)) - 1u : ~0u);
  }
};

// Copies a warp's rows of a tile into its part of a stage, asynchronously where the alignment allows;
// rows at or beyond `rows` and channels at or beyond `left` are filled with zeros.  src points to the
// warp's first row, the block's first channel.  With kMoveVec a lane's pairs come by other lanes'
// copies: __syncwarp() after the wait.
template <typename T, int kMove, int kLanes>
__device__ __forceinline__ void fetch_rows(unsigned char* part, const T* src, long long stride, int rows, int left) {
  typedef typename Pair<T>::raw Raw;
  const int lane = threadIdx.x & 31;
  if (kMove == kMoveVec) {
    constexpr int kChunk = 16 / sizeof(T), kRow = 2 * kLanes / kChunk, kStepRows = 32 / kRow;
    const int col = (lane % kRow) * kChunk, row = lane / kRow;
    src += row * stride + col;
    const unsigned at = scan_smem(part) + lane * 16;
    if (rows == 32 / kLanes * kScanSteps && left == 2 * kLanes) {
#pragma unroll
      for (int j = 0; j < static_cast<int>(sizeof(T)); ++j, src += kStepRows * stride)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(at + j * 512), "l"(src) : "memory");
      return;
    }
#pragma unroll
    for (int j = 0; j < static_cast<int>(sizeof(T)); ++j, src += kStepRows * stride) {
      if (j * kStepRows + row < rows && col < left)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(at + j * 512), "l"(src) : "memory");
      else
        *reinterpret_cast<uint4*>(part + j * 512 + lane * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    return;
  }
  const int pair = lane % kLanes, row0 = lane / kLanes * kScanSteps;
  Raw* slot = reinterpret_cast<Raw*>(part) + row0 * kLanes + pair;
  src += row0 * stride + 2 * pair;
#pragma unroll
  for (int k = 0; k < kScanSteps; ++k, src += stride) {
    const bool on = row0 + k < rows && 2 * pair < left;
    if (kMove == kMovePair) {
      if (on) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" :: "r"(scan_smem(slot + k * kLanes)), "l"(src), "n"(sizeof(Raw)) : "memory");
      else slot[k * kLanes] = 0;
    } else {
      const T zero = from_float<T>(0.0f);
      slot[k * kLanes] = join(on ? src[0] : zero, on && 2 * pair + 1 < left ? src[1] : zero);
    }
  }
}
// The same for a gate that serves both channels; src points to this pair's gate in the warp's first row.
template <typename T, int kLanes>
__device__ __forceinline__ void fetch_shared_gate(unsigned char* part, const T* src, long long stride, int rows, int left) {
  const int lane = threadIdx.x & 31, pair = lane % kLanes, row0 = lane / kLanes * kScanSteps;
  typename Pair<T>::raw* slot = reinterpret_cast<typename Pair<T>::raw*>(part) + row0 * kLanes + pair;
  src += row0 * stride;
#pragma unroll
  for (int k = 0; k < kScanSteps; ++k, src += stride) {
    const T v = row0 + k < rows && 2 * pair < left ? src[0] : from_float<T>(0.0f);
    slot[k * kLanes] = join(v, v);
  }
}

template <typename T, int kMove>
__device__ __forceinline__ void store_pair(T* dst, f32x2 v, int channels) {
  if (kMove != kMoveOne) {
    if (channels > 0) *reinterpret_cast<typename Pair<T>::raw*>(dst) = narrow(v, T{});
  } else {
    const float2 f = unpack2(v);
    if (channels > 0) dst[0] = from_float<T>(f.x);
    if (channels > 1) dst[1] = from_float<T>(f.y);
  }
}

constexpr int kTileElements = kScanThreads * kScanSteps * 2;
__host__ __device__ constexpr size_t scan_stage_bytes(int tensors, size_t elem) { return kTileElements * elem * tensors; }
__host__ __device__ constexpr size_t scan_totals_bytes(int cluster, int channels) {
  return cluster > 1 ? 2 * static_cast<size_t>(cluster) * (channels * sizeof(float2) + sizeof(unsigned)) : 0;
}

// The exchange of a cluster: every CTA sends its tile's map for its channels (and whether it is cut) to
// all others; two buffers, a barrier each.  A buffer is written again two rounds later, by CTAs that
// have by then received the round in between from every other one, which each sent after reading.
template <int kLanes>
struct ScanExchange {
  static constexpr int kChannels = 2 * kLanes;
  float2* totals;    // [2][cluster][kChannels]
  unsigned* cuts;    // [2][cluster]
  unsigned barrier;  // shared address of two barriers
  bool lost;         // a wait ran out (never, unless the hardware fails): states become NaN

  __device__ __forceinline__ ScanExchange(unsigned char* at, unsigned long long* barriers, const ScanPlace<kLanes>& w) {
    totals = reinterpret_cast<float2*>(at);
    cuts = reinterpret_cast<unsigned*>(totals + 2 * w.cluster * kChannels);
    barrier = scan_smem(barriers);
    lost = false;
    if (w.cluster == 1) return;
    if (threadIdx.x == 0) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(barrier) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(barrier + 8) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  // Called by all threads; thread i holds channel i % kChannels' map.
  template <bool kCut>
  __device__ __forceinline__ void send(const ScanPlace<kLanes>& w, int buffer, float a, float b, bool cut) {
    const int ch = threadIdx.x % kChannels;
    if (threadIdx.x == 0) barrier_expect(barrier + 8 * buffer, w.cluster * (kChannels * 8 + (kCut ? 4 : 0)));
    const unsigned at = scan_smem(totals + (buffer * w.cluster + w.rank) * kChannels + ch);
    const unsigned flag = scan_smem(cuts + buffer * w.cluster + w.rank);
    for (int q = threadIdx.x / kChannels; q < w.cluster; q += kScanThreads / kChannels) {
      const unsigned bar = cluster_address(barrier + 8 * buffer, q);
      cluster_store(cluster_address(at, q), bar, make_float2(a, b));
      if (kCut && ch == 0) cluster_store(cluster_address(flag, q), bar, cut ? 1u : 0u);
    }
  }
  // Called by the first kChannels threads, a channel each: the tiles of a round, first to last or last to
  // first; returns what leaves the round, puts what enters this CTA's tile into `enter`.
  template <bool kCut, bool kBackward>
  __device__ __forceinline__ float run(const ScanPlace<kLanes>& w, int buffer, unsigned parity, float e, float* enter) {
    if (!lost) lost = !barrier_wait(barrier + 8 * buffer, parity);
    if (lost) e = __int_as_float(0x7FFFFFFF);
    const float2* all = totals + buffer * w.cluster * kChannels + threadIdx.x;
    const unsigned* cut = cuts + buffer * w.cluster;
    const int last = w.cluster - 1;
#pragma unroll 1
    for (int i = 0; i <= last; i += 4) {   // four at a time: a cluster has 2, 4, 8 or 16
      float2 m[4];
      bool c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int q = min(i + j, last), at = kBackward ? last - q : q;
        m[j] = all[at * kChannels];
        c[j] = kCut && cut[at] != 0;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (i + j > last) break;
        if (i + j == (kBackward ? last - w.rank : w.rank)) enter[threadIdx.x] = e;
        e = through<kCut>(c[j], m[j].x, m[j].y, e);
      }
    }
    return e;
  }
};

// The state that is handed from tile to tile.  With one CTA to a chain the threads of the piece that a
// tile ends with hand it over in shared memory (`hand`, written before one barrier and read after the
// next); in a cluster the first kChannels threads hold a channel each (in the low half).
template <int kLanes>
__device__ __forceinline__ f32x2 get_state(const float* src, const ScanParams& p, const ScanPlace<kLanes>& w) {
  if (!src) return 0;
  src += w.b * p.channels + w.block;
  float a = 0.0f, b = 0.0f;
  if (w.cluster > 1) {
    if (static_cast<int>(threadIdx.x) < w.left) a = src[threadIdx.x];
  } else {
    if (w.channels > 0) a = src[2 * w.pair];
    if (w.channels > 1) b = src[2 * w.pair + 1];
  }
  return pack2(a, b);
}
template <int kLanes>
__device__ __forceinline__ void put_state(float* dst, const ScanParams& p, const ScanPlace<kLanes>& w, int last, f32x2 v) {
  dst += w.b * p.channels + w.block;
  const float2 f = unpack2(v);
  if (w.cluster > 1) {
    if (static_cast<int>(threadIdx.x) < w.left) dst[threadIdx.x] = f.x;
  } else if (w.piece == last) {
    if (w.channels > 0) dst[2 * w.pair] = f.x;
    if (w.channels > 1) dst[2 * w.pair + 1] = f.y;
  }
}
// A kept state: that before the 64-step stretch which holds step t.
template <int kLanes>
__device__ __forceinline__ float* carry_at(const ScanParams& p, const ScanPlace<kLanes>& w, int t) {
  return p.carry + (w.b * ((w.steps + kScanTile - 1) / kScanTile) + t / kScanTile) * p.channels + w.block + 2 * w.pair;
}

// The map of a piece, {A, B} pairs of its lane's channels.
struct __align__(16) ScanMap { f32x2 a, b; };
constexpr int kStretch = kScanTile / kScanSteps;   // pieces between two kept states

// Composes a tile's pieces for one channel (a thread a channel, each channel several times).
__device__ __forceinline__ float map_a(const ScanMap* maps, int ch) { return reinterpret_cast<const float*>(maps + (ch >> 1))[ch & 1]; }
__device__ __forceinline__ float map_b(const ScanMap* maps, int ch) { return reinterpret_cast<const float*>(maps + (ch >> 1))[2 + (ch & 1)]; }

// What bounds it: HBM (2 reads and a write an element); the arithmetic is about 20 lane instructions
// an element.
template <typename T, int kMode, int kMove, int kLanes>
__global__ void __launch_bounds__(kScanThreads, sizeof(T) == 4 ? 2 : 3) scan_kernel(const ScanParams p) {
  typedef typename Pair<T>::raw Raw;
  typedef ScanPlace<kLanes> Place;
  constexpr int kPieces = Place::kPieces;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ ScanMap maps[2][kPieces * kLanes];
  __shared__ __align__(8) float enter[Place::kChannels];   // cluster: the state before this CTA's tile
  __shared__ f32x2 hand[2][kLanes];
  __shared__ unsigned piece_cut[2][kPieces];
  __shared__ unsigned long long barriers[2];
  const Place w(p);
  constexpr int kPart = kTileElements / kScanWarps * sizeof(T);   // a warp's part of a tensor's stage
  unsigned char* stage = dynamic + w.warp * kPart;
  ScanExchange<kLanes> exchange(dynamic + kScanStages * scan_stage_bytes(2, sizeof(T)), barriers, w);
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.block;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + (p.group > 1 ? (w.block + 2 * w.pair) / p.group : w.block);
  T* y = static_cast<T*>(p.y) + w.b * p.yb + w.block + 2 * w.pair;

  // (the row pointers run ahead of what is read; behind the last step nothing is read through them)
  x += w.warp_first(0) * p.xt; gate += w.warp_first(0) * p.gt;
  auto fetch = [&](int s) {
    if (s < w.rounds) {
      unsigned char* part = stage + (s & 1) * (2 * kScanWarps * kPart);
      const int n = Place::clamp_steps(w.len - w.warp_first(s), Place::kParts * kScanSteps);
      fetch_rows<T, kMove, kLanes>(part, x, p.xt, n, w.left);
      part += kScanWarps * kPart;
      if (p.group > 1) fetch_shared_gate<T, kLanes>(part, gate, p.gt, n, w.left);
      else fetch_rows<T, kMove, kLanes>(part, gate, p.gt, n, w.left);
      x += w.stride() * p.xt; gate += w.stride() * p.gt;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  y += w.first(0) * p.yt;

  f32x2 state = get_state(p.h0, p, w);
  if (w.cluster > 1) cluster_sync();   // every CTA of the cluster is there, and has read h0
  else if (w.piece == kPieces - 1) hand[1][w.pair] = state;
  fetch(0);
  unsigned next_reset = w.rounds ? w.reset_byte(p, 0) : 0u;
  for (int s = 0; s < w.rounds; ++s) {
    fetch(s + 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (kMove == kMoveVec) __syncwarp();
    const int live = w.live(s);
    const unsigned resets = w.reset_bits(next_reset);
    next_reset = s + 1 < w.rounds ? w.reset_byte(p, s + 1) : 0u;

    f32x2 a[kScanSteps], u[kScanSteps];
    const Raw* slot = reinterpret_cast<const Raw*>(stage + (s & 1) * (2 * kScanWarps * kPart)) + (w.lane - w.pair) * kScanSteps + w.pair;
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) {
      const f32x2 xv = widen(slot[k * kLanes], T{});
      f32x2 c;
      gate_coefs2<kMode>(widen(slot[kTileElements / 2 + k * kLanes], T{}), a[k], c);
      u[k] = kMode == kGateValue ? xv : mul2(c, xv);
    }
    if (live < kScanSteps) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k)
        if (k >= live) { a[k] = kOnes2; u[k] = 0; }
    }
    f32x2 A = a[0], Bv = u[0];
#pragma unroll
    for (int k = 1; k < kScanSteps; ++k) {
      A = mul2(A, a[k]);
      Bv = fma2(a[k], Bv, u[k]);
    }
    if (resets) {   // what comes before the last reset does not count
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) Bv = through2<true>(resets >> k & 1, a[k], u[k], Bv);
    }
    const ScanMap* tile = maps[s & 1];
    const unsigned* tile_cut = piece_cut[s & 1];
    maps[s & 1][w.piece * kLanes + w.pair] = {held2(A), Bv};
    if (p.reset && w.pair == 0) piece_cut[s & 1][w.piece] = resets;
    __syncthreads();

    f32x2 h;    // the state before this tile, then before this piece
    with_flag(p.reset != nullptr, [&](auto cut) {
      constexpr bool kCut = decltype(cut)::value;
      if (w.cluster > 1) {
        const int ch = threadIdx.x % Place::kChannels;
        float ta = 1.0f, tb = 0.0f;
        bool any = false;
#pragma unroll 4
        for (int v = 0; v < kPieces; ++v) {
          const float ma = map_a(tile + v * kLanes, ch);
          const bool cv = kCut && tile_cut[v] != 0;
          tb = through<kCut>(cv, ma, map_b(tile + v * kLanes, ch), tb);
          ta *= ma;
          any |= cv;
        }
        exchange.template send<kCut>(w, s & 1, held(ta), tb, any);
        if (threadIdx.x < Place::kChannels)
          state = pack2(exchange.template run<kCut, false>(w, s & 1, s >> 1 & 1, unpack2(state).x, enter), 0.0f);
        __syncthreads();
        h = *reinterpret_cast<const f32x2*>(enter + 2 * w.pair);
      } else {
        h = hand[(s & 1) ^ 1][w.pair];
      }
#pragma unroll
      for (int v = 0; v < kPieces - 1; ++v) {
        if (v >= w.piece) break;
        const ScanMap m = tile[v * kLanes + w.pair];
        h = through2<kCut>(kCut && tile_cut[v] != 0, m.a, m.b, h);
      }
    });

    const int t = w.first(s);
    if (p.carry && w.piece % kStretch == 0 && t < w.steps) {
      float* at = carry_at(p, w, t);
      const float2 f = unpack2(h);
      if (w.channels > 0) at[0] = f.x;
      if (w.channels > 1) at[1] = f.y;
    }
    T* out = y;
    y += w.stride() * p.yt;
    if (live == kScanSteps && !resets) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k, out += p.yt) {
        h = fma2(a[k], h, u[k]);
        store_pair<T, kMove>(out, h, w.channels);
      }
    } else {
      const int rows = Place::clamp_steps(w.steps - t, kScanSteps);
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k, out += p.yt) {
        h = through2<true>(resets >> k & 1, a[k], u[k], h);
        if (k < rows) store_pair<T, kMove>(out, k < live ? h : 0, w.channels);
      }
    }
    if (w.cluster == 1 && w.piece == kPieces - 1) hand[s & 1][w.pair] = state = h;
  }
  if (p.h_last && w.rank == 0) put_state(p.h_last, p, w, kPieces - 1, state);
}

// The reverse: the flow of the gradient through the state, tiles from the last to the first.  Each
// stretch of 64 steps starts its states from carry, so only the flow is handed from tile to tile.
template <typename T, int kMode, int kMove, int kLanes>
__global__ void __launch_bounds__(kScanThreads, 2) scan_backward_kernel(const ScanParams p) {
  typedef typename Pair<T>::raw Raw;
  typedef ScanPlace<kLanes> Place;
  constexpr int kPieces = Place::kPieces;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ ScanMap maps[2][kPieces * kLanes];          // of the states
  __shared__ f32x2 flows[2][kPieces * kLanes];           // B of the gradient flow (A is the same)
  __shared__ __align__(8) float enter[Place::kChannels];   // cluster: the flow from behind this CTA's tile
  __shared__ f32x2 hand[2][kLanes];
  __shared__ unsigned piece_cut[2][kPieces];
  __shared__ unsigned long long barriers[2];
  const Place w(p);
  constexpr int kPart = kTileElements / kScanWarps * sizeof(T);
  unsigned char* stage = dynamic + w.warp * kPart;
  ScanExchange<kLanes> exchange(dynamic + kScanStages * scan_stage_bytes(3, sizeof(T)), barriers, w);
  const int c0 = w.block + 2 * w.pair;
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.block;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + (p.group > 1 ? c0 / p.group : w.block);
  const T* dy = static_cast<const T*>(p.dy) + w.b * p.yb + w.block;
  T* dx = static_cast<T*>(p.dx) + w.b * p.dxb + c0;
  T* dgate = static_cast<T*>(p.dgate) + w.b * p.dgb + c0 / p.group;

  const int last = w.rounds - 1;
  x += w.warp_first(last) * p.xt; gate += w.warp_first(last) * p.gt; dy += w.warp_first(last) * p.yt;
  auto fetch = [&](int s) {
    if (s >= 0) {
      unsigned char* part = stage + (s & 1) * (3 * kScanWarps * kPart);
      const int n = Place::clamp_steps(w.len - w.warp_first(s), Place::kParts * kScanSteps);
      fetch_rows<T, kMove, kLanes>(part, x, p.xt, n, w.left);
      part += kScanWarps * kPart;
      if (p.group > 1) fetch_shared_gate<T, kLanes>(part, gate, p.gt, n, w.left);
      else fetch_rows<T, kMove, kLanes>(part, gate, p.gt, n, w.left);
      part += kScanWarps * kPart;
      fetch_rows<T, kMove, kLanes>(part, dy, p.yt, n, w.left);
      x -= w.stride() * p.xt; gate -= w.stride() * p.gt; dy -= w.stride() * p.yt;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  dx += (w.first(last) + kScanSteps - 1) * p.dxt; dgate += (w.first(last) + kScanSteps - 1) * p.dgt;
  auto kept_state = [&](int s) {
    float a = 0.0f, b = 0.0f;
    const int t = w.first(s);
    if (s >= 0 && t < w.steps) {
      const float* at = carry_at(p, w, t);
      if (w.channels > 0) a = at[0];
      if (w.channels > 1) b = at[1];
    }
    return pack2(a, b);
  };

  f32x2 flow = get_state(p.dh_last, p, w);
  if (w.cluster > 1) cluster_sync();
  else if (w.piece == 0) hand[1][w.pair] = flow;
  fetch(w.rounds - 1);
  unsigned next_reset = w.rounds ? w.reset_byte(p, w.rounds - 1) : 0u;
  f32x2 next_state = w.rounds ? kept_state(w.rounds - 1) : 0;
  for (int s = w.rounds - 1; s >= 0; --s) {
    fetch(s - 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (kMove == kMoveVec) __syncwarp();
    const int live = w.live(s);
    const unsigned resets = w.reset_bits(next_reset);
    next_reset = s > 0 ? w.reset_byte(p, s - 1) : 0u;
    f32x2 h = next_state, r;      // the state before this piece, the flow from behind it
    next_state = kept_state(s - 1);

    f32x2 a[kScanSteps], c[kScanSteps];
    const Raw* slot = reinterpret_cast<const Raw*>(stage + (s & 1) * (3 * kScanWarps * kPart)) + (w.lane - w.pair) * kScanSteps + w.pair;
    constexpr int kGate = kTileElements / 2, kDy = kTileElements;
#pragma unroll
    for (int k = 0; k < kScanSteps; ++k) gate_coefs2<kMode>(widen(slot[kGate + k * kLanes], T{}), a[k], c[k]);
    if (live < kScanSteps) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k)
        if (k >= live) { a[k] = kOnes2; c[k] = 0; }
    }
    auto added = [&](int k) {   // what step k adds to the state
      const f32x2 xv = widen(slot[k * kLanes], T{});
      return kMode == kGateValue ? xv : mul2(c[k], xv);
    };
    f32x2 A = kOnes2, Bv = 0, Q = 0;
    with_flag(resets != 0, [&](auto cut) {
      constexpr bool kCut = decltype(cut)::value;
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) {
        A = k ? mul2(A, a[k]) : a[k];
        Bv = through2<kCut>(kCut && resets >> k & 1, a[k], added(k), Bv);
      }
#pragma unroll
      for (int k = kScanSteps - 1; k >= 0; --k) {
        Q = mul2(a[k], add2(widen(slot[kDy + k * kLanes], T{}), Q));
        if (kCut && resets >> k & 1) Q = 0;
      }
    });
    const int round = w.rounds - 1 - s, buffer = round & 1;
    const ScanMap* tile = maps[buffer];
    const f32x2* tile_flow = flows[buffer];
    const unsigned* tile_cut = piece_cut[buffer];
    maps[buffer][w.piece * kLanes + w.pair] = {held2(A), Bv};
    flows[buffer][w.piece * kLanes + w.pair] = Q;
    if (p.reset && w.pair == 0) piece_cut[buffer][w.piece] = resets;
    __syncthreads();

    with_flag(p.reset != nullptr, [&](auto cut) {
      constexpr bool kCut = decltype(cut)::value;
      if (w.cluster > 1) {
        const int ch = threadIdx.x % Place::kChannels;
        float ta = 1.0f, tb = 0.0f;
        bool any = false;
#pragma unroll 4
        for (int v = kPieces - 1; v >= 0; --v) {
          const float ma = map_a(tile + v * kLanes, ch);
          const bool cv = kCut && tile_cut[v] != 0;
          tb = through<kCut>(cv, ma, reinterpret_cast<const float*>(tile_flow + v * kLanes)[ch], tb);
          ta *= ma;
          any |= cv;
        }
        exchange.template send<kCut>(w, buffer, held(ta), tb, any);
        if (threadIdx.x < Place::kChannels)
          flow = pack2(exchange.template run<kCut, true>(w, buffer, round >> 1 & 1, unpack2(flow).x, enter), 0.0f);
        __syncthreads();
        r = *reinterpret_cast<const f32x2*>(enter + 2 * w.pair);
      } else {
        r = hand[buffer ^ 1][w.pair];
      }
#pragma unroll
      for (int v = kPieces - 1; v > 0; --v) {
        if (v <= w.piece) break;
        r = through2<kCut>(kCut && tile_cut[v] != 0, tile[v * kLanes + w.pair].a, tile_flow[v * kLanes + w.pair], r);
      }
      const int from = w.piece / kStretch * kStretch;
#pragma unroll
      for (int v = 0; v < kStretch - 1; ++v) {
        if (from + v >= w.piece) break;
        const ScanMap m = tile[(from + v) * kLanes + w.pair];
        h = through2<kCut>(kCut && tile_cut[from + v] != 0, m.a, m.b, h);
      }
    });

    const int t = w.first(s);
    const int rows = Place::clamp_steps(w.steps - t, kScanSteps);
    // (the sums below shuffle across the warp, so its pieces take the same way)
    with_flag(__all_sync(~0u, resets == 0 && live == kScanSteps), [&](auto whole) {   // every step there, none cut
      constexpr bool kWhole = decltype(whole)::value;
      f32x2 before[kScanSteps];
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) {
        if (!kWhole && resets >> k & 1) h = 0;
        before[k] = h;
        h = fma2(a[k], h, added(k));
      }
      T* gx_at = dx;
      T* gg_at = dgate;
      const int lanes = min(p.group, kScanChannels) / 2;   // that share a gate
#pragma unroll
      for (int k = kScanSteps - 1; k >= 0; --k, gx_at -= p.dxt, gg_at -= p.dgt) {
        const f32x2 dh = add2(widen(slot[kDy + k * kLanes], T{}), r);
        f32x2 gx, gg;
        if (kMode == kGateValue) {
          gx = dh;
          gg = mul2(dh, before[k]);
        } else {
          gx = mul2(dh, c[k]);
          gg = mul2(mul2(gx, a[k]), fma2(widen(slot[k * kLanes], T{}), kMinusOnes2, before[k]));
        }
        r = mul2(a[k], dh);
        if (!kWhole) {
          if (k >= live) gx = gg = 0;
          if (resets >> k & 1) r = 0;
        }
        const bool on = kWhole || k < rows;
        if (on) store_pair<T, kMove>(gx_at, gx, w.channels);
        if (p.group == 1) {
          if (on) store_pair<T, kMove>(gg_at, gg, w.channels);
        } else {
          // sum over the gate's channels: the lanes that share it, by doubling distances
          const float2 f = unpack2(gg);
          float sum = w.channels > 0 ? f.x + (w.channels > 1 ? f.y : 0.0f) : 0.0f;
          for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor_sync(~0u, sum, o);
          if (on && w.channels > 0 && (w.pair & (lanes - 1)) == 0) {
            if (p.partial)
              p.partial[(w.b * p.steps + t + k) * (p.channels / kScanChannels) + c0 / kScanChannels] = sum;
            else
              *gg_at = from_float<T>(sum);
          }
        }
      }
    });
    dx -= w.stride() * p.dxt; dgate -= w.stride() * p.dgt;
    if (w.cluster == 1 && w.piece == 0) hand[buffer][w.pair] = flow = r;
  }
  if (p.dh0 && w.rank == 0) put_state(p.dh0, p, w, 0, flow);
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
