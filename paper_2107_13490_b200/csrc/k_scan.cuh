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
constexpr int kAhead = 2;            // warps' maps read at a time (4: 4 % slower, registers)
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
  bool gate_words;                     // the 4-byte words of a row's gates lie within the row
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
// and reduces them to h -> A h + B; the pieces of a warp join by shuffles, the warps of a tile through
// shared memory.  The CTAs of a cluster take a chain's tiles in turn (tile s K + rank in round s) and send
// each other their tiles' (A, B), so the data is read once whatever the number of chains, and nothing goes
// through global memory.
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
// The product of a piece's decays, held.  Where it ran to infinity on the way and met a decay of 0 (NaN), it is
// formed again, held at every step.  (Decays of the sigmoid form are at most 1.)  The test costs the value form 1 to 2 %:
// 8 x 4096 x 2048 bf16 forward 80.7 -> 81.8 us, backward 132.6 -> 134.4.
template <int kMode>
__device__ __forceinline__ f32x2 held_product(f32x2 product, const f32x2 (&a)[kScanSteps]) {
  product = held2(product);
  if (kMode == kGateValue) {
    const float2 v = unpack2(product);
    if (__builtin_expect(isnan(v.x + v.y), 0)) {
      product = a[0];
#pragma unroll
      for (int k = 1; k < kScanSteps; ++k) product = mul2(held2(product), a[k]);
      product = held2(product);
    }
  }
  return product;
}
// A map h -> a h + b of a lane's two channels; `cut`: what comes before does not count (h -> b).
struct __align__(16) ScanMap { f32x2 a, b; };

// f(true) or f(false), the argument a constant.
template <bool kValue> struct Flag { static constexpr bool value = kValue; };
template <int kValue> struct Number { static constexpr int value = kValue; };
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
__device__ __forceinline__ void cluster_store(unsigned addr, unsigned barrier, float4 v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
               :: "r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(barrier) : "memory");
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
  static constexpr int kStretchWarps = kScanWarps / kParts;   // warps between two kept states
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
// copies: __syncwarp() after the wait, and before the copies where the warp's reads of the part may not be over.
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
// Shared gates are few: a warp copies its rows' gates once, 16 / group for a lane, as the 4-byte words that
// hold them, row by row into its part of the stage.  (Asynchronously: loads into registers a tile ahead
// waited all the same, 8 x 4096 x 2048 bf16 with gates for 64 channels took 137 us, now 105.)
template <typename T, int kLanes>
struct SharedGates {
  int shift, first, mine, left;   // log2 of the gates of a row, the first's number, this pair's, those that exist
  bool odd, words;                // this pair's is the upper half of its word; all words lie within their rows
  __device__ __forceinline__ SharedGates(const ScanParams& p, const ScanPlace<kLanes>& w) {
    shift = p.group < 2 * kLanes ? __ffs(2 * kLanes / p.group) - 1 : 0;   // (a power of two there)
    first = w.block / p.group;
    mine = 2 * w.pair / p.group;
    left = (w.left + p.group - 1) / p.group;
    odd = sizeof(T) == 2 && ((first + mine) & 1);
    words = p.gate_words;
  }
  __device__ __forceinline__ void fetch(unsigned char* part, const T* src, long long stride, int rows) const {
    for (int i = threadIdx.x & 31; i < ((32 / kLanes) * kScanSteps) << shift; i += 32) {
      const int row = i >> shift, g = i - (row << shift);
      unsigned* slot = reinterpret_cast<unsigned*>(part) + i;
      const T* at = src + row * stride + first + g;
      if (row >= rows || g >= left) {
        *slot = 0;
      } else if (words) {
        if (sizeof(T) == 2) at = src + row * stride + ((first + g) & ~1);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(scan_smem(slot)), "l"(at) : "memory");
      } else {
        *slot = both(at[0]);
      }
    }
  }
  __device__ __forceinline__ static unsigned both(float v) { return __float_as_uint(v); }
  template <typename U>
  __device__ __forceinline__ static unsigned both(U v) { return join(v, v); }
  __device__ __forceinline__ f32x2 get(const unsigned char* part, int row) const {
    const unsigned v = reinterpret_cast<const unsigned*>(part)[(row << shift) + mine];
    if (sizeof(T) == 4) return pack2(__uint_as_float(v), __uint_as_float(v));
    const float2 f = unpack2(two(v, T{}));
    return odd ? pack2(f.y, f.y) : pack2(f.x, f.x);
  }
  __device__ __forceinline__ static f32x2 two(unsigned v, float) { return 0; }
  template <typename U>
  __device__ __forceinline__ static f32x2 two(unsigned v, U u) { return widen(v, u); }
};

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
  // Called by the kLanes threads that hold the tile's map.
  template <bool kCut>
  __device__ __forceinline__ void send(const ScanPlace<kLanes>& w, int buffer, const ScanMap& map, bool cut) {
    const float2 a = unpack2(map.a), b = unpack2(map.b);
    const unsigned at = scan_smem(totals + (buffer * w.cluster + w.rank) * kChannels + 2 * w.pair);
    const unsigned flag = scan_smem(cuts + buffer * w.cluster + w.rank);
    for (int q = 0; q < w.cluster; ++q) {
      const unsigned bar = cluster_address(barrier + 8 * buffer, q);
      cluster_store(cluster_address(at, q), bar, make_float4(a.x, b.x, a.y, b.y));
      if (kCut && w.pair == 0) cluster_store(cluster_address(flag, q), bar, cut ? 1u : 0u);
    }
  }
  // Called by one thread, before the round's barrier: the bytes that will come.
  __device__ __forceinline__ void expect(const ScanPlace<kLanes>& w, int buffer, bool flags) {
    barrier_expect(barrier + 8 * buffer, w.cluster * (kChannels * 8 + (flags ? 4 : 0)));
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

// `first`, then `next`.
template <bool kCut>
__device__ __forceinline__ void then_map(ScanMap& first, bool& first_cut, const ScanMap& next, bool next_cut, bool hold) {
  first.b = through2<kCut>(kCut && next_cut, next.a, next.b, first.b);
  first.a = mul2(first.a, next.a);
  if (hold) first.a = held2(first.a);
  first_cut |= kCut && next_cut;
}
__device__ __forceinline__ f32x2 shuffle2(f32x2 v, int from) { return __shfl_sync(~0u, v, from); }

// The pieces of a warp: `map` becomes that of all pieces up to this one (from behind: from this one on),
// the result is that of those before it (behind it), the identity for the first.
template <int kLanes, bool kCut, bool kBackward, bool kHold>
__device__ __forceinline__ ScanMap join_pieces(ScanMap& map, bool& cut, bool& cut_before, int lane) {
  ScanMap before = {kOnes2, 0};
  cut_before = false;
  if constexpr (kLanes < 32) {
#pragma unroll
    for (int o = kLanes; o < 32; o <<= 1) {
      const int from = kBackward ? lane + o : lane - o;
      const bool on = kBackward ? from < 32 : from >= 0;
      ScanMap other = {shuffle2(map.a, from & 31), shuffle2(map.b, from & 31)};
      bool other_cut = kCut && __shfl_sync(~0u, static_cast<int>(cut), from & 31) != 0;
      if (on) {
        then_map<kCut>(other, other_cut, map, cut, kHold);
        map = other;
        cut = other_cut;
      }
    }
    const int from = kBackward ? lane + kLanes : lane - kLanes;
    before = {shuffle2(map.a, from & 31), shuffle2(map.b, from & 31)};
    cut_before = kCut && __shfl_sync(~0u, static_cast<int>(cut), from & 31) != 0;
    if (kBackward ? from >= 32 : from < 0) { before = {kOnes2, 0}; cut_before = false; }
  }
  return before;
}

// What bounds it: HBM (2 reads and a write an element); the arithmetic is about 20 lane instructions
// an element.
template <typename T, int kMode, int kMove, int kLanes>
__global__ void __launch_bounds__(kScanThreads, sizeof(T) == 4 || kLanes < 32 ? 2 : 3) scan_kernel(const ScanParams p) {
  typedef typename Pair<T>::raw Raw;
  typedef ScanPlace<kLanes> Place;
  constexpr int kPieces = Place::kPieces;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ ScanMap maps[2][kScanWarps][kLanes];          // of the warps
  __shared__ __align__(8) float enter[Place::kChannels];   // cluster: the state before this CTA's tile
  __shared__ f32x2 hand[2][kLanes];
  __shared__ bool warp_cut[2][kScanWarps];
  __shared__ unsigned long long barriers[2];
  const Place w(p);
  constexpr int kPart = kTileElements / kScanWarps * sizeof(T);   // a warp's part of a tensor's stage
  unsigned char* stage = dynamic + w.warp * kPart;
  ScanExchange<kLanes> exchange(dynamic + kScanStages * scan_stage_bytes(2, sizeof(T)), barriers, w);
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.block;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + (p.group > 1 ? 0 : w.block);
  T* y = static_cast<T*>(p.y) + w.b * p.yb + w.block + 2 * w.pair;

  const SharedGates<T, kLanes> shared(p, w);
  // (the row pointers run ahead of what is read; behind the last step nothing is read through them)
  x += w.warp_first(0) * p.xt; gate += w.warp_first(0) * p.gt;
  auto fetch = [&](int s) {
    if (s < w.rounds) {
      unsigned char* part = stage + (s & 1) * (2 * kScanWarps * kPart);
      const int n = Place::clamp_steps(w.len - w.warp_first(s), Place::kParts * kScanSteps);
      fetch_rows<T, kMove, kLanes>(part, x, p.xt, n, w.left);
      part += kScanWarps * kPart;
      if (p.group > 1) shared.fetch(part, gate, p.gt, n);
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
    if (kMove == kMoveVec || p.group > 1) __syncwarp();
    const int live = w.live(s);
    const unsigned resets = w.reset_bits(next_reset);
    next_reset = s + 1 < w.rounds ? w.reset_byte(p, s + 1) : 0u;

    f32x2 a[kScanSteps], u[kScanSteps];
    const Raw* slot = reinterpret_cast<const Raw*>(stage + (s & 1) * (2 * kScanWarps * kPart)) + (w.lane - w.pair) * kScanSteps + w.pair;
    const unsigned char* gates = stage + (s & 1) * (2 * kScanWarps * kPart) + kScanWarps * kPart;
    const int row0 = (w.lane / kLanes) * kScanSteps;
    with_flag(p.group > 1, [&](auto group) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) {
        const f32x2 xv = widen(slot[k * kLanes], T{});
        f32x2 c;
        gate_coefs2<kMode>(decltype(group)::value ? shared.get(gates, row0 + k)
                                                      : widen(slot[kTileElements / 2 + k * kLanes], T{}), a[k], c);
        u[k] = kMode == kGateValue ? xv : mul2(c, xv);
      }
    });
    if (live < kScanSteps) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k)
        if (k >= live) { a[k] = kOnes2; u[k] = 0; }
    }
    ScanMap map = {a[0], u[0]};
#pragma unroll
    for (int k = 1; k < kScanSteps; ++k) {
      map.a = mul2(map.a, a[k]);
      map.b = fma2(a[k], map.b, u[k]);
    }
    if (resets) {   // what comes before the last reset does not count
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) map.b = through2<true>(resets >> k & 1, a[k], u[k], map.b);
    }
    map.a = held_product<kMode>(map.a, a);
    const int buffer = s & 1;
    f32x2 h;    // the state before this piece
    with_flag(p.reset != nullptr, [&](auto with_cuts) {
      constexpr bool kCut = decltype(with_cuts)::value;
      bool cut = resets != 0, cut_before;
      const ScanMap before = join_pieces<kLanes, kCut, false, kMode == kGateValue>(map, cut, cut_before, w.lane);
      if (w.lane >= 32 - kLanes) {
        maps[buffer][w.warp][w.pair] = map;
        if (kCut && w.pair == 0) warp_cut[buffer][w.warp] = cut;
      }
      if (w.cluster > 1 && threadIdx.x == 0) exchange.expect(w, buffer, kCut);
      __syncthreads();
      auto tile = [&](int v) { return maps[buffer][v][w.pair]; };
      auto tile_cut = [&](int v) { return kCut && warp_cut[buffer][v]; };
      if (w.cluster > 1) {
        // everything that does not need the other CTAs comes before the wait
        ScanMap pre = {kOnes2, 0};
        bool pre_cut = false;
#pragma unroll
        for (int v0 = 0; v0 < kScanWarps - 1; v0 += kAhead) {
          if (v0 >= w.warp) break;
          ScanMap m[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) m[j] = tile(min(v0 + j, kScanWarps - 1));
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (v0 + j < w.warp) then_map<kCut>(pre, pre_cut, m[j], tile_cut(v0 + j), kMode == kGateValue);
        }
        if (w.warp == kScanWarps - 1 && w.lane >= 32 - kLanes) {
          ScanMap all = pre;
          bool all_cut = pre_cut;
          then_map<kCut>(all, all_cut, map, cut, true);
          exchange.template send<kCut>(w, buffer, all, all_cut);
        }
        then_map<kCut>(pre, pre_cut, before, cut_before, true);
        if (threadIdx.x < Place::kChannels)
          state = pack2(exchange.template run<kCut, false>(w, buffer, s >> 1 & 1, unpack2(state).x, enter), 0.0f);
        __syncthreads();
        h = through2<kCut>(pre_cut, pre.a, pre.b, *reinterpret_cast<const f32x2*>(enter + 2 * w.pair));
      } else {
        h = hand[buffer ^ 1][w.pair];
#pragma unroll
        for (int v0 = 0; v0 < kScanWarps - 1; v0 += kAhead) {
          if (v0 >= w.warp) break;
          ScanMap m[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) m[j] = tile(min(v0 + j, kScanWarps - 1));
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (v0 + j < w.warp) h = through2<kCut>(tile_cut(v0 + j), m[j].a, m[j].b, h);
        }
        if (kLanes < 32) h = through2<kCut>(cut_before, before.a, before.b, h);
      }
    });

    const int t = w.first(s);
    if (p.carry && t % kScanTile == 0 && t < w.steps) {
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
    if (w.cluster == 1 && w.piece == kPieces - 1) hand[buffer][w.pair] = state = h;
  }
  if (p.h_last && w.rank == 0) put_state(p.h_last, p, w, kPieces - 1, state);
}

// The reverse: the flow of the gradient through the state, tiles from the last to the first.  Each
// stretch of 64 steps starts its states from carry, so only the flow is handed from tile to tile.
template <typename T, int kMode, int kMove, int kLanes>
__global__ void __launch_bounds__(kScanThreads, 2) scan_backward_kernel(const ScanParams p) {
  typedef typename Pair<T>::raw Raw;
  typedef ScanPlace<kLanes> Place;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ ScanMap maps[2][kScanWarps][kLanes];          // of the states, warps
  __shared__ f32x2 flows[2][kScanWarps][kLanes];           // b of the gradient flow (a is the same)
  __shared__ __align__(8) float enter[Place::kChannels];   // cluster: the flow from behind this CTA's tile
  __shared__ f32x2 hand[2][kLanes];
  __shared__ bool warp_cut[2][kScanWarps];
  __shared__ unsigned long long barriers[2];
  const Place w(p);
  constexpr int kPart = kTileElements / kScanWarps * sizeof(T);
  unsigned char* stage = dynamic + w.warp * kPart;
  ScanExchange<kLanes> exchange(dynamic + kScanStages * scan_stage_bytes(3, sizeof(T)), barriers, w);
  const int c0 = w.block + 2 * w.pair;
  const T* x = static_cast<const T*>(p.x) + w.b * p.xb + w.block;
  const T* gate = static_cast<const T*>(p.gate) + w.b * p.gb + (p.group > 1 ? 0 : w.block);
  const T* dy = static_cast<const T*>(p.dy) + w.b * p.yb + w.block;
  T* dx = static_cast<T*>(p.dx) + w.b * p.dxb + c0;
  T* dgate = static_cast<T*>(p.dgate) + w.b * p.dgb + c0 / p.group;

  const SharedGates<T, kLanes> shared(p, w);
  const int last = w.rounds - 1;
  x += w.warp_first(last) * p.xt; gate += w.warp_first(last) * p.gt; dy += w.warp_first(last) * p.yt;
  auto fetch = [&](int s) {
    if (s >= 0) {
      unsigned char* part = stage + (s & 1) * (3 * kScanWarps * kPart);
      const int n = Place::clamp_steps(w.len - w.warp_first(s), Place::kParts * kScanSteps);
      fetch_rows<T, kMove, kLanes>(part, x, p.xt, n, w.left);
      part += kScanWarps * kPart;
      if (p.group > 1) shared.fetch(part, gate, p.gt, n);
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
    // the round before read its stage to its end, this fetch fills it again: with other lanes' slots too
    if (kMove == kMoveVec || p.group > 1) __syncwarp();
    fetch(s - 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (kMove == kMoveVec || p.group > 1) __syncwarp();
    const int live = w.live(s);
    const unsigned resets = w.reset_bits(next_reset);
    next_reset = s > 0 ? w.reset_byte(p, s - 1) : 0u;
    f32x2 h = next_state, r;      // the state before this piece, the flow from behind it
    next_state = kept_state(s - 1);

    f32x2 a[kScanSteps], c[kScanSteps];
    const Raw* slot = reinterpret_cast<const Raw*>(stage + (s & 1) * (3 * kScanWarps * kPart)) + (w.lane - w.pair) * kScanSteps + w.pair;
    const unsigned char* gates = stage + (s & 1) * (3 * kScanWarps * kPart) + kScanWarps * kPart;
    const int row0 = (w.lane / kLanes) * kScanSteps;
    constexpr int kGate = kTileElements / 2, kDy = kTileElements;
    with_flag(p.group > 1, [&](auto group) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k)
        gate_coefs2<kMode>(decltype(group)::value ? shared.get(gates, row0 + k)
                                                      : widen(slot[kGate + k * kLanes], T{}), a[k], c[k]);
    });
    if (live < kScanSteps) {
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k)
        if (k >= live) { a[k] = kOnes2; c[k] = 0; }
    }
    auto added = [&](int k) {   // what step k adds to the state
      const f32x2 xv = widen(slot[k * kLanes], T{});
      return kMode == kGateValue ? xv : mul2(c[k], xv);
    };
    ScanMap map = {kOnes2, 0}, back = {kOnes2, 0};   // of the states, of the flow
    with_flag(resets != 0, [&](auto with_cuts) {
      constexpr bool kCut = decltype(with_cuts)::value;
#pragma unroll
      for (int k = 0; k < kScanSteps; ++k) {
        map.a = k ? mul2(map.a, a[k]) : a[k];
        map.b = through2<kCut>(kCut && resets >> k & 1, a[k], added(k), map.b);
      }
#pragma unroll
      for (int k = kScanSteps - 1; k >= 0; --k) {
        back.b = mul2(a[k], add2(widen(slot[kDy + k * kLanes], T{}), back.b));
        if (kCut && resets >> k & 1) back.b = 0;
      }
    });
    back.a = map.a = held_product<kMode>(map.a, a);
    const int round = w.rounds - 1 - s, buffer = round & 1;
    with_flag(p.reset != nullptr, [&](auto with_cuts) {
      constexpr bool kCut = decltype(with_cuts)::value, kHold = kMode == kGateValue;
      bool cut = resets != 0, cut_back = cut, cut_before, cut_behind;
      const ScanMap before = join_pieces<kLanes, kCut, false, kHold>(map, cut, cut_before, w.lane);
      const ScanMap behind = join_pieces<kLanes, kCut, true, kHold>(back, cut_back, cut_behind, w.lane);
      if (w.lane >= 32 - kLanes) {
        maps[buffer][w.warp][w.pair] = map;
        if (kCut && w.pair == 0) warp_cut[buffer][w.warp] = cut;
      }
      if (w.lane < kLanes) flows[buffer][w.warp][w.pair] = back.b;
      if (w.cluster > 1 && threadIdx.x == 0) exchange.expect(w, buffer, kCut);
      __syncthreads();
      auto tile = [&](int v) { return maps[buffer][v][w.pair]; };
      auto tile_back = [&](int v) { return ScanMap{maps[buffer][v][w.pair].a, flows[buffer][v][w.pair]}; };
      auto tile_cut = [&](int v) { return kCut && warp_cut[buffer][v]; };
      if (w.cluster > 1) {
        ScanMap pre = {kOnes2, 0};
        bool pre_cut = false;
#pragma unroll
        for (int v0 = kScanWarps - 1; v0 > 0; v0 -= kAhead) {
          if (v0 <= w.warp) break;
          ScanMap m[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) m[j] = tile_back(max(v0 - j, 0));
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (v0 - j > w.warp) then_map<kCut>(pre, pre_cut, m[j], tile_cut(v0 - j), kHold);
        }
        if (w.warp == 0 && w.lane < kLanes) {
          ScanMap all = pre;
          bool all_cut = pre_cut;
          then_map<kCut>(all, all_cut, back, cut_back, true);
          exchange.template send<kCut>(w, buffer, all, all_cut);
        }
        then_map<kCut>(pre, pre_cut, behind, cut_behind, true);
        if (threadIdx.x < Place::kChannels)
          flow = pack2(exchange.template run<kCut, true>(w, buffer, round >> 1 & 1, unpack2(flow).x, enter), 0.0f);
        __syncthreads();
        r = through2<kCut>(pre_cut, pre.a, pre.b, *reinterpret_cast<const f32x2*>(enter + 2 * w.pair));
      } else {
        r = hand[buffer ^ 1][w.pair];
#pragma unroll
        for (int v0 = kScanWarps - 1; v0 > 0; v0 -= kAhead) {
          if (v0 <= w.warp) break;
          ScanMap m[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) m[j] = tile_back(max(v0 - j, 0));
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (v0 - j > w.warp) r = through2<kCut>(tile_cut(v0 - j), m[j].a, m[j].b, r);
        }
        if (kLanes < 32) r = through2<kCut>(cut_behind, behind.a, behind.b, r);
      }
      // the states from the kept one before this stretch
      const int from = w.warp / Place::kStretchWarps * Place::kStretchWarps;
#pragma unroll
      for (int v0 = 0; v0 < Place::kStretchWarps - 1; v0 += kAhead) {
        if (from + v0 >= w.warp) break;
        ScanMap m[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) m[j] = tile(min(from + v0 + j, kScanWarps - 1));
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (from + v0 + j < w.warp) h = through2<kCut>(tile_cut(from + v0 + j), m[j].a, m[j].b, h);
      }
      if (kLanes < 32) h = through2<kCut>(cut_before, before.a, before.b, h);
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
        // (a decay of the value form may be Inf or NaN at a reset; where one of the sigmoid form is, so is its 1 - a)
        h = through2<!kWhole && kMode == kGateValue>(resets >> k & 1, a[k], added(k), h);
      }
      T* gx_at = dx;
      T* gg_at = dgate;
      float sums[kScanSteps];   // of the gate's gradient over the thread's channels
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
          const float2 f = unpack2(gg);
          sums[k] = w.channels > 0 ? f.x + (w.channels > 1 ? f.y : 0.0f) : 0.0f;
        }
      }
      if (p.group > 1) {
        // the lanes that share a gate add their sums, each keeping half of the steps as long as it has
        // several: 9 shuffles instead of 40 for 32 lanes
        const int lanes = min(p.group, kScanChannels) / 2;
        int kept = 0, count = kScanSteps, o = lanes >> 1;   // first step and number of those kept
        auto halve = [&](auto half_of) {
          constexpr int kHalf = decltype(half_of)::value;
          if (o) {
            const bool upper = w.pair & o;
#pragma unroll
            for (int j = 0; j < kHalf; ++j) {
              const float got = __shfl_xor_sync(~0u, upper ? sums[j] : sums[j + kHalf], o);
              sums[j] = (upper ? sums[j + kHalf] : sums[j]) + got;
            }
            kept += upper ? kHalf : 0;
            count = kHalf;
            o >>= 1;
          }
        };
        halve(Number<4>{});
        halve(Number<2>{});
        halve(Number<1>{});
        const int rest = o ? 2 * o - 1 : 0;
        for (; o; o >>= 1) sums[0] += __shfl_xor_sync(~0u, sums[0], o);
        if (w.channels > 0 && (w.pair & rest) == 0) {
          gg_at = dgate - (kScanSteps - 1) * p.dgt;   // the piece's first row
#pragma unroll
          for (int j = 0; j < kScanSteps; ++j) {
            if (j >= count) break;
            const int k = kept + j;
            if (!kWhole && k >= rows) continue;
            if (p.partial)
              p.partial[(w.b * p.steps + t + k) * (p.channels / kScanChannels) + c0 / kScanChannels] = sums[j];
            else
              gg_at[k * p.dgt] = from_float<T>(sums[j]);
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
