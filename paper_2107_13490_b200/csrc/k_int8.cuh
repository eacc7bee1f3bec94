// Rows to 8-bit codes, and the product of codes with scales for each token and channel.
//
//   m = max |x_k|,  code_k = rne(x_k fl(127 / m)),  scale = m / 127
//   y_ij = (x_scale_i weight_scale_j) sum_k x_ik w_jk (+ bias_j),   the sum in int32: exact
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "k_elem.cuh"
#include "tensor_core.cuh"

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

// The largest of the CTA's threads' values.
__device__ __forceinline__ unsigned cta_max(unsigned v, unsigned* shared) {
  v = __reduce_max_sync(~0u, v);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  for (unsigned w = 0; w < blockDim.x / 32; ++w) v = max(v, shared[w]);
  return v;
}

// A CTA a row, which stays in registers: kChunks 16-byte chunks a thread.
template <typename T, int kChunks>
__global__ __launch_bounds__(kRowsThreads) void int8_rows_kernel(RowsParams q) {
  constexpr int V = 16 / sizeof(T);
  __shared__ unsigned largest_of[kRowsThreads / 32];
  let_next_kernel_start();
  const T* x = static_cast<const T*>(q.x) + blockIdx.x * q.ldx;
  signed char* codes = q.codes + blockIdx.x * q.ld_codes;
  float f[kChunks][V];
  unsigned largest = 0;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (c < q.cols) raw = __ldcs(reinterpret_cast<const uint4*>(x + c));
    unpack16<T>(raw, f[i]);
  }
#pragma unroll
  for (int i = 0; i < kChunks; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) largest = max(largest, __float_as_uint(f[i][k]) & 0x7FFFFFFFu);
  const RowScale s = row_scale(cta_max(largest, largest_of));
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = (i * blockDim.x + threadIdx.x) * V;
    if (c >= q.cols) break;
    unsigned w[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      int t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = to_code(f[i][4 * j + k], s.inverse);
      w[j] = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
      if (s.inverse == 0.0f) w[j] = 0;
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(codes + c) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<unsigned*>(codes + c) = w[0];
  }
  if (threadIdx.x == 0) q.scales[blockIdx.x] = s.scale;
}

// Rows of any length and alignment, read twice.
template <typename T>
__global__ __launch_bounds__(kRowsThreads) void int8_rows_any_kernel(RowsParams q) {
  __shared__ unsigned largest_of[kRowsThreads / 32];
  let_next_kernel_start();
  const T* x = static_cast<const T*>(q.x) + blockIdx.x * q.ldx;
  signed char* codes = q.codes + blockIdx.x * q.ld_codes;
  unsigned largest = 0;
  for (int c = threadIdx.x; c < q.cols; c += kRowsThreads) largest = max(largest, __float_as_uint(to_float(x[c])) & 0x7FFFFFFFu);
  const RowScale s = row_scale(cta_max(largest, largest_of));
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
  bool w_late;         // the kernel in front writes the weights too
};

// 32 results of one token to 32-byte aligned memory, in whole sectors.
template <typename T>
__device__ __forceinline__ void store_run(T* to, const float (&f)[32]) {
  constexpr int kPer = 32 / sizeof(T);   // values of a 32-byte store
#pragma unroll
  for (int i = 0; i < 32; i += kPer) {
    unsigned w[8];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(f[i + k]);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float part[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) part[k] = f[i + 8 * h + k];
        const uint4 p = pack16<T>(part);
        w[4 * h] = p.x; w[4 * h + 1] = p.y; w[4 * h + 2] = p.z; w[4 * h + 3] = p.w;
      }
    }
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" :: "l"(to + i), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
  }
}

// ---- many tokens: tiles of 256 tokens x 256 channels by pairs of CTAs --------------------------------------
//
// A CTA of a pair holds 128 of the tokens and 128 of the channels; the products of both are issued by the first.
// One warp copies tiles ahead, one issues products, four turn finished sums into y while the next tile's
// products run (the sums of two tiles fill the tensor memory).

constexpr int kDepth = 128;              // codes of a row in a stage: one swizzled line
constexpr int kCtaRows = 128;
constexpr int kWideTile = 256;
constexpr int kWideStages = 6;
constexpr int kWideStageBytes = 2 * kCtaRows * kDepth;
constexpr int kWideThreads = 256;
constexpr int kWideSmem = kWideStages * kWideStageBytes + 1024;

struct WideParams {
  LinearParams p;
  int across, down;   // tiles of channels and of tokens
  bool wide_stores;
};

// The tile that comes i-th: bands of kBand tiles of tokens, so that the pairs at work share operands in L2.
constexpr int kBand = 8;
__device__ __forceinline__ int2 wide_tile(int i, int across, int down) {
  const int band = i / (kBand * across), first = band * kBand, height = min(kBand, down - first);
  const int in = i - band * kBand * across;
  return make_int2(first + in % height, in / height);
}

template <typename T>
__global__ __cluster_dims__(2, 1, 1) __launch_bounds__(kWideThreads, 1) void int8_wide_kernel(const __grid_constant__ CUtensorMap x_map,
                                                                                             const __grid_constant__ CUtensorMap w_map,
                                                                                             const WideParams q) {
  extern __shared__ unsigned char wide_smem[];
  __shared__ __align__(8) unsigned long long bars[2 * kWideStages + 4];
  __shared__ unsigned sums_at;
  __shared__ float scale_of[2][kWideTile], bias_of[2][kWideTile];
  __shared__ float turned[4][32][33];   // a warp's 32 x 32 results, for rows that are not aligned
  const unsigned stages = (shared_address(wide_smem) + 1023u) & ~1023u;
  const unsigned full = shared_address(bars), empty = full + 8 * kWideStages, done = empty + 8 * kWideStages, open = done + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned rank = cta_in_cluster();
  const int tiles = q.across * q.down, pairs = gridDim.x / 2, pair = blockIdx.x / 2;
  const int blocks = (q.p.k + kDepth - 1) / kDepth;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kWideStages; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { barrier_init(done + 8 * b, 1); barrier_init(open + 8 * b, 8); }   // open: four warps of both CTAs
    barrier_init_fence();
    tile_map_prefetch(&x_map);
    tile_map_prefetch(&w_map);
  }
  if (warp == 2) tensor_alloc<true>(shared_address(&sums_at), 512);
  tensor_fence_before();
  __syncthreads();
  meet_cluster();
  tensor_fence_after();
  const unsigned sums = sums_at;
  if (warp == 0 && lane == 0) {   // copies
    wait_for_previous_kernel();
    const unsigned bar = peer_address(full, 0);
    unsigned use = 0;
    bool ok = true;
    for (int i = pair; i < tiles && ok; i += pairs) {
      const int2 t = wide_tile(i, q.across, q.down);
      for (int b = 0; b < blocks && ok; ++b, ++use) {
        const unsigned s = use % kWideStages, round = use / kWideStages;
        ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1);
        if (!ok) break;
        const unsigned to = stages + s * kWideStageBytes;
        if (rank == 0) barrier_expect_bytes(full + 8 * s, 2 * kWideStageBytes);
        tile_load<true>(to, &x_map, b * kDepth, t.x * kWideTile + rank * kCtaRows, bar + 8 * s);
        tile_load<true>(to + kCtaRows * kDepth, &w_map, b * kDepth, t.y * kWideTile + rank * kCtaRows, bar + 8 * s);
      }
    }
    // what was copied last has been used (and its barriers have had their last arrival) before the CTA ends
    for (unsigned left = use < kWideStages ? use : kWideStages; left; --left) {
      const unsigned u = use - left;
      ok = barrier_wait(empty + 8 * (u % kWideStages), (u / kWideStages) & 1) && ok;
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {   // products
    constexpr unsigned form = product_form(2 * kCtaRows, kWideTile);
    unsigned use = 0, turn = 0;
    bool ok = true;
    for (int i = pair; i < tiles && ok; i += pairs, ++turn) {
      const unsigned buffer = turn & 1;
      ok = barrier_wait<true>(open + 8 * buffer, ((turn >> 1) & 1) ^ 1);
      if (!ok) break;
      tensor_fence_after();
      for (int b = 0; b < blocks; ++b, ++use) {
        const unsigned s = use % kWideStages;
        ok = barrier_wait(full + 8 * s, (use / kWideStages) & 1);
        if (!ok) break;
        tensor_fence_after();
        const unsigned at = stages + s * kWideStageBytes;
        const unsigned long long a = operand(at), w = operand(at + kCtaRows * kDepth);
#pragma unroll
        for (int k = 0; k < kDepth / 32; ++k) product<true>(sums + buffer * kWideTile, a + 2 * k, w + 2 * k, form, b > 0 || k > 0);
        product_commit<true>(empty + 8 * s);
      }
      if (ok) product_commit<true>(done + 8 * buffer);
    }
  } else if (warp >= 4) {   // sums to y
    wait_for_previous_kernel();
    const int quarter = warp - 4, thread = threadIdx.x - 128;
    const unsigned leader_open = peer_address(open, 0);
    unsigned turn = 0;
    bool ok = true;
    for (int i = pair; i < tiles; i += pairs, ++turn) {
      const unsigned buffer = turn & 1;
      const int2 t = wide_tile(i, q.across, q.down);
      const int row = t.x * kWideTile + static_cast<int>(rank) * kCtaRows + quarter * 32 + lane, col = t.y * kWideTile;
      for (int c = thread; c < kWideTile; c += 128) {
        const bool in = col + c < q.p.n;
        scale_of[buffer][c] = in ? q.p.w_scales[q.p.w_one ? 0 : col + c] : 0.0f;
        bias_of[buffer][c] = in && q.p.bias ? q.p.bias[col + c] : 0.0f;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const float scale = row < q.p.rows ? q.p.x_scales[q.p.x_one ? 0 : row] : 0.0f;
      ok = ok && barrier_wait(done + 8 * buffer, (turn >> 1) & 1);
      ok = __all_sync(~0u, ok);
      tensor_fence_after();
      T* out = static_cast<T*>(q.p.y) + row * q.p.ldy + col;
#pragma unroll 1
      for (int c = 0; c < kWideTile; c += 32) {
        if (col + c >= q.p.n) break;
        int v[32];
        tensor_read32(sums + (static_cast<unsigned>(quarter * 32) << 16) + buffer * kWideTile + c, v);
        tensor_read_wait();
        float f[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          const float y = static_cast<float>(v[k]) * scale * scale_of[buffer][c + k];
          f[k] = ok ? (q.p.bias ? y + bias_of[buffer][c + k] : y) : __int_as_float(0x7FC00000);   // a wait that ran out leaves NaN
        }
        const int count = q.p.n - col - c;
        if (q.wide_stores && count >= 32) {
          if (row < q.p.rows) store_run<T>(out + c, f);
        } else {   // a row of 32 results by the warp
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 32; ++k) turned[quarter][lane][k] = f[k];
          __syncwarp();
          T* line = static_cast<T*>(q.p.y) + (row - lane) * q.p.ldy + col + c + lane;
          const int rows = min(32, q.p.rows - (row - lane));
          if (lane < count)
            for (int r = 0; r < rows; ++r) line[r * q.p.ldy] = from_float<T>(turned[quarter][r][lane]);
        }
      }
      tensor_fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive_cluster(leader_open + 8 * buffer);
    }
  }
  tensor_fence_before();
  __syncthreads();
  meet_cluster();   // nothing of this pair is under way any more
  tensor_fence_after();
  if (warp == 2) tensor_free<true>(sums, 512);
}

// ---- few tokens: the channels are the rows of the products, the sum's index is dealt to a cluster ------------
//
// A tile of 128 channels meets up to 256 tokens, so no row of a tile is idle however few the tokens are, and the
// weights stream once.  The CTAs of a cluster take stretches of the sum's index; each then gets its
// share of the tokens' columns from all of them through shared memory.

constexpr int kNarrowThreads = 128;
__host__ __device__ constexpr int narrow_stage_bytes(int tokens) { return (kCtaRows + tokens) * kDepth; }
__host__ __device__ constexpr int narrow_stages(int tokens) { return tokens <= 64 ? 8 : tokens == 128 ? 6 : 4; }
// CTAs that share a sum at most, and the columns that one of them sends.
__host__ __device__ constexpr int narrow_split(int tokens) { return tokens <= 16 ? 4 : tokens <= 128 ? 8 : 4; }
__host__ __device__ constexpr int narrow_sent(int tokens) { return tokens / narrow_split(tokens) * (narrow_split(tokens) - 1); }
__host__ __device__ constexpr int narrow_smem(int tokens) { return narrow_stages(tokens) * narrow_stage_bytes(tokens) + 1024; }

template <typename T, int kTokens>
__global__ __launch_bounds__(kNarrowThreads) void int8_narrow_kernel(const __grid_constant__ CUtensorMap x_map,
                                                                    const __grid_constant__ CUtensorMap w_map, const LinearParams q) {
  constexpr int kStages = narrow_stages(kTokens), kStageBytes = narrow_stage_bytes(kTokens);
  constexpr unsigned kColumns = kTokens < 32 ? 32 : kTokens;
  static_assert(2 * narrow_sent(kTokens) * kCtaRows * 4 <= kStages * kStageBytes, "what is sent and received fits the stages");
  extern __shared__ unsigned char narrow_smem_[];
  __shared__ __align__(8) unsigned long long bars[2 * kStages + 2];
  __shared__ unsigned sums_at;
  __shared__ float scale_of[kTokens];
  const unsigned aligned = (shared_address(narrow_smem_) + 1023u) & ~1023u;
  const unsigned full = shared_address(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, exchange = done + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned rank = cta_in_cluster(), split = ctas_of_cluster();
  const int channel0 = blockIdx.x / split * kCtaRows, token0 = blockIdx.y * kTokens;
  const int all = (q.k + kDepth - 1) / kDepth;
  const int from = static_cast<int>(static_cast<long long>(all) * rank / split), to = static_cast<int>(static_cast<long long>(all) * (rank + 1) / split);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
    barrier_init(done, 1);
    barrier_init(exchange, 1);
    barrier_init_fence();
    tile_map_prefetch(&w_map);
    tile_map_prefetch(&x_map);
  }
  if (warp == 2) tensor_alloc<false>(shared_address(&sums_at), kColumns);
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const unsigned sums = sums_at;
  if (warp == 0 && lane == 0) {   // copies: the first weights before the tokens' codes are there
    auto weights = [&](int b) {
      const unsigned s = (b - from) % kStages;
      barrier_expect_bytes(full + 8 * s, kStageBytes);
      tile_load<false>(aligned + s * kStageBytes, &w_map, b * kDepth, channel0, full + 8 * s);
    };
    auto tokens = [&](int b) {
      const unsigned s = (b - from) % kStages;
      tile_load<false>(aligned + s * kStageBytes + kCtaRows * kDepth, &x_map, b * kDepth, token0, full + 8 * s);
    };
    const int first = min(to, from + kStages);
    if (q.w_late) wait_for_previous_kernel();
    for (int b = from; b < first; ++b) weights(b);
    wait_for_previous_kernel();
    for (int b = from; b < first; ++b) tokens(b);
    bool ok = true;
    for (int b = first; b < to && ok; ++b) {
      const unsigned use = b - from;
      ok = barrier_wait(empty + 8 * (use % kStages), ((use / kStages) & 1) ^ 1);
      if (!ok) break;
      weights(b);
      tokens(b);
    }
  } else if (warp == 1 && lane == 0) {   // products
    constexpr unsigned form = product_form(kCtaRows, kTokens);
    bool ok = true;
    for (int b = from; b < to; ++b) {
      const unsigned use = b - from, s = use % kStages;
      ok = barrier_wait(full + 8 * s, (use / kStages) & 1);
      if (!ok) break;
      tensor_fence_after();
      const unsigned at = aligned + s * kStageBytes;
      const unsigned long long w = operand(at), x = operand(at + kCtaRows * kDepth);
#pragma unroll
      for (int k = 0; k < kDepth / 32; ++k) product<false>(sums, w + 2 * k, x + 2 * k, form, b > from || k > 0);
      product_commit<false>(empty + 8 * s);
    }
    if (ok) product_commit<false>(done);
  }
  __syncwarp();
  wait_for_previous_kernel();
  const int count = min(kTokens, q.rows - token0);
  for (int c = threadIdx.x; c < count; c += kNarrowThreads) scale_of[c] = q.x_scales[q.x_one ? 0 : token0 + c];
  const int channel = channel0 + threadIdx.x;
  const bool in = channel < q.n;
  const float w_scale = in ? q.w_scales[q.w_one ? 0 : channel] : 0.0f;
  const float bias = in && q.bias ? q.bias[channel] : 0.0f;
  __syncthreads();
  bool ok = barrier_wait(done, 0);   // (then every copy has been used)
  ok = __all_sync(~0u, ok);
  tensor_fence_after();
  const unsigned mine = sums + (static_cast<unsigned>(warp * 32) << 16);
  T* const out = static_cast<T*>(q.y) + token0 * q.ldy + channel;
  auto finish = [&](int sum, int c, bool good) {   // c: the token's column
    float y = static_cast<float>(sum) * scale_of[c] * w_scale;
    if (q.bias) y += bias;
    if (in && c < count) out[c * q.ldy] = from_float<T>(good ? y : __int_as_float(0x7FC00000));
  };
  if (split == 1) {
#pragma unroll 1
    for (int c = 0; c < count; c += 16) {
      int v[16];
      tensor_read16(mine + c, v);
      tensor_read_wait();
#pragma unroll
      for (int k = 0; k < 16; ++k) finish(v[k], c + k, ok);
    }
  } else {
    // Every CTA adds up its share of the columns: those of the others' come by bulk copies, in slots of
    // [four columns][channel].  One whose wait ran out sends nothing, so that the others' run out too.
    const int share = kTokens / static_cast<int>(split), first = static_cast<int>(rank) * share;   // a multiple of 4
    const unsigned slot = share * kCtaRows * 4, received = aligned + (split - 1) * slot;
    if (threadIdx.x == 0) barrier_expect_bytes(exchange, (split - 1) * slot);
#pragma unroll 1
    for (int c = 0; c < count; c += 16) {
      int v[16];
      tensor_read16(mine + c, v);
      tensor_read_wait();
#pragma unroll
      for (int k = 0; k < 16; k += 4) {
        const int owner = (c + k) / share, four = ((c + k) - owner * share) / 4;
        if (owner == static_cast<int>(rank)) continue;
        const unsigned at = aligned + (owner - (owner > static_cast<int>(rank))) * slot + (four * kCtaRows + threadIdx.x) * 16;
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(v[k]), "r"(v[k + 1]), "r"(v[k + 2]), "r"(v[k + 3]) : "memory");
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    meet_cluster();   // everyone's products are done, so that the stages are free, and everyone's sums are in place
    if (threadIdx.x < split && threadIdx.x != rank && ok) {
      const unsigned to_rank = threadIdx.x, out_slot = to_rank - (to_rank > rank), in_slot = rank - (rank > to_rank);
      asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   :: "r"(peer_address(received + in_slot * slot, to_rank)), "r"(aligned + out_slot * slot), "r"(slot),
                      "r"(peer_address(exchange, to_rank)) : "memory");
    }
    bool good = ok && barrier_wait<true>(exchange, 0);
    for (int c = 0; c < share && first + c < count; c += 4) {
      int sum[4];
      tensor_read4(mine + first + c, sum);
      tensor_read_wait();
      for (unsigned r = 0; r + 1 < split; ++r) {
        int4 v;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(received + r * slot + (c / 4 * kCtaRows + threadIdx.x) * 16) : "memory");
        sum[0] += v.x; sum[1] += v.y; sum[2] += v.z; sum[3] += v.w;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) finish(sum[k], first + c + k, good);
    }
    __syncwarp();
    meet_cluster();   // what was sent has arrived
  }
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  if (warp == 2) tensor_free<false>(sums, kColumns);
}

// ---- codes into rows that the TMA unit can read ------------------------------------------------------------

struct CopyRows {
  const signed char* from;
  signed char* to;
  long long ld_from, ld_to;   // ld_to a multiple of 16
  int rows;
};
struct CopyParams { CopyRows part[2]; int cols; };   // activations and weights, either may have no rows

constexpr int kCopyThreads = 128;

// Only aligned blocks that hold a byte of the row are read.
__global__ __launch_bounds__(kCopyThreads) void int8_copy_kernel(CopyParams q) {
  let_next_kernel_start();
  const bool second = blockIdx.x >= static_cast<unsigned>(q.part[0].rows);
  const CopyRows& p = q.part[second];
  const long long r = blockIdx.x - (second ? q.part[0].rows : 0);
  const signed char* row = p.from + r * p.ld_from;
  for (int c = threadIdx.x * 16; c < q.cols; c += kCopyThreads * 16) {
    const unsigned o = static_cast<unsigned>(reinterpret_cast<uintptr_t>(row + c) & 15u);
    const uint4* block = reinterpret_cast<const uint4*>(row + c - o);
    const uint4 lo = __ldg(block);
    uint4 hi = make_uint4(0, 0, 0, 0);
    if (static_cast<int>(o) + min(16, q.cols - c) > 16) hi = __ldg(block + 1);
    *reinterpret_cast<uint4*>(p.to + r * p.ld_to + c) = shift_bytes(lo, hi, o);
  }
}

// ---- a few tokens: dot products on the integer units ---------------------------------------------------------
//
// A warp takes two channels and streams their codes, 16 bytes a lane; the tokens' codes lie in shared memory, where the
// CTA has quantised them while the first weights are on their way.  Weights of any alignment are read in
// the aligned blocks that hold them; the tokens' codes are shifted likewise, and 0 outside the row.

constexpr int kDotThreads = 256;
constexpr int kDotChannels = 2;                    // of a warp
constexpr int kDotStrips = 8;                      // blocks of 16 bytes that a lane has under way for a channel
constexpr int kDotChunk = kDotStrips * 32 * 16;    // codes of a row at a time
// Tokens that take this form.  us, two so and three by the tensor cores: 4096 x 4096 6.8, 9.7; 4096 x 1024 5.0, 6.6; 8192 x 8192 17.7,
// 17.3; 16384 x 4096 18.1, 16.0: for the largest weights it loses with two.
constexpr int kDotMaxRows = 2;

struct DotParams {
  LinearParams p;
  const void* x;       // X: activations that are quantised here, or codes (then p.x_scales)
};

template <typename T, typename X, int kRows, bool kShift>
__global__ __launch_bounds__(kDotThreads) void int8_dot_kernel(const DotParams d) {
  constexpr bool kCodes = sizeof(X) == 1;
  constexpr int kLine = kDotChunk + 32;            // a block of zeros on either side
  constexpr int kChunk = kShift ? kDotChunk - 16 : kDotChunk;   // (the blocks of a shifted chunk are one more)
  __shared__ __align__(16) signed char codes[kRows][kLine];
  __shared__ unsigned largest_of[kRows][kDotThreads / 32];
  const LinearParams& q = d.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int channel0 = (blockIdx.x * (kDotThreads / 32) + warp) * kDotChannels;
  const X* x = static_cast<const X*>(d.x);
  uint4 w[kDotChannels][kDotStrips];
  unsigned off[kDotChannels];
  auto load = [&](int k0) {
    const int len = min(kChunk, q.k - k0);
#pragma unroll
    for (int c = 0; c < kDotChannels; ++c) {
      const signed char* row = q.w + min(channel0 + c, q.n - 1) * q.ldw + k0;
      off[c] = kShift ? static_cast<unsigned>(reinterpret_cast<uintptr_t>(row) & 15u) : 0u;
      const uint4* block = reinterpret_cast<const uint4*>(row - off[c]);
#pragma unroll
      for (int s = 0; s < kDotStrips; ++s) {
        const int at = (s * 32 + lane) * 16;
        w[c][s] = at < len + static_cast<int>(off[c]) ? __ldg(block + s * 32 + lane) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  load(0);
  float inverse[kRows], scale[kRows];
  if constexpr (!kCodes) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      unsigned largest = 0;
      if (r < q.rows)
        for (int c = threadIdx.x; c < q.k; c += kDotThreads) largest = max(largest, __float_as_uint(fabsf(to_float(x[r * q.ldx + c]))));
      largest = __reduce_max_sync(~0u, largest);
      if (lane == 0) largest_of[r][warp] = largest;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      unsigned largest = 0;
#pragma unroll
      for (int i = 0; i < kDotThreads / 32; ++i) largest = max(largest, largest_of[r][i]);
      const RowScale s = row_scale(largest);
      inverse[r] = s.inverse;
      scale[r] = s.scale;
    }
  }
  int sum[kDotChannels][kRows] = {};
  for (int k0 = 0; k0 < q.k; k0 += kChunk) {
    const int len = min(kChunk, q.k - k0);
    if (k0) { __syncthreads(); load(k0); }
    for (int r = 0; r < kRows; ++r) {
      // four codes at a time, and zeros on either side of the row's
      for (int c = static_cast<int>(threadIdx.x) * 4 - 16; c < kDotChunk + 16; c += kDotThreads * 4) {
        unsigned word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          int code = 0;
          if (r < q.rows && c + j >= 0 && c + j < len) {
            if constexpr (kCodes) code = x[r * q.ldx + k0 + c + j];
            else if (inverse[r] != 0.0f) code = to_code(to_float(x[r * q.ldx + k0 + c + j]), inverse[r]);
          }
          word |= (static_cast<unsigned>(code) & 0xFFu) << (8 * j);
        }
        *reinterpret_cast<unsigned*>(&codes[r][c + 16]) = word;
      }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kDotStrips; ++s) {
      if (s * 512 >= len + 16) break;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const uint4* line = reinterpret_cast<const uint4*>(&codes[r][16 + (s * 32 + lane) * 16]);
        const uint4 here = *line;
        uint4 before = make_uint4(0, 0, 0, 0);
        if constexpr (kShift) before = line[-1];
#pragma unroll
        for (int c = 0; c < kDotChannels; ++c) {
          // the block begins off bytes in front of the row's code that stands here
          const uint4 v = !kShift || off[c] == 0 ? here : shift_bytes(before, here, 16 - off[c]);
          sum[c][r] = __dp4a(static_cast<int>(w[c][s].x), static_cast<int>(v.x), sum[c][r]);
          sum[c][r] = __dp4a(static_cast<int>(w[c][s].y), static_cast<int>(v.y), sum[c][r]);
          sum[c][r] = __dp4a(static_cast<int>(w[c][s].z), static_cast<int>(v.z), sum[c][r]);
          sum[c][r] = __dp4a(static_cast<int>(w[c][s].w), static_cast<int>(v.w), sum[c][r]);
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < kDotChannels; ++c)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int total = __reduce_add_sync(~0u, sum[c][r]);
      const int channel = channel0 + c;
      if (lane != 0 || channel >= q.n || r >= q.rows) continue;
      float s;
      if constexpr (kCodes) s = q.x_scales[q.x_one ? 0 : r]; else s = scale[r];
      float y = static_cast<float>(total) * s * q.w_scales[q.w_one ? 0 : channel];
      if (q.bias) y += q.bias[channel];
      static_cast<T*>(q.y)[r * q.ldy + channel] = from_float<T>(y);
    }
}

// ---- no codes at all: y = bias -----------------------------------------------------------------------------------

template <typename T>
__global__ void int8_bias_kernel(const LinearParams q) {
  for (int j = threadIdx.x; j < q.n; j += blockDim.x) static_cast<T*>(q.y)[blockIdx.x * q.ldy + j] = from_float<T>(q.bias ? q.bias[j] : 0.0f);
}

}  // namespace adapt
