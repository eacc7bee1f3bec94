// Token embedding and its gradient.
//
//   out[i] = scale * table[ids[i]],     dtable[v] = scale * sum_{i : ids[i] = v} dy[i]
//
// Both move rows and compute almost nothing: HBM bounds them, and for few tokens the launches.
//
// The gradient takes three launches.  The first sorts the tokens (stable, so that a token's occurrences stay in order) in
// one cluster, whose CTAs exchange their digit counts through shared memory, while the other clusters write the rows of
// tokens that do not occur, most of the table as a rule.  The second sums over blocks of the sorted places, one
// block a team of threads.  A token of up to half a block's places belongs to the team in whose block it begins; more
// frequent ones are cut at the blocks' ends, the sums of their pieces are left in memory, and the third launch joins
// them in the order of the blocks.  So every sum has one order, whatever the timing, and no row of dy is read twice.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "k_elem.cuh"
#include "tensor_core.cuh"

namespace adapt {

struct EmbedParams {
  const void* table;
  const long long* ids;
  void* out;
  long long ld_table, ld_out;
  int n, vocab, dim;
  float scale;
};

// A row's elements from..from+V-1 from registers.
template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, const float (&f)[V]) {
  if constexpr (V == 1) {
    *p = from_float<T>(f[0]);
  } else if constexpr (V * sizeof(T) == 32) {   // fp32 gradients of 16-bit rows
    const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
    __stcs(reinterpret_cast<uint4*>(p), pack16<float>(a));
    __stcs(reinterpret_cast<uint4*>(p) + 1, pack16<float>(b));
  } else {
    __stcs(reinterpret_cast<uint4*>(p), pack16<T>(f));
  }
}

// `lanes` threads (a power of two, up to the CTA) take a row, 16 bytes of the output at a time and four such parts under
// way, as they lie in memory.  kShift: tables or outputs that are not 16-byte aligned.  Then a part is a 16-byte block of the
// output, and the table's is shifted out of the two blocks that hold it; the ends of a row go element by element.
constexpr int kEmbedThreads = 256;

template <typename T, bool kShift>
__global__ __launch_bounds__(kEmbedThreads) void embedding_kernel(EmbedParams q, int lanes) {
  constexpr int V = 16 / static_cast<int>(sizeof(T)), kParts = 4;
  const int i = blockIdx.x * (kEmbedThreads / lanes) + threadIdx.x / lanes;
  if (i >= q.n) return;
  const int lane = threadIdx.x & (lanes - 1);
  const long long id = q.ids[i];
  T* out = static_cast<T*>(q.out) + i * q.ld_out;
  const bool known = id >= 0 && id < q.vocab;
  const T* row = static_cast<const T*>(q.table) + (known ? id : 0) * q.ld_table;
  const float fill = id < 0 ? 0.0f : __int_as_float(0x7FC00000);
  const int skip = kShift ? static_cast<int>((reinterpret_cast<uintptr_t>(out) & 15u) / sizeof(T)) : 0;
  const unsigned shift = kShift ? static_cast<unsigned>(reinterpret_cast<uintptr_t>(row - skip) & 15u) : 0;
  auto whole = [&](int c) { return !kShift || (c >= 0 && c + V <= q.dim); };
  for (int at = lane * V - skip; at < q.dim; at += lanes * V * kParts) {
    uint4 low[kParts], high[kParts];
#pragma unroll
    for (int u = 0; u < kParts; ++u) {
      const int c = at + u * lanes * V;
      low[u] = high[u] = make_uint4(0, 0, 0, 0);
      if (!known || c >= q.dim || !whole(c)) continue;
      const uint4* block = reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(row + c) - shift);
      low[u] = __ldg(block);
      if (kShift && shift) high[u] = __ldg(block + 1);
    }
#pragma unroll
    for (int u = 0; u < kParts; ++u) {
      const int c = at + u * lanes * V;
      if (c >= q.dim) break;
      if (whole(c)) {
        float f[V];
        unpack16<T>(kShift ? shift_bytes(low[u], high[u], shift) : low[u], f);
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = known ? f[k] * q.scale : fill;
        __stcs(reinterpret_cast<uint4*>(out + c), pack16<T>(f));
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (c + k >= 0 && c + k < q.dim) out[c + k] = from_float<T>(known ? to_float(row[c + k]) * q.scale : fill);
      }
    }
  }
}

// ---- gradient -----------------------------------------------------------------------------------

struct EmbedGradParams {
  const void* dy;
  const long long* ids;
  void* dtable;
  long long ld_dy, ld_grad;
  int n, vocab, dim;
  float scale;
  bool accumulate;
  unsigned* keys[2];     // [n] tokens (vocab: none)
  unsigned* places[2];   // [n] their places
  uint2* joins;          // their number, then the blocks in which a token begins that goes on behind them, and the token
  float* partial;        // [blocks][2][dim] sums of a block's first token, which began in front, and of its last, which goes on (where they are cut)
  int width, passes;     // digits of the sort (passes 0: by comparisons)
  int block;             // sorted places of a block
  int cut;               // places of a token (up to a block's) that is cut where a block ends
  int lanes;             // threads of a team
  int slices;            // teams side by side that share a row's columns
  int slot;              // bytes of a row in a stage
};

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortWidth = 10;      // bits of a digit at most: two digits up to a million tokens
constexpr int kSortHeld = 4;        // places of a lane that are held in registers
constexpr int kSortMaxCluster = 16;
constexpr int kSortFew = 1024;      // places that are sorted by comparisons
constexpr int kSortSmem = (kSortWarps + 2) * (1 << kSortWidth) * 4;
constexpr int kAbsentRows = kSortSmem * 8;   // rows of a stretch of the table: a bit each

__device__ __forceinline__ unsigned embed_key(const EmbedGradParams& q, unsigned i) {
  const long long id = q.ids[i];
  return id >= 0 && id < q.vocab ? static_cast<unsigned>(id) : static_cast<unsigned>(q.vocab);
}

// One CTA, up to kSortFew places: a place's rank is the number of smaller (token, place).
__device__ __forceinline__ void embed_sort_few(const EmbedGradParams& q, unsigned* smem) {
  const unsigned i = threadIdx.x, n = static_cast<unsigned>(q.n);
  smem[i] = i < n ? embed_key(q, i) : ~0u;
  __syncthreads();
  if (i >= n) return;
  const unsigned key = smem[i];
  unsigned rank = 0;
  for (unsigned j = 0; j < n; j += 4) {
    const uint4 k = *reinterpret_cast<const uint4*>(smem + j);
    rank += (k.x < key || (k.x == key && j < i)) + (k.y < key || (k.y == key && j + 1 < i)) + (k.z < key || (k.z == key && j + 2 < i)) +
            (k.w < key || (k.w == key && j + 3 < i));
  }
  if (ADAPT_IN_BOUNDS(rank, n, 71)) {
    q.keys[1][rank] = key;   // (where an even number of passes leaves them)
    q.places[1][rank] = i;
  }
}

// By digits from the lowest.  Warp w of the cluster holds places share w .. share (w + 1) - 1 and counts their digits; a
// digit's first place is the count of lower digits plus that of the same digit in the warps before.
__device__ __forceinline__ void embed_sort_many(const EmbedGradParams& q, unsigned* smem, unsigned rank, unsigned parts) {
  __shared__ unsigned warp_sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned buckets = 1u << q.width;
  unsigned* mine = smem + warp * buckets;
  unsigned* totals = smem + kSortWarps * buckets;
  unsigned* first = totals + buckets;
  const unsigned warps = parts * kSortWarps;
  const unsigned n = static_cast<unsigned>(q.n);
  const unsigned share = ((n + warps - 1) / warps + 31) & ~31u;
  const unsigned long long begin = static_cast<unsigned long long>(rank * kSortWarps + warp) * share;
  const unsigned from = begin < n ? static_cast<unsigned>(begin) : n, to = begin + share < n ? from + share : n;
  for (int pass = 0; pass < q.passes; ++pass) {
    const unsigned* keys = q.keys[(pass + 1) & 1];
    const unsigned* places = q.places[(pass + 1) & 1];
    const int shift = pass * q.width;
    auto key_at = [&](unsigned i) { return pass ? __ldcg(keys + i) : embed_key(q, i); };
    unsigned held_key[kSortHeld], held_place[kSortHeld];   // the warp's first places, loaded at once
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k) {
      const unsigned i = from + k * 32 + lane;
      held_key[k] = i < to ? key_at(i) : 0;
      held_place[k] = i < to ? (pass ? __ldcg(places + i) : i) : 0;
    }
    for (unsigned i = threadIdx.x; i < kSortWarps * buckets / 4; i += kSortThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k)
      if (from + k * 32 + lane < to) atomicAdd(mine + ((held_key[k] >> shift) & (buckets - 1)), 1u);
#pragma unroll 4
    for (unsigned i = from + kSortHeld * 32 + lane; i < to; i += 32) atomicAdd(mine + ((key_at(i) >> shift) & (buckets - 1)), 1u);
    __syncthreads();
    if (threadIdx.x < buckets) {
      unsigned count[kSortWarps], total = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) count[w] = smem[w * buckets + threadIdx.x];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        smem[w * buckets + threadIdx.x] = total;
        total += count[w];
      }
      totals[threadIdx.x] = total;
    }
    meet_cluster();   // all totals are there
    unsigned below = 0, all = 0;
    if (threadIdx.x < buckets) {
      const unsigned at = shared_address(totals + threadIdx.x);
#pragma unroll 4
      for (unsigned r = 0; r < parts; ++r) {
        unsigned c;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(peer_address(at, r)) : "memory");
        if (r < rank) below += c;
        all += c;
      }
    }
    unsigned sum = all;   // running sum over the digits
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned v = __shfl_up_sync(~0u, sum, d);
      if (lane >= d) sum += v;
    }
    if (lane == 31) warp_sums[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      unsigned v = warp_sums[lane];
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned w = __shfl_up_sync(~0u, v, d);
        if (lane >= d) v += w;
      }
      warp_sums[lane] = v;
    }
    __syncthreads();
    if (threadIdx.x < buckets) first[threadIdx.x] = sum - all + (warp ? warp_sums[warp - 1] : 0) + below;
    __syncthreads();
    auto put = [&](bool live, unsigned key, unsigned place) {
      const unsigned digit = (key >> shift) & (buckets - 1);
      const unsigned peers = __match_any_sync(~0u, live ? digit : ~0u);
      const unsigned before = peers & ((1u << lane) - 1);
      unsigned goal = 0;
      if (live) goal = first[digit] + mine[digit] + __popc(before);
      __syncwarp();
      if (live && !before) mine[digit] += __popc(peers);
      __syncwarp();
      if (live && ADAPT_IN_BOUNDS(goal, n, 70)) {
        q.keys[pass & 1][goal] = key;
        q.places[pass & 1][goal] = place;
      }
    };
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k)
      if (from + k * 32 < to) put(from + k * 32 + lane < to, held_key[k], held_place[k]);
    unsigned key = 0, place = 0;
    auto load = [&](unsigned i) {
      if (i < to) {
        key = key_at(i);
        place = pass ? __ldcg(places + i) : i;
      }
    };
    load(from + kSortHeld * 32 + lane);
    for (unsigned i = from + kSortHeld * 32; i < to; i += 32) {
      const unsigned this_key = key, this_place = place;
      load(i + 32 + lane);
      put(i + lane < to, this_key, this_place);
    }
    meet_cluster();   // what this pass wrote is there for the next, and its totals have been read
  }
}

// 0 to every element of a row: whole 16-byte blocks, single elements at the ends.
template <typename G>
__device__ __forceinline__ void embed_blank(G* row, int dim, int lane) {
  constexpr int V = 16 / sizeof(G);
  const int skip = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(G));
  for (int c = lane * V - skip; c < dim; c += 32 * V) {
    if (c >= 0 && c + V <= dim) {
      __stcs(reinterpret_cast<uint4*>(row + c), make_uint4(0, 0, 0, 0));
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (c + k >= 0 && c + k < dim) row[c + k] = from_float<G>(0.0f);
    }
  }
}

// The rows of tokens that do not occur, by every CTA from the `rank`-th on, `ctas` of them: a stretch of the table each,
// a bit for each of its rows.
template <typename G>
__device__ __forceinline__ void embed_absent(const EmbedGradParams& q, unsigned* bits, int rank, int ctas) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = min(kAbsentRows, (q.vocab + ctas - 1) / ctas);
  for (long long v0 = static_cast<long long>(rank) * per; v0 < q.vocab; v0 += static_cast<long long>(ctas) * per) {
    const int rows = static_cast<int>(min(static_cast<long long>(per), q.vocab - v0));
    __syncthreads();
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) bits[i] = 0;
    __syncthreads();
#pragma unroll 8
    for (int i = threadIdx.x; i < q.n; i += kSortThreads) {
      const long long v = q.ids[i] - v0;
      if (v >= 0 && v < rows) {
        const unsigned bit = 1u << (v & 31);
        if (!(reinterpret_cast<volatile unsigned*>(bits)[v >> 5] & bit)) atomicOr(bits + (v >> 5), bit);   // (frequent tokens are there already)
      }
    }
    __syncthreads();
    for (int v = warp; v < rows; v += kSortWarps)
      if (!(bits[v >> 5] >> (v & 31) & 1)) embed_blank(static_cast<G*>(q.dtable) + (v0 + v) * q.ld_grad, q.dim, lane);
  }
}

// The first cluster sorts; the others, if there are any, write rows of tokens that do not occur.
template <typename G>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const EmbedGradParams q) {
  extern __shared__ __align__(16) unsigned sort_smem[];
  let_next_kernel_start();
  const unsigned parts = ctas_of_cluster();
  const bool sorts = q.n > 0 && blockIdx.x < parts;
  if (blockIdx.x == 0 && threadIdx.x == 0 && q.n > 0) q.joins->x = 0;
  if (!sorts) {
    const unsigned first = q.n > 0 ? parts : 0;
    embed_absent<G>(q, sort_smem, blockIdx.x - first, gridDim.x - first);
  } else if (q.passes == 0) {
    embed_sort_few(q, sort_smem);
  } else {
    embed_sort_many(q, sort_smem, cta_in_cluster(), parts);
  }
}

// V elements of a gradient's row, in the types' 16 or 32 bytes.
template <typename G, int V>
__device__ __forceinline__ void load_row(const G* p, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = to_float(*p);
  } else {
#pragma unroll
    for (int k = 0; k < V; k += 16 / sizeof(G)) {
      float part[16 / sizeof(G)];
      unpack16<G>(*reinterpret_cast<const uint4*>(p + k), part);
#pragma unroll
      for (int j = 0; j < 16 / static_cast<int>(sizeof(G)); ++j) f[k + j] = part[j];
    }
  }
}

// A team of threads sums over the rows of its block, V elements a thread; CTAs of 256 threads hold one team or several.
// Rows come through stages in shared memory, kStageRows of each team's, which a warp of its own fills ahead by bulk copies:
// whole rows under way cost neither registers nor instructions.  (Filled by the warps that sum, from two stages, narrow rows
// waited for it: 131072 rows of 64 bf16 100 us, so 91.)  Rows between 16-byte boundaries (kAligned false) are copied
// with the aligned blocks around them and read element by element, V of them `lanes` apart.
constexpr int kStageRows = 4;
constexpr int kStages = 4;
constexpr int kSumThreads = kEmbedThreads + 32;

template <typename T, typename G, bool kAligned>
__global__ __launch_bounds__(kSumThreads) void embed_sum_kernel(const EmbedGradParams q) {
  constexpr int V = 16 / static_cast<int>(sizeof(T));
  extern __shared__ __align__(128) unsigned char embed_smem[];
  __shared__ __align__(8) unsigned long long bars[2 * kStages];
  const int teams = kEmbedThreads / q.lanes, team = threadIdx.x / q.lanes, lane = threadIdx.x % q.lanes, warp_lane = threadIdx.x & 31;
  const int slice = blockIdx.x % q.slices, first_column = slice * q.lanes * V, columns = min(q.dim - first_column, q.lanes * V);
  const long long cta_first = static_cast<long long>(blockIdx.x / q.slices) * teams * q.block;
  const int count = static_cast<int>(min(static_cast<long long>(teams) * q.block, q.n - cta_first));
  const int stage_bytes = teams * kStageRows * q.slot;
  // tokens and places of the CTA's places, and of some in front and behind
  const int around = q.cut + 1, held = teams * q.block + 2 * around;
  unsigned* keys = reinterpret_cast<unsigned*>(embed_smem + kStages * stage_bytes) + around;
  unsigned* places = keys + held;
  __shared__ int begins[kEmbedThreads / 8], ends_at[kEmbedThreads / 8];   // what the teams take
  __shared__ bool cut_front[kEmbedThreads / 8];
  const unsigned full = shared_address(bars), empty = full + 8 * kStages, vocab = static_cast<unsigned>(q.vocab);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, kEmbedThreads / 32);
    }
    barrier_init_fence();
  }
  wait_for_previous_kernel();
  {
    const unsigned* all_keys = q.keys[(q.passes + 1) & 1] + cta_first;
    const unsigned* all_places = q.places[(q.passes + 1) & 1] + cta_first;
    for (int i = static_cast<int>(threadIdx.x) - around; i < count + around; i += kSumThreads) {
      const long long p = cta_first + i;
      const bool known = p >= 0 && p < q.n;
      keys[i] = known ? all_keys[i] : ~0u;   // (in front of the first, too: equal to no token)
      places[i] = known ? all_places[i] : 0;
    }
  }
  __syncthreads();
  if (threadIdx.x < static_cast<unsigned>(teams)) {
    const int from = static_cast<int>(threadIdx.x) * q.block, to = min(from + q.block, count);
    int begin = from, end = to;
    bool front = false;
    // the first place in [lo, hi) whose token is not below `least` (there are no places in front of the first)
    auto search = [&](int lo, int hi, unsigned least) {
      lo = max(lo, static_cast<int>(max(-cta_first, static_cast<long long>(-around))));
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (keys[mid] < least) lo = mid + 1; else hi = mid;
      }
      return lo;
    };
    if (from < count) {
      if (keys[from - 1] == keys[from]) {   // its token's places, as far as it matters
        const int first = search(from - around, from, keys[from]), stop = search(from + 1, from + q.cut + 1, keys[from] + 1);
        front = stop - first > q.cut;
        if (!front) begin = stop;   // the team in front takes it
      }
      if (keys[to] == keys[to - 1]) {
        const int first = search(to - around, to, keys[to]), stop = search(to + 1, to + q.cut + 1, keys[to] + 1);
        if (stop - first <= q.cut) end = stop;   // (then it begins in this block)
      }
      begin = min(begin, end);
      end = search(begin, end, vocab);   // (places without a token are sorted to the end)
    } else {
      begin = end = from;
    }
    begins[threadIdx.x] = begin;
    ends_at[threadIdx.x] = end;
    cut_front[threadIdx.x] = front;
  }
  __syncthreads();
  auto row_at = [&](int i) { return static_cast<const T*>(q.dy) + places[i] * q.ld_dy + first_column; };
  int most = 0;
  for (int t = 0; t < teams; ++t) most = max(most, ends_at[t] - begins[t]);
  const int steps = (most + kStageRows - 1) / kStageRows;
  if (threadIdx.x >= kEmbedThreads) {   // the rows of the steps, ahead
    for (int step = 0; step < steps; ++step) {
      const int s = step % kStages;
      const bool ok = barrier_wait(empty + 8 * s, ((step / kStages) & 1) ^ 1);
      if (!__all_sync(~0u, ok)) return;   // (those who sum find no data then)
      auto size_of = [&](const T* row) {
        const unsigned skip = kAligned ? 0 : static_cast<unsigned>(reinterpret_cast<uintptr_t>(row) & 15u);
        return (skip + columns * static_cast<unsigned>(sizeof(T)) + 15) & ~15u;
      };
      auto each = [&](auto f) {
        for (int r = warp_lane; r < teams * kStageRows; r += 32) {
          const int of = r / kStageRows, i = begins[of] + step * kStageRows + r % kStageRows;
          if (i < ends_at[of] && ADAPT_IN_BOUNDS(places[i], q.n, 72)) f(r, i, row_at(i));
        }
      };
      unsigned bytes = 0;   // what will come is said before it is asked for
      each([&](int, int, const T* row) { bytes += size_of(row); });
      bytes = __reduce_add_sync(~0u, bytes);
      if (warp_lane == 0) barrier_expect_bytes(full + 8 * s, bytes);
      __syncwarp();
      each([&](int r, int i, const T* row) {
        const unsigned skip = kAligned ? 0 : static_cast<unsigned>(reinterpret_cast<uintptr_t>(row) & 15u);
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     :: "r"(shared_address(embed_smem) + s * stage_bytes + r * q.slot), "l"(reinterpret_cast<const unsigned char*>(row) - skip),
                        "r"(size_of(row)), "r"(full + 8 * s) : "memory");
        if (q.accumulate && keys[i + 1] != keys[i])   // what the sum will be added to
          asm volatile("prefetch.global.L2 [%0];" :: "l"(static_cast<const G*>(q.dtable) + keys[i] * q.ld_grad + first_column));
      });
    }
    return;
  }
  const int from = begins[team], to = ends_at[team];
  float sum[V] = {};
  bool began = !cut_front[team];   // the token at hand: here, and not in the block in front
  float* partial = q.partial + 2 * (cta_first / q.block + team) * q.dim + first_column;
  auto column = [&](int k) { return kAligned ? lane * V + k : lane + k * q.lanes; };
  const bool in = lane * V < columns;   // (kAligned)
  const unsigned base16 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(static_cast<const T*>(q.dy) + first_column)) & 15u;
  const unsigned step16 = static_cast<unsigned>(q.ld_dy * sizeof(T)) & 15u;
  for (int step = 0; step < steps; ++step) {
    const int s = step % kStages;
    const bool ok = barrier_wait(full + 8 * s, (step / kStages) & 1);
    if (!ok) sum[0] = __int_as_float(0x7FC00000);   // (a wait that ran out leaves NaN)
    const unsigned char* stage = embed_smem + s * stage_bytes + team * kStageRows * q.slot;
    const int i0 = from + step * kStageRows, rows = min(kStageRows, to - i0);
    unsigned last = 0;   // rows after which a sum is written: a token's last, and the team's
#pragma unroll
    for (int r = 0; r < kStageRows; ++r)
      if (r < rows && (keys[i0 + r + 1] != keys[i0 + r] || i0 + r + 1 == to)) last |= 1u << r;
    for (int r = 0; r < rows;) {
      const int stop = last >> r ? r + __ffs(last >> r) : rows;
#pragma unroll 2
      for (; r < stop; ++r) {
        if (kAligned) {
          float f[V];
          unpack16<T>(*reinterpret_cast<const uint4*>(stage + r * q.slot + lane * 16), f);
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += f[k];
        } else {   // (beyond the columns it adds up what lies there, which goes nowhere)
          const T* row = reinterpret_cast<const T*>(stage + r * q.slot + ((base16 + places[i0 + r] * step16) & 15u));
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += to_float(row[column(k)]);
        }
      }
      if (!(last >> (r - 1) & 1)) break;   // the token goes on in the next step
      const unsigned key = keys[i0 + r - 1];
      if (began && keys[i0 + r] != key) {
        G* row = static_cast<G*>(q.dtable) + key * q.ld_grad + first_column;
        if (kAligned) {
          if (in) {
            float f[V] = {};
            if (q.accumulate) load_row<G, V>(row + lane * V, f);
#pragma unroll
            for (int k = 0; k < V; ++k) f[k] += sum[k] * q.scale;
            store_part<G, V>(row + lane * V, f);
          }
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (column(k) < columns) row[column(k)] = from_float<G>(sum[k] * q.scale + (q.accumulate ? to_float(row[column(k)]) : 0.0f));
        }
      } else {
        if (began && lane == 0 && slice == 0)
          q.joins[1 + atomicAdd(&q.joins->x, 1u)] = make_uint2(static_cast<unsigned>(cta_first / q.block) + team, key);
        float* half = partial + (began ? q.dim : 0);
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (column(k) < columns) half[column(k)] = sum[k];
      }
      began = true;
#pragma unroll
      for (int k = 0; k < V; ++k) sum[k] = 0.0f;
    }
    __syncwarp();
    if (warp_lane == 0) barrier_arrive(empty + 8 * s);   // the warp has read the stage
  }
}

// Joins the sums of tokens that go on beyond the block in which they begin: a CTA takes 128 columns of one after the other,
// its warps the blocks behind in turn.
constexpr int kJoinWarps = 8;
constexpr int kJoinColumns = 128;

template <typename G>
__global__ __launch_bounds__(32 * kJoinWarps) void embed_join_kernel(const EmbedGradParams q) {
  __shared__ float part[kJoinWarps][kJoinColumns];
  const unsigned slices = (q.dim + kJoinColumns - 1) / kJoinColumns;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  wait_for_previous_kernel();
  const unsigned* keys = q.keys[(q.passes + 1) & 1];
  const unsigned long long items = static_cast<unsigned long long>(q.joins->x) * slices;
  for (unsigned long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int slice = static_cast<int>(item % slices);
    const uint2 join = q.joins[1 + item / slices];
    const long long b = join.x, end = (b + 1) * q.block;
    const int c0 = slice * kJoinColumns + lane;   // columns 32 apart
    const float* from = q.partial + 2 * (b + 1) * q.dim;
    const float own = q.partial[(2 * b + 1) * q.dim + min(slice * kJoinColumns + static_cast<int>(threadIdx.x % kJoinColumns), q.dim - 1)];
    // the blocks behind that begin with the token: it is the first of those
    const long long blocks = (q.n + q.block - 1) / q.block - b - 1;
    long long count = 1;
    for (bool more = true; more;) {
      const long long j = count + lane;
      const unsigned on = __ballot_sync(~0u, j < blocks && keys[end + j * q.block] == join.y);
      more = on == ~0u;
      count += more ? 32 : __ffs(~on) - 1;
    }
    float sum[4] = {};
#pragma unroll 8
    for (long long j = warp; j < count; j += kJoinWarps)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c0 + 32 * k < q.dim) sum[k] += __ldcg(from + 2 * j * q.dim + c0 + 32 * k);
#pragma unroll
    for (int k = 0; k < 4; ++k) part[warp][lane + 32 * k] = sum[k];
    __syncthreads();
    const int c = slice * kJoinColumns + threadIdx.x;
    if (threadIdx.x < kJoinColumns && c < q.dim) {
      float total = own;
#pragma unroll
      for (int w = 0; w < kJoinWarps; ++w) total += part[w][threadIdx.x];
      total *= q.scale;
      G* to = static_cast<G*>(q.dtable) + join.y * q.ld_grad + c;
      if (q.accumulate) total += to_float(*to);
      *to = from_float<G>(total);
    }
    __syncthreads();
  }
}

}  // namespace adapt
