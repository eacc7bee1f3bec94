// Token embedding and its gradient.
//
//   out[i] = scale * table[ids[i]],     dtable[v] = scale * sum_{i : ids[i] = v} dy[i]
//
// Both move rows and compute almost nothing: HBM bounds them, and for few tokens the launch.
//
// The gradient sorts the tokens (stable, so that a token's occurrences stay in order) in one launch of a
// single cluster, whose CTAs exchange their digit counts through shared memory; the sums then run
// over the sorted places.  A token's occurrences are cut into pieces of kPiece places (a whole number of them, the
// last one takes the rest), so that frequent tokens are summed by many CTAs; the sums of such pieces
// meet in a second launch, in the order of the pieces.  So every sum has one order, whatever the
// timing, and no row of dy is read twice.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "k_elem.cuh"

namespace adapt {

struct EmbedParams {
  const void* table;
  const long long* ids;
  void* out;
  long long ld_table, ld_out;
  int n, vocab, dim;
  float scale;
};

// A row's elements from..from+V-1 (scaled by nothing) to and from registers.
template <typename T, int V>
__device__ __forceinline__ void load_part(const T* p, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = to_float(*p);
  } else {
    unpack16<T>(__ldg(reinterpret_cast<const uint4*>(p)), f);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, const float (&f)[V]) {
  if constexpr (V == 1) {
    *p = from_float<T>(f[0]);
  } else if constexpr (V * sizeof(T) == 32) {   // fp32 gradients of 16-bit rows
    const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
    reinterpret_cast<uint4*>(p)[0] = pack16<float>(a);
    reinterpret_cast<uint4*>(p)[1] = pack16<float>(b);
  } else {
    *reinterpret_cast<uint4*>(p) = pack16<T>(f);
  }
}

// `lanes` threads (a power of two, up to the CTA) take a row; V elements at a time.
constexpr int kEmbedThreads = 256;

template <typename T, int V>
__global__ __launch_bounds__(kEmbedThreads) void embedding_kernel(EmbedParams q, int lanes) {
  const int i = blockIdx.x * (kEmbedThreads / lanes) + threadIdx.x / lanes;
  if (i >= q.n) return;
  const int lane = threadIdx.x & (lanes - 1);
  const long long id = q.ids[i];
  T* out = static_cast<T*>(q.out) + i * q.ld_out;
  const T* row = static_cast<const T*>(q.table) + (id >= 0 && id < q.vocab ? id : 0) * q.ld_table;
  const float fill = id < 0 ? 0.0f : __int_as_float(0x7FC00000);
  const bool known = id >= 0 && id < q.vocab;
  constexpr int kUnroll = 4;
  for (int at = lane * V; at < q.dim; at += lanes * V * kUnroll) {
    float f[kUnroll][V];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = at + u * lanes * V;
      if (known && c < q.dim) load_part<T, V>(row + c, f[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = at + u * lanes * V;
      if (c >= q.dim) break;
#pragma unroll
      for (int k = 0; k < V; ++k) f[u][k] = known ? f[u][k] * q.scale : fill;
      store_part<T, V>(out + c, f[u]);
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
  unsigned* present;     // [ceil(vocab / 32)] bits: the token occurs
  float* partial;        // [n / piece + 1][dim] sums of pieces
  int width, passes;     // digits of the sort
  int piece;             // places of a piece
  int chunk;             // sorted places of a CTA
  int slices;            // CTAs side by side that share a row's columns
  int token_ctas;        // CTAs that sum; the others write the rows of tokens that do not occur
};

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortWidth = 9;       // bits of a digit at most: two digits up to 262142 tokens
constexpr int kSortMaxCluster = 16;
constexpr int kSortSmem = (kSortWarps + 1) * (1 << kSortWidth) * 4;

__device__ __forceinline__ void embed_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A stable sort by digits from the lowest.  Warp w of the cluster holds places share w .. share (w + 1) - 1 and
// counts their digits; where a digit's first place goes is the count of lower digits plus that of the same
// digit in the warps before.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(EmbedGradParams q) {
  extern __shared__ unsigned sort_smem[];
  __shared__ unsigned warp_sums[kSortWarps];
  unsigned rank, parts;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned buckets = 1u << q.width;
  unsigned* mine = sort_smem + warp * buckets;
  unsigned* totals = sort_smem + kSortWarps * buckets;
  const unsigned warps = parts * kSortWarps;
  const unsigned n = static_cast<unsigned>(q.n);
  const unsigned share = ((n + warps - 1) / warps + 31) & ~31u;
  const unsigned long long begin = static_cast<unsigned long long>(rank * kSortWarps + warp) * share;
  const unsigned from = begin < n ? static_cast<unsigned>(begin) : n, to = begin + share < n ? from + share : n;
  const unsigned words = (static_cast<unsigned>(q.vocab) + 31) / 32;
  for (unsigned i = rank * kSortThreads + threadIdx.x; i < words; i += parts * kSortThreads) q.present[i] = 0;
  for (int pass = 0; pass < q.passes; ++pass) {
    const unsigned* keys = q.keys[(pass + 1) & 1];
    const unsigned* places = q.places[(pass + 1) & 1];
    const int shift = pass * q.width;
    auto key_at = [&](unsigned i) -> unsigned {
      if (pass) return __ldcg(keys + i);
      const long long id = q.ids[i];
      return id >= 0 && id < q.vocab ? static_cast<unsigned>(id) : static_cast<unsigned>(q.vocab);
    };
    for (unsigned i = threadIdx.x; i < kSortWarps * buckets; i += kSortThreads) sort_smem[i] = 0;
    __syncthreads();
    for (unsigned i = from + lane; i < to; i += 32) atomicAdd(mine + ((key_at(i) >> shift) & (buckets - 1)), 1u);
    __syncthreads();
    unsigned total = 0;
    if (threadIdx.x < buckets) {
      for (int w = 0; w < kSortWarps; ++w) {
        const unsigned c = sort_smem[w * buckets + threadIdx.x];
        sort_smem[w * buckets + threadIdx.x] = total;
        total += c;
      }
      totals[threadIdx.x] = total;
    }
    embed_cluster_sync();   // all totals are there (and, first, all bits are 0)
    unsigned below = 0, all = 0;
    if (threadIdx.x < buckets) {
      const unsigned at = static_cast<unsigned>(__cvta_generic_to_shared(totals + threadIdx.x));
      for (unsigned r = 0; r < parts; ++r) {
        unsigned a, c;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(r));
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(a) : "memory");
        if (r < rank) below += c;
        all += c;
      }
    }
    unsigned sum = all;   // running sum over the digits
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned v = __shfl_up_sync(~0u, sum, d);
      if (lane >= d) sum += v;
    }
    if (lane == 31) warp_sums[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      unsigned v = warp_sums[lane];
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned w = __shfl_up_sync(~0u, v, d);
        if (lane >= d) v += w;
      }
      warp_sums[lane] = v;
    }
    __syncthreads();
    const unsigned first = sum - all + (warp ? warp_sums[warp - 1] : 0) + below;
    if (threadIdx.x < buckets)
      for (int w = 0; w < kSortWarps; ++w) sort_smem[w * buckets + threadIdx.x] += first;
    embed_cluster_sync();   // the totals have been read; the CTA's first places are there
    for (unsigned i = from; i < to; i += 32) {
      const unsigned at = i + lane;
      const bool live = at < to;
      unsigned key = 0, place = 0;
      if (live) {
        key = key_at(at);
        place = pass ? __ldcg(places + at) : at;
      }
      const unsigned digit = (key >> shift) & (buckets - 1);
      const unsigned peers = __match_any_sync(~0u, live ? digit : ~0u);
      const unsigned before = peers & ((1u << lane) - 1);
      unsigned goal = 0;
      if (live) goal = mine[digit] + __popc(before);
      __syncwarp();
      if (live && !before) mine[digit] += __popc(peers);
      __syncwarp();
      if (live && ADAPT_IN_BOUNDS(goal, n, 40)) {
        q.keys[pass & 1][goal] = key;
        q.places[pass & 1][goal] = place;
        if (pass == 0 && key < static_cast<unsigned>(q.vocab)) atomicOr(q.present + (key >> 5), 1u << (key & 31));
      }
    }
    embed_cluster_sync();   // what this pass wrote is there for the next
  }
}

// The first of the sorted places that holds `key`, which stands at place `at`.
__device__ __forceinline__ int embed_first(const unsigned* keys, int at, unsigned key) {
  int lo = 0, hi = at;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (keys[mid] < key) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// U parts of V columns for each thread, kEmbedThreads V apart.
template <typename T, typename G, int V, int U>
struct EmbedColumns {
  int base;
  int dim;
  __device__ __forceinline__ EmbedColumns(int slice, int dim_) : base(slice * (kEmbedThreads * V * U) + static_cast<int>(threadIdx.x) * V), dim(dim_) {}
  __device__ __forceinline__ int at(int u) const { return base + u * kEmbedThreads * V; }
  __device__ __forceinline__ bool in(int u) const { return at(u) < dim; }
};

template <typename T, typename G, int V, int U>
__device__ __forceinline__ void embed_write(const EmbedGradParams& q, const EmbedColumns<T, G, V, U>& c, unsigned token, float (&sum)[U][V]) {
  G* row = static_cast<G*>(q.dtable) + token * q.ld_grad;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!c.in(u)) continue;
    float f[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      f[k] = sum[u][k] * q.scale;
      if (q.accumulate) f[k] += to_float(row[c.at(u) + k]);
    }
    store_part<G, V>(row + c.at(u), f);
  }
}

template <typename T, typename G, int V, int U>
__global__ __launch_bounds__(kEmbedThreads) void embed_sum_kernel(EmbedGradParams q) {
  const int slice = blockIdx.x % q.slices, block = blockIdx.x / q.slices;
  const EmbedColumns<T, G, V, U> c(slice, q.dim);
  if (block >= q.token_ctas) {   // rows of tokens that do not occur
    float zero[V] = {};
    const int ctas = gridDim.x / q.slices - q.token_ctas;
    for (int v = block - q.token_ctas; v < q.vocab; v += ctas) {
      if (q.n && (q.present[v >> 5] >> (v & 31) & 1)) continue;
      G* row = static_cast<G*>(q.dtable) + v * q.ld_grad;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c.in(u)) store_part<G, V>(row + c.at(u), zero);
    }
    return;
  }
  const unsigned* keys = q.keys[(q.passes + 1) & 1];
  const unsigned* places = q.places[(q.passes + 1) & 1];
  const int begin = block * q.chunk, end = min(begin + q.chunk, q.n);
  int p = begin, first = begin;   // a piece's first place, its token's first place
  unsigned key = keys[p];
  if (p > 0 && keys[p - 1] == key) {   // a token that began in front: its first piece that begins here
    first = embed_first(keys, p, key);
    const int next = first + (p - first + q.piece - 1) / q.piece * q.piece;
    if (next + q.piece <= q.n && keys[next + q.piece - 1] == key) p = next;
    else while (p < q.n && keys[p] == key) ++p;   // (the piece in front takes the rest, fewer than a piece)
  }
  while (p < end) {
    key = keys[p];
    if (key >= static_cast<unsigned>(q.vocab)) return;   // places without a token, sorted to the end
    if (p != begin && keys[p - 1] != key) first = p;
    const bool more = p + 2 * q.piece <= q.n && keys[p + 2 * q.piece - 1] == key;
    int stop = more ? p + q.piece : p + 1;
    if (!more) while (stop < q.n && keys[stop] == key) ++stop;
    float sum[U][V] = {};
    for (int i = p; i < stop; ++i) {
      const T* row = static_cast<const T*>(q.dy) + places[i] * q.ld_dy;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!c.in(u)) continue;
        float f[V];
        load_part<T, V>(row + c.at(u), f);
#pragma unroll
        for (int k = 0; k < V; ++k) sum[u][k] += f[k];
      }
    }
    if (more || p != first) {   // one of several pieces; those begin at least a piece apart
      float* to = q.partial + static_cast<long long>(p / q.piece) * q.dim;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (c.in(u)) to[c.at(u) + k] = sum[u][k];
    } else {
      embed_write<T, G, V, U>(q, c, key, sum);
    }
    p = stop;
  }
}

// Joins the pieces of a token that has several: the CTAs of block b look for a token that begins in places
// b piece .. (b + 1) piece - 1 and has two pieces at least (there is one at most).
template <typename T, typename G, int V, int U>
__global__ __launch_bounds__(kEmbedThreads) void embed_join_kernel(EmbedGradParams q) {
  const int slice = blockIdx.x % q.slices, block = blockIdx.x / q.slices;
  const unsigned* keys = q.keys[(q.passes + 1) & 1];
  const int end = min((block + 1) * q.piece, q.n);
  // the token of the block's last place is the only one that can reach a piece beyond
  const unsigned key = keys[end - 1];
  if (key >= static_cast<unsigned>(q.vocab)) return;
  const int first = embed_first(keys, end - 1, key);
  if (first < block * q.piece || first + 2 * q.piece > q.n || keys[first + 2 * q.piece - 1] != key) return;
  const EmbedColumns<T, G, V, U> c(slice, q.dim);
  float sum[U][V] = {};
  for (int p = first; p + q.piece <= q.n && keys[p + q.piece - 1] == key; p += q.piece) {
    const float* from = q.partial + static_cast<long long>(p / q.piece) * q.dim;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (c.in(u)) sum[u][k] += from[c.at(u) + k];
  }
  embed_write<T, G, V, U>(q, c, key, sum);
}

}  // namespace adapt
