// C-ABI entry points of the token embedding and its gradient.  Declarations and argument contracts live in
// adapt.h.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "k_embedding.cuh"
#include "training_host.cuh"

using namespace adapt;

namespace {

// How the rows of a gradient are dealt out: CTAs of `teams` teams of `lanes` threads, `slices` of them for a row.
struct EmbedTeams {
  int lanes = 8, teams, slices;
  EmbedTeams(int64_t dim, int per_thread) {
    const int64_t threads = (dim + per_thread - 1) / per_thread;
    while (lanes < kEmbedThreads && lanes < threads) lanes *= 2;
    teams = kEmbedThreads / lanes;
    slices = static_cast<int>((threads + lanes - 1) / lanes);
  }
};

constexpr int kEmbedLeast = 8;

// Sorted places of a block: so many that three CTAs an SM take all of them at once, but kEmbedLeast at least, and a 4096th (a token may
// be in all of them).  Two rows
// of sums in fp32 at most go to memory and back for a block.  (By the teams of 16-bit rows, whatever the type.)
int embed_block(int64_t n, int64_t dim) {
  const EmbedTeams t(dim, 8);
  const int64_t places = 3ll * kSms * t.teams, most = 8192 / (t.teams + 2);   // (64 KB of tokens and places)
  return static_cast<int>(std::min(most, std::max({static_cast<int64_t>(kEmbedLeast), n / 4096, (n * t.slices + places - 1) / places})));
}

struct EmbedLayout {
  size_t keys[2], places[2], joins, partial, bytes;
  EmbedLayout(int64_t n, int64_t dim) {
    size_t at = 0;
    auto take = [&](size_t b) { const size_t here = at; at = align_up(at + b, 256); return here; };
    for (int i = 0; i < 2; ++i) { keys[i] = take(4 * n); places[i] = take(4 * n); }
    const int64_t blocks = (n + embed_block(n, dim) - 1) / embed_block(n, dim);
    joins = take(8 * (blocks + 1));
    partial = take(blocks * 2 * dim * 4);
    bytes = at;
  }
};

// Clusters of `parts` CTAs of the sort that the device holds at once.
template <typename G>
int sort_clusters(int parts, int* out) {
  static std::atomic<int> known[64][5];   // by device and the logarithm of parts
  int device = 0, log = 0;
  ADAPT_CUDA(cudaGetDevice(&device));
  while ((1 << log) < parts) ++log;
  std::atomic<int>& slot = known[device & 63][log];
  int n = slot.load();
  if (!n) {
    const auto kernel = embed_sort_kernel<G>;
    ADAPT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmem));
    ADAPT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parts);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = kSortSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ADAPT_CUDA(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
    n = std::max(1, std::min(n, kSms / parts));
    slot.store(n);
  }
  *out = n;
  return ADAPT_OK;
}

// Launches a kernel behind another one of the same call, which it waits for by itself.
template <typename... A, typename... B>
cudaError_t launch_behind(void (*kernel)(A...), unsigned grid, int threads, int smem, cudaStream_t stream, B... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

extern "C" {

int adapt_embedding(const void* table, int64_t vocab, int64_t dim, int64_t ld_table, int dtype, const int64_t* ids,
                    int64_t n, float scale, void* out, int64_t ld_out, void* stream_handle) {
  const int e = elem_bytes(dtype);
  if (!e || !in_int(vocab, 1) || !in_int(dim, 0) || !in_int(n, 0) || !std::isfinite(scale)) return ADAPT_ERR_INVALID_ARG;
  if (n == 0 || dim == 0) return ADAPT_OK;
  if (!table || !ids || !out || misaligned(table, e) || misaligned(out, e) || misaligned(ids, 8)) return ADAPT_ERR_INVALID_ARG;
  if ((vocab > 1 && ld_table < dim) || (n > 1 && ld_out < dim)) return ADAPT_ERR_INVALID_ARG;
  if (vocab == 1) ld_table = dim;
  if (n == 1) ld_out = dim;
  EmbedParams q = {};
  q.table = table; q.ids = reinterpret_cast<const long long*>(ids); q.out = out; q.ld_table = ld_table; q.ld_out = ld_out;
  q.n = static_cast<int>(n); q.vocab = static_cast<int>(vocab); q.dim = static_cast<int>(dim); q.scale = scale;
  const int wide = 16 / e;
  const bool vec = dim % wide == 0 && !misaligned(table, 16) && !misaligned(out, 16) && (vocab == 1 || ld_table % wide == 0) &&
                   (n == 1 || ld_out % wide == 0);
  const int64_t parts = (dim + wide - 1) / wide + (vec ? 0 : 1);
  int lanes = 1;
  while (lanes < kEmbedThreads && lanes * 4 < parts) lanes *= 2;
  const int rows = kEmbedThreads / lanes;
  const unsigned grid = static_cast<unsigned>((n + rows - 1) / rows);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  LaunchScope ls(ADAPT_KERNEL_EMBEDDING, stream);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (vec) embedding_kernel<T, false><<<grid, kEmbedThreads, 0, stream>>>(q, lanes);
    else embedding_kernel<T, true><<<grid, kEmbedThreads, 0, stream>>>(q, lanes);
  });
  ADAPT_LAUNCH_OK("token embedding");
  return ADAPT_OK;
}

size_t adapt_embedding_workspace_bytes(int64_t n, int64_t dim, int64_t vocab) {
  if (!in_int(vocab, 1) || !in_int(dim, 1) || !in_int(n, 1)) return 0;
  return EmbedLayout(n, dim).bytes;
}

int adapt_embedding_backward(const void* dy, int64_t n, int64_t dim, int64_t ld_dy, int dtype, const int64_t* ids,
                             int64_t vocab, float scale, int accumulate, void* dtable, int64_t ld_grad,
                             int grad_dtype, void* workspace, size_t workspace_bytes, void* stream_handle) {
  const int e = elem_bytes(dtype), eg = elem_bytes(grad_dtype);
  if (!e || !eg || (grad_dtype != dtype && grad_dtype != ADAPT_DTYPE_F32)) return ADAPT_ERR_INVALID_ARG;
  if (!in_int(vocab, 1) || !in_int(dim, 0) || !in_int(n, 0) || !std::isfinite(scale)) return ADAPT_ERR_INVALID_ARG;
  if (dim == 0 || (n == 0 && accumulate)) return ADAPT_OK;
  if (!dtable || misaligned(dtable, eg) || (vocab > 1 && ld_grad < dim)) return ADAPT_ERR_INVALID_ARG;
  if (n > 0 && (!dy || !ids || misaligned(dy, e) || misaligned(ids, 8) || (n > 1 && ld_dy < dim))) return ADAPT_ERR_INVALID_ARG;
  if (n == 1) ld_dy = dim;
  if (vocab == 1) ld_grad = dim;
  const EmbedLayout lay(n, dim);
  if (n > 0) {
    if (!workspace || misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    if (workspace_bytes < lay.bytes) return ADAPT_ERR_WORKSPACE;
  }
  EmbedGradParams q = {};
  q.dy = dy; q.ids = reinterpret_cast<const long long*>(ids); q.dtable = dtable; q.ld_dy = ld_dy; q.ld_grad = ld_grad;
  q.n = static_cast<int>(n); q.vocab = static_cast<int>(vocab); q.dim = static_cast<int>(dim); q.scale = scale;
  q.accumulate = accumulate != 0;
  char* ws = static_cast<char*>(workspace);
  for (int i = 0; i < 2; ++i) {
    q.keys[i] = reinterpret_cast<unsigned*>(ws + lay.keys[i]);
    q.places[i] = reinterpret_cast<unsigned*>(ws + lay.places[i]);
  }
  q.joins = reinterpret_cast<uint2*>(ws + lay.joins);
  q.partial = reinterpret_cast<float*>(ws + lay.partial);
  int bits = 1;
  while (bits < 32 && (vocab >> bits)) ++bits;
  q.passes = n <= kSortFew ? 0 : (bits + kSortWidth - 1) / kSortWidth;
  q.width = q.passes ? (bits + q.passes - 1) / q.passes : 0;
  q.block = embed_block(n, dim);
  q.cut = q.block / 2;   // (a team takes three halves of a block at most)
  const int wide = 16 / e;
  const bool vec = dim % wide == 0 && !misaligned(dy, 16) && !misaligned(dtable, 16) && (n <= 1 || ld_dy % wide == 0) &&
                   (vocab == 1 || ld_grad % wide == 0);
  const EmbedTeams team(dim, wide);
  q.lanes = team.lanes; q.slices = team.slices;
  q.slot = team.lanes * 16 + (vec ? 0 : 16);
  const int64_t blocks = (n + q.block - 1) / q.block, sums = (blocks + team.teams - 1) / team.teams * team.slices;
  if (sums > 0x7FFFFFFF) return ADAPT_ERR_INVALID_ARG;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  int rc = ADAPT_OK;
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto g) {
      using G = decltype(g);
      int parts = 1, clusters = 1;
      while (q.passes && parts < kSortMaxCluster && n > 1024ll * parts) parts *= 2;
      if ((rc = sort_clusters<G>(parts, &clusters)) != ADAPT_OK) return;
      // one that sorts, and as many for the rows of tokens that do not occur as there are 64 KB of them for each
      const int64_t bytes = accumulate ? 0 : vocab * dim * eg;
      clusters = accumulate ? 1 : std::max(2, std::min<int>(clusters, static_cast<int>(std::min<int64_t>(1000, bytes / (65536ll * parts) + 2))));
      {
        LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(parts * clusters);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = kSortSmem;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t err = cudaLaunchKernelEx(&cfg, embed_sort_kernel<G>, static_cast<const EmbedGradParams>(q));
        if (err != cudaSuccess) { rc = cuda_fail(err, "sort of tokens"); return; }
      }
      if (n == 0) return;
      const int64_t smem = 1ll * kStages * team.teams * kStageRows * q.slot + 2ll * (team.teams * q.block + 2 * (q.cut + 1)) * 4;
      if (smem > 220 * 1024) { rc = ADAPT_ERR_INVALID_ARG; return; }   // (never: embed_block has a limit)
      {
        LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
        auto sum = [&](auto kernel) {
          if (smem > 48 * 1024) {
            const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
            if (err != cudaSuccess) return err;
          }
          return launch_behind(kernel, static_cast<unsigned>(sums), kSumThreads, static_cast<int>(smem), stream, q);
        };
        const cudaError_t err = vec ? sum(embed_sum_kernel<T, G, true>) : sum(embed_sum_kernel<T, G, false>);
        if (err != cudaSuccess) { rc = cuda_fail(err, "token embedding, backward"); return; }
      }
      if (blocks > 1) {
        const int64_t joins = std::min<int64_t>(kSms * 8, blocks * ((dim + kJoinColumns - 1) / kJoinColumns));
        LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
        const cudaError_t err = launch_behind(embed_join_kernel<G>, static_cast<unsigned>(joins), 32 * kJoinWarps, 0, stream, q);
        if (err != cudaSuccess) rc = cuda_fail(err, "token embedding, joined sums");
      }
    };
    if (grad_dtype == dtype) go(T{}); else go(float{});
  });
  return rc;
}

}  // extern "C"
