// C-ABI entry points of the token embedding and its gradient.  Declarations and argument contracts live in
// adapt.h.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "k_embedding.cuh"
#include "training_host.cuh"

using namespace adapt;

namespace {

bool in_int(int64_t v, int64_t least) { return v >= least && v <= 0x7FFFFFFF; }

// Places of a piece: its sums go to memory and back in fp32 (4 / piece of the bytes of dy in 16 bits), and a
// token's pieces are joined one after the other.
int embed_piece(int64_t n) {
  int piece = 32;
  while (piece < 1024 && n > 256ll * piece) piece *= 2;
  return piece;
}

struct EmbedLayout {
  size_t keys[2], places[2], present, partial, bytes;
  EmbedLayout(int64_t n, int64_t dim, int64_t vocab) {
    size_t at = 0;
    auto take = [&](size_t b) { const size_t here = at; at = align_up(at + b, 256); return here; };
    for (int i = 0; i < 2; ++i) { keys[i] = take(4 * n); places[i] = take(4 * n); }
    present = take((vocab + 31) / 32 * 4);
    partial = take((n / embed_piece(n) + 1) * dim * 4);
    bytes = at;
  }
};

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
  const int64_t parts = vec ? dim / wide : dim;
  int lanes = 1;
  while (lanes < kEmbedThreads && lanes * 4 < parts) lanes *= 2;
  const int rows = kEmbedThreads / lanes;
  const unsigned grid = static_cast<unsigned>((n + rows - 1) / rows);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  LaunchScope ls(ADAPT_KERNEL_EMBEDDING, stream);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (vec) embedding_kernel<T, 16 / sizeof(T)><<<grid, kEmbedThreads, 0, stream>>>(q, lanes);
    else embedding_kernel<T, 1><<<grid, kEmbedThreads, 0, stream>>>(q, lanes);
  });
  ADAPT_LAUNCH_OK("token embedding");
  return ADAPT_OK;
}

size_t adapt_embedding_workspace_bytes(int64_t n, int64_t dim, int64_t vocab) {
  if (!in_int(vocab, 1) || !in_int(dim, 1) || !in_int(n, 1)) return 0;
  return EmbedLayout(n, dim, vocab).bytes;
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
  const EmbedLayout lay(n, dim, vocab);
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
  q.present = reinterpret_cast<unsigned*>(ws + lay.present);
  q.partial = reinterpret_cast<float*>(ws + lay.partial);
  int bits = 1;
  while (bits < 32 && (vocab >> bits)) ++bits;
  q.passes = (bits + kSortWidth - 1) / kSortWidth;
  q.width = (bits + q.passes - 1) / q.passes;
  q.piece = embed_piece(n);
  q.chunk = q.piece / 2;
  const int wide = 16 / e;
  const bool vec = dim % wide == 0 && !misaligned(dy, 16) && !misaligned(dtable, 16) && (n <= 1 || ld_dy % wide == 0) &&
                   (vocab == 1 || ld_grad % wide == 0);
  const int64_t columns = kEmbedThreads * (vec ? wide : 4);
  q.slices = static_cast<int>((dim + columns - 1) / columns);
  q.token_ctas = static_cast<int>((n + q.chunk - 1) / q.chunk);
  const int64_t zero_ctas = accumulate ? 0 : std::min<int64_t>(vocab, 148 * 8);
  const int64_t grid = (q.token_ctas + zero_ctas) * q.slices, joins = (n + q.piece - 1) / q.piece * q.slices;
  if (grid > 0x7FFFFFFF || joins > 0x7FFFFFFF) return ADAPT_ERR_INVALID_ARG;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  if (n > 0) {
    int parts = 1;
    while (parts < kSortMaxCluster && n > 1024ll * parts) parts *= 2;
    LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parts);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = kSortSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ADAPT_CUDA(cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmem));
    if (parts > 8) ADAPT_CUDA(cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    ADAPT_CUDA(cudaLaunchKernelEx(&cfg, embed_sort_kernel, q));
  }
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto g) {
      using G = decltype(g);
      constexpr int V = 16 / sizeof(T);
      {
        LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
        if (vec) embed_sum_kernel<T, G, V, 1><<<static_cast<unsigned>(grid), kEmbedThreads, 0, stream>>>(q);
        else embed_sum_kernel<T, G, 1, 4><<<static_cast<unsigned>(grid), kEmbedThreads, 0, stream>>>(q);
      }
      if (n >= 2 * q.piece) {
        LaunchScope ls(ADAPT_KERNEL_EMBEDDING_BACKWARD, stream);
        if (vec) embed_join_kernel<T, G, V, 1><<<static_cast<unsigned>(joins), kEmbedThreads, 0, stream>>>(q);
        else embed_join_kernel<T, G, 1, 4><<<static_cast<unsigned>(joins), kEmbedThreads, 0, stream>>>(q);
      }
    };
    if (grad_dtype == dtype) go(T{}); else go(float{});
  });
  ADAPT_LAUNCH_OK("token embedding, backward");
  return ADAPT_OK;
}

}  // extern "C"
