// C-ABI entry points of the 8-bit codes and their product.  Declarations and argument contracts live in adapt.h.
#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "k_int8.cuh"
#include "training_host.cuh"

using namespace adapt;

namespace {

int run_rows(const RowsParams& q, int dtype, cudaStream_t stream) {
  const int e = elem_bytes(dtype), wide = 16 / e;
  // a row in the registers of up to 256 threads, 8 chunks each
  const bool vec = q.cols % wide == 0 && q.cols <= kRowsThreads * 8 * wide && !misaligned(q.x, 16) && !misaligned(q.codes, wide) &&
                   (q.rows == 1 || (q.ldx % wide == 0 && q.ld_codes % wide == 0));
  LaunchScope ls(ADAPT_KERNEL_INT8_ROWS, stream);
  const unsigned grid = static_cast<unsigned>(q.rows);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (!vec) { int8_rows_any_kernel<T><<<grid, kRowsThreads, 0, stream>>>(q); return; }
    const int chunks = q.cols / wide;
    auto threads = [&](int per) { return static_cast<unsigned>(std::max(32, (chunks + per * 32 - 1) / (per * 32) * 32)); };
    if (chunks <= kRowsThreads * 2) int8_rows_kernel<T, 2><<<grid, threads(2), 0, stream>>>(q);
    else if (chunks <= kRowsThreads * 4) int8_rows_kernel<T, 4><<<grid, threads(4), 0, stream>>>(q);
    else int8_rows_kernel<T, 8><<<grid, threads(8), 0, stream>>>(q);
  });
  ADAPT_LAUNCH_OK("rows to 8-bit codes");
  return ADAPT_OK;
}

int run_copy(const CopyParams& q, cudaStream_t stream) {
  LaunchScope ls(ADAPT_KERNEL_INT8_ROWS, stream);
  int8_copy_kernel<<<static_cast<unsigned>(q.part[0].rows) + static_cast<unsigned>(q.part[1].rows), kCopyThreads, 0, stream>>>(q);
  ADAPT_LAUNCH_OK("rows of codes");
  return ADAPT_OK;
}

// Whether the TMA unit can read rows of codes as they lie.
bool tma_rows(const void* p, int64_t ld, int64_t rows) {
  return !misaligned(p, 16) && (rows == 1 || (ld > 0 && ld % 16 == 0));
}

// What a product keeps in its workspace: codes of activations that it quantises, and copies of codes that do not
// lie on 16-byte boundaries.  A few tokens need neither.
struct LinearLayout {
  size_t x = 0, scales = 0, w = 0, bytes = 0;
  bool quantise = false, copy_x = false, copy_w = false;
  long long ld = 0;
  LinearLayout(const void* px, int x_dtype, const void* pw, int64_t rows, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    if (rows <= kDotMaxRows || k == 0) return;
    quantise = x_dtype != ADAPT_DTYPE_I8;
    copy_x = !quantise && !tma_rows(px, ldx, rows);
    copy_w = !tma_rows(pw, ldw, n);
    ld = (k + 15) / 16 * 16;
    auto take = [&](size_t b) { const size_t here = bytes; bytes = align_up(bytes + b, 256); return here; };
    if (quantise || copy_x) x = take(static_cast<size_t>(rows) * ld);
    if (quantise) scales = take(4 * static_cast<size_t>(rows));
    if (copy_w) w = take(static_cast<size_t>(n) * ld);
  }
};

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_tiled(EncodeTiled* out) {
  static std::atomic<void*> known{nullptr};
  void* f = known.load();
  if (!f) {
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    ADAPT_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !f) return cuda_fail(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
    known.store(f);
  }
  *out = reinterpret_cast<EncodeTiled>(f);
  return ADAPT_OK;
}

// Tiles of `height` rows by kDepth codes; what lies outside the matrix reads as 0.
int tile_map(CUtensorMap* map, const void* p, int64_t rows, int64_t k, int64_t ld, int height) {
  EncodeTiled encode = nullptr;
  const int rc = encode_tiled(&encode);
  if (rc != ADAPT_OK) return rc;
  const cuuint64_t sizes[2] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(rows == 1 ? (k + 15) / 16 * 16 : ld)};
  const cuuint32_t box[2] = {kDepth, static_cast<cuuint32_t>(height)}, step[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), sizes, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return cuda_fail(cudaErrorInvalidValue, "tensor map of 8-bit codes");
  return ADAPT_OK;
}

// Launches a product.  `early`: it may begin before the kernel in front of it, one of this call's, has ended.
template <auto kKernel, typename... A>
int launch(unsigned x, unsigned y, int threads, int smem, int cluster, bool early, cudaStream_t stream, A... args) {
  static std::atomic<uint64_t> ready{0};   // (one for each kernel) devices that know its shared memory
  int device = 0;
  ADAPT_CUDA(cudaGetDevice(&device));
  const uint64_t bit = 1ull << (device & 63);
  if (!(ready.load() & bit)) {
    ADAPT_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    ready.fetch_or(bit);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(x, y);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  unsigned n = 0;
  if (early) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster; attr[n].val.clusterDim.y = 1; attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  ADAPT_CUDA(cudaLaunchKernelEx(&cfg, kKernel, args...));
  return ADAPT_OK;
}

int run_dot(const LinearParams& q, const void* x, int x_dtype, int dtype, int64_t ldw, cudaStream_t stream) {
  DotParams d = {};
  d.p = q;
  d.x = x;
  const bool shift = misaligned(q.w, 16) || (q.n > 1 && ldw % 16 != 0);
  const unsigned grid = static_cast<unsigned>((q.n + kDotThreads / 32 * kDotChannels - 1) / (kDotThreads / 32 * kDotChannels));
  LaunchScope ls(ADAPT_KERNEL_INT8_LINEAR, stream);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto v) {
      using X = decltype(v);
      auto rows = [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (shift) int8_dot_kernel<T, X, R, true><<<grid, kDotThreads, 0, stream>>>(d);
        else int8_dot_kernel<T, X, R, false><<<grid, kDotThreads, 0, stream>>>(d);
      };
      if (q.rows == 1) rows(std::integral_constant<int, 1>{});
      else rows(std::integral_constant<int, kDotMaxRows>{});
    };
    if (x_dtype == ADAPT_DTYPE_I8) go(static_cast<signed char>(0)); else with_type(x_dtype, go);
  });
  ADAPT_LAUNCH_OK("8-bit product");
  return ADAPT_OK;
}

// How a product is cut: into tiles of pairs (tokens 0), or into tiles of so many tokens by 128 channels whose sums are dealt to
// `split` CTAs.  Estimated in clocks: a code of the sum's index takes a tile the clocks of its products (8192 a
// clock and SM) or those of its operands' way from L2 (about 50 bytes a clock and SM), a CTA some thousand to begin
// and a sum that is dealt some thousand more.  Measured, us: 16384 channels, sums of 4096: 256 tokens (narrow) 20.4, 300 (pairs)
// 29.2.  The estimate errs where a narrow sum is dealt to four: 4096 x 4096 256 tokens (narrow) 22.8, 300 (pairs) 18.6, which would take
// 256 in the same time; 8192 x 8192 32.9 and 29.3.
struct Cut { int tokens, split; };
Cut choose_cut(int64_t rows, int64_t n, int64_t k) {
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const int64_t blocks = up(k, kDepth), across = up(n, kCtaRows);
  Cut best = {0, 1};
  int64_t least = up(up(rows, kWideTile) * up(n, kWideTile), kSms / 2) * (blocks * kDepth * 9 / 2 + 1000) + 6000;
  for (int tokens = 16; tokens <= 256; tokens *= 2) {
    if ((tokens >= 2 * rows && tokens > 16) || up(rows, tokens) > 65535) continue;   // (a grid's second extent)
    for (int split = 1; split <= narrow_split(tokens) && blocks >= 2 * split; split *= 2) {
      const int64_t waves = up(across * up(rows, tokens) * split, kSms), depth = up(blocks, split) * kDepth;
      const int64_t per = std::max<int64_t>(2 * (kCtaRows + tokens), 100 * tokens / 64);   // hundredths of a clock a code
      const int64_t clocks = waves * (depth * per / 100 + 2000 + 12 * tokens) + (split > 1 ? 2000 + 8 * tokens : 0) + 2000;
      if (clocks < least) { least = clocks; best = {tokens, split}; }
    }
  }
  return best;
}

int run_tiles(const LinearParams& q, int dtype, bool early, cudaStream_t stream) {
  const int e = elem_bytes(dtype);
  const Cut cut = choose_cut(q.rows, q.n, q.k);
  CUtensorMap x_map, w_map;
  int rc = ADAPT_OK;
  WideParams wide = {};
  wide.across = (q.n + kWideTile - 1) / kWideTile;
  wide.down = (q.rows + kWideTile - 1) / kWideTile;
  const int64_t tiles = static_cast<int64_t>(wide.across) * wide.down;
  if (tiles > 0x7FFFFFFF) return ADAPT_ERR_INVALID_ARG;
  LaunchScope ls(ADAPT_KERNEL_INT8_LINEAR, stream);
  if (cut.tokens == 0) {
    if ((rc = tile_map(&x_map, q.x, q.rows, q.k, q.ldx, kCtaRows)) != ADAPT_OK || (rc = tile_map(&w_map, q.w, q.n, q.k, q.ldw, kCtaRows)) != ADAPT_OK)
      return rc;
    wide.p = q;
    wide.wide_stores = !misaligned(q.y, 32) && (q.rows == 1 || q.ldy * e % 32 == 0);
    const unsigned grid = 2 * static_cast<unsigned>(std::min<int64_t>(tiles, kSms / 2));
    with_type(dtype, [&](auto t) {
      rc = launch<int8_wide_kernel<decltype(t)>>(grid, 1u, kWideThreads, kWideSmem, 0, early, stream, x_map, w_map, wide);
    });
    return rc;
  }
  const int tokens = cut.tokens, split = cut.split, across = (q.n + kCtaRows - 1) / kCtaRows, down = (q.rows + tokens - 1) / tokens;
  if ((rc = tile_map(&x_map, q.x, q.rows, q.k, q.ldx, tokens)) != ADAPT_OK || (rc = tile_map(&w_map, q.w, q.n, q.k, q.ldw, kCtaRows)) != ADAPT_OK)
    return rc;
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto c) {
      constexpr int N = decltype(c)::value;
      rc = launch<int8_narrow_kernel<T, N>>(static_cast<unsigned>(across * split), static_cast<unsigned>(down), kNarrowThreads, narrow_smem(N), split,
                  early, stream, x_map, w_map, q);
    };
    if (tokens == 16) go(std::integral_constant<int, 16>{});
    else if (tokens == 32) go(std::integral_constant<int, 32>{});
    else if (tokens == 64) go(std::integral_constant<int, 64>{});
    else if (tokens == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 256>{});
  });
  return rc;
}

}  // namespace

extern "C" {

int adapt_int8_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int8_t* codes, int64_t ld_codes,
                    float* scales, void* stream) {
  const int e = elem_bytes(dtype);
  if (!e || !in_int(rows, 0) || !in_int(cols, 0)) return ADAPT_ERR_INVALID_ARG;
  if (rows == 0) return ADAPT_OK;
  if (!scales || misaligned(scales, 4)) return ADAPT_ERR_INVALID_ARG;
  if (cols > 0 && (!x || !codes || misaligned(x, e))) return ADAPT_ERR_INVALID_ARG;
  if (rows > 1 && ((ldx < cols && ldx != 0) || ld_codes < cols)) return ADAPT_ERR_INVALID_ARG;
  RowsParams q = {};
  q.x = x; q.codes = codes; q.scales = scales; q.ldx = ldx; q.ld_codes = ld_codes;
  q.rows = static_cast<int>(rows); q.cols = static_cast<int>(cols);
  return run_rows(q, dtype, static_cast<cudaStream_t>(stream));
}

size_t adapt_int8_linear_workspace_bytes(const void* x, int x_dtype, const int8_t* weight, int64_t rows, int64_t n, int64_t k, int64_t ldx,
                                         int64_t ldw) {
  if (!in_int(rows, 1) || !in_int(n, 1) || k < 0 || k > ADAPT_INT8_MAX_K || (x_dtype != ADAPT_DTYPE_I8 && !elem_bytes(x_dtype))) return 0;
  return LinearLayout(x, x_dtype, weight, rows, n, k, ldx, ldw).bytes;
}

int adapt_int8_linear(const void* x, int x_dtype, const float* x_scales, int64_t x_scale_count, const int8_t* weight,
                      const float* weight_scales, int64_t weight_scale_count, const float* bias, int64_t rows, int64_t n,
                      int64_t k, int64_t ldx, int64_t ldw, void* y, int64_t ldy, int dtype, void* workspace,
                      size_t workspace_bytes, void* stream_handle) {
  const int e = elem_bytes(dtype), ex = x_dtype == ADAPT_DTYPE_I8 ? 1 : elem_bytes(x_dtype);
  const bool coded = x_dtype == ADAPT_DTYPE_I8;
  if (!e || !ex || !in_int(rows, 0) || !in_int(n, 0) || k < 0 || k > ADAPT_INT8_MAX_K) return ADAPT_ERR_INVALID_ARG;
  if (coded ? (x_scale_count != 1 && x_scale_count != rows) : x_scales != nullptr) return ADAPT_ERR_INVALID_ARG;
  if (weight_scale_count != 1 && weight_scale_count != n) return ADAPT_ERR_INVALID_ARG;
  if (rows == 0 || n == 0) return ADAPT_OK;
  if (!y || !weight_scales || (coded && !x_scales) || (k > 0 && (!x || !weight))) return ADAPT_ERR_INVALID_ARG;
  if (misaligned(x, ex) || misaligned(x_scales, 4) || misaligned(weight_scales, 4) || misaligned(bias, 4) || misaligned(y, e))
    return ADAPT_ERR_INVALID_ARG;
  if (rows > 1 && ((ldx < k && ldx != 0) || ldy < n)) return ADAPT_ERR_INVALID_ARG;
  if (n > 1 && ldw < k && ldw != 0) return ADAPT_ERR_INVALID_ARG;
  const LinearLayout lay(x, x_dtype, weight, rows, n, k, ldx, ldw);
  if (lay.bytes) {
    if (!workspace || misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    if (workspace_bytes < lay.bytes) return ADAPT_ERR_WORKSPACE;
  }
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  LinearParams q = {};
  q.x = static_cast<const signed char*>(x); q.x_scales = x_scales; q.ldx = ldx; q.x_one = coded && x_scale_count == 1;
  q.w = weight; q.w_scales = weight_scales; q.bias = bias; q.y = y; q.ldw = ldw; q.ldy = ldy;
  q.rows = static_cast<int>(rows); q.n = static_cast<int>(n); q.k = static_cast<int>(k);
  q.w_one = weight_scale_count == 1;
  if (k == 0) {
    LaunchScope ls(ADAPT_KERNEL_INT8_LINEAR, stream);
    with_type(dtype, [&](auto t) { int8_bias_kernel<decltype(t)><<<static_cast<unsigned>(rows), 256, 0, stream>>>(q); });
    ADAPT_LAUNCH_OK("8-bit product");
    return ADAPT_OK;
  }
  if (rows <= kDotMaxRows) return run_dot(q, x, x_dtype, dtype, ldw, stream);
  signed char* ws = static_cast<signed char*>(workspace);
  int rc = ADAPT_OK;
  if (lay.copy_x || lay.copy_w) {
    CopyParams c = {};
    c.cols = q.k;
    if (lay.copy_x) {
      c.part[0] = {q.x, ws + lay.x, rows > 1 ? ldx : 0, lay.ld, q.rows};
      q.x = c.part[0].to; q.ldx = lay.ld;
    }
    if (lay.copy_w) {
      c.part[1] = {weight, ws + lay.w, n > 1 ? ldw : 0, lay.ld, q.n};
      q.w = c.part[1].to; q.ldw = lay.ld;
    }
    if ((rc = run_copy(c, stream)) != ADAPT_OK) return rc;
  }
  if (lay.quantise) {
    RowsParams r = {};
    r.x = x; r.ldx = ldx; r.ld_codes = lay.ld; r.rows = q.rows; r.cols = q.k;
    r.codes = ws + lay.x;
    r.scales = reinterpret_cast<float*>(ws + lay.scales);
    if ((rc = run_rows(r, x_dtype, stream)) != ADAPT_OK) return rc;
    q.x = r.codes; q.x_scales = r.scales; q.ldx = lay.ld;
  }
  // (where activations are quantised as well, the weights' copies were complete when that kernel began)
  q.w_late = lay.copy_w && !lay.quantise;
  return run_tiles(q, dtype, lay.quantise || lay.copy_x || lay.copy_w, stream);
}

}  // extern "C"
