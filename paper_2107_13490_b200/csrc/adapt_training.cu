// C-ABI entry points of the training-step operators dropout and token log probabilities.  Declarations and
// argument contracts live in adapt.h.
#include <cmath>
#include <cstdint>

#include "dropout_pieces.h"
#include "k_dropout.cuh"
#include "k_logprobs.cuh"
#include "training_host.cuh"

using namespace adapt;

static_assert(ADAPT_MAX_TOP == kMaxTop, "the kernels use the constant of the C interface");

extern "C" {

int adapt_dropout(const void* x, const void* residual, void* y, int64_t rows, int64_t cols, int64_t ldx,
                  int64_t ldr, int64_t ldy, int dtype, double p, uint64_t seed, int32_t layer,
                  uint64_t index_base, void* stream_handle) {
  const int e = elem_bytes(dtype);
  if (!e || rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0)) return ADAPT_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return ADAPT_OK;
  if (!x || !y || misaligned(x, e) || misaligned(y, e) || misaligned(residual, e)) return ADAPT_ERR_INVALID_ARG;
  if (rows > (1ll << 48) / cols || index_base > (1ull << 62)) return ADAPT_ERR_INVALID_ARG;
  if (rows > 1 && (ldx < cols || ldy < cols || (residual && ldr < cols))) return ADAPT_ERR_INVALID_ARG;
  if (rows == 1) ldx = ldr = ldy = cols;
  // whether x, r and y lie alike to the 16-byte boundary, in every row
  auto off = [&](const void* a, const void* b) { return (reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u; };
  const bool vec = !off(x, y) && (!residual || !off(x, residual)) &&
                   (rows == 1 || ((ldx - ldy) % (16 / e) == 0 && (!residual || (ldx - ldr) % (16 / e) == 0)));
  const bool pairs = !vec && rows > 1 && cols < kPairsBelow;
  const int unit = pairs ? 2 : 16 / e;
  DropoutParams q = {};
  q.cols = cols; q.ldx = ldx; q.ldr = ldr; q.ldy = ldy;
  q.base = seed ^ 0xA54FF53A5F1D36F1ull ^ ((static_cast<uint64_t>(static_cast<int64_t>(layer)) + 1ull) * 0x9E3779B97F4A7C15ull);
  const double threshold = std::nearbyint(p * 4294967296.0);
  q.none = threshold >= 4294967296.0;
  q.threshold = q.none ? 0u : static_cast<unsigned>(threshold);
  q.scale = p < 1.0 ? static_cast<float>(1.0 / (1.0 - p)) : 0.0f;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  const DropoutPieces pieces(rows, cols, unit);
  return pieces.each([&](int64_t row, int64_t col, int64_t n_rows, int64_t n_cols) -> int {
    q.x = static_cast<const char*>(x) + (row * ldx + col) * e;
    q.y = static_cast<char*>(y) + (row * ldy + col) * e;
    q.r = residual ? static_cast<const char*>(residual) + (row * ldr + col) * e : nullptr;
    q.x_end = static_cast<const char*>(q.x) + ((n_rows - 1) * ldx + n_cols) * e;
    q.r_end = residual ? static_cast<const char*>(q.r) + ((n_rows - 1) * ldr + n_cols) * e : nullptr;
    q.index_base = static_cast<long long>(index_base) + row * cols + col;
    if (n_rows == 1 && !pairs) {
      q.mis = static_cast<int>((reinterpret_cast<uintptr_t>(q.y) & 15u) / e);
      q.cols = n_cols;
      q.chunks = static_cast<unsigned>((q.mis + n_cols + unit - 1) / unit);
      q.from = q.mis ? 1 : 0;
      q.to = static_cast<unsigned>((q.mis + n_cols) / unit);
    } else {   // whole rows
      q.per_row = static_cast<unsigned>(pieces.per_row);
      q.chunks = static_cast<unsigned>(pieces.per_row * n_rows);
      // i / d for i < 2^31, d >= 2: magic = ceil(2^(32 + s) / d) with 2^s >= d / 2 (Granlund and Montgomery)
      unsigned s = 0;
      while ((2ull << s) < q.per_row) ++s;
      q.shift = s;
      q.magic = static_cast<unsigned>(((1ull << (32 + s)) + q.per_row - 1) / q.per_row);
    }
    const unsigned tile = kDropoutThreads * (pairs ? kPairsUnroll : vec ? kDropoutUnroll : kShiftUnroll);
    const unsigned grid = (q.chunks + tile - 1) / tile;
    LaunchScope ls(ADAPT_KERNEL_DROPOUT, stream);
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      auto go = [&](auto kernel) { kernel<<<grid, kDropoutThreads, 0, stream>>>(q); };
      if (pairs) {
        residual ? go(dropout_pairs_kernel<T, true>) : go(dropout_pairs_kernel<T, false>);
      } else if (n_rows == 1) {
        if (vec) residual ? go(dropout_kernel<T, false, true, false>) : go(dropout_kernel<T, false, false, false>);
        else residual ? go(dropout_kernel<T, true, true, false>) : go(dropout_kernel<T, true, false, false>);
      } else {
        if (vec) residual ? go(dropout_kernel<T, false, true, true>) : go(dropout_kernel<T, false, false, true>);
        else residual ? go(dropout_kernel<T, true, true, true>) : go(dropout_kernel<T, true, false, true>);
      }
    });
    ADAPT_LAUNCH_OK("dropout");
    return ADAPT_OK;
  });
}

}  // extern "C"

namespace {

// CTAs that share a row: enough to fill the device, with two 16-byte loads at least for each thread; and,
// where the gradient comes out of the same call, so many that the rows under way stay in L2 for the
// second reading.
int logprob_parts(const LogprobParams& q, int elem, int sm_count) {
  const long long slots = 6ll * sm_count, least = 2ll * kRowThreads * 16 / elem;
  int parts = 1;
  while (parts < kRowMaxCluster && q.vocab / (2 * parts) >= least) {
    const bool idle = q.rows * parts * 2 <= slots;
    const long long under_way = std::min<long long>(q.rows, slots / parts) * q.vocab * elem;
    const bool spills = q.dlogits && !q.lse_in && under_way > (64ll << 20);
    if (!idle && !spills) break;
    parts *= 2;
  }
  return parts;
}

// Many rows of up to 8192 logits take a warp each, others a CTA each: a CTA's barriers cost about 5 us a
// row, which long rows hide and few rows do not repeat.  Measured on bf16, warp against CTA, us: 16384 x 4096
// 31 / 76, 16384 x 8192 51 / 77, 2048 x 8192 13 / 15, 512 x 8192 with gradient 17 / 11, 2048 x 16384 21 / 19.
constexpr int kTeamRowMax = 8192;
constexpr int kTeamMinRows = 1024;

int run_logprobs(LogprobParams& q, int dtype, void* stream_handle) {
  const int e = elem_bytes(dtype);
  if (!e || q.rows < 0 || q.rows > 0x7FFFFFFF || q.vocab < 1 || !(q.scale > 0.0f) || !std::isfinite(q.scale))
    return ADAPT_ERR_INVALID_ARG;
  if (q.rows == 0) return ADAPT_OK;
  if (!q.logits || misaligned(q.logits, e) || misaligned(q.dlogits, e)) return ADAPT_ERR_INVALID_ARG;
  if (q.rows > 1 && (q.ld < q.vocab || (q.dlogits && q.ld_grad < q.vocab))) return ADAPT_ERR_INVALID_ARG;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  LaunchScope ls(ADAPT_KERNEL_LOGPROBS, stream);
  if (q.vocab <= kWarpRowMax) {
    const unsigned grid = static_cast<unsigned>((q.rows + kRowThreads / 32 - 1) / (kRowThreads / 32));
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      if (q.vocab <= 128) logprob_warp_kernel<T, 4><<<grid, kRowThreads, 0, stream>>>(q);
      else if (q.vocab <= 512) logprob_warp_kernel<T, 16><<<grid, kRowThreads, 0, stream>>>(q);
      else logprob_warp_kernel<T, 32><<<grid, kRowThreads, 0, stream>>>(q);
    });
    ADAPT_LAUNCH_OK("token log probabilities");
    return ADAPT_OK;
  }
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceCache* dc = nullptr;
  int rc = current_cache(&dc);
  if (rc != ADAPT_OK) return rc;
  const int parts = logprob_parts(q, e, dc->sm_count);
  const long long ctas = q.rows * parts;
  if (ctas > 0x7FFFFFFF) return ADAPT_ERR_INVALID_ARG;   // (never: many rows are not split)
  const bool teams = parts == 1 && q.vocab <= kTeamRowMax && q.rows >= kTeamMinRows;
  const unsigned team_grid = static_cast<unsigned>((q.rows + kRowThreads / 32 - 1) / (kRowThreads / 32));
  if (q.lse_in || teams) {
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      if (!q.lse_in) logprob_row_kernel<T, 32><<<team_grid, kRowThreads, 0, stream>>>(q);
      else if (teams) logprob_backward_kernel<T, 32><<<team_grid, kRowThreads, 0, stream>>>(q, 1);
      else logprob_backward_kernel<T, kRowThreads><<<static_cast<unsigned>(ctas), kRowThreads, 0, stream>>>(q, parts);
    });
    ADAPT_LAUNCH_OK("token log probabilities");
    return ADAPT_OK;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kRowThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  with_type(dtype, [&](auto t) {
    const auto kernel = logprob_row_kernel<decltype(t), kRowThreads>;
    cudaError_t err = cudaSuccess;
    if (parts > 8) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err == cudaSuccess) err = cudaLaunchKernelEx(&cfg, kernel, q);
    if (err != cudaSuccess) rc = cuda_fail(err, "token log probabilities");
  });
  if (rc != ADAPT_OK) return rc;
  ADAPT_LAUNCH_OK("token log probabilities");
  return ADAPT_OK;
}

}  // namespace

extern "C" {

int adapt_token_logprobs(const void* logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, float scale,
                         const int64_t* targets, int n_top, float* logprob_out, float* entropy_out,
                         float* lse_out, int32_t* top_ids_out, float* top_logprobs_out,
                         const float* d_logprob, const float* d_entropy, void* dlogits_out,
                         int64_t ld_grad, void* stream) {
  if (vocab < 1 || vocab > 0x7FFFFFFF || n_top < 0 || n_top > kMaxTop || n_top > vocab) return ADAPT_ERR_INVALID_ARG;
  if (rows > 0) {   // (arrays of no rows may have no address)
    if (n_top > 0 && (!top_ids_out || !top_logprobs_out)) return ADAPT_ERR_INVALID_ARG;
    if (!targets && (logprob_out || d_logprob)) return ADAPT_ERR_INVALID_ARG;
    if ((dlogits_out != nullptr) != (d_logprob || d_entropy)) return ADAPT_ERR_INVALID_ARG;
  }
  if (misaligned(targets, 8) || misaligned(logprob_out, 4) || misaligned(entropy_out, 4) || misaligned(lse_out, 4) ||
      misaligned(top_ids_out, 4) || misaligned(top_logprobs_out, 4) || misaligned(d_logprob, 4) || misaligned(d_entropy, 4))
    return ADAPT_ERR_INVALID_ARG;
  LogprobParams q = {};
  q.logits = logits; q.rows = rows; q.ld = ld; q.ld_grad = ld_grad; q.vocab = static_cast<int>(vocab);
  q.n_top = n_top; q.scale = scale; q.targets = reinterpret_cast<const long long*>(targets);
  q.logprob = logprob_out; q.entropy = entropy_out; q.lse = lse_out;
  q.top_ids = top_ids_out; q.top_logprobs = top_logprobs_out;
  q.d_logprob = d_logprob; q.d_entropy = d_entropy; q.dlogits = dlogits_out;
  return run_logprobs(q, dtype, stream);
}

int adapt_token_logprobs_backward(const void* logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                  float scale, const int64_t* targets, const float* lse,
                                  const float* entropy, const float* d_logprob, const float* d_entropy,
                                  void* dlogits_out, int64_t ld_grad, void* stream) {
  if (vocab < 1 || vocab > 0x7FFFFFFF) return ADAPT_ERR_INVALID_ARG;
  if (rows > 0) {
    if (!d_logprob && !d_entropy) return ADAPT_ERR_INVALID_ARG;
    if ((d_logprob && !targets) || (d_entropy && !entropy)) return ADAPT_ERR_INVALID_ARG;
    if (!lse || !dlogits_out) return ADAPT_ERR_INVALID_ARG;
  }
  if (misaligned(targets, 8) || misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(d_logprob, 4) || misaligned(d_entropy, 4))
    return ADAPT_ERR_INVALID_ARG;
  LogprobParams q = {};
  q.logits = logits; q.rows = rows; q.ld = ld; q.ld_grad = ld_grad; q.vocab = static_cast<int>(vocab);
  q.scale = scale; q.targets = reinterpret_cast<const long long*>(targets);
  q.lse_in = lse; q.entropy_in = entropy; q.d_logprob = d_logprob; q.d_entropy = d_entropy; q.dlogits = dlogits_out;
  return run_logprobs(q, dtype, stream);
}

}  // extern "C"
