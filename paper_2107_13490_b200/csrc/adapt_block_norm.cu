// C-ABI entry points of the norms around a block.  Declarations and argument contracts live in adapt.h.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "k_block_norm.cuh"
#include "training_host.cuh"

using namespace adapt;

static_assert(ADAPT_NORM_NONE == kNormNone && ADAPT_NORM_RMS == kNormRms && ADAPT_NORM_LAYER == kNormLayer,
              "the kernels use the constants of the C interface");

namespace {

constexpr int kSms = 148;   // of a B200
constexpr int kNormMaxRow = 16 * kNormMaxThreads;          // elements of a row in a CTA's registers, backward
constexpr int kNormMaxRowForward = 32 * kNormMaxThreads;   // and forward

// Elements of a thread and threads of a CTA for a row, and CTAs of an SM.  Backward: 128 registers a thread.
int norm_elems(int64_t dim) { return dim <= 2048 ? 8 : dim <= kNormMaxRow ? 16 : 32; }
int norm_threads(int64_t dim) {
  const int e = norm_elems(dim);
  return std::min<int>(kNormMaxThreads, static_cast<int>((dim + 32 * e - 1) / (32 * e)) * 32);
}
int norm_per_sm(int64_t dim) { return std::max(1, std::min(8, kNormMaxThreads / norm_threads(dim))); }

// CTAs of a backward pass, each with sums of its own over its rows.
int64_t norm_ctas(int64_t rows, int64_t dim) { return std::min<int64_t>(rows, kSms * norm_per_sm(dim)); }

// How the rows come: through how many stages of shared memory (0: as they lie), of which streams.
struct NormPlan {
  NormRing ring = {};
  int smem = 0;
  bool staged = true;
  // the rows that are read, and what is read or written beside them in 16 bytes
  NormPlan(const NormParams& q, int e, int per_sm, std::initializer_list<std::pair<const void*, long long>> in,
           std::initializer_list<std::pair<const void*, long long>> out) {
    const int unit = 16 / e;
    auto fits = [&](const std::pair<const void*, long long>& p) { return !p.first || (!misaligned(p.first, 16) && (q.rows == 1 || p.second % unit == 0)); };
    staged = q.dim % unit == 0;
    int i = 0;
    for (const auto& p : in) {
      staged = staged && fits(p);
      ring.slot[i++] = p.first ? ring.streams++ : -1;
    }
    for (const auto& p : out) staged = staged && fits(p);
    for (const void* p : {static_cast<const void*>(q.weight_after), static_cast<const void*>(q.weight_before), q.shared ? q.gate : nullptr})
      staged = staged && !misaligned(p, 16);
    const int row = ring.streams * q.dim * e, most = 200 * 1024 / per_sm;
    ring.stages = std::min({kNormMaxStages, most / row, 220 * 1024 / row});
    if (ring.stages < 1 && row <= 220 * 1024) ring.stages = 1;
    staged = staged && ring.stages > 0;
    smem = staged ? ring.stages * row : 0;
  }
};

// Launches a kernel that may need more shared memory than a kernel has by itself.
template <auto kKernel>
int norm_launch(unsigned grid, int threads, int smem, cudaStream_t stream, const NormParams& q, const NormRing& ring) {
  static std::atomic<uint64_t> ready{0};   // devices that know
  int device = 0;
  ADAPT_CUDA(cudaGetDevice(&device));
  const uint64_t bit = 1ull << (device & 63);
  if (!(ready.load() & bit)) {
    ADAPT_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024));
    ready.fetch_or(bit);
  }
  kKernel<<<grid, threads, smem, stream>>>(q, ring);
  ADAPT_LAUNCH_OK("block norm");
  return ADAPT_OK;
}

// What forward and backward share; false where it is refused.
bool norm_common(NormParams& q, int64_t rows, int64_t dim, int dtype, const adapt_norm_args* a, const void* block,
                 const void* residual, const void* gate, const float* weight_after, const float* weight_before) {
  const int e = elem_bytes(dtype);
  if (!e || !a || rows < 0 || rows > 0x7FFFFFFF || dim < 0 || dim > ADAPT_NORM_MAX_DIM) return false;
  auto kind = [](int k) { return k == kNormNone || k == kNormRms || k == kNormLayer; };
  if (!kind(a->after) || !kind(a->before) || (a->gate_mode != ADAPT_GATE_SIGMOID && a->gate_mode != ADAPT_GATE_VALUE)) return false;
  if (!std::isfinite(a->scale) || !std::isfinite(a->residual_scale) || !std::isfinite(a->eps) || a->eps < 0.0f) return false;
  if ((weight_after && a->after == kNormNone) || (weight_before && a->before == kNormNone)) return false;
  if (rows > 0 && dim > 0 && !block) return false;
  const bool shared = a->gate_shared != 0;
  if (misaligned(block, e) || misaligned(residual, e) || misaligned(gate, shared ? 4 : e) || misaligned(weight_after, 4) ||
      misaligned(weight_before, 4)) return false;
  q.block = block; q.residual = residual; q.gate = gate; q.weight_after = weight_after; q.weight_before = weight_before;
  q.rows = static_cast<int>(rows); q.dim = static_cast<int>(dim); q.after = a->after; q.before = a->before;
  q.sigmoid = gate && a->gate_mode == ADAPT_GATE_SIGMOID; q.shared = gate && shared;
  q.scale = a->scale; q.residual_scale = a->residual_scale; q.eps = a->eps;
  return true;
}

// The i-th leading dimension: given, or dim.  Rows that are written must not overlap.
bool norm_line(const int64_t* strides, int i, const void* p, bool out, int64_t rows, int64_t dim, long long& ld) {
  ld = strides && rows > 1 ? strides[i] : dim;
  if (!p || rows <= 1) return true;
  return out ? ld >= dim : ld == 0 || ld >= dim;
}

}  // namespace

extern "C" {

int adapt_block_norm(const void* block, const void* residual, const void* gate, const float* weight_after,
                     const float* weight_before, int64_t rows, int64_t dim, int dtype, const adapt_norm_args* args,
                     const int64_t* strides, void* y, void* normed, float* stats_out, void* stream_handle) {
  NormParams q = {};
  if (!norm_common(q, rows, dim, dtype, args, block, residual, gate, weight_after, weight_before)) return ADAPT_ERR_INVALID_ARG;
  const int e = elem_bytes(dtype);
  if (rows == 0 || dim == 0) return ADAPT_OK;
  if ((!y && !normed) || (normed && q.before == kNormNone)) return ADAPT_ERR_INVALID_ARG;
  if (misaligned(y, e) || misaligned(normed, e) || misaligned(stats_out, 16)) return ADAPT_ERR_INVALID_ARG;
  if (!norm_line(strides, 0, block, false, rows, dim, q.ld_block) || !norm_line(strides, 1, residual, false, rows, dim, q.ld_residual) ||
      !norm_line(strides, 2, q.shared ? nullptr : gate, false, rows, dim, q.ld_gate) ||
      !norm_line(strides, 3, y, true, rows, dim, q.ld_y) || !norm_line(strides, 4, normed, true, rows, dim, q.ld_normed))
    return ADAPT_ERR_INVALID_ARG;
  q.y = y; q.normed = normed; q.stats = stats_out;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  int rc = ADAPT_OK;
  LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM, stream);
  if (dim <= kNormMaxRowForward) {
    const int elems = norm_elems(dim), threads = norm_threads(dim), per_sm = std::max(1, std::min(16, (elems <= 16 ? 1024 : 512) / threads));
    const NormPlan plan(q, e, per_sm, {{block, q.ld_block}, {residual, q.ld_residual}, {q.shared ? nullptr : gate, q.ld_gate}, {nullptr, 0}, {nullptr, 0}},
                        {{y, q.ld_y}, {normed, q.ld_normed}});
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(rows, kSms * per_sm));
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      auto go = [&](auto n) {
        constexpr int N = decltype(n)::value;
        if (plan.staged) rc = norm_launch<norm_row_kernel<T, N, true>>(grid, threads, plan.smem, stream, q, plan.ring);
        else rc = norm_launch<norm_row_kernel<T, N, false>>(grid, threads, 0, stream, q, plan.ring);
      };
      if (elems == 8) go(std::integral_constant<int, 8>{});
      else if (elems == 16) go(std::integral_constant<int, 16>{});
      else go(std::integral_constant<int, 32>{});
    });
    return rc;
  }
  with_type(dtype, [&](auto t) {
    const auto kernel = norm_any_kernel<decltype(t)>;
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ADAPT_NORM_MAX_DIM * 4);
    if (err != cudaSuccess) rc = cuda_fail(err, "block norm");
    else kernel<<<static_cast<unsigned>(rows), kNormThreads, q.dim * 4, stream>>>(q);
  });
  if (rc != ADAPT_OK) return rc;
  ADAPT_LAUNCH_OK("block norm");
  return ADAPT_OK;
}

size_t adapt_block_norm_workspace_bytes(int64_t rows, int64_t dim) {
  if (rows < 1 || rows > 0x7FFFFFFF || dim < 1 || dim > ADAPT_NORM_MAX_DIM) return 0;
  return 3 * sizeof(float) * static_cast<size_t>(norm_ctas(rows, dim)) * dim;
}

int adapt_block_norm_backward(const void* block, const void* residual, const void* gate, const float* weight_after,
                              const float* weight_before, const float* stats, const void* d_y, const void* d_normed,
                              int64_t rows, int64_t dim, int dtype, const adapt_norm_args* args, const int64_t* strides,
                              void* d_block, void* d_residual, void* d_gate, float* d_weight_after, float* d_weight_before,
                              void* workspace, size_t workspace_bytes, void* stream_handle) {
  NormParams q = {};
  if (!norm_common(q, rows, dim, dtype, args, block, residual, gate, weight_after, weight_before)) return ADAPT_ERR_INVALID_ARG;
  const int e = elem_bytes(dtype);
  const bool shared = args->gate_shared != 0;
  if (misaligned(d_y, e) || misaligned(d_normed, e) || misaligned(d_block, e) || misaligned(d_residual, e) ||
      misaligned(d_gate, shared ? 4 : e) || misaligned(d_weight_after, 4) || misaligned(d_weight_before, 4) || misaligned(stats, 16))
    return ADAPT_ERR_INVALID_ARG;
  if ((d_weight_after && q.after == kNormNone) || ((d_weight_before || d_normed) && q.before == kNormNone)) return ADAPT_ERR_INVALID_ARG;
  if (dim == 0) return ADAPT_OK;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  if (rows == 0) {   // sums over no rows
    for (float* p : {shared ? static_cast<float*>(d_gate) : nullptr, d_weight_after, d_weight_before})
      if (p) ADAPT_CUDA(cudaMemsetAsync(p, 0, sizeof(float) * dim, stream));
    return ADAPT_OK;
  }
  if (!stats || (!d_y && !d_normed) || (d_residual && !residual) || (d_gate && !gate)) return ADAPT_ERR_INVALID_ARG;
  if (d_weight_before && !d_normed) return ADAPT_ERR_INVALID_ARG;
  if (!norm_line(strides, 0, block, false, rows, dim, q.ld_block) || !norm_line(strides, 1, residual, false, rows, dim, q.ld_residual) ||
      !norm_line(strides, 2, q.shared ? nullptr : gate, false, rows, dim, q.ld_gate) ||
      !norm_line(strides, 3, d_y, false, rows, dim, q.ld_d_y) || !norm_line(strides, 4, d_normed, false, rows, dim, q.ld_d_normed) ||
      !norm_line(strides, 5, d_block, true, rows, dim, q.ld_d_block) || !norm_line(strides, 6, d_residual, true, rows, dim, q.ld_d_residual) ||
      !norm_line(strides, 7, q.shared ? nullptr : d_gate, true, rows, dim, q.ld_d_gate))
    return ADAPT_ERR_INVALID_ARG;
  q.stats_in = stats; q.d_y = d_y; q.d_normed = d_normed; q.d_block = d_block; q.d_residual = d_residual; q.d_gate = d_gate;
  q.d_weight_after = d_weight_after; q.d_weight_before = d_weight_before;
  const int64_t ctas = norm_ctas(rows, dim);
  NormColumns sum = {};
  sum.out[0] = q.shared ? static_cast<float*>(d_gate) : nullptr;
  sum.out[1] = d_weight_after; sum.out[2] = d_weight_before;
  sum.ctas = static_cast<int>(ctas); sum.dim = q.dim;
  const bool sums = sum.out[0] || sum.out[1] || sum.out[2];
  if (sums) {
    if (!workspace || misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    if (workspace_bytes < adapt_block_norm_workspace_bytes(rows, dim)) return ADAPT_ERR_WORKSPACE;
    q.partial = static_cast<float*>(workspace);
    sum.partial = q.partial;
  }
  int rc = ADAPT_OK;
  {
    LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM_BACKWARD, stream);
    const unsigned grid = static_cast<unsigned>(ctas);
    if (dim <= kNormMaxRow) {
      const int threads = norm_threads(dim);
      const NormPlan plan(q, e, norm_per_sm(dim), {{block, q.ld_block}, {residual, q.ld_residual}, {q.shared ? nullptr : gate, q.ld_gate}, {d_y, q.ld_d_y},
                          {d_normed, q.ld_d_normed}}, {{d_block, q.ld_d_block}, {d_residual, q.ld_d_residual}, {q.shared ? nullptr : d_gate, q.ld_d_gate}});
      with_type(dtype, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto n, auto s) {
          constexpr int N = decltype(n)::value;
          constexpr bool S = decltype(s)::value;
          if (q.shared) rc = norm_launch<norm_row_backward_kernel<T, N, S, true>>(grid, threads, plan.smem, stream, q, plan.ring);
          else rc = norm_launch<norm_row_backward_kernel<T, N, S, false>>(grid, threads, plan.smem, stream, q, plan.ring);
        };
        auto staged = [&](auto n) { plan.staged ? go(n, std::true_type{}) : go(n, std::false_type{}); };
        if (norm_elems(dim) == 8) staged(std::integral_constant<int, 8>{}); else staged(std::integral_constant<int, 16>{});
      });
    } else {
      with_type(dtype, [&](auto t) {
        const auto kernel = norm_any_backward_kernel<decltype(t)>;
        const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ADAPT_NORM_MAX_DIM * 4);
        if (err != cudaSuccess) rc = cuda_fail(err, "block norm, backward");
        else kernel<<<grid, kNormThreads, q.dim * 4, stream>>>(q);
      });
    }
    if (rc != ADAPT_OK) return rc;
    ADAPT_LAUNCH_OK("block norm, backward");
  }
  if (sums) {
    LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM_BACKWARD, stream);
    norm_columns_kernel<<<dim3(static_cast<unsigned>((q.dim + 31) / 32), 3), 32 * kNormColumnWarps, 0, stream>>>(sum);
    ADAPT_LAUNCH_OK("block norm, sums over rows");
  }
  return ADAPT_OK;
}

}  // extern "C"
