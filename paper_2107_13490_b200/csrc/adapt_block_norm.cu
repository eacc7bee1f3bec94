// C-ABI entry points of the norms around a block.  Declarations and argument contracts live in adapt.h.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "k_block_norm.cuh"
#include "training_host.cuh"

using namespace adapt;

static_assert(ADAPT_NORM_NONE == kNormNone && ADAPT_NORM_RMS == kNormRms && ADAPT_NORM_LAYER == kNormLayer,
              "the kernels use the constants of the C interface");

namespace {

// CTAs of a backward pass at most, each with sums of its own over its rows.
constexpr int kNormMaxCtas = 148 * 4;

int64_t norm_ctas(int64_t rows) { return std::min<int64_t>(rows, kNormMaxCtas); }

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
  const int smem = q.dim * 4;
  int rc = ADAPT_OK;
  LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM, stream);
  with_type(dtype, [&](auto t) {
    const auto kernel = norm_any_kernel<decltype(t)>;
    if (smem > 48 * 1024) {
      const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ADAPT_NORM_MAX_DIM * 4);
      if (err != cudaSuccess) { rc = cuda_fail(err, "block norm"); return; }
    }
    kernel<<<static_cast<unsigned>(rows), kNormThreads, smem, stream>>>(q);
  });
  if (rc != ADAPT_OK) return rc;
  ADAPT_LAUNCH_OK("block norm");
  return ADAPT_OK;
}

size_t adapt_block_norm_workspace_bytes(int64_t rows, int64_t dim) {
  if (rows < 1 || rows > 0x7FFFFFFF || dim < 1 || dim > ADAPT_NORM_MAX_DIM) return 0;
  return 3 * sizeof(float) * static_cast<size_t>(norm_ctas(rows)) * dim;
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
  const int64_t ctas = norm_ctas(rows);
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
  const int smem = q.dim * 4;
  int rc = ADAPT_OK;
  {
    LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM_BACKWARD, stream);
    with_type(dtype, [&](auto t) {
      const auto kernel = norm_any_backward_kernel<decltype(t)>;
      if (smem > 48 * 1024) {
        const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ADAPT_NORM_MAX_DIM * 4);
        if (err != cudaSuccess) { rc = cuda_fail(err, "block norm, backward"); return; }
      }
      kernel<<<static_cast<unsigned>(ctas), kNormThreads, smem, stream>>>(q);
    });
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
