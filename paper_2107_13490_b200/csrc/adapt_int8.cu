// C-ABI entry points of the 8-bit codes and their product.  Declarations and argument contracts live in adapt.h.
#include <algorithm>
#include <cstdint>

#include "k_int8.cuh"
#include "training_host.cuh"

using namespace adapt;

namespace {

bool in_int(int64_t v, int64_t least) { return v >= least && v <= 0x7FFFFFFF; }

int run_rows(const RowsParams& q, int dtype, cudaStream_t stream) {
  LaunchScope ls(ADAPT_KERNEL_INT8_ROWS, stream);
  with_type(dtype, [&](auto t) { int8_rows_kernel<decltype(t)><<<static_cast<unsigned>(q.rows), kRowsThreads, 0, stream>>>(q); });
  ADAPT_LAUNCH_OK("rows to 8-bit codes");
  return ADAPT_OK;
}

// Codes (rows of 16-byte multiples) and scales of activations that are quantised within a product.
struct LinearLayout {
  size_t codes = 0, scales = 0, bytes = 0;
  long long ld = 0;
  LinearLayout(int64_t rows, int64_t k, int x_dtype) {
    if (x_dtype == ADAPT_DTYPE_I8) return;
    ld = (k + 15) / 16 * 16;
    scales = align_up(static_cast<size_t>(rows) * ld, 256);
    bytes = align_up(scales + 4 * static_cast<size_t>(rows), 256);
  }
};

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

size_t adapt_int8_linear_workspace_bytes(int64_t rows, int64_t n, int64_t k, int64_t ldw, int x_dtype) {
  (void)ldw;
  if (!in_int(rows, 1) || !in_int(n, 1) || k < 0 || k > ADAPT_INT8_MAX_K || (x_dtype != ADAPT_DTYPE_I8 && !elem_bytes(x_dtype))) return 0;
  return LinearLayout(rows, k, x_dtype).bytes;
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
  const LinearLayout lay(rows, k, x_dtype);
  if (lay.bytes) {
    if (!workspace || misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    if (workspace_bytes < lay.bytes) return ADAPT_ERR_WORKSPACE;
  }
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  LinearParams q = {};
  q.w = weight; q.w_scales = weight_scales; q.bias = bias; q.y = y; q.ldw = ldw; q.ldy = ldy;
  q.rows = static_cast<int>(rows); q.n = static_cast<int>(n); q.k = static_cast<int>(k);
  q.w_one = weight_scale_count == 1;
  if (coded) {
    q.x = static_cast<const signed char*>(x); q.x_scales = x_scales; q.ldx = ldx; q.x_one = x_scale_count == 1;
  } else {
    RowsParams r = {};
    r.x = x; r.ldx = ldx; r.ld_codes = lay.ld; r.rows = q.rows; r.cols = q.k;
    r.codes = static_cast<signed char*>(workspace) + lay.codes;
    r.scales = reinterpret_cast<float*>(static_cast<char*>(workspace) + lay.scales);
    const int rc = run_rows(r, x_dtype, stream);
    if (rc != ADAPT_OK) return rc;
    q.x = r.codes; q.x_scales = r.scales; q.ldx = lay.ld;
  }
  const int64_t across = (n + kTile - 1) / kTile, down = (rows + kTile - 1) / kTile;
  if (down > 65535) return ADAPT_ERR_INVALID_ARG;
  LaunchScope ls(ADAPT_KERNEL_INT8_LINEAR, stream);
  with_type(dtype, [&](auto t) {
    int8_any_kernel<decltype(t)><<<dim3(static_cast<unsigned>(across), static_cast<unsigned>(down)), 256, 0, stream>>>(q);
  });
  ADAPT_LAUNCH_OK("8-bit product");
  return ADAPT_OK;
}

}  // extern "C"
