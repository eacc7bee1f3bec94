// C-ABI entry points of the training-step operators: dropout, token log probabilities, gated
// recurrence.  Declarations and argument contracts live in adapt.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <vector>

#include "../../include/adapt.h"
#include "dropout_pieces.h"
#include "host.cuh"
#include "k_dropout.cuh"
#include "k_logprobs.cuh"
#include "k_scan.cuh"

namespace {

using namespace adapt;

static_assert(ADAPT_SCAN_TILE == kScanTile && ADAPT_MAX_TOP == kMaxTop && ADAPT_GATE_SIGMOID == kGateSigmoid &&
              ADAPT_GATE_VALUE == kGateValue, "the kernels use the constants of the C interface");

// Bytes of an element, 0 for an unknown type.
int elem_bytes(int dtype) {
  return dtype == ADAPT_DTYPE_F32 ? 4 : (dtype == ADAPT_DTYPE_F16 || dtype == ADAPT_DTYPE_BF16) ? 2 : 0;
}

bool misaligned(const void* p, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(bytes - 1)) != 0;
}

// Calls f(T{}) with the element type.
template <typename F>
void with_type(int dtype, F f) {
  if (dtype == ADAPT_DTYPE_F32) f(float{});
  else if (dtype == ADAPT_DTYPE_F16) f(__half{});
  else f(__nv_bfloat16{});
}

}  // namespace

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
  const int unit = 16 / e;
  DropoutParams q = {};
  q.cols = cols; q.ldx = ldx; q.ldr = ldr; q.ldy = ldy;
  q.base = seed ^ 0xA54FF53A5F1D36F1ull ^ ((static_cast<uint64_t>(static_cast<int64_t>(layer)) + 1ull) * 0x9E3779B97F4A7C15ull);
  const double threshold = std::nearbyint(p * 4294967296.0);
  q.none = threshold >= 4294967296.0;
  q.threshold = q.none ? 0u : static_cast<unsigned>(threshold);
  q.scale = p < 1.0 ? static_cast<float>(1.0 / (1.0 - p)) : 0.0f;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  const DropoutPieces pieces(rows, cols, e);
  return pieces.each([&](int64_t row, int64_t col, int64_t n_rows, int64_t n_cols) -> int {
    q.x = static_cast<const char*>(x) + (row * ldx + col) * e;
    q.y = static_cast<char*>(y) + (row * ldy + col) * e;
    q.r = residual ? static_cast<const char*>(residual) + (row * ldr + col) * e : nullptr;
    q.x_end = static_cast<const char*>(q.x) + ((n_rows - 1) * ldx + n_cols) * e;
    q.r_end = residual ? static_cast<const char*>(q.r) + ((n_rows - 1) * ldr + n_cols) * e : nullptr;
    q.index_base = static_cast<long long>(index_base) + row * cols + col;
    if (n_rows == 1) {
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
    const unsigned tile = kDropoutThreads * (vec ? kDropoutUnroll : kShiftUnroll);
    const unsigned grid = (q.chunks + tile - 1) / tile;
    LaunchScope ls(ADAPT_KERNEL_DROPOUT, stream);
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      auto go = [&](auto kernel) { kernel<<<grid, kDropoutThreads, 0, stream>>>(q); };
      if (n_rows == 1) {
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

namespace {

// Checks what forward and backward share.  Fills sizes; strides are set by the caller.
bool scan_shape(ScanParams& q, int64_t batch, int64_t steps, int64_t channels, int group, int dtype, int mode) {
  if (!elem_bytes(dtype) || (mode != ADAPT_GATE_SIGMOID && mode != ADAPT_GATE_VALUE)) return false;
  if (batch < 0 || steps < 0 || channels < 0) return false;
  if (steps > 0x7FFFE000 || channels > 0x7FFFFFFF || batch > 0x7FFFFFFF) return false;
  if (batch > 0 && channels > 0 && batch > (1ll << 27) / ((channels + kScanChannels - 1) / kScanChannels)) return false;
  // a gate of its own, or shared by a power of two of channels up to 64, or by a multiple of 64
  const bool ok = group >= 1 && (group <= 64 ? (group & (group - 1)) == 0 : group % 64 == 0);
  if (!ok || channels % group != 0) return false;
  q.batch = batch; q.steps = steps; q.channels = channels; q.group = group;
  return true;
}

// Stride pair: given, or that of a contiguous [batch][steps][width] array.
void stride_pair(const int64_t* given, int k, int64_t steps, int64_t width, long long& b, long long& t) {
  b = given ? given[2 * k] : steps * width;
  t = given ? given[2 * k + 1] : width;
}

// Rows that are written must not overlap.
bool out_strides_ok(long long b, long long t, const ScanParams& q, int64_t width) {
  if (b < 0 || t < 0) return false;
  if (q.steps > 1 && t < width) return false;
  if (q.batch > 1 && b < width) return false;
  if (q.steps > 1 && q.batch > 1 && b < t * q.steps && t < b * q.batch) return false;
  return true;
}

size_t scan_workspace(const ScanParams& q, bool backward) {
  if (!backward || q.group <= kScanChannels) return 0;
  return sizeof(float) * static_cast<size_t>(q.batch) * q.steps * (q.channels / kScanChannels);
}

// Whether `unit` channels can be moved at a time.
bool scan_fits(const ScanParams& q, int elem, int unit, std::initializer_list<const void*> ptrs, std::initializer_list<long long> strides) {
  if (q.channels % unit) return false;
  for (const void* p : ptrs) if (misaligned(p, unit * elem)) return false;
  for (long long s : strides) if (s % unit) return false;
  return true;
}

// How many channels a tile kernel moves at a time: those of 16 bytes, two, or one.
int scan_move(const ScanParams& q, int elem, std::initializer_list<const void*> ptrs, std::initializer_list<long long> strides) {
  return scan_fits(q, elem, 16 / elem, ptrs, strides) ? kMoveVec : scan_fits(q, elem, 2, ptrs, strides) ? kMovePair : kMoveOne;
}

// Whether shared gates can be copied by the 4-byte words that hold them, none of which leaves its row.
bool scan_gate_words(const ScanParams& q, int elem) {
  return elem == 4 || (q.channels / q.group % 2 == 0 && !misaligned(q.gate, 4) && q.gb % 2 == 0 && q.gt % 2 == 0);
}

// CTAs of a tile kernel that the device holds at once, by kernel (first use: attributes and occupancy).
struct ScanSlots { const void* kernel; int device, slots; };
std::vector<ScanSlots> g_scan_slots;   // under g_mutex

int scan_slots(DeviceCache& dc, const void* kernel, size_t smem, int channels, int* out) {
  int dev = 0;
  ADAPT_CUDA(cudaGetDevice(&dev));
  for (const ScanSlots& s : g_scan_slots)
    if (s.kernel == kernel && s.device == dev) { *out = s.slots; return ADAPT_OK; }
  ADAPT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  static_cast<int>(smem + scan_totals_bytes(kScanMaxCluster, channels))));
  ADAPT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  int per_sm = 0;
  ADAPT_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kScanThreads, smem + scan_totals_bytes(4, channels)));
  const int slots = std::max(1, per_sm) * dc.sm_count;
  g_scan_slots.push_back({kernel, dev, slots});
  *out = slots;
  return ADAPT_OK;
}

typedef void (*ScanKernel)(ScanParams);

// The tile kernels of one type, mode and alignment, for 64, 32 and 16 channels a CTA, and the number of
// CTAs to a chain, by the estimated time: waves of CTAs x rounds of a chain x the time of a round, in units
// of a round without exchange (1.4 to 2.5 us).  An exchange costs 1.35 + 0.03 K of them, narrower tiles
// 10 % a halving.  Measured forward, us: 8 x 4096 x 2048 bf16 (256 chains of 64) 91 with one CTA to a chain,
// 119 with two; 1 x 65536 x 1024 bf16 (16 chains of 64, 32 of 32) 1070 with one, 234 with 16, 134 with 32
// channels and 8 CTAs; over twelve shapes both ways the choice is within 3 % of the best on the mean.
int launch_scan(DeviceCache& dc, const ScanKernel (&kernels)[3], int tensors, int elem, const ScanParams& q, cudaStream_t stream) {
  const size_t stages = kScanStages * scan_stage_bytes(tensors, elem);
  int width = 0, cluster = 1;
  double least = 1e300;
  for (int i = 0; i < 3; ++i) {
    const int channels = kScanChannels >> i;
    if (i && q.group > channels) break;   // a shared gate stays in one CTA
    int slots = 0;
    const int rc = scan_slots(dc, reinterpret_cast<const void*>(kernels[i]), stages, channels, &slots);
    if (rc != ADAPT_OK) return rc;
    const long long chains = q.batch * ((q.channels + channels - 1) / channels);
    const long long tiles = (q.steps * channels + kTileElements - 1) / kTileElements;
    for (int k = 1; k <= kScanMaxCluster; k *= 2) {
      if (k > 1 && k / 2 >= tiles) break;
      const double full = static_cast<double>(chains * k) / slots, waves = full <= 1.0 ? 1.0 : full + 0.5;
      const double rounds = static_cast<double>((tiles + k - 1) / k);
      const double cost = waves * rounds * (k > 1 ? 1.35 + 0.03 * k : 1.0) * (1.0 + 0.1 * i);
      if (cost < least) { least = cost; width = i; cluster = k; }
    }
  }
  const int channels = kScanChannels >> width;
  const long long chains = q.batch * ((q.channels + channels - 1) / channels);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(chains * cluster));
  cfg.blockDim = dim3(kScanThreads);
  cfg.dynamicSmemBytes = stages + scan_totals_bytes(cluster, channels);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADAPT_CUDA(cudaLaunchKernelEx(&cfg, kernels[width], q));
  return ADAPT_OK;
}

#define ADAPT_SCAN_WIDTHS(name, T, mode, move) {name<T, mode, move, 32>, name<T, mode, move, 16>, name<T, mode, move, 8>}
// Launches the kernels `name` of a type for the call's mode and alignment.
#define ADAPT_SCAN_LAUNCH(name, T, tensors)                                                            \
  {                                                                                                    \
    static const ScanKernel kernels[2][3][3] = {                                                       \
        {ADAPT_SCAN_WIDTHS(name, T, 0, 0), ADAPT_SCAN_WIDTHS(name, T, 0, 1), ADAPT_SCAN_WIDTHS(name, T, 0, 2)},  \
        {ADAPT_SCAN_WIDTHS(name, T, 1, 0), ADAPT_SCAN_WIDTHS(name, T, 1, 1), ADAPT_SCAN_WIDTHS(name, T, 1, 2)}}; \
    rc = launch_scan(*dc, kernels[mode][move], tensors, e, q, stream);                                 \
  }
// Short sequences take a thread for every four channels instead of tiles, which would be mostly empty.
// Measured on bf16, us, serial against tiles: 256 x 16 x 4096 36 / 109, 256 x 32 x 4096 68 / 108,
// 64 x 16 x 4096 12 / 29, 64 x 32 x 4096 31 / 29, 8 x 16 x 1024 8 / 8, 8 x 32 x 1024 17 / 8.
bool scan_serial(const ScanParams& q) {
  return q.steps <= 16 || (q.steps <= 32 && q.batch * q.channels >= (1 << 19));
}

// The caller's workspace, or the library's (grown on demand).
int scan_scratch(DeviceCache& dc, void* workspace, size_t have, size_t need, char** out) {
  *out = nullptr;
  if (need == 0) return ADAPT_OK;
  if (workspace) {
    if (have < need) return ADAPT_ERR_WORKSPACE;
    if (misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    *out = static_cast<char*>(workspace);
    return ADAPT_OK;
  }
  const int rc = grow_device(&dc.scan_buf, &dc.scan_buf_bytes, align_up(need, 4096));
  *out = static_cast<char*>(dc.scan_buf);
  return rc;
}

}  // namespace

extern "C" {

size_t adapt_gated_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t channels, int gate_group,
                                        int dtype, int backward) {
  ScanParams q = {};
  if (!scan_shape(q, batch, steps, channels, gate_group, dtype, ADAPT_GATE_SIGMOID)) return 0;
  return scan_workspace(q, backward != 0);
}

int adapt_gated_scan(const void* x, const void* gate, const float* h0, const int32_t* lengths,
                     const uint8_t* reset, int64_t batch, int64_t steps, int64_t channels,
                     int gate_group, int dtype, int mode, const int64_t* strides, void* y,
                     float* h_last, float* carry_out, void* workspace, size_t workspace_bytes,
                     void* stream_handle) {
  ScanParams q = {};
  if (!scan_shape(q, batch, steps, channels, gate_group, dtype, mode)) return ADAPT_ERR_INVALID_ARG;
  if (batch == 0 || channels == 0) return ADAPT_OK;
  const int e = elem_bytes(dtype);
  if (steps > 0 && (!x || !gate || !y)) return ADAPT_ERR_INVALID_ARG;
  if (misaligned(x, e) || misaligned(gate, e) || misaligned(y, e) || misaligned(h0, 4) || misaligned(h_last, 4) ||
      misaligned(carry_out, 4) || misaligned(lengths, 4))
    return ADAPT_ERR_INVALID_ARG;
  stride_pair(strides, 0, steps, channels, q.xb, q.xt);
  stride_pair(strides, 1, steps, channels / gate_group, q.gb, q.gt);
  stride_pair(strides, 2, steps, channels, q.yb, q.yt);
  if (q.xb < 0 || q.xt < 0 || q.gb < 0 || q.gt < 0 || !out_strides_ok(q.yb, q.yt, q, channels)) return ADAPT_ERR_INVALID_ARG;
  q.x = x; q.gate = gate; q.h0 = h0; q.lengths = lengths; q.reset = reset; q.y = y; q.h_last = h_last; q.carry = carry_out;
  (void)workspace; (void)workspace_bytes;   // the tiles meet in shared memory
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceCache* dc = nullptr;
  int rc = current_cache(&dc);
  if (rc != ADAPT_OK) return rc;
  LaunchScope ls(ADAPT_KERNEL_SCAN, stream);
  const bool own = gate_group == 1;   // a gate for every channel
  const std::initializer_list<const void*> ptrs = {x, y, own ? gate : nullptr};
  const std::initializer_list<long long> lines = {q.xb, q.xt, q.yb, q.yt, own ? q.gb : 0, own ? q.gt : 0};
  if (scan_serial(q)) {
    const bool wide = scan_fits(q, e, 4, ptrs, lines) && (own || gate_group % 4 == 0);
    const unsigned grid = static_cast<unsigned>((batch * channels / (wide ? 4 : 1) + 127) / 128);
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      auto go = [&](auto kernel) { kernel<<<grid, 128, 0, stream>>>(q); };
      if (mode == ADAPT_GATE_SIGMOID) wide ? go(scan_serial_kernel<T, kGateSigmoid, 4>) : go(scan_serial_kernel<T, kGateSigmoid, 1>);
      else wide ? go(scan_serial_kernel<T, kGateValue, 4>) : go(scan_serial_kernel<T, kGateValue, 1>);
    });
  } else {
    const int move = scan_move(q, e, ptrs, lines);
    q.gate_words = scan_gate_words(q, e);
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      ADAPT_SCAN_LAUNCH(scan_kernel, T, 2);
    });
    if (rc != ADAPT_OK) return rc;
  }
  ADAPT_LAUNCH_OK("gated scan");
  return ADAPT_OK;
}

int adapt_gated_scan_backward(const void* x, const void* gate, const void* dy, const float* carry,
                              const float* dh_last, const int32_t* lengths, const uint8_t* reset,
                              int64_t batch, int64_t steps, int64_t channels, int gate_group,
                              int dtype, int mode, const int64_t* strides, void* dx, void* dgate,
                              float* dh0, void* workspace, size_t workspace_bytes,
                              void* stream_handle) {
  ScanParams q = {};
  if (!scan_shape(q, batch, steps, channels, gate_group, dtype, mode)) return ADAPT_ERR_INVALID_ARG;
  if (batch == 0 || channels == 0) return ADAPT_OK;
  const int e = elem_bytes(dtype);
  if (steps > 0 && (!x || !gate || !dy || !carry || !dx || !dgate)) return ADAPT_ERR_INVALID_ARG;
  if (misaligned(x, e) || misaligned(gate, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(dgate, e) ||
      misaligned(carry, 4) || misaligned(dh_last, 4) || misaligned(dh0, 4) || misaligned(lengths, 4))
    return ADAPT_ERR_INVALID_ARG;
  stride_pair(strides, 0, steps, channels, q.xb, q.xt);
  stride_pair(strides, 1, steps, channels / gate_group, q.gb, q.gt);
  stride_pair(strides, 2, steps, channels, q.yb, q.yt);
  stride_pair(strides, 3, steps, channels, q.dxb, q.dxt);
  stride_pair(strides, 4, steps, channels / gate_group, q.dgb, q.dgt);
  if (q.xb < 0 || q.xt < 0 || q.gb < 0 || q.gt < 0 || q.yb < 0 || q.yt < 0 ||
      !out_strides_ok(q.dxb, q.dxt, q, channels) || !out_strides_ok(q.dgb, q.dgt, q, channels / gate_group))
    return ADAPT_ERR_INVALID_ARG;
  q.x = x; q.gate = gate; q.dy = dy; q.carry = const_cast<float*>(carry); q.dh_last = dh_last;
  q.lengths = lengths; q.reset = reset; q.dx = dx; q.dgate = dgate; q.dh0 = dh0;
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceCache* dc = nullptr;
  int rc = current_cache(&dc);
  if (rc != ADAPT_OK) return rc;
  char* scratch = nullptr;
  rc = scan_scratch(*dc, workspace, workspace_bytes, scan_workspace(q, true), &scratch);
  if (rc != ADAPT_OK) return rc;
  q.partial = reinterpret_cast<float*>(scratch);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  {
    LaunchScope ls(ADAPT_KERNEL_SCAN_BACKWARD, stream);
    const bool own = gate_group == 1;
    const int move = scan_move(q, e, {x, dy, dx, own ? gate : nullptr, own ? dgate : nullptr},
                                  {q.xb, q.xt, q.yb, q.yt, q.dxb, q.dxt, own ? q.gb : 0, own ? q.gt : 0,
                                   own ? q.dgb : 0, own ? q.dgt : 0});
    q.gate_words = scan_gate_words(q, e);
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      ADAPT_SCAN_LAUNCH(scan_backward_kernel, T, 3);
    });
    if (rc != ADAPT_OK) return rc;
    ADAPT_LAUNCH_OK("gated scan, backward");
  }
  if (q.partial && steps > 0) {
    const long long n = batch * steps * (channels / gate_group);
    LaunchScope ls(ADAPT_KERNEL_SCAN_BACKWARD, stream);
    with_type(dtype, [&](auto t) {
      scan_gate_sum_kernel<decltype(t)><<<static_cast<int>(std::min<long long>((n + 255) / 256, 16ll * dc->sm_count)), 256, 0, stream>>>(q);
    });
    ADAPT_LAUNCH_OK("gate gradient sum");
  }
  return ADAPT_OK;
}

}  // extern "C"
