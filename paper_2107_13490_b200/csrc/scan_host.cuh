// Host side that the forward and the backward entry point of the gated recurrence share.
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <vector>

#include "k_scan.cuh"
#include "training_host.cuh"

namespace adapt {

static_assert(ADAPT_SCAN_TILE == kScanTile && ADAPT_GATE_SIGMOID == kGateSigmoid && ADAPT_GATE_VALUE == kGateValue,
              "the kernels use the constants of the C interface");

// Checks what forward and backward share.  Fills sizes; strides are set by the caller.
inline bool scan_shape(ScanParams& q, int64_t batch, int64_t steps, int64_t channels, int group, int dtype, int mode) {
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
inline void stride_pair(const int64_t* given, int k, int64_t steps, int64_t width, long long& b, long long& t) {
  b = given ? given[2 * k] : steps * width;
  t = given ? given[2 * k + 1] : width;
}

// Rows that are written must not overlap.
inline bool out_strides_ok(long long b, long long t, const ScanParams& q, int64_t width) {
  if (b < 0 || t < 0) return false;
  if (q.steps > 1 && t < width) return false;
  if (q.batch > 1 && b < width) return false;
  if (q.steps > 1 && q.batch > 1 && b < t * q.steps && t < b * q.batch) return false;
  return true;
}

inline size_t scan_workspace(const ScanParams& q, bool backward) {
  if (!backward || q.group <= kScanChannels) return 0;
  return sizeof(float) * static_cast<size_t>(q.batch) * q.steps * (q.channels / kScanChannels);
}

// Whether `unit` channels can be moved at a time.
inline bool scan_fits(const ScanParams& q, int elem, int unit, std::initializer_list<const void*> ptrs, std::initializer_list<long long> strides) {
  if (q.channels % unit) return false;
  for (const void* p : ptrs) if (misaligned(p, unit * elem)) return false;
  for (long long s : strides) if (s % unit) return false;
  return true;
}

// How many channels a tile kernel moves at a time: those of 16 bytes, two, or one.
inline int scan_move(const ScanParams& q, int elem, std::initializer_list<const void*> ptrs, std::initializer_list<long long> strides) {
  return scan_fits(q, elem, 16 / elem, ptrs, strides) ? kMoveVec : scan_fits(q, elem, 2, ptrs, strides) ? kMovePair : kMoveOne;
}

// Whether shared gates can be copied by the 4-byte words that hold them, none of which leaves its row.
inline bool scan_gate_words(const ScanParams& q, int elem) {
  return elem == 4 || (q.channels / q.group % 2 == 0 && !misaligned(q.gate, 4) && q.gb % 2 == 0 && q.gt % 2 == 0);
}

// CTAs of a tile kernel that the device holds at once, by kernel (first use: attributes and occupancy).
struct ScanSlots { const void* kernel; int device, slots; };
inline std::vector<ScanSlots> g_scan_slots;   // under g_mutex

inline int scan_slots(DeviceCache& dc, const void* kernel, size_t smem, int channels, int* out) {
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
inline int launch_scan(DeviceCache& dc, const ScanKernel (&kernels)[3], int tensors, int elem, const ScanParams& q, cudaStream_t stream) {
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

}  // namespace adapt
