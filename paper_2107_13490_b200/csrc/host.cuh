// Host side that the library's translation units share: launch counting and timing, error
// text, per-device caches.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstdio>
#include <mutex>
#include <vector>

#include "../../include/adapt.h"

namespace adapt {

inline std::mutex g_mutex;                     // serialises calls that touch library-owned state
inline std::atomic<uint64_t> g_launches{0};
inline thread_local char g_last_error[512] = "";   // per calling thread

// Optional per-kernel device timing: events around each launch, on its stream.
struct TimedLaunch { int kind; cudaEvent_t start, stop; };
inline std::atomic<bool> g_timing{false};
inline std::mutex g_timing_mutex;
inline std::vector<TimedLaunch> g_pending;
inline std::vector<cudaEvent_t> g_event_pool;
inline double g_kind_ms[ADAPT_KERNEL_KINDS] = {0};
inline uint64_t g_kind_launches[ADAPT_KERNEL_KINDS] = {0};

inline cudaEvent_t pooled_event() {
  if (!g_event_pool.empty()) { cudaEvent_t e = g_event_pool.back(); g_event_pool.pop_back(); return e; }
  cudaEvent_t e = nullptr;
  cudaEventCreate(&e);
  return e;
}

// Brackets one kernel launch; counts it, and times it when timing is on.
struct LaunchScope {
  int kind; cudaStream_t stream; cudaEvent_t start = nullptr;
  LaunchScope(int k, cudaStream_t s) : kind(k), stream(s) {
    if (g_timing.load()) {
      std::lock_guard<std::mutex> l(g_timing_mutex);
      start = pooled_event();
      if (start) cudaEventRecord(start, stream);
    }
  }
  ~LaunchScope() {
    ++g_launches;
    if (start) {
      std::lock_guard<std::mutex> l(g_timing_mutex);
      cudaEvent_t stop = pooled_event();
      if (stop) { cudaEventRecord(stop, stream); g_pending.push_back({kind, start, stop}); }
    }
  }
};

inline int cuda_fail(cudaError_t e, const char* what) {
  std::snprintf(g_last_error, sizeof(g_last_error), "%s: %s", what, cudaGetErrorString(e));
  return ADAPT_ERR_CUDA;
}
#define ADAPT_CUDA(call)                                     \
  do {                                                       \
    cudaError_t e_ = (call);                                 \
    if (e_ != cudaSuccess) return cuda_fail(e_, #call);      \
  } while (0)

// after a kernel launch: report which launch was refused
#define ADAPT_LAUNCH_OK(what)                                \
  do {                                                       \
    cudaError_t e_ = cudaGetLastError();                     \
    if (e_ != cudaSuccess) return cuda_fail(e_, what);       \
  } while (0)

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// ---- per-device caches --------------------------------------------------------

constexpr int kMaxDevices = 64;
constexpr int kRingSlots = 4;

struct PinnedSlot {
  void* host = nullptr;
  size_t bytes = 0;
  cudaEvent_t done = nullptr;
};

struct DeviceCache {
  bool props_ready = false;
  int sm_count = 0;
  int max_smem_optin = 0;
  void* workspace = nullptr;   size_t workspace_bytes = 0;
  void* stage_in = nullptr;    size_t stage_in_bytes = 0;    // host-form calls: inputs
  void* stage_out = nullptr;   size_t stage_out_bytes = 0;   // host-form calls: outputs
  void* batch_tab = nullptr;   size_t batch_tab_bytes = 0;   // batched quantize: layer table
  std::vector<unsigned char> batch_tab_image;   // host copy of what batch_tab holds (empty: unknown)
  cudaStream_t batch_tab_stream = nullptr;      // the stream that uploaded it
  void* stage_codes = nullptr; size_t stage_codes_bytes = 0; // host-form calls: codes
  void* div_buf = nullptr;     size_t div_buf_bytes = 0;     // gradient diversity: tables + sums
  void* scan_buf = nullptr;    size_t scan_buf_bytes = 0;    // gated scan: scratch of calls without their own
  PinnedSlot ring[kRingSlots];
  int ring_next = 0;
  cudaStream_t copy_stream = nullptr;   // host-form calls: downloads that overlap the kernels
  cudaEvent_t slice_done[2] = {nullptr, nullptr};
  cudaEvent_t copies_done = nullptr;
  cudaStream_t side_stream = nullptr;   // search: the direct kernel runs beside the keyed kernels
  cudaEvent_t side_fork = nullptr, side_join = nullptr;
};

inline DeviceCache g_cache[kMaxDevices];

inline int current_cache(DeviceCache** out) {
  int dev = 0;
  ADAPT_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) {
    std::snprintf(g_last_error, sizeof(g_last_error), "device index %d not supported", dev);
    return ADAPT_ERR_CUDA;
  }
  DeviceCache& c = g_cache[dev];
  if (!c.props_ready) {
    ADAPT_CUDA(cudaDeviceGetAttribute(&c.sm_count, cudaDevAttrMultiProcessorCount, dev));
    ADAPT_CUDA(cudaDeviceGetAttribute(&c.max_smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev));
    c.props_ready = true;
  }
  *out = &c;
  return ADAPT_OK;
}

inline int grow_device(void** ptr, size_t* have, size_t need) {
  if (*have >= need) return ADAPT_OK;
  if (*ptr) { ADAPT_CUDA(cudaFree(*ptr)); *ptr = nullptr; *have = 0; }
  ADAPT_CUDA(cudaMalloc(ptr, need));
  *have = need;
  return ADAPT_OK;
}

// A pinned host slot whose previous upload has finished.
inline int acquire_slot(DeviceCache& c, size_t bytes, PinnedSlot** out) {
  PinnedSlot& s = c.ring[c.ring_next];
  c.ring_next = (c.ring_next + 1) % kRingSlots;
  if (!s.done) ADAPT_CUDA(cudaEventCreateWithFlags(&s.done, cudaEventDisableTiming));
  ADAPT_CUDA(cudaEventSynchronize(s.done));
  if (s.bytes < bytes) {
    if (s.host) { ADAPT_CUDA(cudaFreeHost(s.host)); s.host = nullptr; s.bytes = 0; }
    size_t want = align_up(std::max<size_t>(bytes, 16384), 4096);
    ADAPT_CUDA(cudaMallocHost(&s.host, want));
    s.bytes = want;
  }
  *out = &s;
  return ADAPT_OK;
}

}  // namespace adapt
