// C-ABI entry point of the gated recurrence.  Its declaration and argument contract live in adapt.h.
#include "scan_host.cuh"

using namespace adapt;

namespace {

// Short sequences take a thread for every four channels instead of tiles, which would be mostly empty.
// Measured on bf16, us, serial against tiles: 256 x 16 x 4096 36 / 109, 256 x 32 x 4096 68 / 108,
// 64 x 16 x 4096 12 / 29, 64 x 32 x 4096 31 / 29, 8 x 16 x 1024 8 / 8, 8 x 32 x 1024 17 / 8.
bool scan_serial(const ScanParams& q) {
  return q.steps <= 16 || (q.steps <= 32 && q.batch * q.channels >= (1 << 19));
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
  (void)workspace; (void)workspace_bytes;   // not needed: the tiles meet in shared memory
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

}  // extern "C"
