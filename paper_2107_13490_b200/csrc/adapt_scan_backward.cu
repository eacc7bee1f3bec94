// C-ABI entry point of the gated recurrence's backward pass (a unit of its own: its kernels take the longest to
// compile).  Its declaration and argument contract live in adapt.h.
#include "scan_host.cuh"

using namespace adapt;

namespace {

// The caller's workspace, or the library's (grown on demand: a graph would keep an address that a later call frees).
int scan_scratch(DeviceCache& dc, void* workspace, size_t have, size_t need, cudaStream_t stream, char** out) {
  *out = nullptr;
  if (need == 0) return ADAPT_OK;
  if (workspace) {
    if (have < need) return ADAPT_ERR_WORKSPACE;
    if (misaligned(workspace, 256)) return ADAPT_ERR_INVALID_ARG;
    *out = static_cast<char*>(workspace);
    return ADAPT_OK;
  }
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  ADAPT_CUDA(cudaStreamIsCapturing(stream, &capturing));
  if (capturing != cudaStreamCaptureStatusNone) {
    std::snprintf(g_last_error, sizeof(g_last_error),
                  "adapt_gated_scan_backward: the stream is being captured and the call has no workspace of its own");
    return ADAPT_ERR_INVALID_ARG;
  }
  const int rc = grow_device(&dc.scan_buf, &dc.scan_buf_bytes, align_up(need, 4096));
  *out = static_cast<char*>(dc.scan_buf);
  return rc;
}

}  // namespace

extern "C" {

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
  cudaStream_t stream = static_cast<cudaStream_t>(stream_handle);
  rc = scan_scratch(*dc, workspace, workspace_bytes, scan_workspace(q, true), stream, &scratch);
  if (rc != ADAPT_OK) return rc;
  q.partial = reinterpret_cast<float*>(scratch);
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
