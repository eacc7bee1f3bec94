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

// (norm_room is largest one below the limit, where it is odd)
static_assert(norm_room(ADAPT_NORM_MAX_DIM) <= kNormElems * kNormBackwardThreads * kNormMaxParts &&
                  norm_room(ADAPT_NORM_MAX_DIM - 1) <= kNormElems * kNormBackwardThreads * kNormMaxParts,
              "a cluster holds the longest row, and the longest odd one");

// CTAs (or clusters) of a backward pass at most, each with sums of its own over its rows.
int64_t norm_ctas(int64_t rows, int64_t dim) {
  const NormShape shape = norm_backward(dim);
  return std::min<int64_t>(rows, kSms * shape.per_sm / shape.parts);
}
// CTAs of the kernel for any layout, which takes a whole row whatever its length: as many on an SM as have the shared memory for one, up
// to 4, or as many as the kernels above take of short rows.  (us by 1, 2, 4 and 8 on an SM, both norms and a gate, bf16: 16384 x 1024 886,
// 470, 284, 271; 16384 x 4096 3828, 2106, 1140, 1189; 4096 x 16384 4397, 2730, 2173 by 3; 65536 x 384 561 by 8, 461 by 16)
int64_t norm_any_ctas(int64_t rows, int64_t dim) {
  const int fit = static_cast<int>(220 * 1024 / (dim * 4 + 1024));
  return std::min<int64_t>(rows, kSms * std::min(fit, std::max(norm_backward(dim).per_sm, 4)));
}
static_assert(220 * 1024 / (ADAPT_NORM_MAX_DIM * 4 + 1024) >= 1, "an SM holds the longest row");
// A multiple of the period, so that a CTA's rows lie alike; the CTAs that are more have no rows, and sums of 0.
int64_t norm_grid(int64_t ctas, int period) { return (ctas + period - 1) / period * period; }

// How the rows come through shared memory, if they do: all tensors have to lie alike to the 16-byte boundary, row by row.
struct NormPlan {
  NormRing ring = {};
  int smem = 0, copy = 0, copies = 0;
  bool used[3];
  int period = 1;   // rows whose numbers differ by a multiple of the period lie alike
  bool staged = true, edges = false;
  NormPlan(const NormParams& q, int e, const NormShape& shape, std::initializer_list<std::pair<const void*, long long>> in,
           std::initializer_list<std::pair<const void*, long long>> out) {
    auto phase = [](const void* p) { return static_cast<unsigned>(reinterpret_cast<uintptr_t>(p) & 15u); };
    auto step = [&](long long ld) { return q.rows == 1 ? 0u : static_cast<unsigned>(ld * e & 15); };
    const unsigned first = phase(q.block), by = step(q.ld_block);
    auto alike = [&](const std::pair<const void*, long long>& p) { return !p.first || (phase(p.first) == first && step(p.second) == by); };
    int i = 0;
    for (const auto& p : in) {
      staged = staged && alike(p);
      ring.place[i++] = p.first ? ring.streams++ : -1;
    }
    for (const auto& p : out) staged = staged && alike(p);
    edges = first != 0 || by != 0 || q.dim * e % 16 != 0;
    for (const void* p : {static_cast<const void*>(q.weight_after), static_cast<const void*>(q.weight_before), q.shared ? q.gate : nullptr})
      edges = edges || misaligned(p, 16);
    while (period * by % 16) period *= 2;
    ring.parts = shape.parts;
    const int width = shape.elems * shape.threads;   // elements of a part
    if (edges && q.dim + 16 / e - 1 > width * shape.parts) staged = false;   // the elements before a boundary take room too
    ring.stage_row = shape.parts > 1 ? width * e : edges ? (q.dim * e + 15 + 15) / 16 * 16 : q.dim * e;
    for (int& p : ring.place) p = p < 0 ? -1 : p * ring.stage_row;
    copy = edges ? width * 4 : 0;
    used[0] = q.after != kNormNone; used[1] = q.before != kNormNone; used[2] = q.shared;
    for (bool u : used) copies += u ? copy : 0;
    staged = staged && (220 * 1024 - copies) / (ring.streams * ring.stage_row) >= shape.rows;
  }
  // Stages and the rest of shared memory for so many CTAs on an SM.
  void fit(int per_sm, int rows) {
    const int stage = ring.streams * ring.stage_row;
    ring.stages = std::min(kNormMaxStages, std::max((200 * 1024 / per_sm - copies) / stage, rows)) / rows * rows;   // whole turns
    smem = ring.stages * stage;
    smem = (smem + 15) / 16 * 16;
    for (int w = 0; w < 3; ++w) {
      ring.weights[w] = used[w] && edges ? smem : -1;
      if (used[w]) smem += copy;
    }
  }
};

// Calls f with what a kernel is made for.
template <typename F>
void with_form(const NormParams& q, bool edges, F f) {
  auto gates = [&](auto e, auto a, auto b) {
    if (!q.gate) f(e, a, b, std::integral_constant<int, kGateNone>{});
    else if (q.shared) f(e, a, b, std::integral_constant<int, kGateForAll>{});
    else if (q.sigmoid) f(e, a, b, std::integral_constant<int, kGateEachSigmoid>{});
    else f(e, a, b, std::integral_constant<int, kGateEach>{});
  };
  auto norms = [&](auto e) {
    if (q.after == kNormNone) gates(e, std::false_type{}, std::true_type{});
    else if (q.before == kNormNone) gates(e, std::true_type{}, std::false_type{});
    else gates(e, std::true_type{}, std::true_type{});
  };
  if (edges) norms(std::true_type{}); else norms(std::false_type{});
}

// What the device says of a kernel, once for each device; it may use all of an SM's shared memory from then on.
template <auto kKernel>
int norm_registers(int* out) {
  static std::atomic<int> known[kMaxDevices];
  int device = 0;
  ADAPT_CUDA(cudaGetDevice(&device));
  std::atomic<int>& slot = known[device % kMaxDevices];
  int n = slot.load();
  if (!n) {
    cudaFuncAttributes a = {};
    ADAPT_CUDA(cudaFuncGetAttributes(&a, kKernel));
    ADAPT_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024));
    slot.store(n = (a.numRegs + 7) / 8 * 8);
  }
  *out = n;
  return ADAPT_OK;
}

// Clusters of a launch that the device holds at once: of 4 and more CTAs not every SM has a place, since a cluster lies within one of
// the device's groups of SMs (33 clusters of 4, 15 of 8).  The answer to the last question of each device is kept.
template <auto kKernel>
int norm_clusters(const cudaLaunchConfig_t& cfg, int* out) {
  static std::atomic<uint64_t> known[kMaxDevices];   // threads (11 bits), shared memory (18), CTAs of a cluster (4), clusters
  int device = 0, n = 0;
  ADAPT_CUDA(cudaGetDevice(&device));
  std::atomic<uint64_t>& slot = known[device % kMaxDevices];
  const uint64_t asked = cfg.blockDim.x | cfg.dynamicSmemBytes << 11 | static_cast<uint64_t>(cfg.attrs[0].val.clusterDim.x) << 29, last = slot.load();
  if (last && (last & ((1ull << 33) - 1)) == asked) {
    n = static_cast<int>(last >> 33);
  } else {
    ADAPT_CUDA(cudaOccupancyMaxActiveClusters(&n, kKernel, &cfg));
    slot.store(asked | static_cast<uint64_t>(n) << 33);
  }
  *out = n;
  return ADAPT_OK;
}

// Launches a kernel on as many CTAs as the device holds at once, and says how many (clusters) that are: a CTA that had to wait
// for another's end would begin its share of the rows then.  (us, 32768 x 4095 fp16 with 152 CTAs backward 1684, with 144 954;
// 2048 x 32768 bf16 with 37 clusters 765, with 33 443)
template <auto kKernel>
int norm_launch(int64_t rows, const NormShape& shape, NormPlan plan, cudaStream_t stream, const NormParams& q, int* groups) {
  int registers = 0;
  int rc = norm_registers<kKernel>(&registers);
  if (rc != ADAPT_OK) return rc;
  int per_sm = std::max(1, std::min(shape.per_sm, 65536 / (registers * shape.threads)));
  plan.fit(per_sm, shape.rows);
  while (per_sm > 1 && per_sm * (plan.smem + 2048) > 228 * 1024) plan.fit(--per_sm, shape.rows);
  int held = kSms * per_sm / shape.parts;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(held * shape.parts));
  cfg.blockDim = dim3(shape.threads);
  cfg.dynamicSmemBytes = plan.smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = shape.parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = shape.parts > 1 ? 1 : 0;
  if (shape.parts > 1) {
    int clusters = 0;
    if ((rc = norm_clusters<kKernel>(cfg, &clusters)) != ADAPT_OK) return rc;
    held = std::min(held, clusters);
  }
  *groups = static_cast<int>(std::min<int64_t>(norm_grid(rows, plan.period), std::max(1, held / plan.period) * plan.period));
  cfg.gridDim = dim3(static_cast<unsigned>(*groups * shape.parts));
  ADAPT_CUDA(cudaLaunchKernelEx(&cfg, kKernel, q, plan.ring));
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
  const bool known = q.before == kNormNone ? !normed : normed != nullptr;   // (a norm whose output is not wanted: its statistics may be)
  if (known && (q.after != kNormNone || q.before != kNormNone)) {
    const NormShape shape = norm_forward(dim);
    const NormPlan plan(q, e, shape, {{block, q.ld_block}, {residual, q.ld_residual}, {q.shared ? nullptr : gate, q.ld_gate},
                        {nullptr, 0}, {nullptr, 0}}, {{y, q.ld_y}, {normed, q.ld_normed}});
    if (plan.staged) {
      int groups = 0;
      with_type(dtype, [&](auto t) {
        using T = decltype(t);
        with_form(q, plan.edges, [&](auto edges, auto after, auto before, auto kind) {
          rc = norm_launch<norm_row_kernel<T, decltype(edges)::value, decltype(after)::value, decltype(before)::value, decltype(kind)::value>>(
              rows, shape, plan, stream, q, &groups);
        });
      });
      return rc;
    }
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
  return 3 * sizeof(float) * static_cast<size_t>(std::max(norm_grid(norm_ctas(rows, dim), 8), norm_any_ctas(rows, dim))) * dim;
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
  if (!d_normed) q.residual = nullptr;   // (only the norm before the next block looks at it; its gradient needs d_y alone)
  NormColumns sum = {};
  sum.out[0] = q.shared ? static_cast<float*>(d_gate) : nullptr;
  sum.out[1] = d_weight_after; sum.out[2] = d_weight_before;
  sum.dim = q.dim;
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
    auto plan_for = [&](const NormShape& shape) {
      return NormPlan(q, e, shape, {{block, q.ld_block}, {q.residual, q.ld_residual},
                      {q.shared ? nullptr : gate, q.ld_gate}, {d_y, q.ld_d_y}, {d_normed, q.ld_d_normed}},
                      {{d_block, q.ld_d_block}, {d_residual, q.ld_d_residual}, {q.shared ? nullptr : d_gate, q.ld_d_gate}});
    };
    NormShape shape = norm_backward(dim);
    NormPlan plan = plan_for(shape);
    if (norm_in_pairs(dim, (q.after != kNormNone) + (d_normed != nullptr))) {
      const NormPlan pairs = plan_for(norm_backward_pairs(dim));
      if (pairs.staged) {   // (there may be no room before a boundary)
        shape = norm_backward_pairs(dim);
        plan = pairs;
      }
    }
    if (plan.staged && (q.after != kNormNone || d_normed)) {
      if (!d_normed) q.before = kNormNone;   // (its gradient is not given)
      with_type(dtype, [&](auto t) {
        using T = decltype(t);
        with_form(q, plan.edges, [&](auto edges, auto after, auto before, auto kind) {
          constexpr bool E = decltype(edges)::value, A = decltype(after)::value, B = decltype(before)::value;
          constexpr int K = decltype(kind)::value;
          rc = shape.rows == 2 ? norm_launch<norm_pair_backward_kernel<T, E, A, B, K>>(rows, shape, plan, stream, q, &sum.ctas)
                               : norm_launch<norm_row_backward_kernel<T, E, A, B, K>>(rows, shape, plan, stream, q, &sum.ctas);
        });
      });
    } else {
      sum.ctas = static_cast<int>(norm_any_ctas(rows, dim));
      with_type(dtype, [&](auto t) {
        const auto kernel = norm_any_backward_kernel<decltype(t)>;
        const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ADAPT_NORM_MAX_DIM * 4);
        if (err != cudaSuccess) rc = cuda_fail(err, "block norm, backward");
        else kernel<<<static_cast<unsigned>(sum.ctas), kNormThreads, q.dim * 4, stream>>>(q);
      });
    }
    if (rc != ADAPT_OK) return rc;
    ADAPT_LAUNCH_OK("block norm, backward");
  }
  if (sums) {
    LaunchScope ls(ADAPT_KERNEL_BLOCK_NORM_BACKWARD, stream);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((q.dim + 31) / 32), 3);
    cfg.blockDim = dim3(32 * kNormColumnWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // its launch hides behind the rows
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ADAPT_CUDA(cudaLaunchKernelEx(&cfg, norm_columns_kernel, sum));
    ADAPT_LAUNCH_OK("block norm, sums over rows");
  }
  return ADAPT_OK;
}

}  // extern "C"
