// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient of the log probability and the entropy.
//   z = scale x,  lse = m + ln sum e^(z - m),  logprob = z_t - lse,
//   H = ln s - (sum e^(z - m) (z - m)) / s,
//   dx_j = scale (dlp ([j = t] - p_j) - dH p_j (ln p_j + H)).
//
// Forms: rows of up to 1024 logits are held in a warp's registers; longer ones are read once by a
// warp (many rows of up to 8192), by a CTA, or by the CTAs of a cluster, a part each, when there are few
// rows.  All in one launch; the gradient of the same call reads the row again, from L2.
#pragma once

#include "k_elem.cuh"
#include "row_part.h"

namespace adapt {

constexpr int kMaxTop = 32;
constexpr int kRowThreads = 256;
constexpr int kRowMaxCluster = 16;
constexpr int kRowUnroll = 4;            // 16-byte loads of a thread in flight
constexpr int kWarpRowMax = 1024;        // longest row of the warp form

struct LogprobParams {
  const void* logits;
  long long rows, ld, ld_grad;
  int vocab, n_top;
  float scale;
  const long long* targets;  // may be null
  float *logprob, *entropy, *lse;   // each may be null
  int* top_ids;
  float* top_logprobs;
  const float *d_logprob, *d_entropy;   // each may be null
  void* dlogits;                        // may be null
  const float *lse_in, *entropy_in;     // backward alone
};

// Order of the alternatives: larger logit first, equal ones (and +-0) by the lower index, NaN before
// everything.  One 64-bit key, all keys of a row distinct, none 0 and none ~0 (which a selection from above starts
// at: NaN at index 0 would not be below it).
constexpr unsigned kNanOrder = 0xFFFFFFFEu;
static_assert(kNanOrder > (0x7F800000u | 0x80000000u) && kNanOrder != 0xFFFFFFFFu, "above +Inf, below the start");
__device__ __forceinline__ unsigned top_order(float v) {
  const unsigned b = __float_as_uint(__fadd_rn(v, 0.0f));
  return v != v ? kNanOrder : (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ unsigned long long top_key(float v, int j) {
  return (static_cast<unsigned long long>(top_order(v)) << 32) | (0xFFFFFFFFu - static_cast<unsigned>(j));
}
__device__ __forceinline__ int top_index(unsigned long long key) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<unsigned>(key));
}

__device__ __forceinline__ float exp2_approx(float v) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
  return e;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// log2 e scale (v - m), the exponent of v beside the maximum.  (From a scale of 2.4e38 on log2 e scale leaves the range:
// then v and m, which are small there, count twice and the factor half.)
struct Exponent {
  float unit, c;
  __device__ __forceinline__ explicit Exponent(float scale) : unit(scale > 1e38f ? 2.0f : 1.0f), c(scale / unit * kLog2e) {}
  __device__ __forceinline__ float operator()(float v, float unit_m) const { return fmaf(v, unit, -unit_m) * c; }
};

// What a row without a target leaves.
__device__ __forceinline__ void put_ignored(const LogprobParams& p, long long row) {
  if (p.logprob) p.logprob[row] = 0.0f;
  if (p.entropy) p.entropy[row] = 0.0f;
  if (p.lse) p.lse[row] = 0.0f;
  for (int k = 0; k < p.n_top; ++k) {
    p.top_ids[row * p.n_top + k] = -1;
    p.top_logprobs[row * p.n_top + k] = 0.0f;
  }
}

// A row's statistics: m the largest logit, ln_sum = ln sum e^(z - scale m), spread = sum p (ln p) + ln_sum
// (the mean of z - scale m), so that ln p_j = scale (x_j - m) - ln_sum and H = ln_sum - spread.
// Special rows have m = -Inf (nothing but -Inf) or ln_sum = NaN.
struct RowStats { float m, ln_sum, spread; };

__device__ __forceinline__ float row_lse(const RowStats& r, float scale) {
  if (r.ln_sum != r.ln_sum) return r.ln_sum;
  return r.m * scale == -INFINITY ? -INFINITY : fmaf(r.m, scale, r.ln_sum);
}
__device__ __forceinline__ float row_logp(const RowStats& r, float scale, float x) {
  if (r.ln_sum != r.ln_sum) return r.ln_sum;
  if (r.m * scale == -INFINITY) return -INFINITY;
  if (x == -INFINITY) return x;
  return fmaf(x - r.m, scale, -r.ln_sum);
}
__device__ __forceinline__ void put_stats(const LogprobParams& p, long long row, const RowStats& r, long long target, float x_target) {
  if (p.logprob) p.logprob[row] = target < p.vocab ? row_logp(r, p.scale, x_target) : __int_as_float(0x7FFFFFFF);
  const bool dead = r.m * p.scale == -INFINITY && r.ln_sum == r.ln_sum;
  if (p.entropy) p.entropy[row] = dead ? 0.0f : r.ln_sum - r.spread;
  if (p.lse) p.lse[row] = row_lse(r, p.scale);
}

// The gradient of one element from its log probability; dead rows (all -Inf) have none.
struct RowWeights { float dlp, dh; };
__device__ __forceinline__ float element_grad(float logp, bool hot, const RowWeights& g, float h, float scale) {
  const float p = exp2_approx(logp * kLog2e);
  float v = (hot ? g.dlp : 0.0f) - g.dlp * p;
  if (g.dh != 0.0f && !(p == 0.0f)) v -= g.dh * p * (logp + h);
  return v * scale;
}

// ---- short rows: a warp a row, the row in registers ------------------------------------------------

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
  return v;
}

template <typename T, int kPer>
__global__ void __launch_bounds__(kRowThreads) logprob_warp_kernel(const LogprobParams p) {
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  T* dx = p.dlogits ? static_cast<T*>(p.dlogits) + row * p.ld_grad : nullptr;
  const long long target = p.targets ? p.targets[row] : 0;
  if (target < 0) {
    if (!p.lse_in && lane == 0) put_ignored(p, row);
    if (dx) for (int j = lane; j < p.vocab; j += 32) dx[j] = from_float<T>(0.0f);
    return;
  }
  float v[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) v[i] = lane + 32 * i < p.vocab ? to_float(x[lane + 32 * i]) : -INFINITY;
  float lse = 0.0f, h = 0.0f;
  RowStats r = {0.0f, 0.0f, 0.0f};
  if (!p.lse_in) {
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) { m = fmaxf(m, v[i]); nan |= v[i] != v[i]; }
    m = warp_max(m);
    nan = __any_sync(~0u, nan) || m * p.scale == INFINITY;
    r.m = m;
    const Exponent exponent(p.scale);
    const float unit_m = exponent.unit * m;
    float s = 0.0f, w = 0.0f;
    auto sum = [&](auto term) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float t = v[i] * p.scale == -INFINITY ? -200.0f : fmaxf(term(v[i]), -200.0f);
        const float e = exp2_approx(t);
        s += e;
        w = fmaf(e, t, w);
      }
    };
    if (m * p.scale != -INFINITY) {   // (of the two forms the second alone costs 4 % on rows of 1000)
      if (exponent.unit == 1.0f) sum([&](float v) { return (v - m) * exponent.c; });
      else sum([&](float v) { return exponent(v, unit_m); });
    }
    s = warp_sum(s);
    w = warp_sum(w);
    r.ln_sum = logf(s);
    r.spread = kLn2 * w / s;
    if (nan) r.ln_sum = __int_as_float(0x7FFFFFFF);
    float xt = 0.0f;
    if (target < p.vocab) xt = to_float(x[target]);
    if (lane == 0) put_stats(p, row, r, target, xt);
    unsigned long long last = ~0ull;
    for (int k = 0; k < p.n_top; ++k) {
      unsigned long long best = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int j = lane + 32 * i;
        const unsigned long long key = top_key(v[i], j);
        if (j < p.vocab && key < last && key > best) best = key;
      }
      last = best = warp_max(best);
      if (lane == 0) {
        const int j = top_index(best);
        p.top_ids[row * p.n_top + k] = j;
        if (ADAPT_IN_BOUNDS(j, p.vocab, 60)) p.top_logprobs[row * p.n_top + k] = row_logp(r, p.scale, to_float(x[j]));
      }
    }
    h = r.ln_sum - r.spread;
  } else {
    lse = p.lse_in[row];
    h = p.entropy_in ? p.entropy_in[row] : 0.0f;
  }
  if (dx) {
    __syncwarp();   // the row's last reads come before it is overwritten in place
    const RowWeights g = {p.d_logprob ? p.d_logprob[row] : 0.0f, p.d_entropy ? p.d_entropy[row] : 0.0f};
    const bool dead = p.lse_in ? lse == -INFINITY : r.m * p.scale == -INFINITY && r.ln_sum == r.ln_sum;
    const bool lost = p.d_logprob && target >= p.vocab;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = lane + 32 * i;
      if (j >= p.vocab) break;
      const float logp = p.lse_in ? fmaf(v[i], p.scale, -lse) : row_logp(r, p.scale, v[i]);
      float d = dead ? 0.0f : element_grad(logp, j == target, g, h, p.scale);
      if (lost) d = __int_as_float(0x7FFFFFFF);
      dx[j] = from_float<T>(d);
    }
  }
}

// ---- long rows ------------------------------------------------------------------------------------

// Elements as they are read: 16 bytes.  Logits below kFloor count as kFloor, which has probability 0
// beside any larger one that lets the row take this way (checked against the row's maximum).
template <typename T> struct Logits;
template <> struct Logits<float> {
  static constexpr float kFloor = -1e15f;
  __device__ __forceinline__ static float top(const uint4& q) {
    float a, b;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(__uint_as_float(q.x)), "f"(__uint_as_float(q.y)));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(__uint_as_float(q.z)), "f"(__uint_as_float(q.w)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
  }
  __device__ __forceinline__ static uint4 floored(const uint4& q) {
    return make_uint4(__float_as_uint(fmaxf(__uint_as_float(q.x), kFloor)), __float_as_uint(fmaxf(__uint_as_float(q.y), kFloor)),
                      __float_as_uint(fmaxf(__uint_as_float(q.z), kFloor)), __float_as_uint(fmaxf(__uint_as_float(q.w), kFloor)));
  }
  __device__ __forceinline__ static void pairs(const uint4& q, f32x2 (&v)[2]) {
    v[0] = pack2(__uint_as_float(q.x), __uint_as_float(q.y));
    v[1] = pack2(__uint_as_float(q.z), __uint_as_float(q.w));
  }
};
template <> struct Logits<__nv_bfloat16> {
  static constexpr float kFloor = -998356558020608.0f;   // 0xD863: -1.7734375 2^49
  __device__ __forceinline__ static __nv_bfloat162 two(unsigned v) { return *reinterpret_cast<const __nv_bfloat162*>(&v); }
  __device__ __forceinline__ static unsigned floored(unsigned v) {
    const __nv_bfloat162 r = __hmax2(two(v), two(0xD863D863u));
    return *reinterpret_cast<const unsigned*>(&r);
  }
  __device__ __forceinline__ static uint4 floored(const uint4& q) {
    return make_uint4(floored(q.x), floored(q.y), floored(q.z), floored(q.w));
  }
  __device__ __forceinline__ static float top(const uint4& q) {
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(two(q.x), two(q.y)), __hmax2_nan(two(q.z), two(q.w)));
    const float2 f = __bfloat1622float2(m);
    float a;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(f.x), "f"(f.y));
    return a;
  }
  __device__ __forceinline__ static void pairs(const uint4& q, f32x2 (&v)[4]) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = pack2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
    }
  }
};
template <> struct Logits<__half> {
  static constexpr float kFloor = -65504.0f;
  __device__ __forceinline__ static __half2 two(unsigned v) { return *reinterpret_cast<const __half2*>(&v); }
  __device__ __forceinline__ static unsigned floored(unsigned v) {
    const __half2 r = __hmax2(two(v), two(0xFBFFFBFFu));
    return *reinterpret_cast<const unsigned*>(&r);
  }
  __device__ __forceinline__ static uint4 floored(const uint4& q) {
    return make_uint4(floored(q.x), floored(q.y), floored(q.z), floored(q.w));
  }
  __device__ __forceinline__ static float top(const uint4& q) {
    const __half2 m = __hmax2_nan(__hmax2_nan(two(q.x), two(q.y)), __hmax2_nan(two(q.z), two(q.w)));
    const float2 f = __half22float2(m);
    float a;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(f.x), "f"(f.y));
    return a;
  }
  __device__ __forceinline__ static void pairs(const uint4& q, f32x2 (&v)[4]) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = __half22float2(two(w[k]));
      v[k] = pack2(f.x, f.y);
    }
  }
};

// One CTA's part of a row (row_part.h), in chunks of 16 bytes.
template <typename T>
struct RowPart : RowRange {
  static constexpr int kCount = 16 / sizeof(T);
  const uint4* chunks;   // chunk 0 (it may begin before the row)
  const T* x;
  __device__ __forceinline__ RowPart(const T* row, int vocab, int rank, int parts)
      : RowRange(kCount, static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)), vocab, rank, parts),
        chunks(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row) & ~static_cast<uintptr_t>(15))), x(row) {}
};

// Running maximum and sums of a thread; t = c x - mc in units of ln 2, mc = c m rounded up, so that t <= 0
// whatever the size of m: a thread that has met only barred logits (-Inf, the type's lowest, -1e10) sums
// numbers up to 1 until a larger maximum wipes them.  (To nearest, their t could be a rounding error of 10^7,
// and the row took the three-pass form: 64 x 32000 fp32 with a tenth barred 154 us for some masks, 12 for others.)
struct RowSums {
  float m, mc, s, w;
  __device__ __forceinline__ void raise(float to, float c) {
    const float mc2 = __fmul_ru(to, c), d = mc - mc2, f = exp2_approx(d);
    w = f * fmaf(d, s, w);
    s *= f;
    m = to; mc = mc2;
  }
};

__device__ __forceinline__ unsigned cluster_smem(const void* p, unsigned rank) {
  unsigned a = static_cast<unsigned>(__cvta_generic_to_shared(p)), r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

constexpr int kTopSpare = 64;   // candidates that may be there when a round of up to 256 chunks begins

// The threads that work on a row (or a part of one): a CTA or a warp.
template <int kThreads>
struct Team {
  static_assert(kThreads == 32 || kThreads == kRowThreads, "a warp or a CTA");
  __device__ __forceinline__ static int me() { return threadIdx.x % kThreads; }
  __device__ __forceinline__ static void sync() {
    if (kThreads == 32) __syncwarp();
    else __syncthreads();
  }
  __device__ __forceinline__ static bool any(bool v) {
    return kThreads == 32 ? __any_sync(~0u, v) != 0 : __syncthreads_or(v) != 0;
  }
  __device__ __forceinline__ static float reduce(float v, float* red, bool max) {
    v = max ? warp_max(v) : warp_sum(v);
    if (kThreads == 32) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < kRowThreads / 32; ++i) v = max ? fmaxf(v, red[i]) : v + red[i];
    return v;
  }
};

template <typename T, int kThreads>
struct RowShared {
  static constexpr int kCandidates = kThreads * RowPart<T>::kCount + kTopSpare;
  static constexpr int kParts = kThreads == 32 ? 1 : kRowMaxCluster;
  float red[2][kRowThreads / 32];
  float4 parts[kParts];                         // m, mc, s, w of each CTA of the row
  unsigned long long keys[kCandidates];
  unsigned long long best[kMaxTop];
  unsigned long long lists[kParts * kMaxTop];   // the first CTA's: alternatives of every part
  float group[32];
  unsigned char strips[kThreads];
  int n_keys, n_strips;
  float threshold;
};

// The k largest of n keys, sorted, into best[]; n_keys = their number.  All threads.
template <typename T, int kThreads>
__device__ void top_prune(RowShared<T, kThreads>& sh, const unsigned long long* keys, int n, int k) {
  const int me = Team<kThreads>::me();
  for (int i = me; i < n; i += kThreads) {
    const unsigned long long mine = keys[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += keys[j] > mine;
    if (rank < k && ADAPT_IN_BOUNDS(rank, kMaxTop, 61)) sh.best[rank] = mine;
  }
  Team<kThreads>::sync();
}

template <typename T, int kThreads>
__device__ __forceinline__ void add_key(RowShared<T, kThreads>& sh, unsigned long long key) {
  const int at = atomicAdd(&sh.n_keys, 1);
  if (ADAPT_IN_BOUNDS(at, (RowShared<T, kThreads>::kCandidates), 62)) sh.keys[at] = key;
}

// The part's k largest keys into best[].  `bound`: no element of the part below this one's order can be
// among them (0: any can); only the chunks of the threads listed in strips[] can hold larger ones (all of
// them if n_strips is kThreads).  Every round of at most kThreads chunks may add its elements'
// keys; beyond kTopSpare they are cut to the k largest, and the smallest of those bounds the rest.  Where most
// threads' chunks and several rounds are to come, the first round is of kTopSpare keys and is cut as well: equal
// logits, or barred ones where the bound is none, would fill a whole round (about 2000 keys, whose ranks take
// 70 us) and are then below the bound.  (1 x 131072 bf16, all equal, 8 alternatives: 151 -> 14 us.)
template <typename T, int kThreads>
__device__ int top_collect(RowShared<T, kThreads>& sh, const RowPart<T>& part, unsigned bound, int k) {
  const int me = Team<kThreads>::me();
  constexpr int kCount = RowPart<T>::kCount;
  const int n_strips = sh.n_strips, per = (part.q1 - part.q0 + kThreads - 1) / kThreads;
  unsigned long long least = static_cast<unsigned long long>(bound) << 32;   // keys above this one count
  if (me == 0) sh.n_keys = 0;
  Team<kThreads>::sync();
  if (me < part.edges) {
    const int j = part.edge(me);
    const unsigned long long key = top_key(to_float(part.x[j]), j);
    if (key > least) add_key(sh, key);
  }
  const int total = n_strips * per;
  for (int base = 0, width; base < total; base += width) {
    const bool probe = base == 0 && total > kThreads && 2 * n_strips > kThreads;
    width = probe ? min(kThreads, kTopSpare / kCount) : kThreads;
    const int i = base + me;
    if (me < width && i < total) {
      const int step = i / n_strips, s = i - step * n_strips;
      const int q = part.q0 + step * kThreads + (n_strips == kThreads ? s : sh.strips[s]);
      if (q < part.q1) {
        float v[kCount];
        unpack16<T>(part.chunks[q], v);
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
          const unsigned long long key = top_key(v[e], part.element(q) + e);
          if (key > least) add_key(sh, key);
        }
      }
    }
    Team<kThreads>::sync();
    const int n = sh.n_keys;
    Team<kThreads>::sync();   // all have read it before the next round adds to it
    if ((n > kTopSpare || (probe && n >= k)) && base + width < total) {
      top_prune<T, kThreads>(sh, sh.keys, n, k);
      if (me < k) sh.keys[me] = sh.best[me];
      if (me == 0) sh.n_keys = k;
      least = max(least, sh.best[k - 1]);
      Team<kThreads>::sync();
    }
  }
  Team<kThreads>::sync();
  const int n = sh.n_keys;
  top_prune<T, kThreads>(sh, sh.keys, n, k);
  return min(n, k);
}

// Order of the k-th largest of 32 group maxima (the maxima of 8 threads each, or of one): k elements at least are
// as large.  Kept in threshold; the threads whose own maximum reaches it are listed in strips[].
template <typename T, int kThreads>
__device__ void top_threshold(RowShared<T, kThreads>& sh, float m, int k) {
  const int me = Team<kThreads>::me();
  constexpr int kWide = kThreads / 32;
  float g = m;
#pragma unroll
  for (int o = 1; o < kWide; o <<= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, o));
  if (me % kWide == 0) sh.group[me / kWide] = g;
  if (me == 0) sh.n_strips = 0;
  Team<kThreads>::sync();
  if (me < 32) {
    const float mine = sh.group[me];
    int rank = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float v = __shfl_sync(~0u, mine, j);
      rank += v > mine || (v == mine && j < me);
    }
    if (rank == k - 1) sh.threshold = mine;
  }
  Team<kThreads>::sync();
  if (m >= sh.threshold) {
    const int at = atomicAdd(&sh.n_strips, 1);
    if (ADAPT_IN_BOUNDS(at, kThreads, 63)) sh.strips[at] = static_cast<unsigned char>(me);
  }
  Team<kThreads>::sync();
}

// A special row (NaN, Inf, nothing but -Inf, or values where the one-pass sums would lose themselves):
// one CTA, element by element, three passes.
template <typename T, int kThreads>
__device__ void special_row(const LogprobParams& p, RowShared<T, kThreads>& sh, long long row, const T* x, T* dx, long long target) {
  const int me = Team<kThreads>::me();
  const unsigned vocab = p.vocab;   // (a signed count beyond it would overflow near 2^31)
  float m = -INFINITY;
  bool nan = false;
  for (unsigned j = me; j < vocab; j += kThreads) {
    const float v = to_float(x[j]);
    nan |= v != v;
    m = fmaxf(m, v);
  }
  nan = Team<kThreads>::any(nan);
  RowStats r = {Team<kThreads>::reduce(m, sh.red[0], true), 0.0f, 0.0f};
  nan |= r.m * p.scale == INFINITY;
  const bool dead = r.m * p.scale == -INFINITY;
  const Exponent exponent(p.scale);
  const float unit_m = exponent.unit * r.m;
  float s = 0.0f, w = 0.0f;
  if (!dead)
    for (unsigned j = me; j < vocab; j += kThreads) {
      const float v = to_float(x[j]);
      const float t = v * p.scale == -INFINITY ? -200.0f : fmaxf(exponent(v, unit_m), -200.0f);
      const float e = exp2_approx(t);
      s += e;
      w = fmaf(e, t, w);
    }
  s = Team<kThreads>::reduce(s, sh.red[1], false);
  Team<kThreads>::sync();
  w = Team<kThreads>::reduce(w, sh.red[0], false);
  r.ln_sum = logf(s);
  r.spread = kLn2 * w / s;
  if (nan) r.ln_sum = __int_as_float(0x7FFFFFFF);
  if (me == 0) put_stats(p, row, r, target, target < p.vocab ? to_float(x[target]) : 0.0f);
  if (p.n_top) {
    if (me == 0) sh.n_strips = kThreads;
    Team<kThreads>::sync();
    top_collect<T, kThreads>(sh, RowPart<T>(x, p.vocab, 0, 1), 0u, p.n_top);
    if (me < p.n_top) {
      const int j = top_index(sh.best[me]);
      p.top_ids[row * p.n_top + me] = j;
      if (ADAPT_IN_BOUNDS(j, p.vocab, 64)) p.top_logprobs[row * p.n_top + me] = row_logp(r, p.scale, to_float(x[j]));
    }
  }
  if (!dx) return;
  Team<kThreads>::sync();
  const RowWeights g = {p.d_logprob ? p.d_logprob[row] : 0.0f, p.d_entropy ? p.d_entropy[row] : 0.0f};
  const bool lost = p.d_logprob && target >= p.vocab;
  for (unsigned j = me; j < vocab; j += kThreads) {
    float d = dead && !nan ? 0.0f : element_grad(row_logp(r, p.scale, to_float(x[j])), j == target, g, r.ln_sum - r.spread, p.scale);
    if (lost) d = __int_as_float(0x7FFFFFFF);
    dx[j] = from_float<T>(d);
  }
}

// Writes f(x) for the part's elements to dx: 16 bytes at a time where dx is aligned as x is.  From the last
// chunk to the first: what was read last is the likeliest to be in L2 still.
template <typename T, int kThreads, bool kFloored, typename F, typename G>
__device__ __forceinline__ void write_part(const RowPart<T>& part, T* dx, F pairs, G one) {
  constexpr int kCount = RowPart<T>::kCount;
  const bool aligned = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(part.x)) & 15u) == 0;
  uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(dx) & ~static_cast<uintptr_t>(15));
  const int n = part.q1 - part.q0;
  for (int i = Team<kThreads>::me(); i < n; i += kThreads * kRowUnroll) {
    uint4 q[kRowUnroll];
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u)
      if (i + u * kThreads < n) q[u] = __ldcs(part.chunks + part.q1 - 1 - (i + u * kThreads));
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) {
      if (i + u * kThreads >= n) break;
      const int at = part.q1 - 1 - (i + u * kThreads);
      f32x2 v[kCount / 2];
      Logits<T>::pairs(kFloored ? Logits<T>::floored(q[u]) : q[u], v);
      float f[kCount];
#pragma unroll
      for (int e = 0; e < kCount / 2; ++e) {
        const float2 d = unpack2(pairs(v[e]));
        f[2 * e] = d.x; f[2 * e + 1] = d.y;
      }
      if (aligned) {
        __stcs(out + at, pack16<T>(f));
      } else {
#pragma unroll
        for (int e = 0; e < kCount; ++e) dx[part.element(at) + e] = from_float<T>(f[e]);
      }
    }
  }
  if (Team<kThreads>::me() < part.edges) {
    const int j = part.edge(Team<kThreads>::me());
    dx[j] = from_float<T>(one(to_float(part.x[j])));
  }
}
template <typename T, int kThreads>
__device__ __forceinline__ void zero_part(const RowPart<T>& part, T* dx) {
  const bool aligned = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(part.x)) & 15u) == 0;
  uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(dx) & ~static_cast<uintptr_t>(15));
  for (int q = part.q0 + Team<kThreads>::me(); q < part.q1; q += kThreads) {
    if (aligned) __stcs(out + q, make_uint4(0u, 0u, 0u, 0u));
    else for (int e = 0; e < RowPart<T>::kCount; ++e) dx[part.element(q) + e] = from_float<T>(0.0f);
  }
  if (Team<kThreads>::me() < part.edges) dx[part.edge(Team<kThreads>::me())] = from_float<T>(0.0f);
}
// Whether this thread wrote element j of the part (the target's gradient is put right by its writer).
template <typename T, int kThreads>
__device__ __forceinline__ bool wrote(const RowPart<T>& part, int j) {
  const int q = part.chunk(j);
  if (q >= part.q0 && q < part.q1) return Team<kThreads>::me() == (part.q1 - 1 - q) % kThreads;
  return Team<kThreads>::me() < part.edges && part.edge(Team<kThreads>::me()) == j;
}

// What bounds it: HBM (one read of the row; with the gradient one write as well); an element costs about
// 5 lane instructions and one exponential forward, as many for the gradient.
template <typename T, int kThreads>
__global__ void __launch_bounds__(kRowThreads, kThreads == 32 ? 5 : 6) logprob_row_kernel(const LogprobParams p) {
  constexpr int kCount = RowPart<T>::kCount;
  constexpr int kRows = kRowThreads / kThreads;   // of a CTA
  __shared__ RowShared<T, kThreads> shared[kRows];
  RowShared<T, kThreads>& sh = shared[threadIdx.x / kThreads];
  const int me = Team<kThreads>::me();
  unsigned rank = 0, parts = 1;
  if (kRows == 1) {
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  }
  const long long row = kRows == 1 ? blockIdx.x / parts : static_cast<long long>(blockIdx.x) * kRows + threadIdx.x / kThreads;
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  T* dx = p.dlogits ? static_cast<T*>(p.dlogits) + row * p.ld_grad : nullptr;
  const long long target = p.targets ? p.targets[row] : 0;
  const RowPart<T> part(x, p.vocab, rank, parts);
  if (target < 0) {   // the whole cluster
    if (rank == 0 && me == 0) put_ignored(p, row);
    if (dx) zero_part<T, kThreads>(part, dx);
    return;
  }
  if (parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA has started
  const float x_target = target < p.vocab ? to_float(x[target]) : 0.0f;
  const float c = p.scale * kLog2e;

  RowSums a = {Logits<T>::kFloor, __fmul_ru(Logits<T>::kFloor, c), 0.0f, 0.0f};
  f32x2 s2 = 0, w2 = 0;
  const f32x2 cc = pack2(c, c);
  f32x2 shift = pack2(-a.mc, -a.mc);
  auto raise = [&](float top) {
    if (top > a.m || top != top) {   // (a NaN stays: no later value is larger)
      const float2 s = unpack2(s2), w = unpack2(w2);
      a.s = s.x + s.y; a.w = w.x + w.y;
      a.raise(top, c);
      s2 = pack2(a.s, 0.0f); w2 = pack2(a.w, 0.0f);
      shift = pack2(-a.mc, -a.mc);
    }
  };
  auto add = [&](const uint4& q) {
    f32x2 v[kCount / 2];
    Logits<T>::pairs(Logits<T>::floored(q), v);
#pragma unroll
    for (int e = 0; e < kCount / 2; ++e) {
      const f32x2 t = fma2(v[e], cc, shift);
      const float2 tf = unpack2(t);
      const f32x2 ex = pack2(exp2_approx(tf.x), exp2_approx(tf.y));
      s2 = add2(s2, ex);
      w2 = fma2(ex, t, w2);
    }
  };
  int q = part.q0 + me;
  for (; q + (kRowUnroll - 1) * kThreads < part.q1; q += kRowUnroll * kThreads) {
    uint4 v[kRowUnroll];
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) v[u] = part.chunks[q + u * kThreads];
    float top = Logits<T>::top(v[0]);
#pragma unroll
    for (int u = 1; u < kRowUnroll; ++u) {
      const float o = Logits<T>::top(v[u]);
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(o));
    }
    raise(top);
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) add(v[u]);
  }
  for (; q < part.q1; q += kThreads) {
    const uint4 v = part.chunks[q];
    raise(Logits<T>::top(v));
    add(v);
  }
  if (me < part.edges) {
    const float v = to_float(x[part.edge(me)]);
    raise(v);
    const float t = fmaf(fmaxf(v, Logits<T>::kFloor), c, -a.mc), e = exp2_approx(t);
    s2 = add2(s2, pack2(e, 0.0f));
    w2 = add2(w2, pack2(e * t, 0.0f));
  }
  const float own_top = a.m;
  {
    const float2 s = unpack2(s2), w = unpack2(w2);
    a.s = s.x + s.y; a.w = w.x + w.y;
  }
  // one maximum for the CTA, then for the row; NaN shows in the sums
  const bool nan = Team<kThreads>::any(own_top != own_top);
  float m = Team<kThreads>::reduce(own_top, sh.red[0], true);
  a.raise(m, c);
  const float s_cta = Team<kThreads>::reduce(a.s, sh.red[1], false);
  Team<kThreads>::sync();
  float w_sum = Team<kThreads>::reduce(a.w, sh.red[0], false);
  float s_sum = nan ? __int_as_float(0x7FFFFFFF) : s_cta;
  if (parts > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // and so have the others
    if (me < static_cast<int>(parts)) {
      const unsigned at = cluster_smem(&sh.parts[rank], me);
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(at), "f"(m), "f"(a.mc), "f"(s_sum), "f"(w_sum) : "memory");
    }
    cluster_barrier();
    RowSums all = {sh.parts[0].x, sh.parts[0].y, sh.parts[0].z, sh.parts[0].w};
    for (unsigned i = 1; i < parts; ++i) {
      RowSums o = {sh.parts[i].x, sh.parts[i].y, sh.parts[i].z, sh.parts[i].w};
      if (o.m > all.m) all.raise(o.m, c);
      else o.raise(all.m, c);
      all.s += o.s; all.w += o.w;
    }
    m = all.m; a.mc = all.mc; s_sum = all.s; w_sum = all.w;
  }
  // logits at the floor must have been nothing beside the maximum, and c m within 32 of mc
  if (!((m - Logits<T>::kFloor) * c > 160.0f) || !(fabsf(a.mc) < 5e8f) || !(c < 1e7f) || s_sum != s_sum) {
    if (rank == 0) special_row<T, kThreads>(p, sh, row, x, dx, target);
    return;   // (no other CTA's shared memory is touched from here on)
  }
  // s is relative to the rounded c m; delta = c m - fl(c m) takes it to the true one
  const float log2_s = log2f(s_sum), delta = fmaf(m, c, -a.mc);
  const RowStats r = {m, kLn2 * (log2_s - delta), kLn2 * (w_sum / s_sum - delta)};
  if (rank == 0 && me == 0) put_stats(p, row, r, target, x_target);

  if (p.n_top) {
    const int k = p.n_top;
    top_threshold<T, kThreads>(sh, own_top, k);
    const bool few = !(sh.threshold > Logits<T>::kFloor);   // fewer than k above the floor: take any
    if (few) {
      if (me == 0) sh.n_strips = kThreads;
      Team<kThreads>::sync();
    }
    int n = top_collect<T, kThreads>(sh, part, few ? 0u : top_order(sh.threshold), k);
    if (parts > 1) {
      if (me < k) {
        const unsigned at = cluster_smem(&sh.lists[rank * k + me], 0);
        const unsigned long long key = me < n ? sh.best[me] : 0ull;
        asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(at), "l"(key) : "memory");
      }
      cluster_barrier();
      if (rank == 0) top_prune<T, kThreads>(sh, sh.lists, static_cast<int>(parts) * k, k);
    }
    if (rank == 0 && me < k) {
      const int j = top_index(sh.best[me]);
      p.top_ids[row * k + me] = j;
      if (ADAPT_IN_BOUNDS(j, p.vocab, 65)) p.top_logprobs[row * k + me] = row_logp(r, p.scale, to_float(x[j]));
    }
    if (dx && parts > 1) cluster_barrier();   // the alternatives' logits are read before they are overwritten
  }
  if (!dx) return;
  Team<kThreads>::sync();
  const RowWeights g = {p.d_logprob ? p.d_logprob[row] : 0.0f, p.d_entropy ? p.d_entropy[row] : 0.0f};
  const bool lost = p.d_logprob && target >= p.vocab;
  // e (a1 t + a0), e = 2^t, t = c x - fl(c m): ln p + H = ln 2 (t - mean of t)
  const float unit = -p.scale / s_sum, a1 = unit * g.dh * kLn2;
  const float a0 = lost ? __int_as_float(0x7FFFFFFF) : unit * fmaf(-g.dh * kLn2, w_sum / s_sum, g.dlp);
  const f32x2 a1a1 = pack2(a1, a1), a0a0 = pack2(a0, a0), back = pack2(-a.mc, -a.mc);
  auto one = [&](float v) {
    const float t = fmaf(fmaxf(v, Logits<T>::kFloor), c, -a.mc);
    return exp2_approx(t) * fmaf(t, a1, a0);
  };
  write_part<T, kThreads, true>(part, dx, [&](f32x2 v) {
    const f32x2 t = fma2(v, cc, back);
    const float2 f = unpack2(t);
    return mul2(pack2(exp2_approx(f.x), exp2_approx(f.y)), fma2(t, a1a1, a0a0));
  }, one);
  if (!lost && g.dlp != 0.0f && ADAPT_IN_BOUNDS(target, p.vocab, 66) && wrote<T, kThreads>(part, static_cast<int>(target)))
    dx[target] = from_float<T>(fmaf(p.scale, g.dlp, one(x_target)));
}

// The gradient from lse and entropy.
template <typename T, int kThreads>
__global__ void __launch_bounds__(kRowThreads, 5) logprob_backward_kernel(const LogprobParams p, int parts) {
  constexpr int kRows = kRowThreads / kThreads;   // of a CTA
  const long long row = kRows == 1 ? blockIdx.x / parts : static_cast<long long>(blockIdx.x) * kRows + threadIdx.x / kThreads;
  if (row >= p.rows) return;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  T* dx = static_cast<T*>(p.dlogits) + row * p.ld_grad;
  const long long target = p.targets ? p.targets[row] : 0;
  const RowPart<T> part(x, p.vocab, kRows == 1 ? blockIdx.x % parts : 0, kRows == 1 ? parts : 1);
  const float lse = p.lse_in[row];
  if (target < 0 || lse == -INFINITY) { zero_part<T, kThreads>(part, dx); return; }
  const float h = p.entropy_in ? p.entropy_in[row] : 0.0f;
  const RowWeights g = {p.d_logprob ? p.d_logprob[row] : 0.0f, p.d_entropy ? p.d_entropy[row] : 0.0f};
  const bool lost = (p.d_logprob && target >= p.vocab) || lse != lse;
  const bool mine = !lost && g.dlp != 0.0f && ADAPT_IN_BOUNDS(target, p.vocab, 67) &&
                    wrote<T, kThreads>(part, static_cast<int>(target));
  const float x_target = mine ? to_float(x[target]) : 0.0f;   // before it is overwritten in place
  // p (a1 t + a0), t = ln p = z - lse
  const float a1 = -p.scale * g.dh, a0 = lost ? __int_as_float(0x7FFFFFFF) : -p.scale * fmaf(g.dh, h, g.dlp);
  const f32x2 a1a1 = pack2(a1, a1), a0a0 = pack2(a0, a0), ss = pack2(p.scale, p.scale), back = pack2(-lse, -lse), l2 = pack2(kLog2e, kLog2e);
  // t is kept at -1000 (p = 0 there), so that 0 times it is 0
  auto one = [&](float v) {
    const float t = fmaxf(fmaf(v, p.scale, -lse), -1000.0f);
    return exp2_approx(t * kLog2e) * fmaf(t, a1, a0);
  };
  write_part<T, kThreads, false>(part, dx, [&](f32x2 v) {
    const float2 u = unpack2(fma2(v, ss, back));
    const f32x2 t = pack2(fmaxf(u.x, -1000.0f), fmaxf(u.y, -1000.0f));
    const float2 f = unpack2(mul2(t, l2));
    return mul2(pack2(exp2_approx(f.x), exp2_approx(f.y)), fma2(t, a1a1, a0a0));
  }, one);
  if (mine) dx[target] = from_float<T>(fmaf(p.scale, g.dlp, one(x_target)));
}

}  // namespace adapt
