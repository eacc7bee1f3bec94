// How the rows of the norms around a block are dealt to threads and CTAs.  Host arithmetic only.
#pragma once

#include <algorithm>
#include <cstdint>

namespace adapt {

constexpr int kNormElems = 16;             // elements of a thread
constexpr int kNormMaxThreads = 1024;      // of a CTA, forward
constexpr int kNormBackwardThreads = 512;  // and backward
constexpr int kNormMaxParts = 8;           // CTAs of a cluster that share a row
constexpr int kNormPairElems = 8;          // of each of two rows at a time
constexpr int kNormPairThreads = 256;

// Places that a row may take: an odd one has up to 7 elements between a 16-byte boundary and its own first.
constexpr int64_t norm_room(int64_t dim) { return dim + (dim % 8 ? 7 : 0); }

// How a row is held: by CTAs of so many threads, `parts` of them, `per_sm` on an SM (at most; a kernel's registers say how many).
struct NormShape {
  int elems, rows, parts = 1, threads, per_sm;   // of a thread, at a time
  NormShape(int64_t dim, int elems_, int rows_, int most, int of_sm, int ctas) : elems(elems_), rows(rows_) {
    const int64_t room = norm_room(dim);
    while (room > static_cast<int64_t>(elems) * most * parts) parts *= 2;
    const int64_t unit = 32ll * elems * parts;
    threads = static_cast<int>((room + unit - 1) / unit) * 32;
    per_sm = std::max(1, std::min(ctas, of_sm / threads));
  }
};
inline NormShape norm_forward(int64_t dim) { return NormShape(dim, kNormElems, 1, kNormMaxThreads, 1024, 16); }
// (backward: CTAs of one warp, whose rows take a warp's latency each, as many as there is room for; of more, stages pay rather
// than CTAs.  us: 65536 x 256 bf16 with 8 78, with 12 62; 32768 x 1024 fp32 with 8 87, with 10 95)
inline NormShape norm_backward(int64_t dim) {
  return NormShape(dim, kNormElems, 1, kNormBackwardThreads, 512, dim <= 32 * kNormElems ? 16 : 8);
}
// Two rows at a time, by no more CTAs; where they pay.  Above, more CTAs do, and rows of up to 512 are a warp's, 16 CTAs on an SM.
// us, by ones and by pairs, 2^25 elements: 256 bf16 with both norms and a gate 149, 130; 384 152, 167; 640 183, 158; 768 156, 135;
// without the gate 1000 117, 103; 1024 110, 101; with one norm fp32 768 85, 75; 1024 86, 73; 2048 86, 74; 2560 80, 95; 16384 rows of
// 2039 bf16 82, 94.  The rule does not see the gate: with one 896 135, 139; 1000 128, 129; 1024 123, 126
inline NormShape norm_backward_pairs(int64_t dim) {
  return NormShape(dim, kNormPairElems, 2, kNormPairThreads, 512, dim <= 32 * kNormPairElems ? 16 : 8);
}
inline bool norm_in_pairs(int64_t dim, int norms) {
  const int64_t room = norm_room(dim), warp = 32 * kNormPairElems;
  return room <= warp || (room > 2 * warp && room <= (norms == 1 && dim % 8 == 0 ? 8 * warp : 4 * warp));
}
static_assert(8 * 32 * kNormPairElems <= kNormPairElems * kNormPairThreads, "a CTA holds a pair of rows");

}  // namespace adapt
