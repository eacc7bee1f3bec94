// How a row of logits is dealt to the CTAs that share it: whole 16-byte chunks, and beside them the elements before
// the first and behind the last one, which the first CTA takes.  Chunk q begins at element q * count - mis, mis the
// elements by which the row is off a 16-byte boundary.  Good for every vocabulary below 2^31.
#pragma once

#ifdef __CUDACC__
#define ADAPT_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define ADAPT_HOST_DEVICE inline
#endif

namespace adapt {

struct RowRange {
  int count, mis;          // elements of a chunk; before the row in chunk 0
  int q0, q1;              // chunks of this part
  int head, tail_from;     // elements before the chunks; the first behind them
  int edges;               // single elements of this part

  RowRange() = default;
  ADAPT_HOST_DEVICE RowRange(int count, int mis, int vocab, int rank, int parts) : count(count), mis(mis) {
    const int qa = mis ? 1 : 0, whole = static_cast<int>((static_cast<long long>(mis) + vocab) / count);
    const int qb = whole > qa ? whole : qa;
    const int per = (qb - qa + parts - 1) / parts;
    q0 = qa + rank * per;
    q0 = q0 < qb ? q0 : qb;
    q1 = q0 + per < qb ? q0 + per : qb;
    head = mis ? (count - mis < vocab ? count - mis : vocab) : 0;
    const int behind = static_cast<int>(static_cast<long long>(qb) * count - mis);
    tail_from = behind > head ? behind : head;
    edges = rank == 0 ? head + (vocab > tail_from ? vocab - tail_from : 0) : 0;
  }
  ADAPT_HOST_DEVICE int edge(int i) const { return i < head ? i : tail_from + (i - head); }   // element number
  ADAPT_HOST_DEVICE int element(int q) const { return q * count - mis; }   // of a chunk's first
  ADAPT_HOST_DEVICE int chunk(int j) const {   // that holds element j
    return static_cast<int>((static_cast<unsigned>(j) + mis) / count);
  }
};

}  // namespace adapt
