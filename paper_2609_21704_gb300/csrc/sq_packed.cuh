// sq_packed.cuh -- which sequence and position a row of a packed batch has.
#pragma once

#include "sq_serve.h"

namespace sq {

struct PackedRow {
  int b;      // sequence, or -1: the row is none's
  int pos;    // its position in the sequence's cache
  bool ok;    // the sequence's positions lie in the cache
  bool bad;   // the offsets decrease or leave [0, N] (b is then -1)
};

// Called by all threads of a CTA.  With offsets every one is looked at (they
// are as many as sequences, so a pass of the CTA over them costs about as much
// as a binary search and finds a decreasing one besides).
__device__ __forceinline__ PackedRow packed_row(const Packed& p, int64_t row) {
  __shared__ int found;
  PackedRow r = {-1, 0, false, false};
  if (!p.offsets) {
    r.b = (int)(row / p.T);
    const int64_t p0 = p.pos0[r.b];
    r.pos = (int)(p0 + (row - (int64_t)r.b * p.T));
    r.ok = p0 >= 0 && p0 + p.T <= p.max_ctx;
    return r;
  }
  if (threadIdx.x == 0) found = -1;
  __syncthreads();
  bool bad = false;
  for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
    const int lo = p.offsets[b], hi = p.offsets[b + 1];
    bad |= lo < 0 || hi < lo || (int64_t)hi > p.N;
    if (lo <= row && row < hi) found = b;  // (of one sequence, where none is bad)
  }
  r.bad = __syncthreads_or(bad);
  if (r.bad || found < 0) return r;
  r.b = found;
  const int lo = p.offsets[r.b], len = p.offsets[r.b + 1] - lo;
  const int64_t p0 = p.pos0[r.b];
  r.pos = (int)(p0 + (row - lo));
  r.ok = p0 >= 0 && p0 + len <= p.max_ctx;
  return r;
}

}  // namespace sq
