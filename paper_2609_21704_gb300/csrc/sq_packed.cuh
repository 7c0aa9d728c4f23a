// sq_packed.cuh -- which sequence and position the rows of a packed batch have.
#pragma once

#include "sq_serve.h"

namespace sq {

// Rows row0 .. row0 + R - 1: seq[i] their sequence (-1: none's), pos[i] the
// position in its cache (-1: the sequence does not fit, which sets
// SQ_DEV_BAD_POSITION in *status).  True where the offsets decrease or leave
// [0, N].  Called by all threads of a CTA; seq and pos are shared memory and
// valid after it.  With offsets every one is looked at: they are as many as
// sequences, so a pass of the CTA over them costs about as much as a binary
// search, and finds a decreasing one besides.
template <int R>
__device__ __forceinline__ bool packed_rows(const Packed& p, int64_t row0, int* seq, int* pos,
                                            unsigned int* status) {
  if (!p.offsets) {
    if (threadIdx.x < R) {
      const int64_t row = row0 + threadIdx.x;
      int b = -1, at = -1;
      if (row < p.N) {
        b = (int)(row / p.T);
        const int64_t p0 = p.pos0[b];
        if (p0 >= 0 && p0 + p.T <= p.max_ctx)
          at = (int)(p0 + (row - (int64_t)b * p.T));
        else
          atomicOr(status, SQ_DEV_BAD_POSITION);
      }
      seq[threadIdx.x] = b;
      pos[threadIdx.x] = at;
    }
    __syncthreads();
    return false;
  }
  if (threadIdx.x < R) seq[threadIdx.x] = -1;
  __syncthreads();
  bool bad = false;
  for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
    const int lo = p.offsets[b], hi = p.offsets[b + 1];
    bad |= lo < 0 || hi < lo || (int64_t)hi > p.N;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (lo <= row0 + i && row0 + i < hi) {
        const int64_t p0 = p.pos0[b];
        const bool ok = p0 >= 0 && p0 + (hi - lo) <= p.max_ctx;
        seq[i] = b;
        pos[i] = ok ? (int)(p0 + (row0 + i - lo)) : -1;
        if (!ok) atomicOr(status, SQ_DEV_BAD_POSITION);
      }
  }
  bad = __syncthreads_or(bad);
  if (bad && threadIdx.x == 0) atomicOr(status, SQ_DEV_BAD_POSITION);
  return bad;
}

}  // namespace sq
