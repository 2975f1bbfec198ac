// Where the rows of a paged cache lie, as device code shared by the kernels that write and read it.
#pragma once

#include "dp_device.hpp"

namespace dp {

// rows of sequence s
__device__ __forceinline__ int paged_len(const PagedView &c, int s) { return max(0, min(c.seq_lens[s], c.max_seq_len)); }

// Last i in [0, n) with ptr[i] <= x < ptr[n], ptr ascending (n + 1 entries; of equal ones the last i); n where no entry
// holds x.  By the whole wave, x the same in all lanes: 64 entries are looked at per round.
__device__ __forceinline__ int wave_find(const int32_t *ptr, int n, int x) {
  const int lane = lane_id();
  int lo = -1, hi = n;  // ptr[lo] <= x < ptr[hi] (lo = -1: nothing known)
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step;
    const unsigned long long below = __ballot(at <= hi && ptr[min(at, n)] <= x);
    const int c = __builtin_popcountll(below);
    if (lo + c * step >= n) return n;
    lo += c * step;
    hi = min(hi, lo + step);
  }
  return lo < 0 || ptr[n] <= x ? n : lo;
}

}  // namespace dp
