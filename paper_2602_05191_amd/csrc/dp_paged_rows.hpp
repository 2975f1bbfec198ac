// Where the rows of a paged cache lie, and how the kernels that read it are shared out, as device code.
#pragma once

#include "dp_device.hpp"

namespace dp {

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

// The same by every lane for itself.
__device__ __forceinline__ int lane_find(const int32_t *ptr, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ptr[mid] <= x) lo = mid; else hi = mid;
  }
  return ptr[lo] <= x && x < ptr[hi] ? lo : n;
}

__device__ __forceinline__ int paged_len(const PagedView &c, int s) { return max(0, min(c.seq_lens[s], c.max_seq_len)); }

// Rows that sequence s shares with its group (0: none; a sequence that is too short for them shares none).
__device__ __forceinline__ int shared_rows(const SharedView &p, int s, int len) {
  const int g = lane_find(p.group_ptr, p.n_groups, s);
  if (g >= p.n_groups || s - p.group_ptr[g] >= p.max_group_seqs) return 0;
  const int n = max(0, min(p.shared_lens[g], p.max_shared_len));
  return n <= len ? n : 0;
}

}  // namespace dp
