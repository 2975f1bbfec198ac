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

// The sequences [begin, end) of group g that share rows, what they share (0 where none is long enough to hold it) and the
// first of them that holds it, through whose table the rows are read.
struct SharedGroup {
  int begin, end, rows, reader;
};
__device__ __forceinline__ SharedGroup shared_group(const PagedView &c, const SharedView &p, int g) {
  SharedGroup s;
  s.begin = max(0, min(p.group_ptr[g], c.n_seqs));
  s.end = max(s.begin, min(p.group_ptr[g + 1], c.n_seqs));
  s.end = s.begin + min(s.end - s.begin, p.max_group_seqs);
  s.rows = max(0, min(p.shared_lens[g], p.max_shared_len));
  s.reader = s.begin;
  while (s.reader < s.end && paged_len(c, s.reader) < s.rows) ++s.reader;
  if (s.reader == s.end) s.rows = 0;
  return s;
}
// The group of sequence s (n_groups: none) and the rows that s shares (0: none; too short a sequence shares none).
__device__ __forceinline__ int shared_rows(const PagedView &c, const SharedView &p, int s, int len, int &group) {
  group = lane_find(p.group_ptr, p.n_groups, s);
  if (group >= p.n_groups || s - max(0, p.group_ptr[group]) >= p.max_group_seqs) return 0;
  const int n = max(0, min(p.shared_lens[group], p.max_shared_len));
  return n <= len ? n : 0;
}

// ---- work dealt out evenly ----
// n items; item i is subs segments of chunks chunks each, all numbered through in this order.  One round of workgroups
// takes equal shares: workgroup w chunks [w share, (w + 1) share).  A share may end one segment and begin the next, and a
// segment is cut into at most `slots` pieces: ceil(chunks / share) + 1, or as many as it has chunks.
struct Segments {
  int chunks, subs;
  int a, b;  // what the caller wants to know of the item
};
struct Deal {
  int grid, slots;
  __device__ __forceinline__ int share(int total, int longest) const {
    const int least = slots > 1 ? (longest + slots - 2) / (slots - 1) : longest;
    return max(max(1, longest > slots ? least : 1), (total + grid - 1) / grid);
  }
};
struct Dealt {
  Segments item;
  int i, sub, first;      // the segment that holds chunk c, its first chunk's number
  int c, c_end, share;
};
// By every wave for itself: a lane adds up `per` consecutive items, then the lane that holds chunk c has its items spread
// over the lanes.  n <= 64 * 64.  false: no chunk is left.
template <class At>
__device__ __forceinline__ bool deal_start(const Deal &deal, int block, int n, At at, Dealt &d) {
  const int lane = lane_id(), per = (n + 63) / 64;
  Segments item{0, 0, 0, 0};
  auto look = [&](int i, bool valid) {
    item = at(min(i, n - 1));
    if (!valid || i >= n) item.chunks = 0;
    return item.chunks * item.subs;
  };
  int mine = 0, longest = 0;
  for (int u = 0; u < per; ++u) {
    mine += look(lane * per + u, true);
    longest = max(longest, item.chunks);
  }
  int upto = wave_incl_scan(mine);
  const int total = (int)lane_u32((uint32_t)upto, 63);
  d.share = deal.share(total, (int)wave_max((unsigned long long)longest));
  d.c = block * d.share;
  d.c_end = min(total, d.c + d.share);
  if (d.c >= d.c_end) return false;
  int l = __builtin_ctzll(__ballot(upto - mine <= d.c && d.c < upto));
  d.i = l * per;
  int first = (int)lane_u32((uint32_t)(upto - mine), l);
  if (per > 1) {
    mine = look(d.i + lane, lane < per);
    upto = first + wave_incl_scan(mine);
    l = __builtin_ctzll(__ballot(upto - mine <= d.c && d.c < upto));
    d.i += l;
    first = (int)lane_u32((uint32_t)(upto - mine), l);
  }
  d.item.chunks = (int)lane_u32((uint32_t)item.chunks, l);
  d.item.subs = (int)lane_u32((uint32_t)item.subs, l);
  d.item.a = (int)lane_u32((uint32_t)item.a, l);
  d.item.b = (int)lane_u32((uint32_t)item.b, l);
  d.sub = (d.c - first) / d.item.chunks;
  d.first = first + d.sub * d.item.chunks;
  return true;
}
// To the segment behind the one just done (the caller has checked that chunks are left).
template <class At>
__device__ __forceinline__ void deal_next(At at, Dealt &d) {
  d.c = d.first = d.first + d.item.chunks;
  if (++d.sub < d.item.subs) return;
  d.sub = 0;
  do d.item = at(++d.i);
  while (d.item.chunks * d.item.subs == 0);
}
// Number of pieces of the segment.
__device__ __forceinline__ int pieces_of(const Dealt &d) {
  return (d.first + d.item.chunks - 1) / d.share - d.first / d.share + 1;
}

// ---- a call, as its kernels see it ----
constexpr int kSharedBlock = 64;       // shared rows that are attended between two barriers
constexpr int kDealtItems = 64 * 64;  // most sequences, or groups, that the lookup of a share can hold

// Partial results of a head: per slot the accumulator of its 128 dimensions, (maximum, sum).  The slots of its
// own rows come first, then those of the rows that it shares.
struct Partials {
  float *acc;
  float2 *ml;
  int32_t *pieces;   // per head, how many slots of either kind are in use (not written where there are no such rows)
  int32_t own, all;  // slots per head
};

struct PagedArgs {
  PagedView c;
  PagedAttention a;
  AttnOut attn;
  Partials parts;
  int32_t head0;        // this launch serves heads [head0, head0 + 16) of every group
  int32_t whole;        // own rows: nothing dealt out, a workgroup per segment (which writes the output where none are shared)
  int32_t span;         // own rows: KV heads per workgroup, 1 or 4
  Deal own, shared;     // shared.slots == 0: no shared rows
  int32_t shared_cols;  // columns (sequences x query heads of a KV head) per workgroup over shared rows
  float scale_log2;
  float lead;           // 8 / scale_log2: how far a score may lead the reference that is subtracted
};

// what is subtracted from a score whose running maximum is m
__device__ __forceinline__ float finite_max(float m) { return fmaxf(m, -3.402823466e38f); }

// Weights go into the products as bf16 pieces that add up.  A piece that ends up as zero although its weight is not becomes the
// weight's exponent, read as a bf16 pattern: at most 2^-125, for the least weights 2^-133 (the matrix cores take numbers below
// 2^-126 as they are).  An infinite value times a piece of zero would be NaN.  Patterns of numbers that are not negative are in
// the numbers' order.  (1 us of 111 for 64 sequences behind 32768 rows; with the lesser of the pattern and 1 four.)
template <class Bits, class Piece>
__device__ __forceinline__ Piece not_zero(Piece piece, Piece first) {
  return __builtin_bit_cast(Piece, __builtin_elementwise_max(__builtin_bit_cast(Bits, piece),
                                                             __builtin_bit_cast(Bits, first) >> (Bits)7));
}

// Own rows are dealt out in chunks of 64 rows of one KV head, or of 16 of four (span).
__host__ __device__ constexpr int own_chunk(int span) { return kChunkRows / span; }

// Rows [first, len) of a sequence; in chunks of n rows they are [first / n, ceil(len / n)).
struct SeqRows {
  int first, len;
  __device__ __forceinline__ int chunks(int n) const { return first < len ? (len + n - 1) / n - first / n : 0; }
};
template <bool kShared>
__device__ __forceinline__ SeqRows seq_rows(const PagedArgs &p, int s) {
  SeqRows r;
  r.len = paged_len(p.c, s);
  int group;
  if constexpr (kShared)
    r.first = shared_rows(p.c, p.a.shared, s, r.len, group);
  else
    r.first = p.a.first_rows ? max(0, p.a.first_rows[s]) : 0;
  return r;
}
// sequences, and the KV heads (or groups of them) of each
template <bool kShared, int kSpan>
__device__ __forceinline__ auto own_segments(const PagedArgs &p) {
  return [&p](int s) {
    const SeqRows r = seq_rows<kShared>(p, s);
    return Segments{r.chunks(own_chunk(kSpan)), p.c.n_kv_heads / kSpan, r.first, r.len};
  };
}

// Blocks of rows per chunk that is dealt out: a block takes the longer the more of the workgroup's waves have columns (1.4 us
// with one to four, 2.9 with five).  Groups of 4, 13 and 20 sequences, G = 8, 20011 to 8545 rows: 72 us with one block for
// all, 64 so.
__device__ __forceinline__ int shared_blocks(int cols) { return cols <= 128 ? 2 : 1; }

// groups; their KV heads, and of each the column tiles of a workgroup
__device__ __forceinline__ auto shared_segments(const PagedArgs &p) {
  return [&p](int g) {
    const SharedGroup s = shared_group(p.c, p.a.shared, g);
    const int cols = (s.end - s.begin) * p.c.group, tiles = (cols + p.shared_cols - 1) / p.shared_cols;
    const int rows = shared_blocks(cols) * kSharedBlock;
    return Segments{(s.rows + rows - 1) / rows, p.c.n_kv_heads * tiles, s.begin, s.reader};
  };
}

// The attention of shared rows: one launch that leaves partial results (dp_shared.hip).  Columns per workgroup: 256 or 128.
void launch_shared_rows(const PagedArgs &p, hipStream_t stream);

}  // namespace dp
