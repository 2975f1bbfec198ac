// Dense decode attention over the rows of a paged cache, one query token per sequence (Eq. 1 over pages).
//
// HBM-bound streaming kernel (512 B per row and KV head), both contractions on the matrix cores straight from global
// memory in the instructions' layouts, 16 rows x up to 16 query heads of a group per wave and step:
//   scores  S[16 rows x 16 heads] = K Q^T, four v_mfma_f32_16x16x32_bf16: lane l loads chunks l / 16 + 4 j of key row
//           l % 16 and receives the scores of head l % 16 for rows 4 (l / 16) + i, which become weights in place;
//   output  O^T[dims x heads] += V^T P^T, v_mfma_f32_16x16x4_f32 with k = l / 16 standing for row 4 (l / 16) + i: the
//           weights stay fp32, the values are widened; tile n of eight holds dims 8 x + n.  A tile's 16 rows are summed by
//           themselves and then added: the fp32 chain is as long as the wave has tiles, not rows.
// The running maximum is kept and subtracted unscaled, so the largest score has the weight 1 whatever its size; a maximum
// of -inf is taken as the lowest finite number when it is subtracted; weights keep the range below 2^-126 (exp2f).
// Tiles begin at multiples of 16 rows, so a tile of pages of 16 tokens or more lies in one page: its place is a scalar and
// a lane's offsets are the same for every tile.  The numbers of the pages of a wave's next 64 tiles are fetched by its 64
// lanes at once.  Smaller pages: every row's page by the lane that loads the row's key, a tile ahead of the rows.
// A tile has a mask of 16 rows (inside [first, len) and on a page that is there); rows without a bit score -inf and their
// values are made zero: they may hold anything.
// Work split: the rows of all (sequence, KV head) segments, in chunks of 64, are dealt out evenly to one round of resident
// workgroups; pieces are merged by a second kernel.  Short or very many segments are taken whole, a workgroup each, which
// then writes the output itself.
#include "dp_attend.hpp"
#include "dp_device.hpp"
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedThreads = 256;
constexpr int kPagedWaves = kPagedThreads / 64;
constexpr int kPagedHeads = 16;  // query heads per pass: the columns of one MFMA tile
constexpr int kPagedTile = 16;   // rows per wave and step
constexpr int kPartialStride = kHeadDim + 2;
constexpr int kDealtSeqs = 64 * 64;  // most sequences that the lookup can hold

struct PagedArgs {
  PagedView c;
  PagedAttention a;
  AttnOut attn;
  float *partials;   // [heads, splits, kPartialStride]
  int32_t head0;     // this launch serves heads [head0, head0 + 16) of every group
  int32_t splits;    // partial slots per head
  int32_t min_share, grid;
  int32_t whole;     // nothing dealt out: a workgroup per segment
  float scale_log2;
};

// what is subtracted from a score whose running maximum is m
__device__ __forceinline__ float finite_max(float m) { return fmaxf(m, -3.402823466e38f); }

// Rows [first, len) of a sequence; its chunks are [first / 64, ceil(len / 64)).
struct SeqRows {
  int first, len;
  __device__ __forceinline__ int chunk0() const { return first / kChunkRows; }
  __device__ __forceinline__ int chunks() const {
    return first < len ? (len + kChunkRows - 1) / kChunkRows - chunk0() : 0;
  }
};
__device__ __forceinline__ SeqRows seq_rows(const PagedArgs &p, int s) {
  SeqRows r;
  r.len = paged_len(p.c, s);
  r.first = p.a.first_rows ? max(0, p.a.first_rows[s]) : 0;
  return r;
}

// The chunks of all segments, numbered through in (sequence, KV head) order: workgroup w takes [w share, (w + 1) share).
__device__ __forceinline__ int dealt_share(const PagedArgs &p, int total) {
  return max(p.min_share, (total + p.grid - 1) / p.grid);
}
struct PagedStart {
  int seq, kv, first;    // the segment that holds chunk c, its first chunk's number
  SeqRows rows;
  int c, c_end, share;
};
// By every wave for itself: a lane adds up `per` consecutive sequences, then the lane that holds the chunk has its
// sequences spread over the lanes.  false: no chunk is left.
__device__ __forceinline__ bool paged_start(const PagedArgs &p, PagedStart &d) {
  const int lane = lane_id(), n = p.c.n_seqs, per = (n + 63) / 64;
  SeqRows rows{0, 0};
  auto look = [&](int s, bool valid) {
    rows = seq_rows(p, min(s, n - 1));
    return valid && s < n ? rows.chunks() * p.c.n_kv_heads : 0;
  };
  int mine = 0;
  if (per == 1) {
    mine = look(lane, true);
  } else {
    for (int u = 0; u < per; ++u) mine += look(lane * per + u, true);
  }
  int upto = wave_incl_scan(mine);
  const int total = (int)lane_u32((uint32_t)upto, 63);
  d.share = dealt_share(p, total);
  d.c = blockIdx.x * d.share;
  d.c_end = min(total, d.c + d.share);
  if (d.c >= d.c_end) return false;
  int at = __builtin_ctzll(__ballot(upto - mine <= d.c && d.c < upto));
  d.seq = at * per;
  int first = (int)lane_u32((uint32_t)(upto - mine), at);
  if (per > 1) {
    mine = look(d.seq + lane, lane < per);
    upto = first + wave_incl_scan(mine);
    at = __builtin_ctzll(__ballot(upto - mine <= d.c && d.c < upto));
    d.seq += at;
    first = (int)lane_u32((uint32_t)(upto - mine), at);
  }
  d.rows.first = (int)lane_u32((uint32_t)rows.first, at);
  d.rows.len = (int)lane_u32((uint32_t)rows.len, at);
  d.kv = (d.c - first) / d.rows.chunks();
  d.first = first + d.kv * d.rows.chunks();
  return true;
}

// Number of the first piece of segment (my_seq, kv), which has rows, and how many there are; by every wave for itself.
__device__ __forceinline__ int paged_pieces(const PagedArgs &p, int my_seq, int kv, int chunks) {
  int total = 0, before = 0;
  for (int u = 0; u < p.c.n_seqs; u += 64) {
    const int s = u + lane_id();
    const int n = s < p.c.n_seqs ? seq_rows(p, min(s, p.c.n_seqs - 1)).chunks() : 0;
    total += n;
    before += s < my_seq ? n : 0;
  }
  total = wave_sum(total) * p.c.n_kv_heads;
  const int first = wave_sum(before) * p.c.n_kv_heads + kv * chunks;
  const int share = dealt_share(p, total);
  return (first + chunks - 1) / share - first / share + 1;
}

// one wave's 16 rows as the two contractions want them, and which of them count
struct PagedTile {
  uint4 k[4], v[4];
  uint32_t live;
};

// Fetches tiles of one segment: rows t .. t + 15, t a multiple of 16, of the wave's tiles t0, t0 + kStep, ...
template <bool kSmallPages>
struct TileLoader {
  static constexpr int kStep = kPagedWaves * kPagedTile;
  const PagedView &c;
  const int32_t *table;      // of the sequence
  const char *k, *v;         // of the KV head
  SeqRows rows;
  int t0, page;              // page: lane i's, of tile t0 + i kStep (small pages: row lane % 16 of the tile to load next)
  uint32_t k_off, v_off;     // the lane's place in a tile (small pages: in a row)

  __device__ __forceinline__ TileLoader(const PagedView &c, int seq, int kv, SeqRows rows)
      : c(c), table(c.table + (int64_t)seq * c.table_stride), k(c.k_pages + kv * c.head_stride),
        v(c.v_pages + kv * c.head_stride), rows(rows) {
    const int r = lane_id() & 15, kq = lane_id() >> 4;
    k_off = kSmallPages ? kq * 16 : r * c.slot_stride + kq * 16;
    v_off = kSmallPages ? r * 16 : 4 * kq * c.slot_stride + r * 16;
  }
  // (rows behind the last have no entry that may be read)
  __device__ __forceinline__ int page_of(int row) const { return row < rows.len ? table[row >> c.page_shift] : -1; }
  __device__ __forceinline__ void start(int t) {
    t0 = t;
    page = page_of(kSmallPages ? t + (lane_id() & 15) : t + lane_id() * kStep);
  }
  __device__ __forceinline__ bool there(int p) const { return (uint32_t)p < (uint32_t)c.n_pages; }
  __device__ __forceinline__ int64_t place(int p, int row) const {
    return p * c.page_stride + (row & ((1 << c.page_shift) - 1)) * (int64_t)c.slot_stride;
  }

  __device__ __forceinline__ void load(int t, PagedTile &d) {
    // bits of the rows inside [first, len)
    uint32_t live = (0xffffu << min(16, max(0, rows.first - t))) & (0xffffu >> min(16, max(0, t + 16 - rows.len)));
    if constexpr (!kSmallPages) {
      if (t - t0 >= 64 * kStep) start(t);
      int p = (int)lane_u32((uint32_t)page, (t - t0) / kStep);
      if (!there(p)) p = 0, live = 0;
      const int64_t at = place(p, t);
      const char *kr = k + at, *vr = v + at;
#pragma unroll
      for (int j = 0; j < 4; ++j) d.k[j] = load_stream16(kr + (k_off + j * 64));
#pragma unroll
      for (int i = 0; i < 4; ++i) d.v[i] = load_stream16(vr + (v_off + i * c.slot_stride));
    } else {
      const int r = lane_id() & 15, kq = lane_id() >> 4;
      const bool ok = there(page);
      live &= (uint32_t)__ballot(ok);
      const int64_t at = place(ok ? page : 0, t + r);
      const char *kr = k + at + k_off;
#pragma unroll
      for (int j = 0; j < 4; ++j) d.k[j] = load_stream16(kr + j * 64);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 4 * kq + i;
        const int64_t of_row = (int64_t)(((uint64_t)(uint32_t)__shfl((int)(at >> 32), row, 64) << 32) |
                                         (uint32_t)__shfl((int)at, row, 64));
        d.v[i] = load_stream16(v + of_row + v_off);
      }
      page = page_of(t + kStep + r);
    }
    d.live = live;
  }
};

// ---- output of a head: partial results and what was known before, in base 2 ----
struct Merged {
  float m, l, o;  // maximum, sum, accumulator of one dimension
};
__device__ __forceinline__ void store_head(const PagedArgs &p, int64_t head, int d, float prior_lse, float prior_o, Merged x) {
  const float prior = prior_lse * kLog2e;
  const float M = fmaxf(x.m, prior), sub = finite_max(M);
  const float w = exp2f(x.m - sub), wp = exp2f(prior - sub);
  const float L = fmaf(x.l, w, wp);
  float o = x.m > -INFINITY ? x.o * w : 0.f;
  if (prior > -INFINITY) o = fmaf(prior_o, wp, o);  // (a prior without weight may hold anything)
  const bool any = L > 0.f;
  store_out(p.attn.out, p.attn.out_is_bf16, head, d, any ? o / L : 0.f);
  if (p.attn.lse && d == 0) p.attn.lse[head] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
}

template <bool kSmallPages>
__global__ __launch_bounds__(kPagedThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_kernel(PagedArgs p) {
  __shared__ float s_m[kPagedWaves][kPagedHeads], s_l[kPagedWaves][kPagedHeads];
  __shared__ __align__(16) float s_acc[kPagedWaves][kPagedHeads][kHeadDim + 4];
  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int r = lane & 15, kq = lane >> 4;
  const int n_kv = p.c.n_kv_heads, group = p.c.group, n_live = min(kPagedHeads, group - p.head0);
  PagedStart at;
  if (p.whole) {
    at.seq = blockIdx.x / n_kv;
    at.kv = blockIdx.x % n_kv;
    at.rows = seq_rows(p, at.seq);
    at.first = at.c = 0;
    at.c_end = at.rows.chunks();
    at.share = 1;
  } else if (!paged_start(p, at)) {
    return;
  }

  // one piece of a segment after the other, usually one
  while (true) {
    const SeqRows rows = at.rows;
    const int seg_end = at.first + rows.chunks();
    const int ra = (rows.chunk0() + at.c - at.first) * kChunkRows;
    const int rb = min(rows.len, (rows.chunk0() + min(at.c_end, seg_end) - at.first) * kChunkRows);
    const int split = blockIdx.x - at.first / at.share;  // number of the piece inside its segment
    const int64_t head_first = (int64_t)at.seq * p.c.n_q_heads + at.kv * group + p.head0;

    // query head r of the pass (beyond the group: its last head again, not stored), chunks kq + 4 j
    uint4 Q[4];
    {
      const char *row = static_cast<const char *>(p.a.q) + (head_first + min(r, n_live - 1)) * kRowBytes + kq * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) Q[j] = *reinterpret_cast<const uint4 *>(row + j * 64);
    }
    f32x4 acc[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;  // head r: the largest score so far (unscaled), the weights of this lane's rows

    auto attend = [&](PagedTile &d) {
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      f32x4 part[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        part[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, d.k[j]),
                                                          __builtin_bit_cast(bf16x8, Q[j]), zero, 0, 0, 0);
      f32x4 x = (part[0] + part[1]) + (part[2] + part[3]);
      if (d.live != 0xffffu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool on = (d.live >> (4 * kq + i)) & 1;
          x[i] = on ? x[i] : -INFINITY;
          if (!on) d.v[i] = make_uint4(0, 0, 0, 0);
        }
      }
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      top = fmaxf(top, xor16(top));
      top = fmaxf(top, xor32(top));
      top = fmaxf(m, top);
      if (__ballot(top > m)) {
        const float alpha = exp2f((m - finite_max(top)) * p.scale_log2);
        l *= alpha;
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[n] *= alpha;
        m = top;
      }
      const float sub = finite_max(m);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = exp2f((x[i] - sub) * p.scale_log2);
      l += (x[0] + x[1]) + (x[2] + x[3]);
      f32x4 sum[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        unpack8(d.v[i], v);
#pragma unroll
        for (int n = 0; n < 8; ++n)
          sum[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[n], x[i], i == 0 ? zero : sum[n], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < 8; ++n) acc[n] += sum[n];
    };

    // the workgroup's waves take tiles in turn; the next tile's loads are in flight during a tile's arithmetic
    TileLoader<kSmallPages> tiles(p.c, at.seq, at.kv, rows);
    constexpr int kStep = TileLoader<kSmallPages>::kStep;
    int t = ra + wave * kPagedTile;
    if (t < rb) {
      PagedTile d0, d1;
      tiles.start(t);
      tiles.load(t, d0);
      while (true) {
        if (t + kStep >= rb) {
          attend(d0);
          break;
        }
        tiles.load(t + kStep, d1);
        attend(d0);
        t += kStep;
        if (t + kStep >= rb) {
          attend(d1);
          break;
        }
        tiles.load(t + kStep, d0);
        attend(d1);
        t += kStep;
      }
    }
    l += xor16(l);
    l += xor32(l);

    // merge the waves through LDS: lane (r, kq) holds dims 8 (4 kq + i) + n of head r
    if (r < n_live) {
      if (kq == 0) {
        s_m[wave][r] = m * p.scale_log2;
        s_l[wave][r] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 *dst = reinterpret_cast<float4 *>(&s_acc[wave][r][8 * (4 * kq + i)]);
        dst[0] = make_float4(acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
        dst[1] = make_float4(acc[4][i], acc[5][i], acc[6][i], acc[7][i]);
      }
    }
    // (what was known before is read before any of it may be overwritten)
    constexpr int kMost = kPagedHeads / (kPagedThreads / kHeadDim);
    const int d = tid % kHeadDim, j0 = tid / kHeadDim;
    float prior_o[kMost], prior_lse[kMost];
    if (p.whole && p.a.prior_lse) {
#pragma unroll
      for (int u = 0; u < kMost; ++u) {
        const int64_t head = head_first + min(j0 + u * (kPagedThreads / kHeadDim), n_live - 1);
        prior_o[u] = p.a.prior_out[head * kHeadDim + d];
        prior_lse[u] = p.a.prior_lse[head];
      }
    }
    __syncthreads();
    // thread t: dim t % 128 of heads t / 128, t / 128 + 2, ...
#pragma unroll
    for (int u = 0; u < kMost; ++u) {
      const int j = j0 + u * (kPagedThreads / kHeadDim);
      if (j >= n_live) break;
      Merged x{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) x.m = fmaxf(x.m, s_m[w][j]);
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) {
        const float wg = (s_m[w][j] == -INFINITY) ? 0.f : exp2f(s_m[w][j] - x.m);
        x.l += s_l[w][j] * wg;
        x.o += s_acc[w][j][d] * wg;
      }
      if (p.whole) {
        store_head(p, head_first + j, d, p.a.prior_lse ? prior_lse[u] : -INFINITY, p.a.prior_lse ? prior_o[u] : 0.f, x);
        continue;
      }
      float *P = p.partials + ((head_first + j) * p.splits + split) * kPartialStride;
      if (d == 0) {
        P[0] = x.m;
        P[1] = x.l;
      }
      P[2 + d] = x.o;
    }
    at.c = at.first = seg_end;
    if (at.c >= at.c_end) break;
    __syncthreads();  // LDS is reused by the next piece
    if (++at.kv == n_kv) {
      at.kv = 0;
      do at.rows = seq_rows(p, ++at.seq);
      while (at.rows.chunks() == 0);  // (a sequence with rows follows: chunks are left)
    }
  }
}

// One workgroup per head; its groups of 128 threads (one dimension each) take the pieces in turn, so that the partials of
// a head are fetched in a round or two of loads, and meet in LDS.
template <int kGroups>
__global__ __launch_bounds__(kGroups * kHeadDim) void paged_merge_kernel(PagedArgs p) {
  __shared__ float s_m[kGroups], s_l[kGroups], s_o[kGroups][kHeadDim];
  const int head = blockIdx.x, t = threadIdx.x % kHeadDim, grp = threadIdx.x / kHeadDim;
  const int seq = head / p.c.n_q_heads, kv = head % p.c.n_q_heads / p.c.group;
  const int chunks = seq_rows(p, seq).chunks();
  const int n_active = chunks ? paged_pieces(p, seq, kv, chunks) : 0;
  const float prior_lse = p.a.prior_lse ? p.a.prior_lse[head] : -INFINITY;
  const float prior_o = p.a.prior_lse ? p.a.prior_out[(int64_t)head * kHeadDim + t] : 0.f;
  const float *P = p.partials + (int64_t)head * p.splits * kPartialStride;
  constexpr int kBatch = 8;
  Merged x{-INFINITY, 0.f, 0.f};
  for (int s0 = grp; s0 < n_active; s0 += kGroups * kBatch) {
    float ms[kBatch], ll[kBatch], oo[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float *Q = P + min(s0 + kGroups * u, n_active - 1) * kPartialStride;
      ms[u] = Q[0];
      ll[u] = Q[1];
      oo[u] = Q[2 + t];
    }
    float Mn = x.m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + kGroups * u >= n_active) {
        ms[u] = -INFINITY;
        ll[u] = oo[u] = 0.f;
      }
      Mn = fmaxf(Mn, ms[u]);
    }
    const float sub = finite_max(Mn), sc = exp2f(x.m - sub);
    x.l *= sc;
    x.o *= sc;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float w = exp2f(ms[u] - sub);
      x.l = fmaf(ll[u], w, x.l);
      x.o = fmaf(oo[u], w, x.o);
    }
    x.m = Mn;
  }
  s_o[grp][t] = x.o;
  if (t == 0) {
    s_m[grp] = x.m;
    s_l[grp] = x.l;
  }
  __syncthreads();
  if (grp > 0) return;
  Merged all{s_m[0], 0.f, 0.f};
#pragma unroll
  for (int v = 1; v < kGroups; ++v) all.m = fmaxf(all.m, s_m[v]);
#pragma unroll
  for (int v = 0; v < kGroups; ++v) {
    const float w = exp2f(s_m[v] - finite_max(all.m));
    all.l = fmaf(s_l[v], w, all.l);
    all.o = fmaf(s_o[v][t], w, all.o);
  }
  store_head(p, head, t, prior_lse, prior_o, all);
}

// How a call is split; by sizes that the host knows.
struct Split {
  int whole, splits, min_share, grid;
};
Split split_of(const PagedView &c) {
  Split s;
  const long n_seg = (long)c.n_seqs * c.n_kv_heads, nh = (long)c.n_seqs * c.n_q_heads;
  const int max_chunks = (c.max_seq_len + kChunkRows - 1) / kChunkRows;
  s.whole = c.n_seqs > kDealtSeqs || c.max_seq_len <= (n_seg >= 512 ? 1024 : n_seg >= 128 ? 512 : 320);
  // partial slots per head: some thousand pieces in all, never more than a head has chunks
  long slots = 16384 / nh;
  slots = slots < 8 ? 8 : slots > kMaxSplits ? kMaxSplits : slots;
  s.splits = (int)(slots < max_chunks ? slots : max_chunks > 0 ? max_chunks : 1);
  // A segment of n chunks has at most ceil(n / share) + 1 pieces, and never more than n: the share is large enough for
  // the partial slots of a head.  One round of workgroups: two waves per SIMD x 256 CUs.
  s.min_share = 1;
  if (max_chunks > s.splits && s.splits > 1) s.min_share = (max_chunks + s.splits - 2) / (s.splits - 1);
  constexpr int kResident = 2 * 256;
  const long want = (n_seg * max_chunks + s.min_share - 1) / s.min_share;
  s.grid = (int)(want < 1 ? 1 : want < kResident ? want : kResident);
  return s;
}

}  // namespace

size_t paged_partials(const PagedView &c, const SharedView &) {
  const Split s = split_of(c);
  return s.whole ? 1 : (size_t)c.n_seqs * c.n_q_heads * s.splits * kPartialStride;
}

hipError_t launch_paged_decode(const PagedView &c, const PagedAttention &a, float *partials, const AttnOut &attn,
                               hipStream_t stream) {
  const Split s = split_of(c);
  PagedArgs p{c, a, attn, partials, 0, s.splits, s.min_share, s.grid, s.whole, c.sm_scale * kLog2e};
  const int nh = c.n_seqs * c.n_q_heads;
  const dim3 grid(s.whole ? c.n_seqs * c.n_kv_heads : s.grid), block(kPagedThreads);
  for (p.head0 = 0; p.head0 < c.group; p.head0 += kPagedHeads) {  // one pass over the rows for up to 16 heads of a group
    if (c.page_shift < 4)
      hipLaunchKernelGGL(paged_kernel<true>, grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL(paged_kernel<false>, grid, block, 0, stream, p);
  }
  if (s.whole) return hipGetLastError();
  if (nh >= 512 || c.max_seq_len <= 32 * kChunkRows)
    hipLaunchKernelGGL(paged_merge_kernel<1>, dim3(nh), dim3(kHeadDim), 0, stream, p);
  else
    hipLaunchKernelGGL(paged_merge_kernel<8>, dim3(nh), dim3(8 * kHeadDim), 0, stream, p);
  return hipGetLastError();
}

}  // namespace dp
