// Dense decode attention over the rows of a paged cache, one query token per sequence (Eq. 1 over pages).
//
// HBM-bound streaming kernel (512 B per row and KV head), both contractions on the matrix cores straight from global
// memory in the instructions' layouts, 16 rows x up to 16 query heads of a group per wave and step:
//   scores  S[16 rows x 16 heads] = K Q^T, four v_mfma_f32_16x16x32_bf16: lane l loads chunks l / 16 + 4 j of key row
//           l % 16 and receives the scores of head l % 16 for rows 4 (l / 16) + i, which become weights in place;
//   output  O^T[dims x heads] += V^T P^T, v_mfma_f32_16x16x16_bf16, k = 4 (l / 16) + i: the weights are where the scores
//           were, and of the values a lane loads dims 8 (l % 16) .. + 7 of its four rows and puts the rows of a dimension
//           side by side by byte permutes.  Tile n of eight holds dims 8 x + n.
// A weight goes into the product as three bf16 numbers that add up to its 24 bits, the first two cut, not rounded, none of
// them zero (an infinite value would become NaN).  The sum of the weights is taken from the fp32 weights.
// What is subtracted from a head's scores is a score that was its largest at some time, unscaled (the largest weight is in
// order whatever the size of the scores); it moves when one leads it by 8 in base 2: weights up to 2^8 lose nothing in fp32.
// A maximum of -inf is taken as the lowest finite number when it is subtracted.  A weight below 2^-126 of the largest counts
// as zero (v_exp_f32), also times an infinite value.
// Tiles begin at multiples of 16 rows, so a tile of pages of 16 tokens or more lies in one page: its place is a scalar and
// a lane's offsets are the same for every tile.  The numbers of the pages of a wave's next 64 tiles are fetched by its 64
// lanes at once.  Smaller pages: every row's page by the lane that loads the row's key, a tile ahead of the rows (16 sequences
// of up to 65536 rows, pages of 1, 2, 4, 8 tokens 435, 451, 426, 422 us per call, of 16 and 64 412 and 403; tokens outermost
// 435, 425, 419, 416, 410, 410).
// A tile has a mask of 16 rows (inside [first, len) and on a page that is there); rows without a bit score -inf and their
// values are made zero: they may hold anything.
// Work split: the rows of all (sequence, KV head) segments, in chunks of 64, are dealt out evenly to one round of resident
// workgroups; pieces are merged by a second kernel.  Short or very many segments are taken whole, a workgroup each, which
// then writes the output itself.  Where the heads of a token lie side by side a workgroup's waves take the same rows of four
// KV heads (chunks of 16 rows), not a head's rows in turn: what lies next to each other is read at one time.
// Measured (8 KV heads, G = 4): 16 sequences of up to 65536 rows, 2.6 GB, 399 us = 6.5 TB/s, 94 % of what the longest plain
// stream reads here (the matrix cores are busy 16 % of it); one of 131072 rows 82.8 us (6.5 TB/s) and 6.9 for the merge;
// heads side by side, G = 8, four of 131072 rows 332 us (6.5 TB/s; 372 with a head per workgroup).  Two tiles per wave in
// registers, one of them in flight, two waves per SIMD; with a third tile the registers do not suffice (131072 rows: 97 us).
#include "dp_attend.hpp"
#include "dp_device.hpp"
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedThreads = 256;
constexpr int kPagedWaves = kPagedThreads / 64;
constexpr int kPagedHeads = 16;  // query heads per pass: the columns of one MFMA tile
constexpr int kPagedTile = 16;   // rows per wave and step
__device__ __forceinline__ uint32_t part_of(const uint4 &v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// one wave's 16 rows as the two contractions want them, and which of them count
struct PagedTile {
  uint4 k[4], v[4];
  uint32_t live;
};

// Fetches tiles of one segment: rows t .. t + 15, t a multiple of 16, of the wave's tiles t0, t0 + kStep, ...
template <bool kSmallPages, int kStep>
struct TileLoader {
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
  // (a row behind the last, whose entry may not be read: the last one's page)
  __device__ __forceinline__ int page_of(int row) const { return table[min(row, rows.len - 1) >> c.page_shift]; }
  __device__ __forceinline__ void start(int t) {
    t0 = t;
    page = page_of(kSmallPages ? t + (lane_id() & 15) : t + lane_id() * kStep);
    asm volatile("" ::"v"(page));  // waited for here: in front of a tile's loads all loads would be waited for
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
      // (offsets that are widened here, not once for all tiles: the loads then take a scalar base and 32 bits of offset)
      uint32_t ko = k_off, vo = v_off;
      asm volatile("" : "+v"(ko), "+v"(vo));
#pragma unroll
      for (int j = 0; j < 4; ++j) d.k[j] = load_stream16(kr + ko + j * 64);
#pragma unroll
      for (int i = 0; i < 4; ++i) d.v[i] = load_stream16(vr + i * (int64_t)c.slot_stride + vo);
    } else {
      const int r = lane_id() & 15, kq = lane_id() >> 4;
      const int next = page_of(t + kStep + r);  // (in front of the rows: it is waited for before they are)
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
      page = next;
    }
    d.live = live;
  }
};

// ---- output of a head: partial results and what was known before ----
// (maxima as scaled scores: in base 2 the lowest numbers there are would pass the range)
struct Merged {
  float m, l, o;  // maximum, sum, accumulator of one dimension
};
__device__ __forceinline__ float weight_of(float m, float sub) { return exp2f((m - sub) * kLog2e); }
__device__ __forceinline__ void store_head(const PagedArgs &p, int64_t head, int d, float prior, float prior_o, Merged x) {
  const float M = fmaxf(x.m, prior), sub = finite_max(M);
  const float w = weight_of(x.m, sub), wp = weight_of(prior, sub);
  const float L = fmaf(x.l, w, wp);
  float o = x.m > -INFINITY ? x.o * w : 0.f;
  if (prior > -INFINITY) o = fmaf(prior_o, wp, o);  // (a prior without weight may hold anything)
  // Nothing attended: a sum of exactly zero, for a row whose score is subtracted, or the prior, has a weight of one.  A score
  // or a prior of NaN or +inf leaves a sum of NaN, and that is the result.
  const bool none = L == 0.f;
  store_out(p.attn.out, p.attn.out_is_bf16, head, d, none ? 0.f : o / L);
  if (p.attn.lse && d == 0) p.attn.lse[head] = none ? -INFINITY : fmaf(log2f(L), kLn2, M);
}

template <bool kSmallPages, bool kShared, int kSpan>
__global__ __launch_bounds__(kPagedThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_kernel(PagedArgs p) {
  __shared__ float s_m[kPagedWaves][kPagedHeads], s_l[kPagedWaves][kPagedHeads], s_prior[kPagedHeads];
  __shared__ __align__(16) float s_acc[kPagedWaves][kPagedHeads][kHeadDim + 4];
  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int r = lane & 15, kq = lane >> 4;
  constexpr int kRows = own_chunk(kSpan);
  const int n_kv = p.c.n_kv_heads, group = p.c.group, n_live = min(kPagedHeads, group - p.head0);
  Dealt at;
  if (p.whole) {
    at.i = blockIdx.x / n_kv;
    at.sub = blockIdx.x % n_kv;
    at.item = own_segments<kShared, kSpan>(p)(at.i);
    at.first = at.c = 0;
    at.c_end = at.item.chunks;
    at.share = 1;
  } else if (!deal_start(p.own, blockIdx.x, p.c.n_seqs, own_segments<kShared, kSpan>(p), at)) {
    return;
  }

  // one piece of a segment after the other, usually one
  while (true) {
    const SeqRows rows{at.item.a, at.item.b};
    const int seg_end = at.first + at.item.chunks;
    const int ra = (rows.first / kRows + at.c - at.first) * kRows;
    const int rb = min(rows.len, (rows.first / kRows + min(at.c_end, seg_end) - at.first) * kRows);
    const int split = p.whole ? 0 : blockIdx.x - at.first / at.share;  // number of the piece inside its segment
    const int kv = kSpan == 1 ? at.sub : at.sub * kSpan + wave;
    const int64_t head_first = (int64_t)at.i * p.c.n_q_heads + kv * group + p.head0;

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
    float m = -INFINITY, l = 0.f;  // head r: the score that is subtracted, the weights of this lane's rows

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
      if (__ballot(top > m + p.lead)) {
        const float alpha = __builtin_amdgcn_exp2f((m - finite_max(top)) * p.scale_log2);
        l *= alpha;
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[n] *= alpha;
        m = top;
      }
      const float sub = finite_max(m);
      bf16x4 piece[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = __builtin_amdgcn_exp2f((x[i] - sub) * p.scale_log2);
        x[i] = w;
        float rest = w;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          piece[q][i] = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(rest) >> 16));
          rest -= __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
        }
        piece[2][i] = (__bf16)rest;
      }
#pragma unroll
      for (int q = 1; q < 3; ++q) piece[q] = not_zero<u16x4>(piece[q], piece[0]);
      l += (x[0] + x[1]) + (x[2] + x[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // dims 2 j, 2 j + 1 of the lane's eight: the four rows' values side by side
        const uint32_t w0 = part_of(d.v[0], j), w1 = part_of(d.v[1], j), w2 = part_of(d.v[2], j), w3 = part_of(d.v[3], j);
        const s16x4 even = __builtin_bit_cast(s16x4, make_uint2(__builtin_amdgcn_perm(w1, w0, 0x05040100),
                                                                __builtin_amdgcn_perm(w3, w2, 0x05040100)));
        const s16x4 odd = __builtin_bit_cast(s16x4, make_uint2(__builtin_amdgcn_perm(w1, w0, 0x07060302),
                                                               __builtin_amdgcn_perm(w3, w2, 0x07060302)));
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          const s16x4 w = __builtin_bit_cast(s16x4, piece[q]);
          acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(even, w, acc[2 * j], 0, 0, 0);
          acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(odd, w, acc[2 * j + 1], 0, 0, 0);
        }
      }
    };

    // the workgroup's waves take tiles in turn, or a KV head each; the next tile's loads are in flight during a tile's arithmetic
    constexpr int kStep = kSpan == 1 ? kPagedWaves * kPagedTile : kPagedTile;
    TileLoader<kSmallPages, kStep> tiles(p.c, at.i, kv, rows);
    int t = kSpan == 1 ? ra + wave * kPagedTile : ra;
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
        s_m[wave][r] = m * p.c.sm_scale;
        s_l[wave][r] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 *dst = reinterpret_cast<float4 *>(&s_acc[wave][r][8 * (4 * kq + i)]);
        dst[0] = make_float4(acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
        dst[1] = make_float4(acc[4][i], acc[5][i], acc[6][i], acc[7][i]);
      }
    }
    const bool direct = kSpan == 1 && !kShared && p.whole;
    if (kSpan == 1 && !kShared) {  // (read before any of it may be overwritten)
      if (tid < n_live) s_prior[tid] = direct && p.a.prior_lse ? p.a.prior_lse[head_first + tid] : -INFINITY;
    }
    __syncthreads();
    if constexpr (kSpan > 1) {  // a KV head per wave: nothing to merge
      for (int j = 0; j < n_live; ++j) {
        const int64_t slot = (head_first + j) * p.parts.all + split;
        reinterpret_cast<float2 *>(p.parts.acc + slot * kHeadDim)[lane] = reinterpret_cast<const float2 *>(s_acc[wave][j])[lane];
        if (lane == 0) {
          p.parts.ml[slot] = make_float2(s_m[wave][j], s_l[wave][j]);
          if (split == 0) p.parts.pieces[2 * (head_first + j)] = pieces_of(at);
        }
      }
    }
    // thread t: dim t % 128 of heads t / 128, t / 128 + 2, ...
    const int d = tid % kHeadDim;
#pragma unroll 2
    for (int j = tid / kHeadDim; kSpan == 1 && j < n_live; j += kPagedThreads / kHeadDim) {
      const float prior_o = direct && p.a.prior_lse ? p.a.prior_out[(head_first + j) * kHeadDim + d] : 0.f;
      Merged x{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) x.m = fmaxf(x.m, s_m[w][j]);
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) {
        const float wg = weight_of(s_m[w][j], finite_max(x.m));
        x.l += s_l[w][j] * wg;
        x.o += s_acc[w][j][d] * wg;
      }
      if (direct) {
        store_head(p, head_first + j, d, s_prior[j], prior_o, x);
        continue;
      }
      const int64_t slot = (head_first + j) * p.parts.all + split;
      p.parts.acc[slot * kHeadDim + d] = x.o;
      if (d == 0) {
        p.parts.ml[slot] = make_float2(x.m, x.l);
        if (split == 0) p.parts.pieces[2 * (head_first + j)] = p.whole ? 1 : pieces_of(at);
      }
    }
    if (seg_end >= at.c_end) break;
    __syncthreads();  // LDS is reused by the next piece
    deal_next(own_segments<kShared, kSpan>(p), at);
  }
}

// One workgroup per head: sum over its slots of e^(m - M) (sum, accumulator).  A chain of dependent loads and launch bound:
// a slot's 128 dimensions are taken by 32 lanes, four each, so that a head's partials are fetched in a round or two of loads;
// the groups of 32 meet in LDS.  32 heads of some 64 slots 6.2 us, 2048 heads of 36 slots (38 MB) 8.9, of which 3 are any
// launch's.
template <int kThreads, bool kShared>
__global__ __launch_bounds__(kThreads) void paged_merge_kernel(PagedArgs p) {
  constexpr int kGroups = kThreads / 32, kBatch = 8;
  __shared__ float s_m[kGroups], s_l[kGroups];
  __shared__ __align__(16) float s_o[kGroups][kHeadDim];
  const int head = blockIdx.x, t = threadIdx.x % 32, grp = threadIdx.x / 32;
  const int2 pieces = reinterpret_cast<const int2 *>(p.parts.pieces)[head];  // (left alone where there are no rows)
  const float prior_lse = p.a.prior_lse ? p.a.prior_lse[head] : -INFINITY;
  const float prior_o = p.a.prior_lse && threadIdx.x < kHeadDim ? p.a.prior_out[(int64_t)head * kHeadDim + threadIdx.x] : 0.f;
  const SeqRows rows = seq_rows<kShared>(p, head / p.c.n_q_heads);
  const int n_own = rows.first < rows.len || p.whole ? pieces.x : 0;
  const int n_active = n_own + (kShared && rows.first > 0 ? pieces.y : 0);
  const int64_t slot0 = (int64_t)head * p.parts.all;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = grp; s0 < n_active; s0 += kGroups * kBatch) {
    float2 ml[kBatch];
    float4 oo[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      int s = min(s0 + kGroups * u, n_active - 1);
      s = s < n_own ? s : s - n_own + p.parts.own;
      ml[u] = p.parts.ml[slot0 + s];
      oo[u] = reinterpret_cast<const float4 *>(p.parts.acc + (slot0 + s) * kHeadDim)[t];
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + kGroups * u >= n_active) ml[u] = make_float2(-INFINITY, 0.f);
      top = fmaxf(top, ml[u].x);
    }
    const float sub = finite_max(top), sc = weight_of(m, sub);
    l *= sc;
    o.x *= sc; o.y *= sc; o.z *= sc; o.w *= sc;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float w = weight_of(ml[u].x, sub);
      l = fmaf(ml[u].y, w, l);
      if (s0 + kGroups * u < n_active) {
        o.x = fmaf(oo[u].x, w, o.x);
        o.y = fmaf(oo[u].y, w, o.y);
        o.z = fmaf(oo[u].z, w, o.z);
        o.w = fmaf(oo[u].w, w, o.w);
      }
    }
    m = top;
  }
  reinterpret_cast<float4 *>(s_o[grp])[t] = o;
  if (t == 0) {
    s_m[grp] = m;
    s_l[grp] = l;
  }
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  Merged all{s_m[0], 0.f, 0.f};
#pragma unroll
  for (int v = 1; v < kGroups; ++v) all.m = fmaxf(all.m, s_m[v]);
#pragma unroll
  for (int v = 0; v < kGroups; ++v) {
    const float w = weight_of(s_m[v], finite_max(all.m));
    all.l = fmaf(s_l[v], w, all.l);
    all.o = fmaf(s_o[v][threadIdx.x], w, all.o);
  }
  store_head(p, head, threadIdx.x, prior_lse, prior_o, all);
}

// How a call is split; by sizes that the host knows.
struct Split {
  int whole, span, cols;  // own rows; shared rows: columns of a workgroup
  Deal own, shared;
};
int at_most(long n, long most) { return (int)(n < most ? n : most); }
int at_least(long n, long least) { return (int)(n > least ? n : least); }

Split split_of(const PagedView &c, const SharedView &shared) {
  Split s{};
  const long n_seg = (long)c.n_seqs * c.n_kv_heads, nh = (long)c.n_seqs * c.n_q_heads;
  const int max_chunks = (c.max_seq_len + kChunkRows - 1) / kChunkRows;
  // Whole segments against dealt-out chunks, us, G = 4, pages of 16 (segments of equal length): 8 segments of 512 rows 9.1 /
  // 10.0, of 768 11.3 / 9.9; 64 of 512 10.8 / 11.9, of 768 14.3 / 13.5; 128 of 768 15.7 / 15.7, of 1024 19.6 / 18.6; 256 of
  // 1536 33.4 / 38.1, ragged ones of up to 2048 36.0 / 34.2; 512 of 1024 43.2 / 48.0, ragged of up to 2048 67.6 / 63.6.
  // (By the bound of the lengths.  One of 131072 instead of the longest: 1 x 1000 rows of one KV head 9.3 -> 10.7 us per call, of 8
  // KV heads 1 x 4096 11.7 -> 13.7, 32 ragged of up to 700 14.9 -> 19.5, 64 x 512 23.3 -> 28.1, 16 x 4096 no change.)
  s.whole = c.n_seqs > kDealtItems || c.max_seq_len <= (n_seg >= 256 ? 1536 : n_seg >= 128 ? 768 : 640);
  // Shared rows are read once where that saves more than 48 MiB of reads and 4 MiB per sequence: below, the launches that it
  // takes cost more than the reads, which find much of what is shared in the caches.  us, shared once / every sequence for
  // itself (G = 4, 8 KV heads, 100 rows of their own): 4 sequences, 4096 rows 22.4 / 21.6, 8192 rows 25.0 / 30.7; 16
  // sequences, 1024 rows 22.1 / 19.8, 2048 rows 26.0 / 29.0; 64 sequences, 1024 rows 36.5 / 29.3, 2048 rows 42.1 / 53.7;
  // 1 KV head: 64 sequences, 4096 rows 29.3 / 24.3, 8192 rows 33.6 / 42.2.
  const long saved = ((long)c.n_seqs - at_most(shared.n_groups, kDealtItems)) * shared.max_shared_len * c.n_kv_heads * (2 * kRowBytes);
  const bool any_shared = shared.n_groups > 0 && shared.max_shared_len > 0 && shared.n_groups <= kDealtItems &&
                          (shared.once || saved > (48l << 20) + (4l << 20) * c.n_seqs);
  // Where the heads of a token lie side by side (pages with the tokens outermost) a workgroup takes the same rows of four
  // heads, a wave each: 1 KB next to each other, and neighbouring workgroups the rest, where waves of one head alone read
  // 256 bytes here and there.  us, a head per workgroup / four (8 KV heads, G = 4): 16 sequences of up to 65536 rows 450 /
  // 397, one of 131072 102 / 92, of 32768 33.4 / 31.7, 64 of 2048 99 / 91.  Shorter, the steps of a wave are too few and the
  // pieces to merge too many: one of 8192 16.7 / 17.3, four of 4096 20.1 / 21.5; 4 KV heads, one of 65536 30.8 / 32.1.
  // (Behind shared rows: by the rows beyond them.)
  const int own_chunks = max_chunks - (any_shared ? shared.max_shared_len / kChunkRows : 0);
  const bool heads_together = c.head_stride < (c.page_shift ? (int64_t)c.slot_stride : c.page_stride);
  s.span = !s.whole && heads_together && c.n_kv_heads % kPagedWaves == 0 && n_seg >= 2 * kPagedWaves && n_seg * own_chunks >= 4096
               ? kPagedWaves : 1;
  // one round of workgroups (two waves per SIMD x 256 CUs), and partial slots for some thousand pieces in all
  s.own.grid = at_least(at_most(n_seg * max_chunks, 2 * 256), 1);
  // (four heads per workgroup: a quarter of the segments, so four times as many pieces of each)
  const int pieces = s.span > 1 ? at_most(at_least(32768 / nh, 8), kMaxSplits + 1) : at_most(at_least(16384 / nh, 8), kMaxSplits);
  s.own.slots = s.whole ? 1 : at_least(at_most(s.span * max_chunks, pieces), 1);
  if (!any_shared) return s;
  const long cols = (long)(shared.max_group_seqs < c.n_seqs ? shared.max_group_seqs : c.n_seqs) * c.group;
  s.cols = cols <= 128 ? 128 : 256;
  // one workgroup per CU; a segment has at most ceil(grid / KV heads) + 1 pieces
  s.shared.grid = 256;
  const int max_blocks = (shared.max_shared_len + kSharedBlock - 1) / kSharedBlock;
  s.shared.slots = at_most(at_most(max_blocks, s.shared.grid / c.n_kv_heads + 2), at_least(131072 / nh, 8));
  return s;
}

template <bool kShared>
void launch_own(const PagedArgs &p, hipStream_t stream) {
  const dim3 grid(p.whole ? p.c.n_seqs * p.c.n_kv_heads : p.own.grid);
  const bool small = p.c.page_shift < 4;
  const auto kernel = p.span > 1 ? small ? paged_kernel<true, kShared, kPagedWaves> : paged_kernel<false, kShared, kPagedWaves>
                                 : small ? paged_kernel<true, kShared, 1> : paged_kernel<false, kShared, 1>;
  hipLaunchKernelGGL(kernel, grid, dim3(kPagedThreads), 0, stream, p);
}

template <bool kShared>
void launch_merge(const PagedArgs &p, hipStream_t stream) {
  const int nh = p.c.n_seqs * p.c.n_q_heads;
  if (p.parts.all <= 32)
    hipLaunchKernelGGL((paged_merge_kernel<128, kShared>), dim3(nh), dim3(128), 0, stream, p);
  else if (p.parts.all <= 64 || nh >= 256)
    hipLaunchKernelGGL((paged_merge_kernel<256, kShared>), dim3(nh), dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((paged_merge_kernel<1024, kShared>), dim3(nh), dim3(1024), 0, stream, p);
}

}  // namespace

size_t paged_partials(const PagedView &c, const SharedView &shared) {
  const Split s = split_of(c, shared);
  const size_t slots = s.whole && !s.shared.slots ? 0 : (size_t)s.own.slots + s.shared.slots;
  return slots ? (size_t)c.n_seqs * c.n_q_heads * (slots * (kHeadDim + 2) + 2) : 1;
}

hipError_t launch_paged_decode(const PagedView &c, const PagedAttention &a, float *partials, const AttnOut &attn,
                               hipStream_t stream) {
  const Split s = split_of(c, a.shared);
  PagedArgs p{};
  p.c = c;
  p.a = a;
  p.attn = attn;
  p.parts.own = s.own.slots;
  p.parts.all = s.own.slots + s.shared.slots;
  p.parts.acc = partials;
  p.parts.ml = reinterpret_cast<float2 *>(partials + (size_t)c.n_seqs * c.n_q_heads * p.parts.all * kHeadDim);
  p.parts.pieces = reinterpret_cast<int32_t *>(p.parts.ml + (size_t)c.n_seqs * c.n_q_heads * p.parts.all);
  p.whole = s.whole;
  p.span = s.span;
  p.own = s.own;
  p.shared = s.shared;
  p.shared_cols = s.cols;
  p.scale_log2 = c.sm_scale * kLog2e;
  p.lead = fminf(8.f / p.scale_log2, 3e38f);
  if (s.shared.slots) launch_shared_rows(p, stream);
  // one pass over the rows for up to 16 heads of a group (131072 rows of 8 KV heads, G = 16 92 us, 17 175, 32 180)
  for (p.head0 = 0; p.head0 < c.group; p.head0 += kPagedHeads) {
    if (s.shared.slots)
      launch_own<true>(p, stream);
    else
      launch_own<false>(p, stream);
  }
  if (s.shared.slots)
    launch_merge<true>(p, stream);
  else if (!s.whole)
    launch_merge<false>(p, stream);
  return hipGetLastError();
}

}  // namespace dp
