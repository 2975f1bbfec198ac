// Dense decode attention over the rows of a paged cache, one query token per sequence (Eq. 1 over pages): device code of
// the kernels that attend each sequence's own rows.
//
// HBM-bound streaming kernel (512 B per row and KV head), both contractions on the matrix cores straight from global
// memory in the instructions' layouts, 16 rows x up to 16 query heads of a group per wave and step:
//   scores  S[16 rows x 16 heads] = K Q^T, four v_mfma_f32_16x16x32_bf16: lane l loads chunks l / 16 + 4 j of key row
//           l % 16 and receives the scores of head l % 16 for rows 4 (l / 16) + i, which become weights in place;
//   output  O^T[dims x heads] += V^T P^T, v_mfma_f32_16x16x4_f32 with k = l / 16 standing for row 4 (l / 16) + i: the
//           weights stay fp32, the values are widened; tile n of eight holds dims 8 x + n.  A tile's 16 rows are summed by
//           themselves and then added: the fp32 chain is as long as the wave has tiles, not rows.
// What is subtracted from a head's scores is a score that was its largest at some time, unscaled (the largest weight is in
// order whatever the size of the scores); it moves when one leads it by 8 in base 2: weights up to 2^8 lose nothing in fp32.
// A maximum of -inf is taken as the lowest finite number when it is subtracted; weights keep the range below 2^-126 (exp2f).
// Tiles begin at multiples of 16 rows, so a tile of pages of 16 tokens or more lies in one page: its place is a scalar and
// a lane's offsets are the same for every tile.  The numbers of the pages of a wave's next 64 tiles are fetched by its 64
// lanes at once.  Smaller pages: every row's page by the lane that loads the row's key, a tile ahead of the rows.
// A tile has a mask of 16 rows (inside [first, len) and on a page that is there); rows without a bit score -inf and their
// values are made zero: they may hold anything.
// Work split: the rows of all (sequence, KV head) segments, in chunks of 64, are dealt out evenly to one round of resident
// workgroups; pieces are merged by a second kernel.  Short or very many segments are taken whole, a workgroup each, which
// then writes the output itself.
#pragma once

#include "dp_attend.hpp"
#include "dp_device.hpp"
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedHeads = 16;  // query heads per pass: the columns of one MFMA tile
constexpr int kPagedTile = 16;   // rows per wave and step
// one wave's 16 rows as the two contractions want them, and which of them count
struct PagedTile {
  uint4 k[4], v[4];
  uint32_t live;
};

// Fetches tiles of one segment: rows t .. t + 15, t a multiple of 16, of the wave's tiles t0, t0 + kStep, ...
template <bool kSmallPages, int kWaves>
struct TileLoader {
  static constexpr int kStep = kWaves * kPagedTile;
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
#pragma unroll
      for (int j = 0; j < 4; ++j) d.k[j] = load_stream16(kr + (k_off + j * 64));
#pragma unroll
      for (int i = 0; i < 4; ++i) d.v[i] = load_stream16(vr + (v_off + i * c.slot_stride));
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

template <int kWaves>
struct PagedLds {
  float m[kWaves][kPagedHeads], l[kWaves][kPagedHeads], prior[kPagedHeads];
  __attribute__((aligned(16))) float acc[kWaves][kPagedHeads][kHeadDim + 4];
};

// The `block`-th workgroup's share of the own rows of all sequences.
template <bool kSmallPages, bool kShared, int kWaves>
__device__ __forceinline__ void paged_rows(const PagedArgs &p, int block, PagedLds<kWaves> &lds) {
  constexpr int kThreads = 64 * kWaves;
  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int r = lane & 15, kq = lane >> 4;
  const int n_kv = p.c.n_kv_heads, group = p.c.group, n_live = min(kPagedHeads, group - p.head0);
  Dealt at;
  if (p.whole) {
    at.i = block / n_kv;
    at.sub = block % n_kv;
    at.item = own_segments<kShared>(p)(at.i);
    at.first = at.c = 0;
    at.c_end = at.item.chunks;
    at.share = 1;
  } else if (!deal_start(p.own, block, p.c.n_seqs, own_segments<kShared>(p), at)) {
    return;
  }

  // one piece of a segment after the other, usually one
  while (true) {
    const SeqRows rows{at.item.a, at.item.b};
    const int seg_end = at.first + at.item.chunks;
    const int ra = (rows.chunk0() + at.c - at.first) * kChunkRows;
    const int rb = min(rows.len, (rows.chunk0() + min(at.c_end, seg_end) - at.first) * kChunkRows);
    const int split = p.whole ? 0 : block - at.first / at.share;  // number of the piece inside its segment
    const int64_t head_first = (int64_t)at.i * p.c.n_q_heads + at.sub * group + p.head0;

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
    TileLoader<kSmallPages, kWaves> tiles(p.c, at.i, at.sub, rows);
    constexpr int kStep = kWaves * kPagedTile;
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
        lds.m[wave][r] = m * p.scale_log2;
        lds.l[wave][r] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 *dst = reinterpret_cast<float4 *>(&lds.acc[wave][r][8 * (4 * kq + i)]);
        dst[0] = make_float4(acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
        dst[1] = make_float4(acc[4][i], acc[5][i], acc[6][i], acc[7][i]);
      }
    }
    const bool direct = !kShared && p.whole;
    if (!kShared) {  // (read before any of it may be overwritten)
      if (tid < n_live) lds.prior[tid] = direct && p.a.prior_lse ? p.a.prior_lse[head_first + tid] : -INFINITY;
    }
    __syncthreads();
    // thread t: dim t % 128 of heads t / 128, t / 128 + 2, ...
    const int d = tid % kHeadDim;
#pragma unroll 2
    for (int j = tid / kHeadDim; j < n_live; j += kThreads / kHeadDim) {
      const float prior_o = direct && p.a.prior_lse ? p.a.prior_out[(head_first + j) * kHeadDim + d] : 0.f;
      Merged x{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x.m = fmaxf(x.m, lds.m[w][j]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float wg = (lds.m[w][j] == -INFINITY) ? 0.f : exp2f(lds.m[w][j] - x.m);
        x.l += lds.l[w][j] * wg;
        x.o += lds.acc[w][j][d] * wg;
      }
      if (direct) {
        store_head(p, head_first + j, d, lds.prior[j], prior_o, x);
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
    deal_next(own_segments<kShared>(p), at);
  }
}

}  // namespace dp
