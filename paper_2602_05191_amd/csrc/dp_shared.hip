// Decode attention over rows that a group of sequences shares (a common beginning of their contexts), once for all of them.
//
// The columns are the queries of all sequences of the group, G per sequence: with tens of columns and more the products
// are large enough for the matrix cores' bf16 rate, and the rows are read once for all of them.
//   scores  S^T[32 rows x 32 columns] = K Q^T, v_mfma_f32_32x32x16_bf16, the keys from LDS, the queries in registers: a
//           lane holds 16 scores of column lane % 32, rows 8 (i / 4) + 4 (lane / 32) + i % 4;
//   output  O^T[dims x columns] += V^T P^T, the same instruction: weights i = 8 n .. 8 n + 7 of a lane are the k = 8
//           (lane / 32) .. + 7 of the n-th 16 rows if the values come in that order of rows, and they do: ds_read_tr16_b64
//           hands a lane one dimension of four consecutive rows, two of them the eight rows 16 n + 4 (lane / 32) + {0 .. 3,
//           8 .. 11}.  Nothing moves between lanes but the two halves' maxima.
// Weights go into the product in bf16 pieces that add up: two (16 bits) for a bf16 output, three (all 24) for fp32; their
// sum is taken from the fp32 weights.  (One piece rounds a weight by up to 2^-9, as much as the output itself is rounded.)
// All but the last piece are cut, not rounded, and none is zero (an infinite value would become NaN).
// A weight below 2^-126 of the largest counts as zero here (v_exp_f32), also times an infinite value.
// What is subtracted from a column's scores is a score that was its largest at some time; it moves when one leads it by 8 in
// base 2 (weights up to 2^8 lose nothing in fp32 or in pieces).  Moving with every new maximum, some of a wave's columns
// had one in most tiles.
//
// A workgroup is eight waves, two per SIMD.  A wave owns 32 columns of all rows of a block (256 columns per workgroup) or of
// half of them (128).  The scores of a tile of 32 rows are taken while the weights of the tile before are made: the matrix
// cores and the vector ALU have work of the same wave at the same time.
// Blocks of 64 rows go global -> registers -> LDS, two blocks ahead of the products (three buffers, one barrier per block);
// LDS rows are padded to 272 (keys) and 288 (values) bytes.
// Measured: 64 sequences x 4 heads, 32768 rows, 8 KV heads (256 columns, 134 MB, 34 GFLOP, 52 with the weights' second
// piece): 67 to 73 us = 0.77 to 0.71 PFLOP/s of instructions, the rows read once (135 MB).  No unit is full: matrix cores 41 %
// busy, vector ALU 38, LDS 24; a loop of the matrix instruction would take 31 us, HBM 20.
#include "dp_attend.hpp"
#include "dp_device.hpp"
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 *LdsTile;

constexpr int kSharedWaves = 8, kSharedThreads = 64 * kSharedWaves;
constexpr int kWaveCols = 32;
constexpr int kKPitch = 272, kVPitch = 288;  // bytes of a row in LDS
constexpr int kBuffer = kSharedBlock * (kKPitch + kVPitch);
constexpr int kLoads = kSharedBlock * 16 / kSharedThreads;  // 16-byte loads of a thread per block, of keys and of values
typedef unsigned long long Mask;                            // one bit per row of a block

// kCols waves along the columns, 8 / kCols along the rows of a block
template <int kCols, int kPieces>
__global__ __launch_bounds__(kSharedThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_kernel(PagedArgs p) {
  constexpr int kParts = kSharedWaves / kCols, kSubs = 2 / kParts;  // kSubs: 32-row tiles of a wave in a block
  __shared__ __align__(16) char s_rows[3][kBuffer];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int col_wave = wave / kParts, part = wave % kParts, half = lane >> 5;
  const PagedView &c = p.c;
  Dealt at;
  if (!deal_start(p.shared, blockIdx.x, p.a.shared.n_groups, shared_segments(p), at)) return;

  while (true) {
    const SharedGroup grp = shared_group(c, p.a.shared, at.i);
    const int tiles = at.item.subs / c.n_kv_heads, kv = at.sub / tiles;
    const int col0 = at.sub % tiles * p.shared_cols + kWaveCols * col_wave, n_cols = (grp.end - grp.begin) * c.group;
    const int split = blockIdx.x - at.first / at.share, seg_end = at.first + at.item.chunks;
    const int per = shared_blocks(n_cols), block0 = (at.c - at.first) * per;
    const int block1 = min((min(at.c_end, seg_end) - at.first) * per, (grp.rows + kSharedBlock - 1) / kSharedBlock);
    const int32_t *table = c.table + (int64_t)grp.reader * c.table_stride;
    const bool busy = col0 < n_cols;

    // ---- a block's rows: 16 lanes per row, four rows per wave and load; the pages of its 64 rows are looked up by 64
    // lanes, a block ahead of the rows.  (A lane that has no page to read from reads page 0.)
    const char *k_head = c.k_pages + kv * c.head_stride, *v_head = c.v_pages + kv * c.head_stride;
    const int in_page = (1 << c.page_shift) - 1;
    const uint32_t lane_off = (lane >> 4) * c.slot_stride + (lane & 15) * 16;
    int page;
    struct Rows {
      uint4 k[kLoads], v[kLoads];
      Mask there;
    };
    auto look_up = [&](int block) { page = table[min(block * kSharedBlock + lane, grp.rows - 1) >> c.page_shift]; };
    auto fetch = [&](int block, Rows &r) {
      const bool there = (uint32_t)page < (uint32_t)c.n_pages;
      r.there = __ballot(there && block * kSharedBlock + lane < grp.rows);
      page = there ? page : 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int quad = i * (4 * kSharedWaves) + 4 * wave;
        if (c.page_shift >= 2) {  // four rows in one page
          const int64_t at = lane_u32(page, quad) * c.page_stride +
                             ((block * kSharedBlock + quad) & in_page) * (int64_t)c.slot_stride;
          r.k[i] = load_stream16(k_head + at + lane_off);
          r.v[i] = load_stream16(v_head + at + lane_off);
        } else {
          const int row = quad + (lane >> 4);
          const int64_t at = __shfl(page, row, 64) * c.page_stride +
                             ((block * kSharedBlock + row) & in_page) * (int64_t)c.slot_stride + (lane & 15) * 16;
          r.k[i] = load_stream16(k_head + at);
          r.v[i] = load_stream16(v_head + at);
        }
      }
    };
    auto put = [&](Rows &r, char *buffer) {  // (values of rows that are not there: zero)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = i * (4 * kSharedWaves) + 4 * wave + (lane >> 4);
        if (r.there != ~0ull && !(r.there >> row & 1)) r.v[i] = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(buffer + row * kKPitch + (lane & 15) * 16) = r.k[i];
        *reinterpret_cast<uint4 *>(buffer + kSharedBlock * kKPitch + row * kVPitch + (lane & 15) * 16) = r.v[i];
      }
    };
    Mask live, live1;  // rows that are there, of the block being attended and of the next one
    look_up(block0);

    // the lane's column: a query head of one of the sequences
    const int col = col0 + (lane & 31), col_in = min(col, n_cols - 1), col_seq = grp.begin + col_in / c.group;
    const int64_t head = (int64_t)col_seq * c.n_q_heads + kv * c.group + col_in % c.group;
    const bool mine = col < n_cols && paged_len(c, col_seq) >= grp.rows;
    uint4 Q[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      Q[k] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(p.a.q) + head * kRowBytes + k * 32 + half * 16);
    {
      Rows r0, r1;
      fetch(block0, r0);
      look_up(block0 + 1);
      fetch(block0 + 1, r1);
      look_up(block0 + 2);
      put(r0, s_rows[0]);
      put(r1, s_rows[1]);
      live = r0.there;
      live1 = r1.there;
    }
    // (the queries are waited for here: a load that is pending when the loop begins would be waited for in it, and the
    // next block's rows with it)
#pragma unroll
    for (int k = 0; k < 8; ++k) asm volatile("" ::"v"(Q[k].x), "v"(Q[k].y), "v"(Q[k].z), "v"(Q[k].w));
    __syncthreads();

    // ---- attention of the wave's columns ----
    f32x16 O[4], x;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) O[n] = f32x16(0.f);

    auto tile_row = [&](int u) { return (u * kParts + part) * 32; };
    auto scores = [&](const char *buffer, int u) {
      const char *k = buffer + (tile_row(u) + (lane & 31)) * kKPitch + half * 16;
      uint4 key[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) key[j] = *reinterpret_cast<const uint4 *>(k + 32 * j);
      f32x16 y;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, key[j]), __builtin_bit_cast(bf16x8, Q[j]),
                                                    j == 0 ? f32x16(0.f) : y, 0, 0, 0);
      return y;
    };
    auto largest = [&](const f32x16 &y) {
      float top = y[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, y[i]);
      return fmaxf(m, fmaxf(top, xor32(top)));
    };
    // rows that are not there leave the scores (top: the largest with them); the reference moves where a score leads it
    auto settle = [&](f32x16 &y, float top, uint32_t rows) {
      if (rows != 0xffffffffu) {
        const uint32_t on = rows >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = on & 1u << (8 * (i / 4) + i % 4) ? y[i] : -INFINITY;
        top = largest(y);
      }
      if (top > m + p.lead) {
        const float alpha = __builtin_amdgcn_exp2f((m - finite_max(top)) * p.scale_log2);
        l *= alpha;
#pragma unroll
        for (int n = 0; n < 4; ++n) O[n] *= alpha;
        m = top;
      }
    };
    auto attend = [&](const char *buffer, int u) {
      // the value rows 4 half + (lane % 16) / 4 of a quad, dims 16 (lane / 16 % 2) + 4 (lane % 4)
      const char *v = buffer + kSharedBlock * kKPitch + (tile_row(u) + 4 * half + (lane & 15) / 4) * kVPitch +
                      (lane >> 4 & 1) * 32 + (lane & 3) * 8;
      const float sub = finite_max(m);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = __builtin_amdgcn_exp2f((x[i] - sub) * p.scale_log2);
        sum += x[i];
      }
      l += sum;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        bf16x8 piece[kPieces];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float rest = x[8 * n + e];
#pragma unroll
          for (int q = 0; q + 1 < kPieces; ++q) {
            piece[q][e] = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(rest) >> 16));
            rest -= __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
          }
          piece[kPieces - 1][e] = (__bf16)rest;
        }
#pragma unroll
        for (int q = 1; q < kPieces; ++q) piece[q] = not_zero<u16x8>(piece[q], piece[0]);
        bf16x8 value[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const char *at = v + n * 16 * kVPitch + dt * 64;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTile)(at));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTile)(at + 8 * kVPitch));
          value[dt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int q = 0; q < kPieces; ++q)
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
            O[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value[dt], piece[q], O[dt], 0, 0, 0);
      }
    };

    if (busy) {
      x = scores(s_rows[0], 0);
      settle(x, largest(x), (uint32_t)(live >> tile_row(0)));
    }
    int now = 0;
    for (int b = block0; b < block1; ++b) {
      const int next = now == 2 ? 0 : now + 1, last = next == 2 ? 0 : next + 1;
      Rows r;
      const bool more = b + 2 < block1;
      if (more) {
        fetch(b + 2, r);
        look_up(b + 3);
      }
      if (busy) {
#pragma unroll
        for (int u = 0; u < kSubs; ++u) {
          // (behind the last block: rows of an old one, or of none; their scores are not used)
          const bool inside = u + 1 < kSubs;
          f32x16 y = inside ? scores(s_rows[now], u + 1) : scores(s_rows[next], 0);
          attend(s_rows[now], u);
          const uint32_t rows = inside ? (uint32_t)(live >> tile_row(u + 1)) : b + 1 < block1 ? (uint32_t)(live1 >> tile_row(0)) : 0u;
          settle(y, largest(y), rows);
          x = y;
        }
      }
      live = live1;
      if (more) {
        put(r, s_rows[last]);
        live1 = r.there;
      }
      __syncthreads();
      now = next;
    }
    l += xor32(l);
    m *= c.sm_scale;

    if constexpr (kParts == 2) {  // the two halves of the rows meet in LDS
      float *slot = reinterpret_cast<float *>(&s_rows[0][0]) + col_wave * (66 * 64) + lane;
      static_assert(kCols * 66 * 64 * 4 <= 3 * kBuffer, "the halves fit the buffers");
      if (part == 1) {
        slot[64 * 64] = m;
        slot[65 * 64] = l;
#pragma unroll
        for (int i = 0; i < 64; ++i) slot[i * 64] = O[i / 16][i % 16];
      }
      __syncthreads();
      if (part == 0) {
        const float mo = slot[64 * 64], top = fmaxf(m, mo), sub = finite_max(top);
        const float w = __builtin_amdgcn_exp2f((m - sub) * kLog2e), wo = __builtin_amdgcn_exp2f((mo - sub) * kLog2e);
        l = fmaf(l, w, slot[65 * 64] * wo);
#pragma unroll
        for (int i = 0; i < 64; ++i) O[i / 16][i % 16] = fmaf(O[i / 16][i % 16], w, slot[i * 64] * wo);
        m = top;
      }
      __syncthreads();
    }

    if (busy && mine && part == 0) {
      const int64_t slot = head * p.parts.all + p.parts.own + split;
      if (half == 0) {
        p.parts.ml[slot] = make_float2(m, l);
        if (split == 0) p.parts.pieces[2 * head + 1] = pieces_of(at);
      }
      float4 *dst = reinterpret_cast<float4 *>(p.parts.acc + slot * kHeadDim + 4 * half);
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          dst[8 * n + 2 * i] = make_float4(O[n][4 * i], O[n][4 * i + 1], O[n][4 * i + 2], O[n][4 * i + 3]);
    }
    if (seg_end >= at.c_end) break;
    deal_next(shared_segments(p), at);
  }
}

}  // namespace

void launch_shared_rows(const PagedArgs &p, hipStream_t stream) {
  const dim3 grid(p.shared.grid), block(kSharedThreads);
  if (p.shared_cols == 256) {
    if (p.attn.out_is_bf16)
      hipLaunchKernelGGL((shared_kernel<8, 2>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((shared_kernel<8, 3>), grid, block, 0, stream, p);
  } else {
    if (p.attn.out_is_bf16)
      hipLaunchKernelGGL((shared_kernel<4, 2>), grid, block, 0, stream, p);
    else
      hipLaunchKernelGGL((shared_kernel<4, 3>), grid, block, 0, stream, p);
  }
}

}  // namespace dp
