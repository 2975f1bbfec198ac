// Appending to a paged cache: keys rotated to their positions, values as they are, into the pages; queries rotated.
//
// Rotation of a pair (a, b) at position p with frequency f: (a cos t - b sin t, a sin t + b cos t), t = p f.  t is taken
// in turns in 64 bits (p f / 2 pi, the nearest whole number of turns off), so the angle handed to the fp32 sine and cosine
// is exact to 2^-25 of a turn whatever the position; products in fp32, one rounding to bf16.
//
// A wave owns one token (or one of `parts` shares of its rows): its 64 lanes find the token's sequence, page and slot
// and take the sines and cosines of the up to 64 pairs, one each, which all heads of the token then share through LDS.
// A row (one head) is 16 lanes x 8 dimensions, four rows per wave and load.
// Bound by HBM: 131072 tokens of 48 bf16 rows (3.2 GB read and written) 571 us = 5.6 TB/s, 14771 from fp32 (0.54 GB) 107 us
// = 5.1 TB/s, as much as a large copy; one token by the chain of loads, sine and stores (3.7 us).
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / 64;

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// kStream: 16 bytes that no cache is to keep
template <bool kStream>
__device__ __forceinline__ uint4 load16(const char *p) {
  if constexpr (kStream) return load_stream16(p);
  return *reinterpret_cast<const uint4 *>(p);
}
template <bool kStream>
__device__ __forceinline__ void store16(char *p, const uint4 &v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (kStream)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(p));
  else
    *reinterpret_cast<uint4 *>(p) = v;
}

// 8 dimensions of a row, widened
template <bool kF32, bool kStream>
struct Slice {
  uint4 a, b;  // b: fp32 only
  __device__ __forceinline__ void load(const char *row, int lane16) {
    a = load16<kStream>(row + lane16 * (kF32 ? 32 : 16));
    if constexpr (kF32) b = load16<kStream>(row + lane16 * 32 + 16);
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
    if constexpr (kF32) {
      const float4 f = __builtin_bit_cast(float4, a), g = __builtin_bit_cast(float4, b);
      x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
      x[4] = g.x; x[5] = g.y; x[6] = g.z; x[7] = g.w;
    } else {
      unpack8(a, x);
    }
  }
};

__device__ __forceinline__ uint4 round8(const float (&x)[8]) {  // to nearest even, NaN stays NaN
  const f32x8 v = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
  return __builtin_bit_cast(uint4, __builtin_convertvector(v, bf16x8));
}

// the r-th row of a token: keys, then values, then queries
struct TokenRow {
  int head;
  bool is_v, is_q;
};
__device__ __forceinline__ TokenRow token_row(const PagedView &c, int r) {
  TokenRow t;
  t.is_v = r >= c.n_kv_heads && r < 2 * c.n_kv_heads;
  t.is_q = r >= 2 * c.n_kv_heads;
  t.head = t.is_q ? r - 2 * c.n_kv_heads : t.is_v ? r - c.n_kv_heads : r;
  return t;
}

template <bool kF32, bool kStream>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(PagedView c, AppendTokens t, int parts) {
  __shared__ float2 s_turn[kAppendWaves][kHeadDim / 2];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int t16 = lane & 15, grp = lane >> 4;
  const int64_t task = (int64_t)blockIdx.x * kAppendWaves + wave;
  const int token = (int)min(task / parts, (int64_t)t.n_tokens - 1), part = (int)(task % parts);
  bool live = task < (int64_t)t.n_tokens * parts;

  // four rows per batch and wave; the first two batches are on their way while the token's place is found
  const int rows = 2 * c.n_kv_heads + (t.q ? c.n_q_heads : 0), step = 4 * parts;
  auto fetch = [&](int r, Slice<kF32, kStream> &s) {
    const TokenRow row = token_row(c, min(r, rows - 1));
    s.load(static_cast<const char *>(row.is_q ? t.q : row.is_v ? t.v : t.k) +
               token * (row.is_q ? t.q_stride : row.is_v ? t.v_stride : t.k_stride) + row.head * (kHeadDim * (kF32 ? 4 : 2)),
           t16);
  };
  int r = 4 * part + grp;
  Slice<kF32, kStream> s0, s1;
  fetch(r, s0);
  fetch(r + step, s1);

  const int found = t.tok_ptr ? wave_find(t.tok_ptr, c.n_seqs, token) : token;
  live = live && found < c.n_seqs;
  const int seq = min(found, c.n_seqs - 1);
  const int64_t at = (int64_t)c.seq_lens[seq] - (t.tok_ptr ? (int64_t)t.tok_ptr[seq + 1] - token : 1);
  bool stored = at >= 0 && at < c.max_seq_len;
  int64_t page = 0;
  if (stored) {
    page = c.table[(int64_t)seq * c.table_stride + (at >> c.page_shift)];
    stored = page >= 0 && page < c.n_pages;
  }
  const int64_t place = page * c.page_stride + (at & ((1 << c.page_shift) - 1)) * c.slot_stride;
  const double position = t.positions ? (double)t.positions[token] : (double)at;

  const int half = t.rope_dims / 2;
  if (lane < half) {
    const double turns = position * ((double)t.freqs[lane] * 0.15915494309189535);  // 1 / 2 pi
    float2 cs;
    sincospif(2.f * (float)(turns - rint(turns)), &cs.y, &cs.x);
    s_turn[wave][lane] = cs;
  }
  __syncthreads();
  if (!live) return;

  // what the lane's 8 dimensions are multiplied with, and the partner dimension of each
  const int lanes_half = half / 8;  // lanes that hold the first dimensions of the pairs (i, i + half)
  const bool turns = t16 < 2 * lanes_half;
  float cosine[8], sine[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int pair = t.adjacent ? 4 * t16 + e / 2 : 8 * (t16 < lanes_half ? t16 : t16 - lanes_half) + e;
    const float2 cs = s_turn[wave][turns ? pair : 0];
    const bool first = t.adjacent ? e % 2 == 0 : t16 < lanes_half;
    cosine[e] = cs.x;
    sine[e] = first ? -cs.y : cs.y;
  }
  const int partner = (lane & 48) + (!turns ? t16 : t16 < lanes_half ? t16 + lanes_half : t16 - lanes_half);

  auto finish = [&](int r, const Slice<kF32, kStream> &s) {
    const TokenRow row = token_row(c, min(r, rows - 1));
    float x[8], y[8];
    s.widen(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = t.adjacent ? x[e ^ 1] : __shfl(x[e], partner, 64);
      const float turned = fmaf(x[e], cosine[e], other * sine[e]);
      y[e] = turns && !row.is_v ? turned : x[e];
    }
    if (r >= rows || (!row.is_q && !stored)) return;
    char *dst = row.is_q ? static_cast<char *>(t.q_out) + ((int64_t)token * c.n_q_heads + row.head) * kRowBytes
                         : (row.is_v ? c.v_pages : c.k_pages) + place + row.head * c.head_stride;
    store16<kStream>(dst + t16 * 16, round8(y));
  };
  for (int left = rows - 4 * part; left > 0; left -= 2 * step, r += 2 * step) {
    Slice<kF32, kStream> n0, n1;
    fetch(r + 2 * step, n0);
    fetch(r + 3 * step, n1);
    finish(r, s0);
    finish(r + step, s1);
    s0 = n0;
    s1 = n1;
  }
}

}  // namespace

hipError_t launch_append(const PagedView &c, const AppendTokens &t, hipStream_t s) {
  // A token's rows by one wave where there are enough tokens to fill the chip, else by several, down to four rows each: a
  // call is then one round of loads.  us: one token of 48 rows 7.6 with one wave, 3.7 with twelve; 64 tokens 8.7 / 4.2.
  constexpr int kChipWaves = 8192;
  const int rows = 2 * c.n_kv_heads + (t.q ? c.n_q_heads : 0), most = (rows + 3) / 4, want = kChipWaves / t.n_tokens;
  const int parts = want < 1 ? 1 : want < most ? want : most;
  const int64_t tasks = (int64_t)t.n_tokens * parts;
  const dim3 grid((unsigned)((tasks + kAppendWaves - 1) / kAppendWaves)), block(kAppendThreads);
  // What no cache could hold goes by without the caches, counted by the rows as they are stored; below, what is written is read
  // from the caches by the attention that follows.  us through the caches / past them, 48 rows a token: bf16 21500 tokens (252
  // MiB) 105 / 97, 131072 601 / 568, fp32 21500 152 / 150, 131072 915 / 896; short of it, bf16 4096 18.1 / 20.8, fp32 25.1 / 31.8.
  const bool stream = (int64_t)t.n_tokens * rows * kRowBytes > (int64_t)256 << 20;
  const auto kernel = t.is_f32 ? stream ? append_kernel<true, true> : append_kernel<true, false>
                               : stream ? append_kernel<false, true> : append_kernel<false, false>;
  hipLaunchKernelGGL(kernel, grid, block, 0, s, c, t, parts);
  return hipGetLastError();
}

}  // namespace dp
