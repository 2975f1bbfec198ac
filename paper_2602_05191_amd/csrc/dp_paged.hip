// Dense decode attention over the rows of a paged cache: the launch over each sequence's own rows, the merge of partial
// results, and how a call is split.
#include "dp_paged_body.hpp"

namespace dp {
namespace {

constexpr int kPagedThreads = 256;

template <bool kSmallPages, bool kShared>
__global__ __launch_bounds__(kPagedThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_kernel(PagedArgs p) {
  __shared__ PagedLds<kPagedThreads / 64> lds;
  paged_rows<kSmallPages, kShared, kPagedThreads / 64>(p, blockIdx.x, lds);
}

// One workgroup per head.  A slot's 128 dimensions are taken by 32 lanes, four each, so that a head's partials are fetched in
// a round or two of loads; the groups of 32 meet in LDS.
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
  const int n_own = rows.chunks() > 0 || p.whole ? pieces.x : 0;
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
    const float sub = finite_max(top), sc = exp2f(m - sub);
    l *= sc;
    o.x *= sc; o.y *= sc; o.z *= sc; o.w *= sc;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float w = exp2f(ml[u].x - sub);
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
    const float w = exp2f(s_m[v] - finite_max(all.m));
    all.l = fmaf(s_l[v], w, all.l);
    all.o = fmaf(s_o[v][threadIdx.x], w, all.o);
  }
  store_head(p, head, threadIdx.x, prior_lse, prior_o, all);
}

// How a call is split; by sizes that the host knows.
struct Split {
  int whole, cols;  // own rows; shared rows: columns of a workgroup
  Deal own, shared;
};
int at_most(long n, long most) { return (int)(n < most ? n : most); }
int at_least(long n, long least) { return (int)(n > least ? n : least); }

Split split_of(const PagedView &c, const SharedView &shared) {
  Split s{};
  const long n_seg = (long)c.n_seqs * c.n_kv_heads, nh = (long)c.n_seqs * c.n_q_heads;
  const int max_chunks = (c.max_seq_len + kChunkRows - 1) / kChunkRows;
  s.whole = c.n_seqs > kDealtItems || c.max_seq_len <= (n_seg >= 512 ? 1024 : n_seg >= 128 ? 512 : 320);
  const bool any_shared = shared.n_groups > 0 && shared.max_shared_len > 0 && shared.n_groups <= kDealtItems;
  // one round of workgroups (two waves per SIMD x 256 CUs), and partial slots for some thousand pieces in all
  s.own.grid = at_least(at_most(n_seg * max_chunks, 2 * 256), 1);
  s.own.slots = s.whole ? 1 : at_least(at_most(max_chunks, at_most(at_least(16384 / nh, 8), kMaxSplits)), 1);
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
  const dim3 grid(p.whole ? p.c.n_seqs * p.c.n_kv_heads : p.own.grid), block(kPagedThreads);
  if (p.c.page_shift < 4)
    hipLaunchKernelGGL((paged_kernel<true, kShared>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((paged_kernel<false, kShared>), grid, block, 0, stream, p);
}

template <bool kShared>
void launch_merge(const PagedArgs &p, hipStream_t stream) {
  const int nh = p.c.n_seqs * p.c.n_q_heads;
  if (p.parts.all <= 32)
    hipLaunchKernelGGL((paged_merge_kernel<128, kShared>), dim3(nh), dim3(128), 0, stream, p);
  else if (p.parts.all <= 64 || nh >= 512)
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
  p.own = s.own;
  p.shared = s.shared;
  p.shared_cols = s.cols;
  p.scale_log2 = c.sm_scale * kLog2e;
  p.lead = fminf(8.f / p.scale_log2, 3e38f);
  if (s.shared.slots) launch_shared_rows(p, stream);
  for (p.head0 = 0; p.head0 < c.group; p.head0 += kPagedHeads) {  // one pass over the rows for up to 16 heads of a group
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
