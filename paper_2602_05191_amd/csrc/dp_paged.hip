// Dense decode attention over the rows of a paged cache, one query token per sequence.
#include "dp_attend.hpp"
#include "dp_device.hpp"
#include "dp_kernels.hpp"
#include "dp_paged_rows.hpp"

namespace dp {
namespace {

constexpr int kPagedThreads = 256;

// One workgroup per head; every 16-lane row takes rows in turn, one online softmax each, merged at the end.
__global__ __launch_bounds__(kPagedThreads) void paged_kernel(PagedView c, PagedAttention a, AttnOut attn) {
  constexpr int kGroups = kPagedThreads / 16;
  __shared__ float s_m[kGroups], s_l[kGroups], s_acc[kGroups][kHeadDim];
  const int t16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const int head = blockIdx.x, seq = head / c.n_q_heads, kv = head % c.n_q_heads / c.group;
  float q[8];
  unpack8(load_row_slice(a.q, head, t16), q);
  const int len = paged_len(c, seq), first = a.first_rows ? max(0, a.first_rows[seq]) : 0;
  const float scale_log2 = c.sm_scale * kLog2e;
  float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int r = first + grp; r < len; r += kGroups) {
    const int page = c.table[(int64_t)seq * c.table_stride + (r >> c.page_shift)];
    if (page < 0 || page >= c.n_pages) continue;
    const int64_t row = page * c.page_stride + kv * c.head_stride + (r & ((1 << c.page_shift) - 1)) * (int64_t)c.slot_stride;
    const uint4 k = reinterpret_cast<const uint4 *>(c.k_pages + row)[t16];
    const uint4 v = reinterpret_cast<const uint4 *>(c.v_pages + row)[t16];
    float kf[8];
    unpack8(k, kf);
    // (the maximum is kept and subtracted unscaled: the largest score has the weight 1 whatever its size)
    const float x = row16_sum(dot8(q, kf));
    const float top = fmaxf(m, x), sub = fmaxf(top, -3.402823466e38f);
    const float alpha = exp2f((m - sub) * scale_log2), p = exp2f((x - sub) * scale_log2);
    float vf[8];
    unpack8(v, vf);
    l = l * alpha + p;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = fmaf(p, vf[i], acc[i] * alpha);
    m = top;
  }
  if (t16 == 0) {
    s_m[grp] = m * scale_log2;
    s_l[grp] = l;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) s_acc[grp][8 * t16 + i] = acc[i];
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  const int d = threadIdx.x;
  float M = a.prior_lse ? a.prior_lse[head] * kLog2e : -INFINITY, L = 0.f, o = 0.f;
  const float prior = M;
  for (int g = 0; g < kGroups; ++g) M = fmaxf(M, s_m[g]);
  const float sub = fmaxf(M, -3.402823466e38f);
  for (int g = 0; g < kGroups; ++g) {
    const float w = exp2f(s_m[g] - sub);
    L = fmaf(s_l[g], w, L);
    o = fmaf(s_acc[g][d], w, o);
  }
  if (prior > -INFINITY) {
    const float w = exp2f(prior - sub);
    L += w;
    o = fmaf(a.prior_out[head * (int64_t)kHeadDim + d], w, o);
  }
  const bool any = L > 0.f;
  store_out(attn.out, attn.out_is_bf16, head, d, any ? o / L : 0.f);
  if (attn.lse && d == 0) attn.lse[head] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
}

}  // namespace

hipError_t launch_paged_decode(const PagedView &c, const PagedAttention &a, const AttnOut &attn, hipStream_t s) {
  hipLaunchKernelGGL(paged_kernel, dim3(c.n_seqs * c.n_q_heads), dim3(kPagedThreads), 0, s, c, a, attn);
  return hipGetLastError();
}

}  // namespace dp
