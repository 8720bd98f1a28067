// k_tree_attn.cu -- attention of a tree of drafted tokens over a cache
// (as2d_tree_attention).
//
// Row i of request b sees the prefix [0, L_b) and those of its request's rows j,
// at L_b + j, whose bit j its mask has.  With s_t = scale q k_t over what it sees:
//   m = max s_t, l = sum e^(s_t - m), out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// One CTA per (row, query head); its four warps take every fourth key, a lane
// holding D / 32 dims, with a running maximum and sum each, joined at the end.
#include "ops.h"
#include "ptx_sm100.cuh"
#include "small_dev.cuh"

namespace as2d {
namespace {

template <int D>
__global__ void __launch_bounds__(128) tree_attn_kernel(const __grid_constant__ TreeArgs a) {
  constexpr int E = D / 32, W = 4;
  __shared__ float s_m[W], s_l[W], s_o[W][D];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int r = blockIdx.x, h = blockIdx.y, w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = row_request(a.rm, r), r0 = a.rm.start[b], i = r - r0, rows = a.rm.start[b + 1] - r0;
  const int L = a.len[b];
  if (!rows_fit(L, rows, a.cap)) {
    if (threadIdx.x == 0 && a.err) atomicOr(a.err, kErrCapacity);
    return;
  }
  const uint64_t vis = a.visible ? a.visible[r] : ~0ull >> (63 - i);
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t at = r * a.q_stride + (int64_t)h * D + lane * E + e;
    q[e] = a.q_f32 ? ((const float*)a.q)[at] : __bfloat162float(((const bf16*)a.q)[at]);
    o[e] = 0.f;
  }
  const size_t base = ((size_t)b * a.nkv + h / (a.nq / a.nkv)) * a.cap * D;
  for (int t = w; t < L + rows; t += W) {
    if (t >= L && !((vis >> (t - L)) & 1)) continue;
    const bf16 *k = a.k + base + (size_t)t * D + lane * E, *v = a.v + base + (size_t)t * D + lane * E;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], __bfloat162float(k[e]), s);
    s = warp_sum(s) * a.scale_log2;
    const float mn = fmaxf(m, s);
    const float c = m == -INFINITY ? 0.f : exp2f(m - mn), p = exp2f(s - mn);
    l = fmaf(l, c, p);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], c, p * __bfloat162float(v[e]));
    m = mn;
  }
  if (lane == 0) s_m[w] = m, s_l[w] = l;
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[w][lane * E + e] = o[e];
  __syncthreads();
  float M = -INFINITY, l_all = 0.f;
  for (int j = 0; j < W; ++j) M = fmaxf(M, s_m[j]);
  float wt[W];
  for (int j = 0; j < W; ++j) {
    wt[j] = s_l[j] == 0.f ? 0.f : exp2f(s_m[j] - M);
    l_all += s_l[j] * wt[j];
  }
  if ((int)threadIdx.x < D) {
    float x = 0.f;
    for (int j = 0; j < W; ++j)
      if (wt[j] != 0.f) x += s_o[j][threadIdx.x] * wt[j];
    x = l_all == 0.f ? 0.f : x / l_all;
    const size_t at = ((size_t)r * a.nq + h) * D + threadIdx.x;
    if (a.q_f32)
      ((float*)a.out)[at] = x;
    else
      ((bf16*)a.out)[at] = __float2bfloat16_rn(x);
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[(size_t)r * a.nq + h] = l_all == 0.f ? -INFINITY : (M + log2f(l_all)) * 0.69314718055994531f;
}

}  // namespace

size_t tree_attention_workspace(int) { return 256; }

cudaError_t launch_tree_attention(const TreeArgs& a, int head_dim, int64_t, void*, cudaStream_t st) {
  const dim3 grid(a.rm.rows, a.nq);
  return head_dim == 128 ? launch_pdl(tree_attn_kernel<128>, grid, dim3(128), 0, st, 1, a)
                         : launch_pdl(tree_attn_kernel<64>, grid, dim3(128), 0, st, 1, a);
}

}  // namespace as2d
