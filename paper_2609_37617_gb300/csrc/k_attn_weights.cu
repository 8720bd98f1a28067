// k_attn_weights.cu -- the weight that attention gives each cache entry
// (as2d_attention_weights): over a request's rows i and the query heads h of a
// kv head, w_t (+)= sum e^(scale q_ih k_t - lse_ih).
//
// A thread per key, which goes through the queries one after another.
#include "ops.h"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

template <int D>
__global__ void __launch_bounds__(128) attn_weights_kernel(const __grid_constant__ WeightArgs wa) {
  const TreeArgs& a = wa.t;
  __shared__ float s_q[D];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int g = blockIdx.y, b = blockIdx.z, G = a.nq / a.nkv;
  const int r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0;
  if (rows == 0) return;
  const int L = a.len[b];
  if (!rows_fit(L, rows, a.cap)) {
    if (threadIdx.x == 0 && a.err) atomicOr(a.err, kErrCapacity);
    return;
  }
  for (int t0 = blockIdx.x * 128; t0 < L + rows; t0 += gridDim.x * 128) {
    const int t = t0 + threadIdx.x;
    const bool live = t < L + rows;
    float k[D], sum = 0.f;
    const size_t head = (size_t)b * a.nkv + g;
    for (int e = 0; e < D; ++e) k[e] = live ? __bfloat162float(a.k[(head * a.cap + t) * D + e]) : 0.f;
    for (int n = 0; n < rows * G; ++n) {
      const int r = r0 + n / G, h = g * G + n % G;
      __syncthreads();
      for (int e = threadIdx.x; e < D; e += 128) {
        const int64_t at = r * a.q_stride + (int64_t)h * D + e;
        s_q[e] = a.q_f32 ? ((const float*)a.q)[at] : __bfloat162float(((const bf16*)a.q)[at]);
      }
      __syncthreads();
      const uint64_t vis = a.visible ? a.visible[r] : ~0ull >> (63 - (r - r0));
      if (!live || (t >= L && !((vis >> (t - L)) & 1))) continue;
      float s = 0.f;
      for (int e = 0; e < D; ++e) s = fmaf(s_q[e], k[e], s);
      sum += exp2f(s * a.scale_log2 - a.lse[(size_t)r * a.nq + h] * 1.4426950408889634f);
    }
    if (live) {
      float* w = wa.w + head * a.cap + t;
      *w = t < L ? *w + sum : sum;
    }
  }
}

}  // namespace

cudaError_t launch_attention_weights(const WeightArgs& a, int head_dim, int64_t max_keys, cudaStream_t st) {
  const dim3 grid((unsigned)((max_keys + 127) / 128), a.t.nkv, a.t.rm.batch);
  return head_dim == 128 ? launch_pdl(attn_weights_kernel<128>, grid, dim3(128), 0, st, 1, a)
                         : launch_pdl(attn_weights_kernel<64>, grid, dim3(128), 0, st, 1, a);
}

}  // namespace as2d
