// k_sampled.cu -- probabilities at a temperature (as2d_token_probs) and the
// acceptance of drafted tokens from given random numbers (as2d_accept_sampled).
//
// probs_kernel, one CTA per row: p_v = e^((x_v - max x) / T) / sum, in three
// passes over the row.
// accept_kernel, one CTA per request: the candidates' tests, then the sum of the
// weights max(p_n - q_n, 0) in chunks of a thread each, the chunk that holds the
// border u_k total, and the token within it.
#include "ops.h"
#include "ptx_sm100.cuh"
#include "small_dev.cuh"

namespace as2d {
namespace {

template <int N>
__device__ __forceinline__ float block_max(float v, float* s) {
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  for (int i = 0; i < N / 32; ++i) v = fmaxf(v, s[i]);
  return v;
}
template <int N>
__device__ __forceinline__ float block_sum(float v, float* s) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
  for (int i = 0; i < N / 32; ++i) v += s[i];
  return v;
}

__global__ void __launch_bounds__(1024) probs_kernel(const float* logits, int vocab, float c, float* probs) {
  __shared__ float s[32];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const float* x = logits + (size_t)blockIdx.x * vocab;
  float* p = probs + (size_t)blockIdx.x * vocab;
  float m = -INFINITY, bad = 0.f;
  for (int v = threadIdx.x; v < vocab; v += 1024) {
    m = fmaxf(m, x[v]);
    if (x[v] != x[v]) bad = 1.f;
  }
  m = block_max<1024>(m, s);
  if (block_max<1024>(bad, s) != 0.f) m = NAN;
  float l = 0.f;
  const float ref = m == -INFINITY ? 0.f : m;
  for (int v = threadIdx.x; v < vocab; v += 1024) l += exp2f((x[v] - ref) * c);
  l = block_sum<1024>(l, s);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int v = threadIdx.x; v < vocab; v += 1024) p[v] = exp2f((x[v] - ref) * c) * inv;
}

__global__ void __launch_bounds__(1024) accept_sampled_kernel(const __grid_constant__ SampledArgs a) {
  __shared__ double s_sum[1024];
  __shared__ int s_n, s_chunk, s_any;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int b = blockIdx.x, r0 = a.start[b], k = a.start[b + 1] - r0 - 1, c0 = r0 - b, tid = threadIdx.x;
  const size_t V = a.vocab;
  if (tid < 32) {
    bool stands = false;
    if (tid < k) {
      const int c = a.cand[c0 + tid];
      if (c >= 0 && c < a.vocab) {
        const double q = a.draft ? (double)a.draft[(size_t)(c0 + tid) * V + c] : 1.0;
        stands = (double)a.u[r0 + tid] * q < (double)a.probs[(size_t)(r0 + tid) * V + c];
      }
    }
    const unsigned m = __ballot_sync(~0u, stands);
    if (tid == 0) s_n = __ffs(~m) - 1;
  }
  __syncthreads();
  const int n = s_n, gone = n < k && !a.draft ? a.cand[c0 + n] : -1;
  const float* p = a.probs + (size_t)(r0 + n) * V;
  const float* q = n < k && a.draft ? a.draft + (size_t)(c0 + n) * V : nullptr;
  const int per = (a.vocab + 1023) / 1024;
  const double u = a.u[r0 + k];
  int token = -1;
  for (int plain = n < k ? 0 : 1; plain < 2 && token < 0; ++plain) {
    auto weight = [&](int v) -> double {
      double x = p[v];
      if (!plain) x = q ? x - (double)q[v] : (v == gone ? 0.0 : x);
      return x > 0.0 ? x : 0.0;
    };
    const int v0 = min(tid * per, a.vocab), v1 = min(v0 + per, a.vocab);
    double sum = 0.0;
    for (int v = v0; v < v1; ++v) sum += weight(v);
    __syncthreads();
    s_sum[tid] = sum;
    if (tid == 0) s_chunk = -1;
    __syncthreads();
    if (tid == 0) {
      double total = 0.0, at = 0.0;
      for (int i = 0; i < 1024; ++i) total += s_sum[i];
      const double border = u * total;
      int pick = -1;
      for (int i = 0; i < 1024; ++i) {
        if (s_sum[i] > 0.0) pick = i;
        if (at + s_sum[i] > border) break;
        at += s_sum[i];
      }
      if (pick >= 0) {
        at = 0.0;
        for (int i = 0; i < pick; ++i) at += s_sum[i];
        for (int v = pick * per; v < min((pick + 1) * per, a.vocab); ++v) {
          const double x = weight(v);
          if (x > 0.0) s_chunk = v;
          if (at + x > border) break;
          at += x;
        }
      }
    }
    __syncthreads();
    token = s_chunk;
  }
  if (tid == 0) {
    a.n_out[b] = n;
    a.token_out[b] = token;
  }
}

}  // namespace

cudaError_t launch_token_probs(const float* logits, int rows, int vocab, float temperature, float* probs,
                               cudaStream_t st) {
  return launch_pdl(probs_kernel, dim3(rows), dim3(1024), 0, st, 1, logits, vocab,
                    (float)(1.4426950408889634 / temperature), probs);
}

cudaError_t launch_accept_sampled(const SampledArgs& a, cudaStream_t st) {
  return launch_pdl(accept_sampled_kernel, dim3(a.batch), dim3(1024), 0, st, 1, a);
}

}  // namespace as2d
