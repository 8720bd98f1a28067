// k_evict.cu -- eviction of cache entries by gathered weight, in place
// (as2d_cache_evict).
//
// evict_select_kernel, one CTA per unit (layer, request, kv head): the threshold
// among the older entries' weights by radix selection (order keys of 32 bits,
// 8 bits a pass, counted in shared memory), then the entries that stay, in
// order: those above it, those equal to it from the lowest position up to the
// number wanted, the latest `recent`.  It writes their old positions and moves
// their weights.
// evict_move_kernel, one CTA per unit and cache: entry j comes from position
// at[j] >= j.  Tiles of entries in order, a tile read before it is written: what
// a tile's writes cover, [j0, j0 + T), no later tile reads, as its entries
// come from their own positions or later.
#include "ops.h"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

constexpr int kSel = 1024;  // threads of the selection

// An unsigned key in the order of the float values; NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t evict_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if (w != w) return 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix of v over the block (warps in order, every thread of a warp
// passing the warp's value); total: the sum.
__device__ __forceinline__ int warp_prefix(int v, int* s, int* total) {
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  if (lane == 0) s[w] = v;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kSel / 32; ++i) {
    before += i < w ? s[i] : 0;
    all += s[i];
  }
  *total = all;
  return before;
}

__global__ void __launch_bounds__(kSel) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ int hist[256], s_w[32], s_pick[2];
  ptx::griddep_wait();
  const int unit = blockIdx.x, b = (unit / a.nkv) % a.batch;
  const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
  const int L = a.len[b], keep = a.keep[b];
  if (L < 0 || L > a.cap || L <= keep) {
    if (tid == 0) a.first[unit] = -1;
    return;
  }
  float* wt = a.w + (size_t)unit * a.cap;
  uint16_t* at = a.at + (size_t)unit * a.cap;
  const int late = min(a.recent, keep), old = L - late;  // [old, L) stay
  int want = keep - late;                                // of [0, old)
  uint32_t prefix = 0, mask = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSel) hist[i] = 0;
    __syncthreads();
    for (int t = tid; t < old; t += kSel) {
      const uint32_t key = evict_key(wt[t]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int n = 0, bin = 255;
      while (bin > 0 && n + hist[bin] < want) n += hist[bin--];
      s_pick[0] = bin;
      s_pick[1] = n;
    }
    __syncthreads();
    prefix |= (uint32_t)s_pick[0] << shift;
    mask |= 255u << shift;
    want -= s_pick[1];
    __syncthreads();
  }
  // entries above the threshold stay, and the first `want` equal to it
  const int per = (L + kSel - 1) / kSel * 32, t0 = w * per, t1 = min(t0 + per, L);
  int ties = 0;
  for (int c = t0; c < t1; c += 32)
    ties += __popc(__ballot_sync(~0u, c + lane < min(t1, old) && evict_key(wt[c + lane]) == prefix));
  int all;
  int tie = warp_prefix(ties, s_w, &all);
  const int tie0 = tie;
  auto stays = [&](int t, float x, int& tie_at) {
    const uint32_t key = evict_key(x);
    const bool in = t < t1 && t < old, eq = in && key == prefix;
    const unsigned m = __ballot_sync(~0u, eq);
    const bool yes = (in && key > prefix) || (eq && tie_at + __popc(m & ((1u << lane) - 1)) < want) ||
                     (t < t1 && t >= old);
    tie_at += __popc(m);
    return yes;
  };
  int n = 0;
  for (int c = t0; c < t1; c += 32)
    n += __popc(__ballot_sync(~0u, stays(c + lane, c + lane < t1 ? wt[c + lane] : 0.f, tie)));
  int j = warp_prefix(n, s_w, &all);
  // old positions first, then the weights by them: a weight is read before its
  // place is written
  tie = tie0;
  for (int c = t0; c < t1; c += 32) {
    const bool yes = stays(c + lane, c + lane < t1 ? wt[c + lane] : 0.f, tie);
    const unsigned m = __ballot_sync(~0u, yes);
    if (yes) at[j + __popc(m & ((1u << lane) - 1))] = (uint16_t)(c + lane);
    j += __popc(m);
  }
  __syncthreads();
  if (tid == 0) s_pick[0] = keep;
  __syncthreads();
  for (int c = 0; c < keep; c += kSel) {
    const bool in = c + tid < keep;
    const int from = in ? at[c + tid] : 0;
    const float x = in ? wt[from] : 0.f;
    __syncthreads();
    if (in) wt[c + tid] = x;
    if (in && from != c + tid) atomicMin(&s_pick[0], c + tid);
    __syncthreads();
  }
  if (tid == 0) a.first[unit] = s_pick[0] < keep ? s_pick[0] : -1;
}

template <int D>
__global__ void __launch_bounds__(256) evict_move_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int C = D / 8, T = 256 / C;  // 16-byte pieces of an entry, entries of a tile
  ptx::griddep_wait();
  const int unit = blockIdx.x, b = (unit / a.nkv) % a.batch, keep = a.keep[b];
  bf16* x = (blockIdx.y ? a.v : a.k) + (size_t)unit * a.cap * D;
  const uint16_t* at = a.at + (size_t)unit * a.cap;
  const int first = a.first[unit], c = threadIdx.x % C;
  if (first < 0) return;
  for (int j0 = first; j0 < keep; j0 += T) {
    const int j = j0 + threadIdx.x / C;
    uint4 v;
    if (j < keep) v = *reinterpret_cast<const uint4*>(x + (size_t)at[j] * D + 8 * c);
    __syncthreads();
    if (j < keep) *reinterpret_cast<uint4*>(x + (size_t)j * D + 8 * c) = v;
    __syncthreads();
  }
}

__global__ void evict_len_kernel(const __grid_constant__ EvictArgs a) {
  ptx::griddep_wait();
  const int b = threadIdx.x;
  if (b < a.batch && a.len[b] > a.keep[b] && a.len[b] <= a.cap) a.len[b] = a.keep[b];
}

}  // namespace

size_t cache_evict_workspace(int64_t units, int cap) {
  return ((size_t)units * cap * 2 + 255) / 256 * 256 + ((size_t)units * 4 + 255) / 256 * 256;
}

void cache_evict_carve(EvictArgs& a, int64_t units, void* workspace) {
  a.at = (uint16_t*)workspace;
  a.first = (int32_t*)((char*)workspace + ((size_t)units * a.cap * 2 + 255) / 256 * 256);
}

cudaError_t launch_cache_evict(const EvictArgs& a, int head_dim, cudaStream_t st) {
  const unsigned units = (unsigned)(a.n_layers * a.batch * a.nkv);
  cudaError_t e = launch_pdl(evict_select_kernel, dim3(units), dim3(kSel), 0, st, 1, a);
  if (e != cudaSuccess) return e;
  e = head_dim == 128 ? launch_pdl(evict_move_kernel<128>, dim3(units, 2), dim3(256), 0, st, 1, a)
                      : launch_pdl(evict_move_kernel<64>, dim3(units, 2), dim3(256), 0, st, 1, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(evict_len_kernel, dim3(1), dim3(kMaxBatch), 0, st, 1, a);
}

}  // namespace as2d
