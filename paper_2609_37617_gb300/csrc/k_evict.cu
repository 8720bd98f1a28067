// k_evict.cu -- eviction of cache entries by gathered weight, in place
// (as2d_cache_evict).
//
// evict_select_kernel, one CTA per unit (layer, request, kv head): the threshold
// among the older entries' weights by radix selection (order keys of 32 bits,
// counted in shared memory), then the entries that stay, in
// order: those above it, those equal to it from the lowest position up to the
// number wanted, the latest `recent`.  It writes their old positions and moves
// their weights.  Each thread reads its weights once and holds them over all passes: in
// registers up to a capacity of 16384 (16 a thread), mostly in local memory beyond (64 a
// thread of 64 registers: 880 bytes of stack, not timed).
// evict_move_kernel, one CTA per unit, cache and 128 bytes of an entry: entry j comes
// from position at[j] >= j.  Tiles of entries in order, a tile read wholly before
// it is written: what its writes cover, [j0, j0 + T), no later tile reads, as
// those entries come from their own positions or later; so the next tile's
// reads are on their way while a tile is written.  Bound by memory: each entry that
// moves is read and written once (28 layers x 4 kv heads of 15128 entries cut to
// 11346: 225 us, 17 of them the selection; 1.31 GB at 6.3 TB/s in the move).
#include "ops.h"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

// Digits of the radix selection, 11 + 11 + 10 bits from the top: the first takes
// in the exponent and two bits of the mantissa, so that weights of one size still
// fall into several bins (8-bit digits put them into one or two, whose counts
// are then added one after another).
constexpr int kPasses = 3, kBins = 2048;

// An unsigned key in the order of the float values; NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t evict_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if (w != w) return 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix of v over the block's W warps in order (every thread of a warp
// passing the warp's value).
template <int W>
__device__ __forceinline__ int warp_prefix(int v, int* s) {
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  if (lane == 0) s[w] = v;
  __syncthreads();
  const int mine = lane < W ? s[lane] : 0;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < W; o <<= 1) {
    const int t = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += t;
  }
  return __shfl_sync(~0u, upto - mine, w);
}

// T threads, E entries of a thread (a warp's are consecutive, 32 at a time), which
// it holds.
template <int T, int E>
__global__ void __launch_bounds__(T) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int W = T / 32, B = kBins / T;  // warps, bins of a thread
  __shared__ int hist[kPasses * kBins], s_w[W], s_pick[2];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
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
  const int t0 = w * 32 * E + lane;
  float x[E];
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = t0 + 32 * i < L ? wt[t0 + 32 * i] : 0.f;
  for (int i = tid; i < kPasses * kBins; i += T) hist[i] = 0;
  __syncthreads();
  uint32_t prefix = 0, mask = 0;
#pragma unroll 1
  for (int pass = 0; pass < kPasses; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digit = pass < 2 ? kBins - 1 : kBins / 2 - 1;
    int* h = hist + pass * kBins;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint32_t key = evict_key(x[i]);
      if (t0 + 32 * i < old && (key & mask) == prefix) atomicAdd(&h[(key >> shift) & digit], 1);
    }
    __syncthreads();
    // the bin in which the count from above reaches `want`: B bins a thread, the
    // highest first
    const int bin = kBins - 1 - B * tid;
    int c[B], sum = 0;
#pragma unroll
    for (int i = 0; i < B; ++i) sum += c[i] = h[bin - i];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += t;
    }
    int n = warp_prefix<W>(__shfl_sync(~0u, upto, 31), s_w) + upto - sum;
    if (n < want && want <= n + sum) {
      int i = 0;
#pragma unroll
      for (int k = 0; k < B - 1; ++k)
        if (i == k && n + c[k] < want) n += c[k], ++i;
      s_pick[0] = bin - i;
      s_pick[1] = n;
    } else if (want == 0 && tid == 0) {  // none of them: nothing is above the highest key
      s_pick[0] = digit;
      s_pick[1] = 0;
    }
    __syncthreads();
    prefix |= (uint32_t)s_pick[0] << shift;
    mask |= digit << shift;
    want -= s_pick[1];
  }
  // entries above the threshold stay, and the first `want` equal to it
  const unsigned below = (1u << lane) - 1;
  int ties = 0;
#pragma unroll
  for (int i = 0; i < E; ++i)
    ties += __popc(__ballot_sync(~0u, t0 + 32 * i < old && evict_key(x[i]) == prefix));
  int tie = warp_prefix<W>(ties, s_w);
  uint32_t stay[(E + 31) / 32] = {};
  int n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int t = t0 + 32 * i;
    const uint32_t key = evict_key(x[i]);
    const bool eq = t < old && key == prefix;
    const unsigned m = __ballot_sync(~0u, eq);
    const bool yes = t < L && (t >= old || key > prefix || (eq && tie + __popc(m & below) < want));
    tie += __popc(m);
    if (yes) stay[i / 32] |= 1u << (i % 32);
    n += __popc(__ballot_sync(~0u, yes));
  }
  int j = warp_prefix<W>(n, s_w), first = keep;
  // (every weight has been read by now: their places can be written)
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const bool yes = (stay[i / 32] >> (i % 32)) & 1;
    const unsigned m = __ballot_sync(~0u, yes);
    const int to = j + __popc(m & below);
    if (yes) {
      at[to] = (uint16_t)(t0 + 32 * i);
      wt[to] = x[i];
      if (to != t0 + 32 * i) first = min(first, to);
    }
    j += __popc(m);
  }
  if (tid == 0) s_pick[0] = keep;
  __syncthreads();
  if (first < keep) atomicMin(&s_pick[0], first);
  __syncthreads();
  if (tid == 0) a.first[unit] = s_pick[0] < keep ? s_pick[0] : -1;
}

// (and the new lengths: nothing after the selection reads the old ones)
constexpr int kMove = 256, kSteps = 8;  // threads, entries of a thread in a tile
template <int D>
__global__ void __launch_bounds__(kMove) evict_move_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int P = 8, E = kMove / P, T = E * kSteps;  // 16-byte pieces, entries of a step, of a tile
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int unit = blockIdx.x, b = (unit / a.nkv) % a.batch, keep = a.keep[b];
  if (threadIdx.x == 0 && blockIdx.y == 0 && unit < a.batch * a.nkv && unit % a.nkv == 0) {
    const int L = a.len[b];
    if (L > keep && L <= a.cap) a.len[b] = keep;
  }
  const int first = a.first[unit];
  if (first < 0) return;
  constexpr int kSlices = D / 64;
  bf16* x = (blockIdx.y >= kSlices ? a.v : a.k) + (size_t)unit * a.cap * D + (blockIdx.y % kSlices) * 64 +
            (threadIdx.x % P) * 8;
  const uint16_t* at = a.at + (size_t)unit * a.cap;
  const int e0 = threadIdx.x / P;
  uint4 v[kSteps];
  int from[kSteps];
  auto places = [&](int j0) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int j = j0 + s * E + e0;
      from[s] = j < keep ? at[j] : -1;
    }
  };
  auto read = [&]() {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (from[s] >= 0) v[s] = *reinterpret_cast<const uint4*>(x + (size_t)from[s] * D);
  };
  places(first);
  read();
  for (int j0 = first; j0 < keep; j0 += T) {
    uint4 w[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) w[s] = v[s];
    places(j0 + T);
    read();
    __syncthreads();  // every thread has read this tile
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int j = j0 + s * E + e0;
      if (j < keep) *reinterpret_cast<uint4*>(x + (size_t)j * D) = w[s];
    }
  }
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
  // (an eviction of 200 entries of the tiny decoder took 17.0 us with 1024 threads and
  // 13.5 with 256 on one machine: fewer warps wait for one another.  14.4 to 18.3 over machines.)
  const cudaError_t e =
      a.cap <= 4096    ? launch_pdl(evict_select_kernel<256, 16>, dim3(units), dim3(256), 0, st, 1, a)
      : a.cap <= 16384 ? launch_pdl(evict_select_kernel<1024, 16>, dim3(units), dim3(1024), 0, st, 1, a)
                       : launch_pdl(evict_select_kernel<1024, 64>, dim3(units), dim3(1024), 0, st, 1, a);
  if (e != cudaSuccess) return e;
  return head_dim == 128 ? launch_pdl(evict_move_kernel<128>, dim3(units, 4), dim3(kMove), 0, st, 1, a)
                         : launch_pdl(evict_move_kernel<64>, dim3(units, 2), dim3(kMove), 0, st, 1, a);
}

}  // namespace as2d
