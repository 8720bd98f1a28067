// k_sampled.cu -- probabilities at a temperature (as2d_token_probs) and the
// acceptance of drafted tokens from given random numbers (as2d_accept_sampled).
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "ops.h"
#include "ptx_sm100.cuh"
#include "small_dev.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- probabilities -----------------------------------------------------------
//
// p_v = e^((x_v - max x) / T) / sum: bound by memory, each value read and written
// once.  A cluster of CTAs per row, a slice of it in the registers of each: a
// thread's maximum m_t, e^((x - m_t) / T) and their sum, then one reduction of
// (maximum, sum) over the block and, through distributed shared memory, the
// cluster, and the factor that is left to each thread.  Slices that the registers
// do not hold (kHeld values a thread) are read again.  VEC: rows in pieces of 16
// bytes.

// Bound by latency for few rows (9 of 152064 values 5.2 us), by memory for many (145:
// 35.4 us, 5.0 TB/s).
//
// Threads, values a thread holds, CTAs per SM.  145 rows of 152064 values, us: 512 /
// 40 / 2 39, 256 / 40 / 4 42, 256 / 48 / 3 41, 128 / 40 / 8 45, 1024 / 24 / 1 55
// (the copy peak takes 26).
constexpr int kProbs = 512, kHeld = 40, kProbsCtas = 2, kProbsWarps = kProbs / 32;

// (maximum, sum relative to it) of two parts; -inf: nothing there.
__device__ __forceinline__ float2 join(float2 a, float2 b, float c) {
  const float M = fmaxf(a.x, b.x);
  const float wa = a.x == -INFINITY ? 0.f : ex2((a.x - M) * c), wb = b.x == -INFINITY ? 0.f : ex2((b.x - M) * c);
  return make_float2(M, (a.x == -INFINITY ? a.y : a.y * wa) + (b.x == -INFINITY ? b.y : b.y * wb));
}

// (maximum, sum) of the row from each thread's, over the block and the cluster.  start: the
// first row of a cluster whose CTAs have arrived at its barrier; their shared memory is written once
// all of them have started.
__device__ __forceinline__ float2 join_row(float2 all, float c, uint32_t rank, uint32_t ranks, float2* s_warp,
                                           float2* s_part, bool start) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    all = join(all, make_float2(__shfl_xor_sync(~0u, all.x, o), __shfl_xor_sync(~0u, all.y, o)), c);
  if (lane == 0) s_warp[warp] = all;
  __syncthreads();
  all = s_warp[lane % kProbsWarps];
#pragma unroll
  for (int o = kProbsWarps / 2; o > 0; o >>= 1)
    all = join(all, make_float2(__shfl_xor_sync(~0u, all.x, o), __shfl_xor_sync(~0u, all.y, o)), c);
  if (ranks > 1) {
    if (start) ptx::cluster_wait();
    if (tid < (int)ranks) {
      const uint32_t to = ptx::dsmem_map(ptx::smem_u32(&s_part[rank]), tid);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(all.x), "f"(all.y) : "memory");
    }
    ptx::cluster_sync();
    all = s_part[lane % ranks];
    for (int o = ranks / 2; o > 0; o >>= 1)
      all = join(all, make_float2(__shfl_xor_sync(~0u, all.x, o), __shfl_xor_sync(~0u, all.y, o)), c);
  }
  return all;
}

template <bool VEC>
__global__ void __launch_bounds__(kProbs, kProbsCtas) probs_kernel(const float* logits, int vocab, int slice, float c,
                                                          float* probs) {
  constexpr int W = VEC ? 4 : 1, R = kHeld / W;
  __shared__ float2 s_warp[kProbsWarps], s_part[16];
  const int tid = threadIdx.x;
  const uint32_t rank = ptx::cluster_rank(), ranks = gridDim.x;
  const int v0 = min((int)rank * slice, vocab), n = (min(v0 + slice, vocab) - v0) / W;  // pieces
  const float* x = logits + (size_t)blockIdx.y * vocab + v0;
  float* p = probs + (size_t)blockIdx.y * vocab + v0;
  if (ranks > 1) ptx::cluster_arrive_relaxed();
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  float v[R][W];
  auto load = [&](int i, float (&to)[W]) {
    if constexpr (VEC) {
      const float4 t = __ldcs(reinterpret_cast<const float4*>(x) + i);
      to[0] = t.x, to[1] = t.y, to[2] = t.z, to[3] = t.w;
    } else {
      to[0] = __ldcs(x + i);
    }
  };
  auto store = [&](int i, const float (&from)[W]) {
    if constexpr (VEC)
      __stcs(reinterpret_cast<float4*>(p) + i, make_float4(from[0], from[1], from[2], from[3]));
    else
      __stcs(p + i, from[0]);
  };
  float m = -INFINITY;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = r * kProbs + tid;
#pragma unroll
    for (int e = 0; e < W; ++e) v[r][e] = -INFINITY;
    if (i < n) load(i, v[r]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < W; ++e) m = fmaxf(m, v[r][e]);
  for (int i = R * kProbs + tid; i < n; i += kProbs) {
    float t[W];
    load(i, t);
#pragma unroll
    for (int e = 0; e < W; ++e) m = fmaxf(m, t[e]);
  }
  const float ref = m == -INFINITY ? 0.f : m;  // (e^-inf = 0; NaN passes the maximum by and reaches the sum)
  float l = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < W; ++e) {
      v[r][e] = ex2((v[r][e] - ref) * c);
      l += v[r][e];
    }
  for (int i = R * kProbs + tid; i < n; i += kProbs) {
    float t[W];
    load(i, t);
#pragma unroll
    for (int e = 0; e < W; ++e) l += ex2((t[e] - ref) * c);
  }
  const float2 all = join_row(make_float2(m, l), c, rank, ranks, s_warp, s_part, true);
  // (a thread that holds nothing has zeros, a row that holds nothing gets them)
  const float f = all.y == 0.f ? 0.f : (m == -INFINITY ? 1.f : ex2((m - all.x) * c)) / all.y;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = r * kProbs + tid;
#pragma unroll
    for (int e = 0; e < W; ++e) v[r][e] *= f;
    if (i < n) store(i, v[r]);
  }
  for (int i = R * kProbs + tid; i < n; i += kProbs) {
    float t[W];
    load(i, t);
#pragma unroll
    for (int e = 0; e < W; ++e) t[e] = ex2((t[e] - ref) * c) * f;
    store(i, t);
  }
}

// The same for more rows than clusters run at once (rows in pieces of 16 bytes,
// slices that the registers hold): the clusters stay, each goes from row to row,
// and while a row is worked on and written the next one is on its way into shared
// memory (each thread's own pieces, so that only the sums are waited for).
__global__ void __launch_bounds__(kProbs, kProbsCtas) probs_rows_kernel(const float* logits, int rows, int vocab,
                                                                       int slice, float c, float* probs) {
  constexpr int R = kHeld / 4;
  extern __shared__ float4 s_next[];  // [R][kProbs]
  __shared__ float2 s_warp[2][kProbsWarps], s_part[2][16];
  const int tid = threadIdx.x;
  const uint32_t rank = ptx::cluster_rank(), ranks = gridDim.x;
  const int v0 = min((int)rank * slice, vocab), n = (min(v0 + slice, vocab) - v0) / 4;  // pieces
  if (ranks > 1) ptx::cluster_arrive_relaxed();
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  auto fetch = [&](int row) {
    const float4* x = reinterpret_cast<const float4*>(logits + (size_t)row * vocab + v0);
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * kProbs + tid < n) ptx::cp_async16(&s_next[r * kProbs + tid], x + r * kProbs + tid);
  };
  if ((int)blockIdx.y < rows) fetch(blockIdx.y);
  for (int row = blockIdx.y, turn = 0; row < rows; row += gridDim.y, turn ^= 1) {
    float4 v[R];
    float m = -INFINITY;
    ptx::cp_async_wait_all();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      v[r] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (r * kProbs + tid < n) v[r] = s_next[r * kProbs + tid];
      m = fmaxf(m, fmaxf(fmaxf(v[r].x, v[r].y), fmaxf(v[r].z, v[r].w)));
    }
    if (row + (int)gridDim.y < rows) fetch(row + gridDim.y);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      v[r] = make_float4(ex2((v[r].x - ref) * c), ex2((v[r].y - ref) * c), ex2((v[r].z - ref) * c),
                         ex2((v[r].w - ref) * c));
      l += (v[r].x + v[r].y) + (v[r].z + v[r].w);
    }
    const float2 all =
        join_row(make_float2(m, l), c, rank, ranks, s_warp[turn], s_part[turn], row == (int)blockIdx.y);
    const float f = all.y == 0.f ? 0.f : (m == -INFINITY ? 1.f : ex2((m - all.x) * c)) / all.y;
    float4* p = reinterpret_cast<float4*>(probs + (size_t)row * vocab + v0);
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * kProbs + tid < n)
        __stcs(p + r * kProbs + tid, make_float4(v[r].x * f, v[r].y * f, v[r].z * f, v[r].w * f));
  }
}

// ---- acceptance ------------------------------------------------------------------
//
// A cluster of CTAs per request.  Each finds n from the candidates' tests (one
// gather), then sums its slice of row n's weights w_v = max(p_v - q_v, 0): the
// slice lies in shared memory and a thread adds a contiguous chunk of it, each
// difference exactly (as the sum of two floats, Knuth's two-sum) and the sum in
// two floats, so that the border u total falls between the same two tokens as in
// 64 bits but for differences of some 2^-46.  The threads' sums are
// scanned by shuffles, the CTAs exchange their totals, and the thread whose sums
// the border lies between finds the token in its chunk.  All of it in pairs of
// floats: in 64 bits, at this card's rate and latency for them, the additions of
// one request took 9 of 22 us.  Bound by latency for a few requests (three
// dependent round trips to memory: one without draft 7.0 us).  What bounds more of them has
// not been found: 16 with draft take 15.0 us with 16 CTAs each, of which 14 clusters run at
// once, and 14.1, 17.7 and 14.4 with 12, 10 and 9, of which all run.

// a + b = s + e exactly.
__device__ __forceinline__ void two_sum(float a, float b, float& s, float& e) {
  s = a + b;
  const float t = s - a;
  e = (a - (s - t)) + (b - t);
}

// A number as the sum of two floats, |y| at most half a step of x.
__device__ __forceinline__ float2 pair_of(float x, float y) {
  const float s = x + y;
  return make_float2(s, y - (s - x));
}
__device__ __forceinline__ float2 add(float2 a, float2 b) {
  float s, e;
  two_sum(a.x, b.x, s, e);
  return pair_of(s, e + (a.y + b.y));
}
__device__ __forceinline__ bool less(float2 a, float2 b) { return a.x < b.x || (a.x == b.x && a.y < b.y); }
// Inclusive sums over the first N lanes of each N.
template <int N>
__device__ __forceinline__ float2 scan(float2 v, int lane) {
#pragma unroll
  for (int o = 1; o < N; o <<= 1) {
    const float2 t = make_float2(__shfl_up_sync(~0u, v.x, o, N), __shfl_up_sync(~0u, v.y, o, N));
    if ((lane & (N - 1)) >= o) v = add(t, v);
  }
  return v;
}
__device__ __forceinline__ float2 from_lane(float2 v, int lane) {
  return make_float2(__shfl_sync(~0u, v.x, lane), __shfl_sync(~0u, v.y, lane));
}

constexpr int kMostChunk = 53;    // values of a thread's chunk at most: two rows of a slice fit shared memory
constexpr int kMostPieces = 128;  // pieces of a slice that shared memory holds one after another
static_assert(kWarps == 16, "the warps' sums and the CTAs' are scanned by 16 lanes");

// VEC: rows in pieces of 16 bytes.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) accept_sampled_kernel(const __grid_constant__ SampledArgs a, int chunk,
                                                                  int pieces) {
  extern __shared__ __align__(16) float s_row[];  // [512 chunks] p, then q
  __shared__ float2 s_part[2][16], s_warp[kWarps], s_piece[kMostPieces];
  __shared__ int s_n, s_pick, s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.y, ranks = gridDim.x, rank = (int)ptx::cluster_rank();
  const int r0 = a.start[b], k = a.start[b + 1] - r0 - 1, c0 = r0 - b;
  const size_t V = a.vocab;
  const int piece = chunk * kThreads;
  ptx::cluster_arrive_relaxed();
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  if (warp == 0) {
    bool stands = false;
    if (lane < k) {
      const int c = a.cand[c0 + lane];
      if (c >= 0 && c < a.vocab) {
        // (products of two floats and their comparison are exact in 64 bits)
        const double q = a.draft ? (double)a.draft[(size_t)(c0 + lane) * V + c] : 1.0;
        stands = (double)a.u[r0 + lane] * q < (double)a.probs[(size_t)(r0 + lane) * V + c];
      }
    }
    const unsigned m = __ballot_sync(~0u, stands);
    if (lane == 0) s_n = __ffs(~m) - 1;
  }
  __syncthreads();
  const int n = s_n, gone = n < k && !a.draft ? a.cand[c0 + n] : -1;
  const float* p = a.probs + (size_t)(r0 + n) * V;
  const float* q = n < k && a.draft ? a.draft + (size_t)(c0 + n) * V : nullptr;
  // (within [0, 1): the border is below the total)
  const float u = fminf(fmaxf(a.u[r0 + k], 0.f), 0x1.fffffep-1f);
  float *sp = s_row, *sq = s_row + piece;

  auto weight = [&](int j, bool minus, float& hi, float& lo) {
    hi = sp[j], lo = 0.f;
    if (minus) two_sum(hi, -sq[j], hi, lo);
    if (!(hi > 0.f && hi < INFINITY)) hi = lo = 0.f;
  };
  // Piece i of the slice into shared memory: its first token, the thread's sum
  // and the sum up to and with it, and of all threads.
  float2 mine, upto, all;
  auto stage = [&](int i, bool plain) {
    const int v0 = (int)min((long long)(rank * pieces + i) * piece, (long long)a.vocab), len = min(piece, a.vocab - v0);
    const bool minus = q && !plain;
    using T = std::conditional_t<VEC, float4, float>;
    constexpr int W = VEC ? 4 : 1, U = VEC ? 5 : 20;
    const T *pv = reinterpret_cast<const T*>(p + v0), *qv = reinterpret_cast<const T*>(q + v0);
    __syncthreads();
    if (tid == 0) s_pick = 0x7fffffff, s_last = -1;
    for (int j0 = tid; j0 < len / W; j0 += U * kThreads) {
      T x[U], y[U];
#pragma unroll
      for (int t = 0; t < U; ++t)
        if (j0 + t * kThreads < len / W) {
          x[t] = __ldcs(pv + j0 + t * kThreads);
          if (minus) y[t] = __ldcs(qv + j0 + t * kThreads);
        }
#pragma unroll
      for (int t = 0; t < U; ++t) {
        const int j = j0 + t * kThreads;
        if (j < len / W) {
          reinterpret_cast<T*>(sp)[j] = x[t];
          if (minus) reinterpret_cast<T*>(sq)[j] = y[t];
        }
      }
    }
    __syncthreads();
    if (!plain && gone >= v0 && gone < v0 + len) {
      if (tid == 0) sp[gone - v0] = 0.f;
      __syncthreads();
    }
    float s = 0.f, e = 0.f;
    for (int j = tid * chunk; j < min((tid + 1) * chunk, len); ++j) {
      float hi, lo, t;
      weight(j, minus, hi, lo);
      two_sum(s, hi, s, t);
      e += t + lo;
    }
    mine = pair_of(s, e);
    upto = scan<32>(mine, lane);
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    const float2 w = scan<16>(s_warp[lane & 15], lane);
    all = from_lane(w, 15);
    if (warp > 0) upto = add(from_lane(w, warp - 1), upto);
    return v0;
  };
  for (int plain = n < k ? 0 : 1, first = 1; plain < 2; ++plain, first = 0) {
    float2 sum = make_float2(0.f, 0.f);
    int v0 = 0;
    for (int i = 0; i < pieces; ++i) {
      v0 = stage(i, plain);
      if (tid == 0) s_piece[i] = all;
      sum = add(sum, all);
    }
    if (first) ptx::cluster_wait();  // every CTA has started: its shared memory can be written
    if (tid < ranks) {
      const uint32_t to = ptx::dsmem_map(ptx::smem_u32(&s_part[plain][rank]), tid);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(sum.x), "f"(sum.y) : "memory");
    }
    ptx::cluster_sync();
    const bool part = (lane & 15) < ranks;
    const float2 own = part ? s_part[plain][lane & 15] : make_float2(0.f, 0.f), ends = scan<16>(own, lane);
    const float2 total = from_lane(ends, 15);
    if (!(total.x > 0.f)) continue;  // nothing: once more without q
    // border = u total
    const float h = u * total.x;
    const float2 border = pair_of(h, fmaf(u, total.x, -h) + u * total.y);
    // the first slice that ends above the border, else the last that holds
    // anything; of it the first piece, of that the first thread, and so on
    const unsigned over = __ballot_sync(~0u, own.x > 0.f && less(border, ends)) & 0xFFFFu;
    const unsigned any = __ballot_sync(~0u, own.x > 0.f) & 0xFFFFu;
    if (rank != (over ? __ffs(over) - 1 : 31 - __clz(any))) return;
    float2 base = rank > 0 ? from_lane(ends, rank - 1) : make_float2(0.f, 0.f);
    if (pieces > 1) {
      int pick = 0;
      float2 at = base, t = base;
      for (int i = 0; i < pieces; ++i) {
        const float2 end = add(t, s_piece[i]);
        if (s_piece[i].x > 0.f) {
          pick = i, at = t;
          if (less(border, end)) break;
        }
        t = end;
      }
      base = at;
      v0 = stage(pick, plain);
    }
    if (mine.x > 0.f) {
      if (less(border, add(base, upto))) atomicMin(&s_pick, tid);
      atomicMax(&s_last, tid);
    }
    __syncthreads();
    if (tid != (s_pick < kThreads ? s_pick : s_last)) return;
    float2 at = add(base, add(upto, make_float2(-mine.x, -mine.y)));
    int token = -1;
    for (int j = tid * chunk; j < min((tid + 1) * chunk, a.vocab - v0); ++j) {
      float hi, lo;
      weight(j, q && !plain, hi, lo);
      if (hi > 0.f) {
        token = v0 + j;
        at = add(at, make_float2(hi, lo));
        if (less(border, at)) break;
      }
    }
    a.n_out[b] = n;
    a.token_out[b] = token;
    return;
  }
  if (rank == 0 && tid == 0) {
    a.n_out[b] = n;
    a.token_out[b] = -1;
  }
}

}  // namespace

cudaError_t launch_token_probs(const float* logits, int rows, int vocab, float temperature, float* probs,
                               cudaStream_t st) {
  constexpr int kNext = kHeld * kProbs * 4;
  static PerDevice opted[3], clusters;
  cudaError_t e = opt_in(opted[0], probs_kernel<true>, 0, true);
  if (e == cudaSuccess) e = opt_in(opted[1], probs_kernel<false>, 0, true);
  if (e == cudaSuccess) e = opt_in(opted[2], probs_rows_kernel, kNext);
  if (e != cudaSuccess) return e;
  // CTAs per row: as many as hold it in registers, twice as many (up to 16) while
  // all of them run at once and a slice is no smaller than 2048 values
  int ranks = 1;
  while (ranks < 16 && (ranks * kProbs * kHeld < vocab ||
                        (ranks * 4096 <= vocab && (int64_t)rows * 2 * ranks <= device_sms())))
    ranks *= 2;
  const bool vec = vocab % 4 == 0 && ((uintptr_t)logits | (uintptr_t)probs) % 16 == 0;
  const int slice = ((vocab + ranks - 1) / ranks + 3) / 4 * 4;
  // (finite: at the smallest temperatures the maximum's own 0 c is 0, not NaN)
  const float c = (float)std::min(1.4426950408889634 / temperature, (double)FLT_MAX);
  // the clusters of eight that run at once, by the occupancy calculator less two: with
  // all of them, 36, some started late (250 rows 67 us, not 56)
  const int resident = resident_clusters(clusters, probs_rows_kernel, kProbs, kNext, 8) - 2;
  // us, a cluster to a row / this, vocab 152064: 73 rows 22.7 / 21.9, 100 27.1 / 25.6,
  // 145 38.5 / 35.4, 300 73 / 66, 400 96 / 86; 72 rows in two rounds 19.8 / 23.3, which
  // stay with the first.
  if (vec && ranks == 8 && rows > 2 * resident && resident > 0 && slice <= kHeld * kProbs) {
    const int rounds = (rows + resident - 1) / resident;
    return launch_pdl(probs_rows_kernel, dim3(8, (rows + rounds - 1) / rounds), dim3(kProbs), kNext, st, 8, logits,
                      rows, vocab, slice, c, probs);
  }
  for (int r0 = 0; r0 < rows; r0 += 65535) {  // (a grid's rows)
    const int n = rows - r0 < 65535 ? rows - r0 : 65535;
    const float* x = logits + (size_t)r0 * vocab;
    float* p = probs + (size_t)r0 * vocab;
    e = vec ? launch_pdl(probs_kernel<true>, dim3(ranks, n), dim3(kProbs), 0, st, ranks, x, vocab, slice, c, p)
            : launch_pdl(probs_kernel<false>, dim3(ranks, n), dim3(kProbs), 0, st, ranks, x, vocab, slice, c, p);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_accept_sampled(const SampledArgs& a, cudaStream_t st) {
  constexpr int kSmem = 2 * kMostChunk * kThreads * 4;
  static PerDevice opted[2];
  cudaError_t e = opt_in(opted[0], accept_sampled_kernel<true>, kSmem, true);
  if (e == cudaSuccess) e = opt_in(opted[1], accept_sampled_kernel<false>, kSmem, true);
  if (e != cudaSuccess) return e;
  // 16 CTAs a request, but 8 for many requests without a draft's rows.  us, 8 / 16,
  // vocab 152064: 4 requests 12.9 / 8.7, 16 with draft 22.3 / 17.0, 64 with draft
  // 58 / 48, 24 without 18.8 / 19.4, 64 without 33 / 43.
  const int ranks = a.draft || a.batch * 16 <= 2 * device_sms() ? 16 : 8;
  const int slice = (a.vocab + ranks - 1) / ranks;
  // (odd chunks: the threads' chunks start in different banks)
  int chunk = (slice + kThreads - 1) / kThreads | 1, pieces = 1;
  if (chunk > kMostChunk) {
    chunk = kMostChunk;
    pieces = (slice + chunk * kThreads - 1) / (chunk * kThreads);
  }
  const size_t smem = (size_t)(a.draft ? 2 : 1) * chunk * kThreads * 4;
  const bool vec = a.vocab % 4 == 0 && ((uintptr_t)a.probs | (uintptr_t)a.draft) % 16 == 0;
  return launch_pdl(vec ? accept_sampled_kernel<true> : accept_sampled_kernel<false>, dim3(ranks, a.batch),
                    dim3(kThreads), smem, st, ranks, a, chunk, pieces);
}

}  // namespace as2d
