// k_attn_weights.cu -- the weight that attention gives each cache entry
// (as2d_attention_weights): over a request's rows i and the query heads h of a
// kv head, w_t (+)= sum e^(scale q_ih k_t - lse_ih).
//
// The product is taken with the keys as the MMA's rows, S^T = K Q^T (M = 128 keys,
// N = the queries, padded to 16): a thread owns a key and adds the exponentials
// of its row of TMEM, so that no sum crosses threads, the order of every sum is
// fixed, and each weight is read and written once by one thread.  32-bit queries
// are bf16 hi and lo parts, two products.
//
// Work is cut as in k_tree_attn.cu: the key tiles of every (request, kv head),
// weighted by the tiles of 128 queries that go over them, in even shares over one
// CTA per SM; a tile belongs to the CTA in whose share its first unit falls.
// Per CTA: warp 0 loads key tiles by TMA through a ring (and the next one into L2
// while the ring is full), warp 1 issues the products into four TMEM buffers, warps
// 2-9 bring in the queries and their sums (a pass ahead, into registers: with two
// warps, after the last product of a pass, turning took 6 us), warps 10-13 and
// 14-17 take the tiles in turn.  More than 128 queries: one pass over the CTA's
// tiles for each 128 (the keys then come from L2).
//
// Bound by memory: each key is read once (16 ragged requests, 64 MB: 21.5 us, of
// which 10 at 6 TB/s in the loop, 4 until the first product, 2 for each turn), for few
// entries by latency (9 rows over 814 entries of two kv heads: 8.0 to 9.2 us).
#include <type_traits>

#include "ops.h"
#include "ptx_sm100.cuh"
#include "tree_dev.cuh"

namespace as2d {
namespace {

// Threads that bring in queries: those of 128 in registers at once.
constexpr int kBring = 256, kThreads = 64 + kBring + 256;
// What turning to another head costs a CTA, in tiles (where a CTA has several): 16
// ragged requests take 24.1 / 22.5 / 22.2 / 22.4 / 22.6 us with 1 / 2 / 3 / 4 / 5.
constexpr int kTurn = 3;

template <int D, bool F32>
struct Shape {
  static constexpr uint32_t STAGE = 128 * D * 2;
  static constexpr uint32_t Q = (F32 ? 2 : 1) * 128 * D * 2;
  static constexpr int NST = D == 64 ? 8 : F32 ? 4 : 5;
  static constexpr uint32_t SMEM = 1024 + Q + NST * STAGE + 2 * 128 * (4 + 8) + (2 * NST + 16) * 8 + 16;
  static_assert(SMEM + sizeof(UnitPlan) <= 232448, "shared memory of one CTA");
};

// The tiles of one (request, kv head) in units [u, u1): [t0, t1); the first unit
// after them.  A head's units: what its passes' turns count (UnitPlan::extra), then
// its tiles one after another, `passes` units each.
struct Segment {
  Unit it;
  int next, passes;
};
__device__ __forceinline__ Segment segment_at(const UnitPlan& p, const TreeArgs& a, int u, int u1) {
  Segment s;
  s.it = unit_at(p, a, u, u1);  // (for the request; the rest is in another order here)
  const int b = s.it.b, extra = p.qts[b] * p.extra, per = p.tiles[b] * p.qts[b] + extra, rel = u - p.unit[b];
  s.passes = p.qts[b];
  s.it.g = rel / per;
  const int r0 = rel - s.it.g * per, r1 = min(per, r0 + (u1 - u));
  s.next = u + r1 - r0;
  s.it.t0 = (max(r0 - extra, 0) + s.passes - 1) / s.passes;
  s.it.t1 = (max(r1 - extra, 0) + s.passes - 1) / s.passes;
  s.it.qt = 0;
  return s;
}
// The same of the first head from u on of which there is a tile to do; u: the first
// unit after it.
__device__ __forceinline__ bool next_segment(const UnitPlan& p, const TreeArgs& a, int& u, int u1, Segment& s) {
  while (u < u1) {
    s = segment_at(p, a, u, u1);
    u = s.next;
    if (s.it.t0 < s.it.t1) return true;
  }
  return false;
}

// Adds the exponentials of 16 queries from column q0 on; masked: of those, q < n,
// that see the thread's key.  need: its bit in a word of seen's masks (0: all see it),
// upper: in their upper words.
template <bool MASKED>
__device__ __forceinline__ void add_weights(const uint32_t (&v)[16], uint64_t c2, const float* lse, const uint2* seen,
                                            int q0, int n, uint32_t need, bool upper, uint64_t (&sum)[2]) {
#pragma unroll
  for (int e = 0; e < 16; e += 4) {
    const float4 l = *reinterpret_cast<const float4*>(lse + q0 + e);  // (negated)
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const uint64_t less = k == 0 ? two(l.x, l.y) : two(l.z, l.w);
      const float2 y = of_two(fma2(two(__uint_as_float(v[e + k]), __uint_as_float(v[e + k + 1])), c2, less));
      float p0 = ex2(y.x), p1 = ex2(y.y);
      if (MASKED) {
        const int q = q0 + e + k;
        const uint4 m = *reinterpret_cast<const uint4*>(seen + q);
        const uint32_t w0 = upper ? m.y : m.x, w1 = upper ? m.w : m.z;
        p0 = q < n && (w0 & need) == need ? p0 : 0.f;
        p1 = q + 1 < n && (w1 & need) == need ? p1 : 0.f;
      }
      sum[k >> 1] = add2(sum[k >> 1], two(p0, p1));
    }
  }
}

// The weight of one key of 32-bit queries q0 .. q0 + n - 1 of a head, that came out as NaN, by a whole warp:
// if the key holds infinities (and no NaN) once more in 32-bit arithmetic, as in hi and lo
// parts a score of -inf may be NaN.
template <int D>
__device__ __forceinline__ float weight_of(const TreeArgs& a, const Unit& it, int q0, int n, int key, const float* lse,
                                           const uint2* seen, uint32_t need, bool upper, int lane) {
  const bf16* k = a.k + (((size_t)it.b * a.nkv + it.g) * a.cap + key) * D;
  if (!infinite_key<D>(k, lane)) return NAN;
  const int G = a.nq / a.nkv;
  float sum = 0.f;
#pragma unroll 1
  for (int q = lane; q < n; q += 32) {
    const uint32_t w = upper ? seen[q].y : seen[q].x;
    if ((w & need) != need) continue;
    const int i = divide_group(a, q0 + q);
    const float* x = (const float*)a.q + (it.r0 + i) * a.q_stride + (int64_t)(it.g * G + (q0 + q - i * G)) * D;
    sum += ex2(fmaf(exact_product<D>(x, k), a.scale_log2, lse[q]));
  }
  __syncwarp();
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  return sum;
}

template <int D, bool F32>
__global__ void __launch_bounds__(kThreads, 1)
    attn_weights_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ WeightArgs wa, int turn) {
  using S = Shape<D, F32>;
  constexpr int NST = S::NST, NR = D / 64;
  constexpr int kInFlight = 128 * (D / 8) / kBring;  // all of 128 queries
  const TreeArgs& a = wa.t;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* qimg = sm;
  uint8_t* ring = sm + S::Q;
  // of a pass, by its parity
  float* s_lse = reinterpret_cast<float*>(ring + NST * S::STAGE);  // [2][128] base 2, negated
  uint64_t* s_vis = reinterpret_cast<uint64_t*>(s_lse + 2 * 128);  // [2][128]
  uint64_t* full = s_vis + 2 * 128;
  uint64_t* empty = full + NST;
  uint64_t* s_full = empty + NST;   // [4]
  uint64_t* s_empty = s_full + 4;   // [4]
  uint64_t* q_first = s_empty + 4;
  uint64_t* q_full = q_first + 1;
  uint64_t* q_empty = q_full + 1;
  uint64_t* e_empty = q_empty + 1;  // [2]
  uint64_t* e_full = e_empty + 2;   // [2]
  uint64_t* drain = e_full + 2;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(drain + 1);
  __shared__ UnitPlan plan;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      ptx::mbar_init(&full[i], 1);
      ptx::mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(&s_full[i], 1);
      ptx::mbar_init(&s_empty[i], 4);
    }
    ptx::mbar_init(q_first, kThreads / 32 - 2);
    ptx::mbar_init(q_full, kBring / 32);
    ptx::mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&e_empty[i], 8);
      ptx::mbar_init(&e_full[i], 4);
    }
    ptx::mbar_init(drain, 1);
    ptx::fence_mbar_init();
  }
  if (warp == 1) ptx::tmem_alloc(tslot, 512);
  if (warp == 0 && lane == 0) ptx::prefetch_tmap(&tmK);
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  if (warp == 0) make_plan(a, 128, turn, lane, plan, blockIdx.x == 0, wa.skip);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tslot;
  const int G = a.nq / a.nkv;
  int u0, u1;
  unit_range(plan, blockIdx.x, gridDim.x, u0, u1);
  const unsigned long long limit = a.timeout_ns;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok && !ptx::mbar_spin(bar, parity, limit)) {
      ok = false;
      if (a.err) atomicOr(a.err, kErrTimeout);
    }
    return ok;
  };
  // queries of a pass (zeros up to the next 16th), by N threads from t on
  auto bring = [&](const Unit& it, int t, auto n_threads, auto in_flight, auto later, auto ready) {
    constexpr int N = decltype(n_threads)::value;
    load_queries<D, F32, N, decltype(in_flight)::value, decltype(later)::value>(a, it, t, qimg, ready);
    const int n0 = it.qt * 128, n = min(128, it.rows * G - n0), pad = (n + 15) & ~15;
    for (int c = t; c < (pad - n) * (D / 8); c += N) {
      uint8_t* to = qimg + chunk_off(n + c / (D / 8), c % (D / 8));
      *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
      if (F32) *reinterpret_cast<uint4*>(to + 128 * D * 2) = make_uint4(0, 0, 0, 0);
    }
    ptx::fence_proxy_async_smem();
  };
  // the sum of query q of a pass and which rows it sees
  auto sums_of = [&](const Unit& it, int q, float& l, uint64_t& vis) {
    const int n0 = it.qt * 128, n = min(128, it.rows * G - n0);
    l = 0.f;
    vis = 0;
    if (q >= n) return;
    const int i = divide_group(a, n0 + q), h = it.g * G + (n0 + q - i * G);
    l = a.lse[(size_t)(it.r0 + i) * a.nq + h] * -1.4426950408889634f;
    vis = visible_rows(a, it.r0 + i, i, it.rows);
  };
  Segment s;
  if (int u = u0; warp >= 2 && next_segment(plan, a, u, u1, s)) {
    // the first pass, by every warp that has nothing to do yet
    const int q = tid - 64;
    bring(s.it, q, std::integral_constant<int, kThreads - 64>{}, std::integral_constant<int, 4>{}, std::false_type{},
          [&] {
            if (q < 128) sums_of(s.it, q, s_lse[q], s_vis[q]);
          });
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(q_first);
  }

  if (warp == 0) {
    if (lane == 0) {
      const uint64_t pol = ptx::policy_evict_first();
      Stage at;
      uint32_t n = 0;
      auto load = [&](int t, int z) {
        const uint32_t k = at.next<NST>(), i = Stage::slot(k);
        if (n >= NST && !wait(&empty[i], Stage::parity(k) ^ 1)) return;
        ptx::mbar_arrive_expect_tx(&full[i], S::STAGE);
#pragma unroll
        for (int h = 0; h < NR; ++h)
          ptx::tma_load_3d(ring + i * S::STAGE + h * kRegion, &tmK, &full[i], 64 * h, t * 128, z, pol);
        ++n;
      };
      int before = -1, z_before = 0;  // the tile that is on its way to L2 while the ring is full
      for (int u = u0; next_segment(plan, a, u, u1, s);) {
        const int z = s.it.b * a.nkv + s.it.g;
        for (int qt = 0; qt < s.passes; ++qt)
          for (int t = s.it.t0; t < s.it.t1 && ok; ++t) {
            if (before >= 0) load(before, z_before);
#pragma unroll
            for (int h = 0; h < NR; ++h) ptx::tma_prefetch_3d(&tmK, 64 * h, t * 128, z);
            before = t;
            z_before = z;
          }
      }
      if (ok && before >= 0) load(before, z_before);
      // no copy is in flight when the CTA ends
      for (uint32_t i = n > NST ? n - NST : 0; i < n; ++i)
        ptx::mbar_wait(&full[i % NST], (i / NST) & 1, ptx::kDrainNs);
    }
  } else if (warp == 1) {
    // the whole warp, for operands in uniform registers; one thread issues
    const uint32_t lead = ptx::elect_one(), tm = __shfl_sync(~0u, tmem, 0);
    const uint32_t q_lo = ptx::desc_lo(ptx::smem_u32(qimg), 16u);
    auto whole = [&](bool) { return ok = __all_sync(~0u, ok); };
    Stage at;
    uint32_t done[2] = {0, 0}, pass = 0;  // tiles of each group so far
    for (int u = u0; ok && next_segment(plan, a, u, u1, s);) {
      const int tiles = __shfl_sync(~0u, s.it.t1 - s.it.t0, 0), queries = __shfl_sync(~0u, s.it.rows * G, 0);
      for (int qt = 0; qt * 128 < queries && ok; ++qt, ++pass) {
        whole(pass == 0 ? wait(q_first, 0) : wait(q_full, (pass - 1) & 1));
        const uint32_t idesc = ptx::idesc_bf16_f32(128, (min(128, queries - qt * 128) + 15) & ~15);
        for (int t = 0; t < tiles && ok; ++t) {
          const int odd = t & 1;
          const uint32_t d = odd ? done[1] : done[0], buf = odd + 2 * (d & 1);
          const uint32_t k = at.next<NST>(), i = Stage::slot(k);
          wait(&full[i], Stage::parity(k));
          if (d >= 2) wait(&s_empty[buf], ((d >> 1) - 1) & 1);
          if (!whole(ok)) break;
          ptx::tc_fence_after();
          const uint32_t kt = ptx::desc_lo(ptx::smem_u32(ring + i * S::STAGE), 16u), ds = tm + 128 * buf;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t to = ((kk >> 2) * kRegion + 32u * (kk & 3)) >> 4;
            ptx::mma_bf16_lo(lead, ds, kt + to, q_lo + to, idesc, kk > 0 ? 1u : 0u);
            if (F32) ptx::mma_bf16_lo(lead, ds, kt + to, q_lo + to + (128u * D * 2 >> 4), idesc, 1u);
          }
          ptx::mma_commit_if(lead, &s_full[buf]);
          ptx::mma_commit_if(lead, &empty[i]);
          if (t == tiles - 1) ptx::mma_commit_if(lead, q_empty);
          if (odd)
            ++done[1];
          else
            ++done[0];
        }
      }
    }
    // no product is running when TMEM is freed
    ptx::mma_commit_if(lead, drain);
    ptx::mbar_wait(drain, 0, ptx::kDrainNs);
  } else if (warp < 2 + kBring / 32) {
    const int q = tid - 64;
    uint32_t pass = 0;
    for (int u = u0; next_segment(plan, a, u, u1, s);) {
      for (int qt = 0; qt < s.passes; ++qt, ++pass) {
        if (pass == 0) continue;
        s.it.qt = qt;
        float l;
        uint64_t vis;
        if (q < 128) sums_of(s.it, q, l, vis);
        bring(s.it, q, std::integral_constant<int, kBring>{}, std::integral_constant<int, kInFlight>{},
              std::true_type{}, [&] { wait(q_empty, (pass - 1) & 1); });
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(q_full);
        if (q < 128) {
          // the sums of the pass before the last have been read
          if (pass > 1) wait(&e_empty[pass & 1], ((pass >> 1) - 1) & 1);
          s_lse[128 * (pass & 1) + q] = l;
          s_vis[128 * (pass & 1) + q] = vis;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&e_full[pass & 1]);
        }
      }
    }
  } else {
    const int group = (warp - 2 - kBring / 32) >> 2, row = 32 * (warp & 3) + lane;  // key of the tile, TMEM lane
    const uint32_t tl = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint64_t c2 = two(a.scale_log2, a.scale_log2);
    uint32_t d = 0, pass = 0;
    for (int u = u0; next_segment(plan, a, u, u1, s);) {
      float* w = wa.w + ((size_t)s.it.b * a.nkv + s.it.g) * a.cap;
      for (int qt = 0; qt < s.passes; ++qt, ++pass) {
        const int n = min(128, s.it.rows * G - qt * 128);
        const float* lse = s_lse + 128 * (pass & 1);
        const uint2* seen = reinterpret_cast<const uint2*>(s_vis + 128 * (pass & 1));
        pass == 0 ? wait(q_first, 0) : wait(&e_full[pass & 1], ((pass - 1) >> 1) & 1);
        for (int t = s.it.t0 + group; t < s.it.t1; t += 2, ++d) {
          const int key = t * 128 + row, j = key - s.it.L;
          const bool live = j < s.it.rows;
          // its weight so far, on its way while the product runs
          const float before = live && (j < 0 || qt > 0) ? w[key] : 0.f;
          const uint32_t buf = group + 2 * (d & 1);
          wait(&s_full[buf], (d >> 1) & 1);
          ok = __all_sync(~0u, ok);
          ptx::tc_fence_after();
          const bool tail = t * 128 + 128 > s.it.L, upper = j >= 32;
          const uint32_t need = j < 0 ? 0u : 1u << (j & 31);
          uint64_t sum[2] = {0, 0};
#pragma unroll 1
          for (int q = 0; q < n; q += 32) {
            uint32_t v[2][16];
            ptx::tmem_ld16(tl + 128 * buf + q, v[0]);
            if (q + 16 < n) ptx::tmem_ld16(tl + 128 * buf + q + 16, v[1]);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
              if (q + h >= n) break;
              if (tail || q + h + 16 > n)
                add_weights<true>(v[h >> 4], c2, lse, seen, q + h, n, need, upper, sum);
              else
                add_weights<false>(v[h >> 4], c2, lse, seen, q + h, n, need, upper, sum);
            }
          }
          const float2 sums = of_two(add2(sum[0], sum[1]));
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&s_empty[buf]);
          float more = sums.x + sums.y;
          if (F32)
            for (unsigned left = __ballot_sync(~0u, ok && live && more != more); left; left &= left - 1) {
              const int of = __ffs(left) - 1;
              const float y = weight_of<D>(a, s.it, qt * 128, n, __shfl_sync(~0u, key, of), lse, seen,
                                           __shfl_sync(~0u, need, of), __shfl_sync(~0u, (int)upper, of), lane);
              if (lane == of) more = y;
            }
          if (live && ok) w[key] = before + more;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&e_empty[pass & 1]);
      }
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

template <int D, bool F32>
cudaError_t launch(const CUtensorMap& tk, const WeightArgs& a, int ctas, int turn, cudaStream_t st) {
  using S = Shape<D, F32>;
  static PerDevice opted;
  const cudaError_t e = opt_in(opted, attn_weights_kernel<D, F32>, S::SMEM);
  if (e != cudaSuccess) return e;
  return launch_pdl(attn_weights_kernel<D, F32>, dim3(ctas), dim3(kThreads), S::SMEM, st, 1, tk, a, turn);
}

}  // namespace

cudaError_t launch_attention_weights(const WeightArgs& a, int head_dim, int64_t max_keys, cudaStream_t st) {
  const int sms = device_sms();
  CUtensorMap tk;
  if (!encode_cache_map(&tk, a.t.k, head_dim, a.t.cap, (int64_t)a.t.rm.batch * a.t.nkv)) return cudaErrorInvalidValue;
  const int64_t units = (max_keys + 127) / 128 * tree_items(a.t);
  const int ctas = (int)(units < sms ? units : sms), turn = units > sms ? kTurn : 0;
  if (head_dim == 128)
    return a.t.q_f32 ? launch<128, true>(tk, a, ctas, turn, st) : launch<128, false>(tk, a, ctas, turn, st);
  return a.t.q_f32 ? launch<64, true>(tk, a, ctas, turn, st) : launch<64, false>(tk, a, ctas, turn, st);
}

}  // namespace as2d
