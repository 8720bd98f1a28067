// k_tree_attn.cu -- attention of a tree of drafted tokens over a cache
// (as2d_tree_attention).
//
// Row i of request b sees the prefix [0, L_b) and those of its request's rows j,
// at L_b + j, whose bit j its mask has.  With s_t = scale q k_t over what it sees:
//   m = max s_t, l = sum e^(s_t - m), out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// All G = n_q / n_kv query heads of a kv head, for all rows of a request, form
// one query matrix of rows G queries, cut into query tiles of 128 (the MMA's M),
// so each key and value is read from memory once per call (by further query
// tiles from L2).  An item is one (request, kv head, query tile), a unit one tile of
// 128 keys of an item.  The units of all items, in order, are split evenly over
// one CTA per SM (UnitPlan), from the lengths on the device: whatever the
// requests' lengths, every SM streams the same number of bytes.  An item cut
// between CTAs leaves partial results, which tree_combine_kernel joins in CTA order;
// so results repeat bit for bit.  Small calls go other ways, without the second
// kernel (Mode): one CTA to an item of up to two tiles, or a cluster of eight, which
// joins its parts through distributed shared memory.
//
// Per CTA (20 warps, TMEM full: two score buffers, two accumulators):
//   warp 0     loads key and value tiles by TMA (3D map over the layer, 128-byte
//              swizzle) through a ring of shared-memory stages;
//   warp 1     issues the products: S = Q K^T (M = 128 queries, N = 128 keys),
//              O += P V (A = P from TMEM, V read MN-major);
//   warps 2-3  prepare the value tiles that hold entries of the call's own rows
//              (clean_tile);
//   warps 4-19 two sets of eight that take the item's key tiles in turn, half of
//              a query's keys per thread: S from TMEM, mask, running maximum (of
//              both halves, exchanged through shared memory), P = 2^(S - m) back
//              into TMEM over S as bf16 hi and lo parts (P to 2^-17), both
//              multiplied by V.  Each set has its own accumulator, maximum and sum,
//              and O is rescaled only where the maximum grew by more than 2^8 (P
//              stays below 2^8, in 32-bit sums).
// The first item's queries are brought in by warps 2-19, another's by the set that
// has no part in the last tile of the item before, while the other has.
// 32-bit queries are bf16 hi and lo parts too (two products with K; scores to 2^-17
// of |q| |k|), 16-bit ones are exact.
//
// Bound by memory for the rows of a chain or a small tree (a key and value are
// read once: 16 ragged requests, 126 MB, 39.3 us; in the loop 5.3 TB/s of a copy's
// 6.8, the rest is start, turns and join), by the products and what stands
// between them for more than 128 queries to a kv head (64 rows of seven over 15128
// entries 29.5 us, the tensor pipe 3/4 busy in the loop), by the latency of one
// chain of launch, load, products for few entries (one row over 1564: 9 to 10.7 us).
//
// What is not finite.  NaN scores pass the maxima by and reach the sums, so a row that sees NaN
// is NaN in out and lse.  Parts of bf16 products take infinities apart (hi inf + lo inf with lo
// negative or 0): a NaN in a tile's sum, and an accumulator that is not finite, make the
// warp look at the keys or values once more (mend_weights, not_finite_values), at 1.8 % of the
// ragged requests' time and none of the tree's where all is finite; an infinite value in
// 15128 entries costs 64 rows of 32-bit queries some 90 us, NaN everywhere some 100.
#include <algorithm>
#include <cfloat>

#include "ops.h"
#include "ptx_sm100.cuh"
#include "small_dev.cuh"
#include "tree_dev.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 640;
// What turning to another item costs a CTA, in tiles (where a CTA has several): its
// queries, its epilogue.  us with 3 / 4 / 5 / 6: 16 ragged requests (60 items) 46.9 /
// 42.7 / 41.4 / 42.7, a tree of 64 rows (16 items) 32.1 / 31.4 / 32.1 / 32.6.
constexpr int kTurn = 5;
// P may grow to 2^kLazy before the accumulator is rescaled.
constexpr float kLazy = 8.f;
// References from here on (base 2) are rounded by 32 and more (exponent_of); below, weights stay within 2^41.
constexpr float kFar = 1073741824.f;

// How the items go over the CTAs.
enum Mode : int {
  kShares = 0,   // even shares of all units
  kWhole = 1,    // an item to a CTA
  kCluster = 2,  // an item to a cluster of kRanks CTAs
};
constexpr int kRanks = 8;

template <int D, bool F32>
struct Shape {
  static constexpr uint32_t STAGE = 128 * D * 2;            // one K or V tile
  static constexpr uint32_t Q = (F32 ? 2 : 1) * 128 * D * 2;  // hi (and lo) image
  static constexpr int NST = D == 64 ? 8 : F32 ? 4 : 5;
  static constexpr uint32_t SMEM =
      1024 + Q + NST * STAGE + 4 * 128 * 8 + 2 * 4 * 128 * 4 + (3 * NST + 12) * 8 + 8 + 16 + 2 * sizeof(Unit);
  static_assert(SMEM + sizeof(UnitPlan) + sizeof(First) <= 232448, "shared memory of one CTA");
};

// An accumulator of weight w; infinities and NaN as they are, as no weight of the
// formula is 0.
__device__ __forceinline__ float weighted(float x, float w) { return is_finite(x) ? x * w : x; }

// Adds a part's sum and four of its dims to those of maximum M.  NaN scores pass every
// maximum by and are in the sum alone, so the sum counts whatever the part's weight (without
// NaN it is 0 where the maximum is -inf): the row is NaN wherever the work is cut.
__device__ __forceinline__ void add_part(float2 ml, float4 v, float M, float& l, float (&x)[4]) {
  const float w = part_weight(ml.x, M);
  l = fmaf(ml.y, w, l);
  x[0] += weighted(v.x, w);
  x[1] += weighted(v.y, w);
  x[2] += weighted(v.z, w);
  x[3] += weighted(v.w, w);
}

__device__ __forceinline__ void dsmem_st4(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void dsmem_st(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void dsmem_st2(uint32_t addr, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory");
}

// A value tile that holds entries from L on, before it is multiplied: entries
// past the request's last are zeroed (a stale NaN would reach O through 0 V), and
// in the entries of the call's own rows, which not every row sees, values that
// are not finite are zeroed too and their rows noted in bad: the epilogue adds
// them to the rows that do see them.
template <int D>
__device__ __forceinline__ void clean_tile(uint8_t* v, int p0, int L, int kend, int tid, unsigned long long* bad) {
  constexpr int C = D / 8, B = 4;  // chunks of a row, of a thread at once
  const int z = max(L - p0, 0), end = min(kend - p0, 128);
#pragma unroll 1
  for (int c0 = z * C + tid; c0 < end * C; c0 += 64 * B) {
    uint4 x[B];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int c = c0 + 64 * u;
      x[u] = make_uint4(0, 0, 0, 0);
      if (c < end * C) x[u] = *reinterpret_cast<const uint4*>(v + chunk_off(c / C, c % C));
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&x[u]);
      // an exponent of ones, and no other, carries into its value's sign bit
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= (w[e] & 0x7F807F80u) + 0x00800080u;
      if (!(any & 0x80008000u)) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
        if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0xFFFFu;
      }
      const int c = c0 + 64 * u;
      *reinterpret_cast<uint4*>(v + chunk_off(c / C, c % C)) = x[u];
      atomicOr(bad, 1ull << (p0 + c / C - L));
    }
  }
#pragma unroll 1
  for (int c = max(end, z) * C + tid; c < 128 * C; c += 64)
    *reinterpret_cast<uint4*>(v + chunk_off(c / C, c % C)) = make_uint4(0, 0, 0, 0);
}

// 32-bit queries are hi and lo parts, so a score of -inf (infinite keys) may come out as NaN.
// The weights P of 64 keys of a head, k the first, by a whole warp whose threads with `mine`
// found NaN in their sum: those of keys that hold infinities (and no NaN), whose score in 32 bits
// leaves them nothing beside the reference, are set to 0.  Returns the thread's sum.
template <int D>
__device__ __forceinline__ float mend_weights(uint32_t ts, bool mine, const float* q, const bf16* k, float c, float ref,
                                              float sum) {
  const int lane = threadIdx.x & 31;
  float l = 0.f;
  ptx::tmem_st_wait();
#pragma unroll 1
  for (int x = 0; x < 64; x += 16) {
    uint32_t p[16], nan = 0;  // of each 16 keys the hi parts, two in a word, then the lo parts
    ptx::tmem_ld16(ts + x, p);
    ptx::tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = __uint_as_float(e & 1 ? p[e / 2] & 0xFFFF0000u : p[e / 2] << 16);
      nan |= (y != y ? 1u : 0u) << e;
    }
    uint32_t gone = 0;  // of them
    if (!mine) nan = 0;
#pragma unroll 1
    for (uint32_t left = __reduce_or_sync(~0u, nan); left; left &= left - 1) {
      const int e = __ffs(left) - 1;
      const bf16* key = k + (size_t)(x + e) * D;
      if (!infinite_key<D>(key, lane)) continue;
      if (((nan >> e) & 1) && exact_product<D>(q, key) * c < ref - 160.f) gone |= 1u << e;
      __syncwarp();
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t other = e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      if ((gone >> e) & 1) p[e / 2] &= other, p[8 + e / 2] &= other;
      l += __uint_as_float(e & 1 ? p[e / 2] & 0xFFFF0000u : p[e / 2] << 16) +
           __uint_as_float(e & 1 ? p[8 + e / 2] & 0xFFFF0000u : p[8 + e / 2] << 16);
    }
    __syncwarp();
    ptx::tmem_st16(ts + x, p);
  }
  return mine ? l : sum;
}

// Sum of the infinities and NaN among one dim of prefix entries [t0, t1) (their values from v on, D
// apart), by a whole warp; 0 if there are none.
template <int D>
__device__ __forceinline__ float not_finite_values(const bf16* v, int t0, int t1, int lane) {
  float sum = 0.f;
#pragma unroll 4
  for (int t = t0 + lane; t < t1; t += 32) {
    const float y = __bfloat162float(v[(size_t)t * D]);
    if (!is_finite(y)) sum += y;
  }
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  return sum;
}

// N consecutive results x inv at element `at` of the output: 32-bit (F32), bf16, or
// bf16 hi and lo parts (F32 with out_lo).
template <int N, bool F32>
__device__ __forceinline__ void write_out(const TreeArgs& a, const float* x, float inv, size_t at) {
  if (F32 && a.out_lo) {
    bf16* out = (bf16*)a.out + at;
    bf16* lo = a.out_lo + at;
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      uint2 h, l;
      hi_lo(x[e] * inv, x[e + 1] * inv, h.x, l.x);
      hi_lo(x[e + 2] * inv, x[e + 3] * inv, h.y, l.y);
      *reinterpret_cast<uint2*>(out + e) = h;
      *reinterpret_cast<uint2*>(lo + e) = l;
    }
  } else if (F32) {
    float* out = (float*)a.out + at;
#pragma unroll
    for (int e = 0; e < N; e += 4)
      *reinterpret_cast<float4*>(out + e) = make_float4(x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv);
  } else {
    bf16* out = (bf16*)a.out + at;
#pragma unroll
    for (int e = 0; e < N; e += 4)
      *reinterpret_cast<uint2*>(out + e) =
          make_uint2(pack2(x[e] * inv, x[e + 1] * inv), pack2(x[e + 2] * inv, x[e + 3] * inv));
  }
}

// DIRECT: kWhole, kCluster; else kShares.
template <int D, bool F32, bool DIRECT>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ TreeArgs a, TreeWork ws, int mode, int turn) {
  using S = Shape<D, F32>;
  constexpr int NST = S::NST, NR = D / 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* qimg = sm;
  uint8_t* ring = sm + S::Q;
  // kCluster, over the ring once it is read: each rank's part of this CTA's dims,
  // four of a query together, and its (maximum, sum)
  constexpr int kQuads = D / kRanks / 4;
  static_assert(kRanks * 128 * (kQuads * 16 + 8) <= NST * S::STAGE, "the parts fit the ring");
  float4* recv = reinterpret_cast<float4*>(ring);                          // [rank][quad][128]
  float2* recv_ml = reinterpret_cast<float2*>(recv + kRanks * kQuads * 128);  // [rank][128]
  float2* s_ml = reinterpret_cast<float2*>(ring + NST * S::STAGE);  // [4 groups][128] (maximum, sum)
  float* s_mx = reinterpret_cast<float*>(s_ml + 4 * 128);           // [4 groups][128] a tile's maxima
  float* s_ref = s_mx + 4 * 128;                                    // [4 groups][128] the scores that references are of
  uint64_t* full = reinterpret_cast<uint64_t*>(s_ref + 4 * 128);
  uint64_t* empty = full + NST;
  uint64_t* tail_full = empty + NST;  // in full's place for value tiles that clean_tile prepares
  uint64_t* q_full = tail_full + NST;
  uint64_t* q_empty = q_full + 1;
  uint64_t* s_full = q_empty + 1;   // [2]
  uint64_t* p_full = s_full + 2;    // [2]
  uint64_t* v_clean = p_full + 2;   // [2]
  uint64_t* o_full = v_clean + 2;
  uint64_t* o_empty = o_full + 1;
  uint64_t* drain = o_empty + 1;
  uint64_t* q_first = drain + 1;  // in q_full's place for the CTA's first item
  unsigned long long* s_bad = reinterpret_cast<unsigned long long*>(q_first + 1);
  uint32_t* tslot = reinterpret_cast<uint32_t*>(s_bad + 1);
  Unit* s_next = reinterpret_cast<Unit*>(tslot + 2);  // [2] the item after one of this parity
  __shared__ UnitPlan s_plan;
  __shared__ First s_first;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      ptx::mbar_init(&full[i], 1);
      ptx::mbar_init(&empty[i], 1);
      ptx::mbar_init(&tail_full[i], 1);
    }
    ptx::mbar_init(q_first, (kThreads - 64) / 32);
    ptx::mbar_init(q_full, 8);
    ptx::mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&s_full[i], 1);
      ptx::mbar_init(&p_full[i], 8);
      ptx::mbar_init(&v_clean[i], 64);
    }
    ptx::mbar_init(o_full, 1);
    ptx::mbar_init(o_empty, 16);
    ptx::mbar_init(drain, 1);
    ptx::fence_mbar_init();
  }
  if (warp == 1) ptx::tmem_alloc(tslot, 512);
  if (warp == 0 && lane == 0) {
    ptx::prefetch_tmap(&tmK);
    ptx::prefetch_tmap(&tmV);
  }
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  int u1 = 0;
  Unit it;
  if constexpr (DIRECT) {
    // grid: (query tile and rank, kv head, request)
    it.b = blockIdx.z;
    it.g = blockIdx.y;
    it.qt = mode == kCluster ? blockIdx.x / kRanks : blockIdx.x;
    it.r0 = a.rm.start[it.b];
    it.rows = a.rm.start[it.b + 1] - it.r0;
    it.L = a.len[it.b];
    it.tiles = 0;
    const bool some = it.qt * 128 < it.rows * (a.nq / a.nkv);
    if (some && rows_fit(it.L, it.rows, a.cap))
      it.tiles = (it.L + it.rows + 127) / 128;
    else if (some && tid == 0 && a.err)
      atomicOr(a.err, kErrCapacity);
    const int per = mode == kCluster ? (it.tiles + kRanks - 1) / kRanks : it.tiles;
    it.t0 = mode == kCluster ? min((int)ptx::cluster_rank() * per, it.tiles) : 0;
    it.t1 = min(it.t0 + per, it.tiles);
    u1 = it.t0 < it.t1 ? 1 : 0;
  } else {
    if (warp == 0) {
      make_plan(a, 128, turn, lane, s_plan, blockIdx.x == 0);
      first_item(s_plan, a, blockIdx.x, gridDim.x, lane, s_first);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tslot;
  if constexpr (!DIRECT) it = s_first.it, u1 = s_first.u1;
  const bool some = DIRECT ? u1 > 0 : it.rows > 0;
  // The CTA's items one after another, each with its tiles, in `it` (the first is there).
  auto next = [&] {
    if constexpr (DIRECT)
      return false;
    else {
      int u = it.next;
      return next_item(s_plan, a, u, u1, it);
    }
  };
  if (warp >= 2 && some) {
    // the first item's queries, by every warp that has nothing to do yet (by two
    // warps 32-bit queries of 119 rows took 5 us)
    load_queries<D, F32, kThreads - 64, 4, false>(a, it, tid - 64, qimg, [] {});
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(q_first);
  }
  // every wait is bounded; a role that gives up flags the call and waits for
  // nothing more, so that all of them come to the end
  const unsigned long long limit = a.timeout_ns;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok && !ptx::mbar_spin(bar, parity, limit)) {
      ok = false;
      if (a.err) atomicOr(a.err, kErrTimeout);
    }
    return ok;
  };
  // two at once: their first looks overlap
  auto wait2 = [&](uint64_t* a_bar, uint32_t a_parity, uint64_t* b_bar, uint32_t b_parity) {
    const bool a_done = ptx::mbar_try_wait(a_bar, a_parity), b_done = ptx::mbar_try_wait(b_bar, b_parity);
    if (!a_done) wait(a_bar, a_parity);
    if (!b_done) wait(b_bar, b_parity);
    return ok;
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint64_t pol = ptx::policy_evict_first();
      uint32_t n = 0, tail = 0, turn = 0;  // slots whose last tile is on tail_full, its parity
      for (bool more = some; more; more = next()) {
        const int z = it.b * a.nkv + it.g;
        for (int t = it.t0; t < it.t1 && ok; ++t)
          for (int kv = 0; kv < 2; ++kv, ++n) {
            const uint32_t s = n % NST, bit = 1u << s;
            if (n >= NST && !wait(&empty[s], (n / NST - 1) & 1)) break;
            uint64_t* bar = &full[s];
            tail &= ~bit;
            if (kv && t >= it.L / 128) {
              ptx::mbar_arrive(bar);  // (this tile's phase of it)
              bar = &tail_full[s];
              tail |= bit;
              turn ^= bit;
            }
            ptx::mbar_arrive_expect_tx(bar, S::STAGE);
#pragma unroll
            for (int h = 0; h < NR; ++h)
              ptx::tma_load_3d(ring + s * S::STAGE + h * kRegion, kv ? &tmV : &tmK, bar, 64 * h, t * 128, z, pol);
          }
      }
      // no copy is in flight when the CTA ends
      for (uint32_t i = n > NST ? n - NST : 0; i < n; ++i) {
        const uint32_t s = i % NST;
        if ((tail >> s) & 1)
          ptx::mbar_wait(&tail_full[s], ((turn >> s) & 1) ^ 1, ptx::kDrainNs);
        else
          ptx::mbar_wait(&full[s], (i / NST) & 1, ptx::kDrainNs);
      }
    }
  } else if (warp == 1) {
    // the whole warp, for operands in uniform registers; one thread issues
    const uint32_t lead = ptx::elect_one(), tm = __shfl_sync(~0u, tmem, 0);
    auto whole = [&](bool) { return ok = __all_sync(~0u, ok); };
    constexpr uint32_t IDESC1 = ptx::idesc_bf16_f32(128, 128);
    constexpr uint32_t IDESC2 = ptx::idesc_bf16_f32(128, D, true);
    const uint32_t q_lo = ptx::desc_lo(ptx::smem_u32(qimg), 16u);
    constexpr uint32_t kNone = ~0u;
    Stage at;
    uint32_t items = 0, p_turn = 0, c_turn = 0;    // parities of p_full and v_clean
    uint32_t last0 = kNone, last1 = kNone, v = 0;  // value stages of the sets' last tiles, of the last tile
    for (bool more = some; ok && more; more = next(), ++items) {
      const int cnt = __shfl_sync(~0u, it.t1 - it.t0, 0), first_tail = __shfl_sync(~0u, it.L / 128 - it.t0, 0);
      whole(items == 0 ? wait(q_first, 0) : wait(q_full, (items - 1) & 1));
      for (int j = 0; j <= cnt && ok; ++j) {
        const uint32_t v_before = v;
        if (j < cnt) {
          const uint32_t k = at.next<NST>(), last = j & 1 ? last1 : last0;
          v = at.next<NST>();
          // the last P that stood where these scores go has been read: its
          // product released the stage of its values
          uint64_t* there = &full[Stage::slot(k)];
          if (!whole(last == kNone ? wait(there, Stage::parity(k))
                                   : wait2(there, Stage::parity(k), &empty[Stage::slot(last)], Stage::parity(last))))
            break;
          ptx::tc_fence_after();
          const uint32_t kt = ptx::desc_lo(ptx::smem_u32(ring + Stage::slot(k) * S::STAGE), 16u);
          const uint32_t ds = tm + 128 * (j & 1);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t to = ((kk >> 2) * kRegion + 32u * (kk & 3)) >> 4;
            ptx::mma_bf16_lo(lead, ds, q_lo + to, kt + to, IDESC1, kk > 0 ? 1u : 0u);
            if (F32) ptx::mma_bf16_lo(lead, ds, q_lo + to + (128u * D * 2 >> 4), kt + to, IDESC1, 1u);
          }
          ptx::mma_commit_if(lead, &s_full[j & 1]);
          if (j == cnt - 1) ptx::mma_commit_if(lead, q_empty);
          if (j & 1)
            last1 = v;
          else
            last0 = v;
        }
        if (j > 0) {
          const uint32_t i = (j - 1) & 1;
          const int tail = j - 1 - first_tail;  // the tiles that hold entries from L on
          uint64_t* there = tail < 0 ? &full[Stage::slot(v_before)] : &v_clean[tail];
          const uint32_t parity = tail < 0 ? Stage::parity(v_before) : (c_turn >> tail) & 1;
          if (!whole(wait2(there, parity, &p_full[i], (p_turn >> i) & 1))) break;
          p_turn ^= 1u << i;
          if (tail >= 0) c_turn ^= 1u << tail;
          if (j <= 2 && items > 0 && !whole(wait(o_empty, (items - 1) & 1))) break;
          ptx::tc_fence_after();
          const uint32_t vt = ptx::desc_lo(ptx::smem_u32(ring + Stage::slot(v_before) * S::STAGE), kRegion);
          const uint32_t ds = tm + 256 + 128 * i, ps = tm + 128 * i;
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) {
            ptx::mma_bf16_ta_lo(lead, ds, ps + 16u * kk, vt + 128u * kk, IDESC2, j > 2 || kk > 0 ? 1u : 0u);
            ptx::mma_bf16_ta_lo(lead, ds, ps + 16u * kk + 8, vt + 128u * kk, IDESC2, 1u);
          }
          ptx::mma_commit_if(lead, &empty[Stage::slot(v_before)]);
          if (j == cnt) ptx::mma_commit_if(lead, o_full);
        }
      }
    }
    // no product is running when TMEM is freed
    ptx::mma_commit_if(lead, drain);
    ptx::mbar_wait(drain, 0, ptx::kDrainNs);
  } else if (warp < 4) {
    const int t64 = tid - 64;
    uint32_t n = 0, items = 0, turn = 0;
    for (bool more = some; more; more = next(), ++items) {
      const int first = it.L / 128;
      // the epilogue of the item before has read what was noted for it
      if (items > 0) wait(o_empty, (items - 1) & 1);
      if (it.t1 > first) {
        if (t64 == 0) *s_bad = 0;
        ptx::named_bar_sync(2, 64);
        for (int t = max(first, it.t0); t < it.t1; ++t) {
          const uint32_t s = (n + 2 * (t - it.t0) + 1) % NST;
          const bool here = wait(&tail_full[s], (turn >> s) & 1);
          turn ^= 1u << s;
          if (!here) continue;  // (nor is this one let go)
          clean_tile<D>(ring + s * S::STAGE, t * 128, it.L, it.L + it.rows, t64, s_bad);
          ptx::fence_proxy_async_smem();
          ptx::mbar_arrive(&v_clean[t - first]);
        }
      }
      n += 2 * (it.t1 - it.t0);
    }
  } else {
    const int group = (warp - 4) >> 2;           // of four warps
    const int set = group & 1, half = group >> 1;  // tiles of this parity, keys of this half of them
    const int quad = warp & 3, row = 32 * quad + lane;  // query of the tile, TMEM lane
    const uint32_t tl = tmem + ((uint32_t)(32 * quad) << 16);
    const uint32_t ts = tl + 128 * set + 64 * half, to = tl + 256 + 128 * set + half * (D / 2);
    const int G = a.nq / a.nkv;
    const float c = a.scale_log2;
    uint32_t ns = 0, items = 0, c_turn = 0, before = 0;  // tiles of this CTA before the item
    for (bool more = some; more;) {
      const int cnt = it.t1 - it.t0, nqs = it.rows * G;
      const bool live = it.qt * 128 + row < nqs;
      // the row and query head of the thread's query (computed where they are needed: they would take
      // registers over the tiles)
      auto place = [&](int& i, int& h) {
        int q = it.qt * 128 + row;
        asm volatile("" : "+r"(q));
        i = divide_group(a, q);
        h = it.g * G + (q - i * G);
      };
      const bool warp_live = it.qt * 128 + 32 * quad < nqs;  // a query of the warp is
      uint64_t vis = 0;
      if (live && it.t1 > it.L / 128) {
        int i, h;
        place(i, h);
        vis = visible_rows(a, it.r0 + i, i, it.rows);
      }
      float m = -INFINITY, l = 0.f;
      for (int j = set; j < cnt; j += 2, ++ns) {
        wait(&s_full[set], ns & 1);
        // (the tile's keys have been read; after a wait that gave up they may not be there
        // yet, and their stage is not given back)
        if (ok && half == 0 && quad == 0 && lane == 0) ptx::mbar_arrive(&empty[2 * (before + j) % NST]);
        ok = __all_sync(~0u, ok);
        // (a warp without a query leaves what it has in the place of P: it reaches
        // the accumulators of rows that are not read)
        if (warp_live) {
          ptx::tc_fence_after();
          const int p0 = (it.t0 + j) * 128 + 64 * half;
          const bool tail = p0 + 64 > it.L;
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
          for (int x = 0; x < 64; x += 32) {
            uint32_t v[32];
            ptx::tmem_ld32(ts + x, v);
            ptx::tmem_ld_wait();
            if (tail) {
              // -inf where the row does not see, for the second reading too
              mask_scores(v, key_bits(p0 + x, it.L, vis));
              ptx::tmem_st16(ts + x, v);
              ptx::tmem_st16(ts + x + 16, v + 16);
            }
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              mx[0] = max3(mx[0], __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
              mx[1] = max3(mx[1], __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
            }
          }
          if (tail) ptx::tmem_st_wait();
          const float mine = fmaxf(mx[0], mx[1]);
          s_mx[group * 128 + row] = mine;
          ptx::named_bar_sync(3 + 4 * set + quad, 64);
          const float top = fmaxf(mine, s_mx[(group ^ 2) * 128 + row]), mt = top * c;
          // (NaN scores pass the maximum by, and reach the sums)
          const bool grow = mt > m + kLazy || (m == -INFINITY && mt > m);
          if (__any_sync(~0u, grow)) {
            const float m_new = grow ? mt : m;
            const float f = m == -INFINITY ? 0.f : ex2(m - m_new);
            l = grow ? l * f : l;
            if (j >= 2) {
#pragma unroll 1
              for (int x = 0; x < D / 2; x += 16) {
                uint32_t o[16];
                ptx::tmem_ld16(to + x, o);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = grow ? __float_as_uint(__uint_as_float(o[e]) * f) : o[e];
                ptx::tmem_st16(to + x, o);
              }
            }
            m = m_new;
            if (grow) s_ref[group * 128 + row] = top;
          }
          // (a greater score that did not move m has the same product with c)
          const Exponent x2 = exponent_of([&] { return fmaxf(s_ref[group * 128 + row], top); }, m, c, kFar);
          const uint64_t c2 = two(x2.by, x2.by), ref2 = two(-x2.at, -x2.at), less = two(-1.f, -1.f);
          uint64_t ls[2] = {0, 0};
          // P: of each 16 keys the hi parts, then the lo parts, in the place of
          // their scores (which are read a second time: they do not fit the
          // registers)
#pragma unroll 1
          for (int x = 0; x < 64; x += 16) {
            uint32_t v[16], p[16];
            ptx::tmem_ld16(ts + x, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 y = of_two(fma2(two(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), c2, ref2));
              const uint64_t w = two(ex2(y.x), ex2(y.y));
              ls[e & 1] = add2(ls[e & 1], w);
              const float2 f = of_two(w);
              p[e] = pack2(f.x, f.y);
              const float2 r = of_two(
                  fma2(two(__uint_as_float(p[e] << 16), __uint_as_float(p[e] & 0xFFFF0000u)), less, w));
              p[8 + e] = pack2(r.x, r.y);
            }
            ptx::tmem_st16(ts + x, p);
          }
          const float2 sums = of_two(add2(ls[0], ls[1]));
          float more = sums.x + sums.y;
          if (F32 && ok && __any_sync(~0u, live && more != more)) {
            int i, h;
            place(i, h);
            more = mend_weights<D>(ts, live && more != more,
                                   (const float*)a.q + (it.r0 + i) * a.q_stride + (int64_t)h * D,
                                   a.k + (((size_t)it.b * a.nkv + it.g) * a.cap + p0) * D, c, m == -INFINITY ? 0.f : m, more);
          }
          l += more;
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[set]);
      }
      // the next item and its queries, by the set that has no part in the last tile
      if constexpr (!DIRECT) {
        if (set == (cnt & 1)) {
          Unit then;
          if (int v = it.next; next_item(s_plan, a, v, u1, then)) {
            load_queries<D, F32, 256, 4, true>(a, then, half * 128 + row, qimg, [&] { wait(q_empty, items & 1); });
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(q_full);
          } else {
            then.rows = 0;
          }
          if (half == 0 && row == 0) s_next[items & 1] = then;
        }
      }
      // ---- the item's end: the two sets' parts, each group a quarter of the dims ----
      const bool tails = it.t1 > it.L / 128;
      wait(o_full, items & 1);
      if (tails)
        for (int t = max(it.L / 128, it.t0); t < it.t1; ++t) {
          const int x = t - it.L / 128;
          wait(&v_clean[x], (c_turn >> x) & 1);
          c_turn ^= 1u << x;
        }
      ok = __all_sync(~0u, ok);
      ptx::tc_fence_after();
      s_ml[group * 128 + row] = make_float2(m, l);
      ptx::named_bar_sync(1, 512);
      const float m0 = s_ml[row].x, m1 = s_ml[128 + row].x;
      const float l0 = s_ml[row].y + s_ml[256 + row].y, l1 = s_ml[128 + row].y + s_ml[384 + row].y;
      const float M = fmaxf(m0, m1);
      const float w0 = part_weight(m0, M), w1 = cnt > 1 ? part_weight(m1, M) : 0.f;
      const float lt = l0 * w0 + (cnt > 1 ? l1 * w1 : 0.f);
      const unsigned long long bad = tails ? *s_bad & vis : 0ull;
      int i, h;
      place(i, h);
      // every CTA of the cluster has read its ring: the parts go there
      if (DIRECT && mode == kCluster) ptx::cluster_sync();
      if (ok && warp_live) {
        const bool done = DIRECT || (it.t0 == 0 && it.t1 == it.tiles);
        const size_t part = (size_t)blockIdx.x * 2 + (it.t0 > 0 ? 0 : 1);
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
        float zero[2] = {0.f, 0.f};  // 0 times each accumulator
#pragma unroll 1
        for (int d0 = group * (D / 4); d0 < (group + 1) * (D / 4); d0 += 16) {
          uint32_t o0[16], o1[16];
          ptx::tmem_ld16(tl + 256 + d0, o0);
          if (cnt > 1) ptx::tmem_ld16(tl + 384 + d0, o1);
          ptx::tmem_ld_wait();
          float o[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            zero[e & 1] = fmaf(__uint_as_float(o0[e]), 0.f, zero[e & 1]);
            if (cnt > 1) zero[e & 1] = fmaf(__uint_as_float(o1[e]), 0.f, zero[e & 1]);
            o[e] = w0 != 0.f ? __uint_as_float(o0[e]) * w0 : 0.f;
            if (cnt > 1 && w1 != 0.f) o[e] = fmaf(__uint_as_float(o1[e]), w1, o[e]);
          }
          for (unsigned long long left = bad; left; left &= left - 1) {
            const int r = __ffsll((long long)left) - 1;
            const bf16* v = a.v + (((size_t)it.b * a.nkv + it.g) * a.cap + it.L + r) * D + d0;
            if (it.L + r >= it.t0 * 128 && it.L + r < it.t1 * 128)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float y = __bfloat162float(v[e]);
                if (!(fabsf(y) <= 3.4e38f)) o[e] += y;
              }
          }
          if (DIRECT && live && mode == kCluster) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int quad = d0 / 4 + e;
              dsmem_st4(ptx::dsmem_map(ptx::smem_u32(recv + (ptx::cluster_rank() * kQuads + quad % kQuads) * 128 + row),
                                       quad / kQuads),
                        make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]));
            }
          } else if (!DIRECT && live && !done) {
            float4* dst = ws.o + (part * (D / 4) + d0 / 4) * 128 + row;
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[e * 128] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          } else if (live) {
            write_out<16, F32>(a, o, inv, ((size_t)(it.r0 + i) * a.nq + h) * D + d0);
          }
          __syncwarp();
        }
        // An infinite value of the prefix times hi and lo parts of P, of which lo may be 0 or
        // negative, or times a P that is 0 in 32 bits, is NaN where the formula has that
        // infinity; and a set of weight 0 beside the other is left out.  Such dims once more.
        if (__any_sync(~0u, live && zero[0] + zero[1] != 0.f && lt == lt)) {
          const bf16* v = a.v + ((size_t)it.b * a.nkv + it.g) * a.cap * D;
#pragma unroll 1
          for (int d = group * (D / 4); d < (group + 1) * (D / 4); ++d) {
            float y = not_finite_values<D>(v + d, it.t0 * 128, min(it.t1 * 128, it.L), lane);
            if (is_finite(y) || !live || lt != lt) continue;
#pragma unroll 1
            for (unsigned long long left = bad; left; left &= left - 1) {
              const int t = it.L + __ffsll((long long)left) - 1;
              const float z = __bfloat162float(v[(size_t)t * D + d]);
              if (t >= it.t0 * 128 && t < it.t1 * 128 && !is_finite(z)) y += z;
            }
            if (DIRECT && mode == kCluster) {
              const float* to = &recv[(ptx::cluster_rank() * kQuads + d / 4 % kQuads) * 128 + row].x + d % 4;
              dsmem_st(ptx::dsmem_map(ptx::smem_u32(to), d / 4 / kQuads), y);
            } else if (!DIRECT && !done) {
              (&ws.o[(part * (D / 4) + d / 4) * 128 + row].x)[d % 4] = y;
            } else {
              const size_t at = ((size_t)(it.r0 + i) * a.nq + h) * D + d;
              if (F32 && !a.out_lo)
                ((float*)a.out)[at] = y;
              else
                ((bf16*)a.out)[at] = __float2bfloat16_rn(y);
              if (F32 && a.out_lo) a.out_lo[at] = __float2bfloat16_rn(0.f);
            }
          }
          __syncwarp();
        }
        if (DIRECT && live && mode == kCluster) {
          for (int r = 2 * group; r < 2 * group + 2; ++r)
            dsmem_st2(ptx::dsmem_map(ptx::smem_u32(recv_ml + ptx::cluster_rank() * 128 + row), r), make_float2(M, lt));
        } else if (live && group == 0) {
          if (!done)
            ws.ml[part * 128 + row] = make_float2(M, lt);
          else if (a.lse)
            a.lse[(size_t)(it.r0 + i) * a.nq + h] = row_lse(M, lt);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(o_empty);
      if constexpr (!DIRECT) it = s_next[items & 1];
      before += cnt;
      more = !DIRECT && it.rows > 0;
      ++items;
    }
  }
  if (DIRECT && mode == kCluster) {
    // (the groups of a CTA with tiles have passed the first barrier above)
    __syncwarp();
    if (warp < 4 || !some) ptx::cluster_sync();
    ptx::cluster_sync();
    // the parts of four dims of a query, in rank order
    const int t = tid - 128, quad = t >> 7, row = t & 127, q = it.qt * 128 + row, G = a.nq / a.nkv;
    if (t >= 0 && quad < kQuads && q < it.rows * G && it.tiles > 0) {
      const int per = (it.tiles + kRanks - 1) / kRanks, n = (it.tiles + per - 1) / per;
      float M = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int r = 0; r < n; ++r) M = fmaxf(M, recv_ml[r * 128 + row].x);
#pragma unroll 1
      for (int r = 0; r < n; ++r) add_part(recv_ml[r * 128 + row], recv[(r * kQuads + quad) * 128 + row], M, l, x);
      const int i = divide_group(a, q), h = it.g * G + (q - i * G);
      write_out<4, F32>(a, x, l == 0.f ? 0.f : 1.f / l,
                        ((size_t)(it.r0 + i) * a.nq + h) * D + ptx::cluster_rank() * (D / kRanks) + 4 * quad);
      if (quad == 0 && ptx::cluster_rank() == 0 && a.lse) a.lse[(size_t)(it.r0 + i) * a.nq + h] = row_lse(M, l);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

// The parts of items cut between CTAs, joined in CTA order: a CTA per 32 queries and
// 32 dims of an item, a lane per query (16 bytes each side by side in a part), a
// warp per four dims, U parts in flight.  (One CTA for all dims, a quarter of
// the CTAs: a tree of 64 rows 50 us, then 35.)  U: as many of 12, 8 and 4 as let all
// CTAs run at once, 2, 3 and 5 per SM.  us with 12 / 8, 256 CTAs: a tree of 64 rows
// 29.3 / 30.4, one item of 60000 entries 25.4 / 26.6; with 4 / 8, 384 CTAs: six requests
// of 4000 entries 20.4 / 19.3; 1024 CTAs: 16 ragged requests 39.9 / 41.4.
constexpr int kCombineWarps = 8;
template <int D, bool F32, int U>
__global__ void __launch_bounds__(32 * kCombineWarps, U == 12 ? 2 : U == 8 ? 3 : 5)
    tree_combine_kernel(const __grid_constant__ TreeArgs a, TreeWork ws, int ctas, int turn) {
  constexpr int Z = D / 4 / kCombineWarps;
  __shared__ UnitPlan plan;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.z, g = blockIdx.y, quad = blockIdx.x % Z * kCombineWarps + warp;
  const int qt = blockIdx.x / Z >> 2, row = 32 * (blockIdx.x / Z & 3) + lane, q = qt * 128 + row;
  const int r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0, G = a.nq / a.nkv;
  // The lengths before the wait: the products' kernel let this one start after
  // its own wait, so what ran before that kernel is done, and it writes none.
  // (No CTA ends before it: what follows in the stream waits for this kernel.)
  ptx::griddep_launch_dependents();
  if (q - lane >= rows * G) {
    ptx::griddep_wait();
    return;
  }
  if (warp == 0) make_plan(a, 128, turn, lane, plan, false);
  __syncthreads();
  const int tiles = plan.tiles[b];
  const int first = plan.unit[b] + (g * plan.qts[b] + qt) * (tiles + turn) + turn;
  const int c0 = tiles > 0 ? unit_owner(plan, first, ctas) : 0;
  const int n = tiles > 0 ? unit_owner(plan, first + tiles - 1, ctas) - c0 + 1 : 0;
  ptx::griddep_wait();
  if (n <= 1 || q >= rows * G) return;  // skipped, or written by its CTA
  auto part = [&](int k) { return (size_t)(c0 + k) * 2 + (k == 0 ? 1 : 0); };
  float M = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int k0 = 0; k0 < n; k0 += U) {
    float2 ml[U];
    float4 v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      ml[k] = make_float2(-INFINITY, 0.f);
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k0 + k < n) {
        ml[k] = __ldcg(&ws.ml[part(k0 + k) * 128 + row]);
        v[k] = __ldcg(&ws.o[(part(k0 + k) * (D / 4) + quad) * 128 + row]);
      }
    }
    const float before = M;
#pragma unroll
    for (int k = 0; k < U; ++k) M = fmaxf(M, ml[k].x);
    const float w = part_weight(before, M);
    l *= w;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = weighted(x[e], w);
#pragma unroll
    for (int k = 0; k < U; ++k) add_part(ml[k], v[k], M, l, x);
  }
  const int i = divide_group(a, q), h = g * G + (q - i * G);
  write_out<4, F32>(a, x, l == 0.f ? 0.f : 1.f / l, ((size_t)(r0 + i) * a.nq + h) * D + 4 * quad);
  if (quad == 0 && a.lse) a.lse[(size_t)(r0 + i) * a.nq + h] = row_lse(M, l);
}

template <int D, bool F32>
cudaError_t launch_join(const TreeArgs& a, const TreeWork& ws, int most_rows, int ctas, int turn, int sms,
                        cudaStream_t st) {
  const dim3 join((most_rows * (a.nq / a.nkv) + 127) / 128 * 4 * (D / 4 / kCombineWarps), a.nkv, a.rm.batch);
  const int64_t joins = (int64_t)join.x * join.y * join.z;
  return launch_pdl(joins <= 2 * sms   ? tree_combine_kernel<D, F32, 12>
                    : joins <= 3 * sms ? tree_combine_kernel<D, F32, 8>
                                       : tree_combine_kernel<D, F32, 4>,
                    join, dim3(32 * kCombineWarps), 0, st, 1, a, ws, ctas, turn);
}

// Items of at most this many key tiles are each done by one CTA.  us, in one CTA /
// by clusters: four items of two tiles 6.7 / 6.9, of three 8.2 / 7.2.
constexpr int kWholeTiles = 2;
// A call whose clusters all run at once is done by clusters, unless its items are
// longer than this.  us, even shares / clusters, rows of seven queries: 4 items of
// 1564 entries 10.2 / 8.9, 15 14.0 / 9.6, 16 (one more than run at once) 13.6 / 13.7; 4
// of 6000 14.9 / 13.9; one of 8100 14.0 / 15.7, 4 15.8 / 16.3, 15 22.0 / 18.5; 4 of
// 15128 19.6 / 23.2.
constexpr int kClusterTiles = 6 * kRanks;

template <int D, bool F32>
cudaError_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const TreeArgs& a, const TreeWork& ws,
                   int64_t items, int most_rows, int64_t most_tiles, int sms, cudaStream_t st, int64_t& launches) {
  using S = Shape<D, F32>;
  static PerDevice opted[2], clusters;
  cudaError_t e = opt_in(opted[0], tree_attn_kernel<D, F32, true>, S::SMEM);
  if (e == cudaSuccess) e = opt_in(opted[1], tree_attn_kernel<D, F32, false>, S::SMEM);
  if (e != cudaSuccess) return e;
  const int64_t units = items * most_tiles;
  ++launches;
  const dim3 direct((most_rows * (a.nq / a.nkv) + 127) / 128, a.nkv, a.rm.batch);
  if (most_tiles <= kWholeTiles)
    return launch_pdl(tree_attn_kernel<D, F32, true>, direct, dim3(kThreads), S::SMEM, st, 1, tk, tv, a, ws,
                      (int)kWhole, 0);
  if (most_tiles <= kClusterTiles &&
      items <= resident_clusters(clusters, tree_attn_kernel<D, F32, true>, kThreads, S::SMEM, kRanks))
    return launch_pdl(tree_attn_kernel<D, F32, true>, dim3(direct.x * kRanks, direct.y, direct.z), dim3(kThreads),
                      S::SMEM, st, kRanks, tk, tv, a, ws, (int)kCluster, 0);
  // No more CTAs to an item than pay for the joining of their parts.  us, one item
  // of 8100 / 15128 / 60000 entries: at most 16 14.3 / 18.9 / 46.7, 32 13.4 / 16.3 / 30.4,
  // 64 16.5 / 17.7 / 26.0, as many as there are SMs 16.5 / 24.0 / 42.5; so 13.8 / 16.1 / 26.7
  // (all with eight parts of the join in flight).
  const int64_t most_ctas = items * (16 + most_tiles / 8);
  const int ctas = (int)std::min(std::min<int64_t>(units, sms), most_ctas), turn = units > sms ? kTurn : 0;
  e = launch_pdl(tree_attn_kernel<D, F32, false>, dim3(ctas), dim3(kThreads), S::SMEM, st, 1, tk, tv, a, ws,
                 (int)kShares, turn);
  if (e != cudaSuccess) return e;
  ++launches;
  return launch_join<D, F32>(a, ws, most_rows, ctas, turn, sms, st);
}

}  // namespace

int device_sms() {
  static PerDevice sms;
  const int n = sms.get([] {
    int dev = 0, count = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return -1;
    return count;
  });
  return n > 0 ? n : 1;
}

int64_t tree_items(const TreeArgs& a) {
  const int G = a.nq / a.nkv;
  int64_t items = 0;
  for (int b = 0; b < a.rm.batch; ++b)
    items += (int64_t)((a.rm.start[b + 1] - a.rm.start[b]) * G + 127) / 128 * a.nkv;
  return items;
}

TreeWork tree_work(void* workspace, int head_dim) {
  TreeWork ws;
  ws.o = (float4*)workspace;
  ws.ml = (float2*)(ws.o + (size_t)device_sms() * 2 * 128 * head_dim / 4);
  return ws;
}

cudaError_t launch_tree_join(const TreeArgs& a, int head_dim, const TreeWork& ws, int ctas, int turn, cudaStream_t st) {
  const int sms = device_sms();
  int most = 0;
  for (int b = 0; b < a.rm.batch; ++b) most = std::max(most, a.rm.start[b + 1] - a.rm.start[b]);
  if (head_dim == 128)
    return a.q_f32 ? launch_join<128, true>(a, ws, most, ctas, turn, sms, st)
                   : launch_join<128, false>(a, ws, most, ctas, turn, sms, st);
  return a.q_f32 ? launch_join<64, true>(a, ws, most, ctas, turn, sms, st)
                 : launch_join<64, false>(a, ws, most, ctas, turn, sms, st);
}

size_t tree_attention_workspace(int head_dim) {
  return (size_t)device_sms() * 2 * 128 * (head_dim * 4 + 8);
}

cudaError_t launch_tree_attention(const TreeArgs& a, int head_dim, int64_t max_keys, void* workspace,
                                  cudaStream_t st, int64_t* launches) {
  const int sms = device_sms();
  int64_t uncounted = 0, &n = launches ? *launches : uncounted;
  const int64_t items = tree_items(a);
  int most = 0;  // rows of a request
  for (int b = 0; b < a.rm.batch; ++b) most = std::max(most, a.rm.start[b + 1] - a.rm.start[b]);
  const TreeWork ws = tree_work(workspace, head_dim);
  CUtensorMap tk, tv;
  if (!encode_cache_map(&tk, a.k, head_dim, a.cap, (int64_t)a.rm.batch * a.nkv) ||
      !encode_cache_map(&tv, a.v, head_dim, a.cap, (int64_t)a.rm.batch * a.nkv))
    return cudaErrorInvalidValue;
  const int64_t tiles = (max_keys + 127) / 128;
  if (head_dim == 128)
    return a.q_f32 ? launch<128, true>(tk, tv, a, ws, items, most, tiles, sms, st, n)
                   : launch<128, false>(tk, tv, a, ws, items, most, tiles, sms, st, n);
  return a.q_f32 ? launch<64, true>(tk, tv, a, ws, items, most, tiles, sms, st, n)
                 : launch<64, false>(tk, tv, a, ws, items, most, tiles, sms, st, n);
}

}  // namespace as2d
