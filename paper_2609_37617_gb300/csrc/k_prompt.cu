// k_prompt.cu -- causal attention of whole prompts over a cache
// (as2d_prompt_attention).
//
// Row i of request b sees the entries 0 .. L_b + i.  With s_t = scale q k_t over them:
//   m = max s_t, l = sum e^(s_t - m), out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// The G = n_q / n_kv query heads of a kv head, for all rows of a request, form one
// query matrix (row by row, so that 256 queries stand for few rows and little of a tile on
// the diagonal is masked), cut into pairs of query tiles of 128 (the MMA's M): as many whole rows
// as fit 256 queries (of more than 256 heads: 256 of a row).  An item is one (request, kv head,
// pair); a CTA takes it through its key tiles of 128.  One CTA per SM takes the items in turn,
// those of most key tiles first, back and forth over the CTAs (by the lengths on the device: eight
// prompts of 1 to 2029 rows took 102 us in the order of their rows where they took 90 so; 84 now).
//
// Per CTA (12 warps, TMEM full: two score buffers, two accumulators):
//   warp 0     loads key and value tiles by TMA through a ring of shared-memory stages;
//   warp 1     issues the products: S = Q K^T, O += P V (P from TMEM) of the two query
//              tiles in turn, so that one's products run under the other's softmax;
//   warp 2     looks for the next item while this one runs, and has its queries brought in (TMA) when the
//              last scores of this one are there;
//   warp 3     prepares the value tiles that hold entries not every row sees;
//   warps 4-11 four to a query tile, a query a thread: S from TMEM, mask, P = 2^(S - m) back into
//              TMEM in bf16 over S.  The next item's scores are computed while an item's
//              results are written.
// m is not looked for: a tile's weights are computed with the reference there is, and only where
// their sum passes kMost (or there is none yet) is the tile's maximum taken for the new one, the accumulator
// rescaled and the weights computed again.  That keeps the chain from scores to weights, which the
// products of one query tile wait for while the other's run, at one exponential a score.
// Bound by the tensor cores and the chain between them.  7564 rows of 28 / 4 heads of 128 (floor 212 us): 304 to 309, the
// tensor pipe 60 % busy; a key tile's four products read shared memory for as many cycles as they compute. Sixteen
// softmax warps, which have to agree on a reference: 315 and more; a quarter of the exponentials by
// polynomials: 363.  Clocks of an item (cycles): 2970 a key tile, of which the softmax of a query tile is 1900 and its two
// products 1024; at its end 1300 until the results are there and 3700 to write them.
// P in one bf16 part: each weight is off by at most 2^-8 of itself, as the result's own
// rounding is; the sums l are of the weights in 32 bits.
#include <algorithm>

#include "ops.h"
#include "ptx_sm100.cuh"
#include "tree_dev.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 384;
constexpr int kMaxTails = 3;  // key tiles that not all rows of 256 queries see whole
// Items that are described at a time (a power of two): the one whose results are written, the one before and the one after.
constexpr int kItems = 4;
// The sum of a tile's 128 weights that makes its maximum the reference.
constexpr float kMost = 8192.f;
// References from here on (base 2) are rounded by 32 and more (exponent_of); below, weights stay within 2^45.
constexpr float kFar = 1073741824.f;

// How queries are cut into items.
struct Cut {
  int rows_each, chunks;  // whole rows of an item, or items of a row
  int parts;              // of an item's key tiles; more than one where there are fewer items than SMs
  int last;               // the round over the CTAs that has fewer items, or parts of them, than CTAs; -1: none
};
// Partial results of an item's parts; at most kSlots an SM, of parts of kPartTiles tiles at least (but
// for requests shorter than the host's bound).
constexpr int kSlots = 2, kPartTiles = 4;
struct Parts {
  float4* o;   // [slot][D / 4][256], four dims of a query together; slot: item parts + part
  float2* ml;  // [slot][256] (reference base 2, sum)
};

struct Item {
  int b, g, r0, L;
  int i_min, h0, nq;  // row and head (of the group) of its first query, queries
  int end, from;      // entries that some row sees; from the first that not every row does
  int t0, cnt;        // key tiles: the first, how many (0: there are no more items)
  int tail0;          // the first that holds such entries, from t0
  int slot;           // of its partial results
};

template <int D>
struct Shape {
  static constexpr uint32_t STAGE = 128 * D * 2;  // one K or V tile, and one query tile
  static constexpr int NST = D == 64 ? 8 : 5;
  static constexpr uint32_t SMEM =
      (2 + NST) * STAGE + (3 * NST + 10 + 2 * kMaxTails) * 8 + 8 * kMaxTails * 4 + kItems * sizeof(Item) + 16;
  static_assert(SMEM <= 232448, "shared memory of one CTA");
};

// An item of all requests' in the order of their key tiles, most first, by a whole warp.  (No
// tiles: there are no more.)  A request's k-th item has (end of its last row + 127) / 128 tiles,
// so that those with at least T need no list to be counted.
__device__ __forceinline__ Item item_at(const TreeArgs& a, Cut cut, int64_t at, int lane) {
  const int G = a.nq / a.nkv;
  int L[2], rows[2], items[2], most = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int b = 32 * h + lane;
    L[h] = rows[h] = items[h] = 0;
    if (b < a.rm.batch) {
      const int r = a.rm.start[b + 1] - a.rm.start[b], len = a.len[b];
      if (rows_fit(len, r, a.cap)) {
        L[h] = len, rows[h] = r;
        items[h] = cut.chunks > 1 ? r * cut.chunks : (r + cut.rows_each - 1) / cut.rows_each;
        if (r > 0) most = max(most, (len + r + 127) / 128);
      }
    }
  }
  most = __reduce_max_sync(~0u, most);
  // of a request, the first item with at least T tiles
  auto first = [&](int h, int T) {
    const int x = (T - 1) * 128 - L[h];  // rows that end before
    return x >= rows[h] ? items[h] : x <= 0 ? 0 : cut.chunks > 1 ? x * cut.chunks : x / cut.rows_each;
  };
  auto count = [&](int T) {
    return (int64_t)a.nkv * __reduce_add_sync(~0u, items[0] - first(0, T) + items[1] - first(1, T));
  };
  Item it;
  it.cnt = 0;
  if (most == 0 || count(1) <= at) return it;
  int T = 1, hi = most;  // the most tiles that the item has
  while (T < hi) {
    const int mid = (T + hi + 1) >> 1;
    if (count(mid) > at)
      T = mid;
    else
      hi = mid - 1;
  }
  const int in = (int)(at - count(T + 1)), x = in / a.nkv;  // among those with T tiles
  it.g = in - x * a.nkv;
  int before = 0, b = -1, item = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int from = first(h, T), mine = first(h, T + 1) - from;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += y;
    }
    const uint32_t past = __ballot_sync(~0u, before + sum > x);
    if (b < 0 && past) {
      const int l = __ffs(past) - 1;
      b = 32 * h + l;
      item = __shfl_sync(~0u, from + x - before - (sum - mine), l);
      it.L = __shfl_sync(~0u, L[h], l);
    }
    before += __shfl_sync(~0u, sum, 31);
  }
  it.b = b;
  it.r0 = a.rm.start[b];
  if (cut.chunks > 1) {
    it.i_min = item / cut.chunks;
    it.h0 = item % cut.chunks * 256;
    it.nq = min(256, G - it.h0);
  } else {
    it.i_min = item * cut.rows_each;
    it.h0 = 0;
    it.nq = min(cut.rows_each, a.rm.start[b + 1] - it.r0 - it.i_min) * G;
  }
  it.end = it.L + it.i_min + divide_group(a, it.h0 + it.nq - 1) + 1;
  it.from = it.L + it.i_min + 1;
  it.t0 = 0;
  it.cnt = T;
  it.tail0 = it.from / 128;
  return it;
}

// The n-th item, or part of one, of this CTA: back and forth over the CTAs, and the last ones, which not all CTAs have,
// to those whose first was shortest (tiles, and 2.6 for each item, of the busiest CTA with the eight prompts: 47 without
// that, 45 so, of 42.6 on average); of parts, those without tiles are passed by (n: the one after it).  Not inlined: two
// roles run it, once an item.
static __device__ __noinline__ Item item_of_cta(const TreeArgs& a, Cut cut, int& n, int lane, const Parts& parts) {
  const int ctas = gridDim.x, c = blockIdx.x;
  for (;;) {
    const int64_t at = (int64_t)n * ctas + ((n & 1) || n == cut.last ? ctas - 1 - c : c);
    ++n;
    Item it = item_at(a, cut, at / cut.parts, lane);
    if (cut.parts == 1 || it.cnt == 0) return it;
    const int T = it.cnt, part = (int)(at % cut.parts);
    it.slot = (int)at;
    it.t0 = T * part / cut.parts;
    it.cnt = T * (part + 1) / cut.parts - it.t0;
    it.tail0 -= it.t0;
    if (it.cnt > 0) return it;
    for (int r = lane; r < 256; r += 32) parts.ml[at * 256 + r] = make_float2(-INFINITY, 0.f);
  }
}

// Whether a value tile has values that are not finite in rows z .. e - 1, by a warp: 0 times one is NaN, and
// stays in the sum.
template <int D>
__device__ __forceinline__ bool not_finite(const uint8_t* v, int z, int e, int lane) {
  const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
  __nv_bfloat162 s[4] = {zero, zero, zero, zero};
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    const uint8_t* end = v + h * kRegion + e * 128;
#pragma unroll 4
    for (const uint8_t* at = v + h * kRegion + z * 128 + lane * 16; at < end; at += 512) {
      const uint4 x = *reinterpret_cast<const uint4*>(at);
      s[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.x), zero, s[0]);
      s[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.y), zero, s[1]);
      s[2] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.z), zero, s[2]);
      s[3] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.w), zero, s[3]);
    }
  }
  const float2 t = __bfloat1622float2(__hadd2(__hadd2(s[0], s[1]), __hadd2(s[2], s[3])));
  return __any_sync(~0u, t.x != 0.f || t.y != 0.f);  // (true of NaN)
}

// Of a value tile the entries from `from` on, which not every row of the item sees: values
// that are not finite become 0 and their rows are noted in bad (bit: entry - from0); entries
// from `end` on become 0, if any of both are not finite.  By a warp; of most tiles it is a look (by
// two warps, value by value, one prompt of 36 rows took 11.2 us, not 10.0, 16 of 100 20.4, not 18.6).
template <int D>
static __device__ __noinline__ void clean_tile(uint8_t* v, int p0, int from, int end, int from0, int lane, uint32_t* bad) {
  constexpr int C = D / 8;
  const int z = max(from - p0, 0), e0 = min(max(end - p0, z), 128);
  if (!not_finite<D>(v, z, 128, lane)) return;
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll 8
    for (int x = e0 * 128 + lane * 16; x < kRegion; x += 512) *reinterpret_cast<uint4*>(v + h * kRegion + x) = make_uint4(0, 0, 0, 0);
  if (!not_finite<D>(v, z, e0, lane)) return;
#pragma unroll 1
  for (int c = z * C + lane; c < e0 * C; c += 32) {
    uint4* at = reinterpret_cast<uint4*>(v + chunk_off(c / C, c % C));
    uint4 x = *at;
    uint32_t* w = reinterpret_cast<uint32_t*>(&x);
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
    *at = x;
    const int bit = p0 + c / C - from0;
    atomicOr(&bad[bit >> 5], 1u << (bit & 31));
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ TreeArgs a, const Cut cut, const Parts parts) {
  using S = Shape<D>;
  constexpr int NST = S::NST, NR = D / 64;
  extern __shared__ __align__(1024) uint8_t sm[];  // (the kernel has no other shared memory)
  uint8_t* qimg = sm;
  uint8_t* ring = sm + 2 * S::STAGE;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + NST * S::STAGE);
  uint64_t* empty = full + NST;
  uint64_t* tail_full = empty + NST;  // in full's place for value tiles that clean_tile prepares
  uint64_t* q_full = tail_full + NST;
  uint64_t* q_empty = q_full + 1;
  uint64_t* s_full = q_empty + 1;   // [2]
  uint64_t* p_full = s_full + 2;    // [2]
  uint64_t* o_full = p_full + 2;    // [2]
  uint64_t* o_empty = o_full + 2;
  uint64_t* drain = o_empty + 1;
  uint64_t* v_clean = drain + 1;    // [2][kMaxTails] of items of this parity
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(v_clean + 2 * kMaxTails);  // [2][4 kMaxTails]
  Item* s_item = reinterpret_cast<Item*>(s_bad + 8 * kMaxTails);           // [kItems]
  uint32_t* tslot = reinterpret_cast<uint32_t*>(s_item + kItems);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      ptx::mbar_init(&full[i], 1);
      ptx::mbar_init(&empty[i], 1);
      ptx::mbar_init(&tail_full[i], 1);
    }
    ptx::mbar_init(q_full, 1);
    // (all that look at q_full let go of an item's queries, so that none of them is an item behind)
    ptx::mbar_init(q_empty, 10);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&s_full[i], 1);
      ptx::mbar_init(&p_full[i], 4);
      ptx::mbar_init(&o_full[i], 1);
    }
    ptx::mbar_init(o_empty, 8);
    ptx::mbar_init(drain, 1);
    for (int i = 0; i < 2 * kMaxTails; ++i) ptx::mbar_init(&v_clean[i], 32);
    ptx::fence_mbar_init();
  }
  if (warp == 1) ptx::tmem_alloc(tslot, 512);
  if (warp == 0 && lane == 0) {
    ptx::prefetch_tmap(&tmQ);
    ptx::prefetch_tmap(&tmK);
    ptx::prefetch_tmap(&tmV);
  }
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  Item it;  // of the two roles that look for the items
  int next_item = 0;
  if (warp == 0 || warp == 2) it = item_of_cta(a, cut, next_item, lane, parts);
  if (tid == 64) s_item[0] = it;
  if (warp == 3 && blockIdx.x == 0) {
    bool over = false;
    for (int b = lane; b < a.rm.batch; b += 32) {
      const int rows = a.rm.start[b + 1] - a.rm.start[b];
      over = over || (rows > 0 && !rows_fit(a.len[b], rows, a.cap));
    }
    if (__any_sync(~0u, over) && lane == 0 && a.err) atomicOr(a.err, kErrCapacity);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tslot;
  // every wait is bounded; a role that gives up flags the call and waits for
  // nothing more, so that all of them come to the end
  const unsigned long long limit = a.timeout_ns;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok && !ptx::mbar_sleep(bar, parity, limit)) {
      ok = false;
      if (a.err) atomicOr(a.err, kErrTimeout);
    }
    return ok;
  };

  if (warp == 0) {
    const uint64_t pol = ptx::policy_evict_last();
    uint32_t n = 0, tail = 0, turn = 0;  // slots whose last tile is on tail_full, its parity
    auto load = [&](int from, int to) {  // by one thread
      const int z = it.b * a.nkv + it.g;
      for (int t = from; t < to && ok; ++t)
        for (int kv = 0; kv < 2; ++kv, ++n) {
          const uint32_t s = n % NST, bit = 1u << s;
          if (n >= NST && !wait(&empty[s], (n / NST - 1) & 1)) break;
          uint64_t* bar = &full[s];
          tail &= ~bit;
          if (kv && t >= it.tail0) {
            ptx::mbar_arrive(bar);  // (this tile's phase of it)
            bar = &tail_full[s];
            tail |= bit;
            turn ^= bit;
          }
          ptx::mbar_arrive_expect_tx(bar, S::STAGE);
#pragma unroll
          for (int h = 0; h < NR; ++h)
            ptx::tma_load_3d(ring + s * S::STAGE + h * kRegion, kv ? &tmV : &tmK, bar, 64 * h, (it.t0 + t) * 128, z, pol);
        }
    };
    while (it.cnt > 0) {
      // (the next item is looked for while this one's first tiles are on their way)
      if (lane == 0) load(0, min(it.cnt, 2));
      __syncwarp();
      const Item next = item_of_cta(a, cut, next_item, lane, parts);
      if (lane == 0) load(2, it.cnt);
      ok = __all_sync(~0u, ok);
      it = next;
      if (!ok) break;
    }
    // no copy is in flight when the CTA ends
    if (lane == 0)
      for (uint32_t i = n > NST ? n - NST : 0; i < n; ++i) {
        const uint32_t s = i % NST;
        if ((tail >> s) & 1)
          ptx::mbar_wait(&tail_full[s], ((turn >> s) & 1) ^ 1, ptx::kDrainNs);
        else
          ptx::mbar_wait(&full[s], (i / NST) & 1, ptx::kDrainNs);
      }
  } else if (warp == 1) {
    // the whole warp, for operands in uniform registers; one thread issues
    const uint32_t lead = ptx::elect_one(), tm = __shfl_sync(~0u, tmem, 0);
    auto whole = [&](bool) { return ok = __all_sync(~0u, ok); };
    constexpr uint32_t IDESC1 = ptx::idesc_bf16_f32(128, 128);
    constexpr uint32_t IDESC2 = ptx::idesc_bf16_f32(128, D, true);
    // (shuffled, so that the compiler knows them to be the same in all threads and has a
    // product's descriptors computed in uniform registers: 20 cycles a product, not 44)
    auto uniform = [](uint32_t x) { return __shfl_sync(~0u, x, 0); };
    const uint32_t q_lo = uniform(ptx::desc_lo(ptx::smem_u32(qimg), 16u));
    Stage at;
    uint32_t p_turn = 0, c_turn = 0;  // parities of p_full and v_clean
    auto stage_of = [&](uint32_t x) { return ptx::smem_u32(ring + Stage::slot(x) * S::STAGE); };
    auto scores = [&](int t, uint32_t kt) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        ptx::mma_bf16_lo(lead, tm + 128 * t, q_lo + (((kk >> 2) * 2 * kRegion + t * kRegion + 32u * (kk & 3)) >> 4),
                         kt + (((kk >> 2) * kRegion + 32u * (kk & 3)) >> 4), IDESC1, kk > 0 ? 1u : 0u);
      ptx::mma_commit_if(lead, &s_full[t]);
    };
    for (uint32_t n = 0; ok; ++n) {
      if (n == 0 && s_item[0].cnt == 0) break;
      if (!whole(wait(q_full, n & 1))) break;
      const int cnt = __shfl_sync(~0u, s_item[n % kItems].cnt, 0), tail0 = __shfl_sync(~0u, s_item[n % kItems].tail0, 0);
      const bool two = __shfl_sync(~0u, s_item[n % kItems].nq, 0) > 128;
      if (cnt == 0) break;
      uint32_t k = at.next<NST>(), v = at.next<NST>();
      if (!whole(wait(&full[Stage::slot(k)], Stage::parity(k)))) break;
      // (products run in the order of their issue: scores come after the products that
      // read weights in their place)
      ptx::tc_fence_after();
      const uint32_t first = uniform(ptx::desc_lo(stage_of(k), 16u));
      scores(0, first);
      if (two) scores(1, first);
      ptx::mma_commit_if(lead, &empty[Stage::slot(k)]);
      if (cnt == 1) ptx::mma_commit_if(lead, q_empty);
      for (int j = 0; j < cnt && ok; ++j) {
        const int tail = j - tail0;
        const bool more = j + 1 < cnt;
        const uint32_t v_now = v;
        if (more) k = at.next<NST>(), v = at.next<NST>();
        // the values, the first tile's weights and the next keys: their first looks overlap
        const int tail_bar = (n & 1) * kMaxTails + tail;
        uint64_t* v_bar = tail < 0 ? &full[Stage::slot(v_now)] : &v_clean[tail_bar];
        const uint32_t v_parity = tail < 0 ? Stage::parity(v_now) : (c_turn >> tail_bar) & 1;
        const bool v_there = ptx::mbar_try_wait(v_bar, v_parity), p_there = ptx::mbar_try_wait(&p_full[0], p_turn & 1);
        const bool k_there = !more || ptx::mbar_try_wait(&full[Stage::slot(k)], Stage::parity(k));
        if (!v_there) wait(v_bar, v_parity);
        if (!p_there) wait(&p_full[0], p_turn & 1);
        if (!k_there) wait(&full[Stage::slot(k)], Stage::parity(k));
        if (j == 0 && n > 0) wait(o_empty, (n - 1) & 1);
        if (!whole(ok)) break;
        if (tail >= 0) c_turn ^= 1u << tail_bar;
        p_turn ^= two ? 3u : 1u;
        ptx::tc_fence_after();
        const uint32_t vt = uniform(ptx::desc_lo(stage_of(v_now), kRegion)), kt = uniform(ptx::desc_lo(stage_of(k), 16u));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (t == 1) {
            if (!two) break;
            if (!whole(wait(&p_full[1], ((p_turn >> 1) & 1) ^ 1))) break;
            ptx::tc_fence_after();
          }
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            ptx::mma_bf16_ta_lo(lead, tm + 256 + 128 * t, tm + 128 * t + 8u * kk, vt + 128u * kk, IDESC2,
                                j > 0 || kk > 0 ? 1u : 0u);
          if (more)
            scores(t, kt);
          else
            ptx::mma_commit_if(lead, &o_full[t]);
        }
        // (what was loaded is let go when all products up to here are done)
        ptx::mma_commit_if(lead, &empty[Stage::slot(v_now)]);
        if (more) ptx::mma_commit_if(lead, &empty[Stage::slot(k)]);
        if (j + 2 == cnt) ptx::mma_commit_if(lead, q_empty);
      }
    }
    // no product is running when TMEM is freed
    ptx::mma_commit_if(lead, drain);
    ptx::mbar_wait(drain, 0, ptx::kDrainNs);
  } else if (warp == 2) {
    auto load_queries = [&](const Item& it) {  // by one thread
      const int heads = min(256, a.nq / a.nkv);
      ptx::mbar_arrive_expect_tx(q_full, NR * 128 * heads * cut.rows_each);
#pragma unroll
      for (int h = 0; h < NR; ++h)
        ptx::tma_load_3d(qimg + 2 * h * kRegion, &tmQ, q_full, 64 * h, it.g * (a.nq / a.nkv) + it.h0, it.r0 + it.i_min,
                         ptx::policy_evict_first());
    };
    if (lane == 0 && it.cnt > 0) load_queries(it);
    uint32_t n = 0;  // items whose queries are on their way, or were
    while (it.cnt > 0) {
      it = item_of_cta(a, cut, next_item, lane, parts);
      // this item's queries, when the last one's have been read.  (Its results are not written yet, but those of the one
      // before are: who writes them has let go of the last one's queries.)
      if (lane == 0 && wait(q_empty, n & 1)) {
        s_item[(n + 1) % kItems] = it;
        if (it.cnt > 0)
          load_queries(it);
        else
          ptx::mbar_arrive(q_full);
      }
      ok = __all_sync(~0u, ok);
      if (!ok) break;
      ++n;
    }
    // no copy is in flight when the CTA ends (q_empty says so of those that were waited for)
    if (lane == 0 && !ok) ptx::mbar_wait(q_full, n & 1, ptx::kDrainNs);
  } else if (warp == 3) {
    uint32_t tiles = 0, turn = 0;
    for (uint32_t n = 0; ok; ++n) {
      if (n == 0 && s_item[0].cnt == 0) break;
      wait(q_full, n & 1);
      ok = __all_sync(~0u, ok);
      it = s_item[n % kItems];
      if (!ok || it.cnt == 0) break;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(q_empty);
      // (what was noted for the item before the last has been read)
      uint32_t* bad = s_bad + (n & 1) * 4 * kMaxTails;
      if (lane < 4 * kMaxTails) bad[lane] = 0;
      __syncwarp();
      for (int t = max(it.tail0, 0); t < it.cnt; ++t) {
        const uint32_t s = (2 * (tiles + t) + 1) % NST;
        // (what follows is done by the whole warp, or by none of it; nor is a tile let go that did not come)
        ok = __all_sync(~0u, wait(&tail_full[s], (turn >> s) & 1));
        turn ^= 1u << s;
        if (!ok) break;
        clean_tile<D>(ring + s * S::STAGE, (it.t0 + t) * 128, it.from, it.end, it.from, lane, bad);
        ptx::fence_proxy_async_smem();
        ptx::mbar_arrive(&v_clean[(n & 1) * kMaxTails + t - it.tail0]);
      }
      tiles += it.cnt;
    }
  } else {
    const int quad = warp & 3, t = (warp - 4) >> 2, row = 32 * quad + lane;
    const uint32_t tl = tmem + ((uint32_t)(32 * quad) << 16);
    const uint32_t ts = tl + 128 * t, to = tl + 256 + 128 * t;
    const int G = a.nq / a.nkv;
    const float c = a.scale_log2;
    uint32_t ns = 0, mine_items = 0, c_turn = 0;
    for (uint32_t n = 0;; ++n) {
      if (n == 0 && s_item[0].cnt == 0) break;
      wait(q_full, n & 1);
      ok = __all_sync(~0u, ok);
      const int cnt = s_item[n % kItems].cnt;
      if (!ok || cnt == 0) break;
      const int tail0 = s_item[n % kItems].tail0, nq = s_item[n % kItems].nq, t0 = s_item[n % kItems].t0;
      const int of_parity = n & 1;
      const bool some = nq > 128 * t;  // the tile has queries
      // the last entry that the row sees
      const int last = s_item[n % kItems].L + s_item[n % kItems].i_min + divide_group(a, s_item[n % kItems].h0 + min(128 * t + row, nq - 1));
      // (a row that is no query's has what was in its place before, of no consequence)
      const bool live = 128 * t + row < nq;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(q_empty);
      float ref = live ? -INFINITY : 0.f, l = 0.f;  // the reference, a score
      bool fresh = __any_sync(~0u, live);  // a row has no reference yet
      if (some) {
#pragma unroll 1
        for (int j = 0; j < cnt; ++j, ++ns) {
          wait(&s_full[t], ns & 1);
          __syncwarp();
          ptx::tc_fence_after();
          const bool tail = j >= tail0;
          const int seen = last + 1 - (t0 + j) * 128;  // entries of the tile that the row sees
          uint32_t p[64];
          float sum;
          // looked: the row's reference may have been moved, and is what this tile gives
          float m = __fmul_rn(ref, c);
          bool need = m == -INFINITY, again = fresh, looked = false;
#pragma unroll 1
          for (;;) {
            if (again) {
              float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
              for (int x = 0; x < 128; x += 32) {
                uint32_t v[32];
                ptx::tmem_ld32(ts + x, v);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (!tail || x + e < seen) mx[e & 1] = fmaxf(mx[e & 1], __uint_as_float(v[e]));
              }
              // (NaN scores pass the maximum by, and reach the sums)
              const float top = fmaxf(mx[0], mx[1]), mt = __fmul_rn(top, c);
              // (a row whose sum is fine keeps its reference: what another row sees changes nothing for it)
              const bool grow = need && top > ref && mt > -INFINITY;
              const float m_new = grow ? mt : m, f = m == -INFINITY ? 0.f : ex2(m - m_new);
              l = grow ? l * f : l;
              if (j > 0) {
#pragma unroll 1
                for (int x = 0; x < D; x += 16) {
                  uint32_t o[16];
                  ptx::tmem_ld16(to + x, o);
                  ptx::tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = grow ? __float_as_uint(__uint_as_float(o[e]) * f) : o[e];
                  ptx::tmem_st16(to + x, o);
                }
              }
              m = m_new;
              ref = grow ? top : ref;
              looked = looked || need;
              fresh = __any_sync(~0u, m == -INFINITY);
            }
            const Exponent x2 = exponent_of([&] { return ref; }, m, c, kFar);
            const uint64_t c2 = as2d::two(x2.by, x2.by), ref2 = as2d::two(-x2.at, -x2.at);
            uint64_t ls[2] = {0, 0};
            uint32_t v[2][32];
            ptx::tmem_ld32(ts, v[0]);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              ptx::tmem_ld_wait();
              if (x < 3) ptx::tmem_ld32(ts + 32 * (x + 1), v[(x + 1) & 1]);
              uint32_t(&u)[32] = v[x & 1];
              if (tail) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (32 * x + e >= seen) u[e] = 0xFF800000u;  // -inf
              }
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float2 y = of_two(fma2(as2d::two(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1])), c2, ref2));
                const uint64_t w = as2d::two(ex2(y.x), ex2(y.y));
                ls[e & 1] = add2(ls[e & 1], w);
                const float2 f = of_two(w);
                p[16 * x + e] = pack2(f.x, f.y);
              }
            }
            const float2 sums = of_two(add2(ls[0], ls[1]));
            sum = sums.x + sums.y;
            // (a pass for rows without a reference, of which NaN rows are never rid, was none for the others)
            need = live && !looked && !(sum <= kMost);
            if (!__any_sync(~0u, need)) break;
            again = true;
          }
#pragma unroll
          for (int x = 0; x < 64; x += 16) ptx::tmem_st16(ts + x, p + x);
          l += sum;
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&p_full[t]);
          __syncwarp();
        }
        // ---- the item's end ----
        wait(&o_full[t], mine_items & 1);
        ++mine_items;
      } else {
        wait(&o_full[0], n & 1);  // (not an item ahead of the others)
      }
      for (int x = max(-tail0, 0); x < cnt - tail0; ++x) {
        const int bar = of_parity * kMaxTails + x;
        if (some) wait(&v_clean[bar], (c_turn >> bar) & 1);
        c_turn ^= 1u << bar;
      }
      ok = __all_sync(~0u, ok);
      ptx::tc_fence_after();
      if (some && ok) {
        const float m = __fmul_rn(ref, c), inv = l == 0.f ? 0.f : 1.f / l;
        it = s_item[n % kItems];
        const int q = it.h0 + min(128 * t + row, nq - 1), of = divide_group(a, q), h = it.g * G + (q - of * G);
        const size_t at = (size_t)(it.r0 + it.i_min + of) * a.nq + h;
        bf16* out = (bf16*)a.out + at * D;
        const uint32_t* bad = s_bad + of_parity * 4 * kMaxTails;
        uint32_t any = 0;
        if (cnt > tail0)
          for (int x = 0; x < 4 * kMaxTails; ++x) any |= bad[x];
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 32) {
          uint32_t o[32];
          ptx::tmem_ld32(to + d0, o);
          ptx::tmem_ld_wait();
          if (any) {
            // values that are not finite in entries that not every row sees: added where they are seen
            for (int x = 0; x < 4 * kMaxTails; ++x)
              for (uint32_t left = bad[x]; left; left &= left - 1) {
                const int e = it.from + 32 * x + __ffs(left) - 1;
                if (e > last) continue;
                const bf16* u = a.v + (((size_t)it.b * a.nkv + it.g) * a.cap + e) * D + d0;
#pragma unroll
                for (int y = 0; y < 32; ++y) {
                  const float z = __bfloat162float(u[y]);
                  if (!(fabsf(z) <= 3.4e38f)) o[y] = __float_as_uint(__uint_as_float(o[y]) + z);
                }
              }
            __syncwarp();
          }
          if (live && cut.parts > 1) {
            float4* to_part = parts.o + ((size_t)it.slot * (D / 4) + d0 / 4) * 256 + 128 * t + row;
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              to_part[e / 4 * 256] = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]),
                                                 __uint_as_float(o[e + 3]));
          } else if (live) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
              uint32_t w[8];
#pragma unroll
              for (int y = 0; y < 8; ++y)
                w[y] = pack2(__uint_as_float(o[e + 2 * y]) * inv, __uint_as_float(o[e + 2 * y + 1]) * inv);
              ptx::store_8(out + d0 + e, w);
            }
          }
          __syncwarp();
        }
        if (live && cut.parts > 1)
          parts.ml[(size_t)it.slot * 256 + 128 * t + row] = make_float2(m, l);
        else if (live && a.lse)
          a.lse[at] = row_lse(m, l);
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(o_empty);
      __syncwarp();
    }
  }
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// The parts of items joined, in the order of their tiles: a block for 32 queries of an item, a lane to a
// query.
constexpr int kJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps)
    prompt_join_kernel(const __grid_constant__ TreeArgs a, const Cut cut, const Parts parts) {
  __shared__ Item s_item;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockIdx.x / 8, row = blockIdx.x % 8 * 32 + lane;
  ptx::griddep_launch_dependents();
  // (the lengths before the wait: the kernel before lets this one start after its own, and writes none)
  if (warp == 0) {
    const Item it = item_at(a, cut, n, lane);
    if (lane == 0) s_item = it;
  }
  __syncthreads();
  ptx::griddep_wait();
  if (s_item.cnt == 0 || row >= s_item.nq) return;
  const int G = a.nq / a.nkv;
  const int q = s_item.h0 + row, of = divide_group(a, q), h = s_item.g * G + (q - of * G);
  const size_t at = (size_t)(s_item.r0 + s_item.i_min + of) * a.nq + h;
  constexpr int Z = D / 4 / kJoinWarps, U = 4;  // of a lane; parts in flight
  float M = -INFINITY, l = 0.f;
  float4 o[Z];
#pragma unroll
  for (int z = 0; z < Z; ++z) o[z] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < cut.parts; k0 += U) {
    float2 ml[U];
    float4 v[U][Z];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t slot = n * cut.parts + min(k0 + u, cut.parts - 1);
      ml[u] = __ldcg(&parts.ml[slot * 256 + row]);
      if (k0 + u >= cut.parts) ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int z = 0; z < Z; ++z) v[u][z] = __ldcg(&parts.o[(slot * (D / 4) + warp * Z + z) * 256 + row]);
    }
    const float before = M;
#pragma unroll
    for (int u = 0; u < U; ++u) M = fmaxf(M, ml[u].x);
    const float w = part_weight(before, M);
    // (what a part has that is not finite stays, whatever its weight; one without tiles has nothing)
    auto weighted = [](float x, float f) { return is_finite(x) ? x * f : x; };
    l *= w;  // (a NaN stays)
#pragma unroll
    for (int z = 0; z < Z; ++z)
      o[z] = make_float4(weighted(o[z].x, w), weighted(o[z].y, w), weighted(o[z].z, w), weighted(o[z].w, w));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = part_weight(ml[u].x, M);
      l = fmaf(ml[u].y, f, l);
      if (ml[u].x == -INFINITY && ml[u].y == 0.f) continue;
#pragma unroll
      for (int z = 0; z < Z; ++z) {
        o[z].x += weighted(v[u][z].x, f);
        o[z].y += weighted(v[u][z].y, f);
        o[z].z += weighted(v[u][z].z, f);
        o[z].w += weighted(v[u][z].w, f);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16* out = (bf16*)a.out + at * D + warp * Z * 4;
#pragma unroll
  for (int z = 0; z < Z; ++z)
    *reinterpret_cast<uint2*>(out + 4 * z) =
        make_uint2(pack2(o[z].x * inv, o[z].y * inv), pack2(o[z].z * inv, o[z].w * inv));
  if (warp == 0 && a.lse) a.lse[at] = row_lse(M, l);
}

template <int D>
cudaError_t launch(const TreeArgs& a, Cut cut, int64_t n, void* workspace, cudaStream_t st) {
  static PerDevice opted;
  cudaError_t e = opt_in(opted, prompt_kernel<D>, Shape<D>::SMEM);
  if (e != cudaSuccess) return e;
  CUtensorMap tq, tk, tv;
  const int64_t heads = (int64_t)a.rm.batch * a.nkv;
  if (!encode_rows_map(&tq, a.q, D, a.nq, a.rm.rows, a.q_stride, std::min(256, a.nq / a.nkv), cut.rows_each) ||
      !encode_cache_map(&tk, a.k, D, a.cap, heads) || !encode_cache_map(&tv, a.v, D, a.cap, heads))
    return cudaErrorInvalidValue;
  Parts parts;
  parts.o = (float4*)workspace;
  parts.ml = (float2*)(parts.o + (size_t)kSlots * device_sms() * 256 * D / 4);
  e = launch_pdl(prompt_kernel<D>, dim3((unsigned)std::min<int64_t>(n * cut.parts, device_sms())), dim3(kThreads),
                 Shape<D>::SMEM, st, 1, tq, tk, tv, a, cut, parts);
  if (e != cudaSuccess || cut.parts == 1) return e;
  return launch_pdl(prompt_join_kernel<D>, dim3((unsigned)n * 8), dim3(32 * kJoinWarps), 0, st, 1, a, cut, parts);
}

}  // namespace

size_t prompt_attention_workspace(int head_dim) {
  return (size_t)kSlots * device_sms() * 256 * (head_dim * 4 + 8);
}

cudaError_t launch_prompt_attention(const TreeArgs& a, int head_dim, int64_t max_keys, void* workspace,
                                    cudaStream_t st) {
  const int G = a.nq / a.nkv, sms = device_sms();
  Cut cut = {std::max(1, 256 / G), (G + 255) / 256, 1, -1};
  int64_t n = 0;
  for (int b = 0; b < a.rm.batch; ++b) {
    const int64_t r = a.rm.start[b + 1] - a.rm.start[b];
    n += (cut.chunks > 1 ? r * cut.chunks : (r + cut.rows_each - 1) / cut.rows_each) * a.nkv;
  }
  // Few items of many tiles: one part a CTA, or where that is less than two, parts for two
  // rounds.  us, 28 query and 4 kv heads, 128 rows after 15000 / 4000 / 1000 entries: whole 189 / 60 / 24, parts of
  // four tiles at least 42 / 26 / 22, of eight 42 / 29 / 24.
  const int64_t tiles = (max_keys + 127) / 128;
  if (n <= sms) cut.parts = (int)std::max<int64_t>(1, std::min<int64_t>((2 * n <= sms ? 1 : kSlots) * sms / n, tiles / kPartTiles));
  const int64_t all = n * cut.parts, ctas = std::min<int64_t>(all, sms);
  if (all % ctas != 0) cut.last = (int)(all / ctas);
  return head_dim == 128 ? launch<128>(a, cut, n, workspace, st) : launch<64>(a, cut, n, workspace, st);
}

}  // namespace as2d
