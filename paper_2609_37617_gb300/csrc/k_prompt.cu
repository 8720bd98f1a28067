// k_prompt.cu -- causal attention of whole prompts over a cache
// (as2d_prompt_attention).
//
// Row i of request b sees the entries 0 .. L_b + i.  With s_t = scale q k_t over them:
//   m = max s_t, l = sum e^(s_t - m), out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// The G = n_q / n_kv query heads of a kv head, for all rows of a request, form one
// query matrix of rows G queries (row by row, so that 256 queries stand for few rows and
// little of a tile on the diagonal is masked), cut into pairs of query tiles of 128
// (the MMA's M).  An item is one (request, kv head, pair); a CTA takes it through its key
// tiles of 128.
//
// Per CTA (12 warps, TMEM full: two score buffers, two accumulators):
//   warp 0     loads key and value tiles by TMA through a ring of shared-memory stages;
//   warp 1     issues the products: S = Q K^T, O += P V (P from TMEM) of the two query
//              tiles in turn, so that one's products run under the other's softmax;
//   warps 2-3  prepare the value tiles that hold entries not every row sees;
//   warps 4-7 and 8-11 a query tile each, a query a thread: S from TMEM, mask, running
//              maximum, P = 2^(S - m) back into TMEM in bf16 over S; O is rescaled only where
//              the maximum grew by more than 2^8.
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
// P may grow to 2^kLazy before the accumulator is rescaled.
constexpr float kLazy = 8.f;

// The items of a call, longest first: requests by their rows, of a request its last rows first.
struct Items {
  int first[kMaxBatch + 1];   // items before the n-th request of the order
  uint8_t request[kMaxBatch];
};

template <int D>
struct Shape {
  static constexpr uint32_t STAGE = 128 * D * 2;  // one K or V tile, and one query tile
  static constexpr int NST = D == 64 ? 8 : 5;
  static constexpr uint32_t SMEM = 1024 + (2 + NST) * STAGE + (3 * NST + 8 + kMaxTails) * 8 + 4 * kMaxTails * 4 + 16;
  static_assert(SMEM <= 232448, "shared memory of one CTA");
};

// Of a value tile the entries from `from` on, which not every row of the item sees: values
// that are not finite become 0 and their rows are noted in bad (bit: entry - from0); entries
// from `end` on become 0.
template <int D>
__device__ __forceinline__ void clean_tile(uint8_t* v, int p0, int from, int end, int from0, int tid, uint32_t* bad) {
  constexpr int C = D / 8;
  const int z = max(from - p0, 0), e0 = min(max(end - p0, z), 128);
#pragma unroll 1
  for (int c = z * C + tid; c < 128 * C; c += 64) {
    uint4* at = reinterpret_cast<uint4*>(v + chunk_off(c / C, c % C));
    if (c >= e0 * C) {
      *at = make_uint4(0, 0, 0, 0);
      continue;
    }
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
    prompt_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ TreeArgs a, const __grid_constant__ Items items) {
  using S = Shape<D>;
  constexpr int NST = S::NST, NR = D / 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* qimg = sm;
  uint8_t* ring = sm + 2 * S::STAGE;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + NST * S::STAGE);
  uint64_t* empty = full + NST;
  uint64_t* tail_full = empty + NST;  // in full's place for value tiles that clean_tile prepares
  uint64_t* q_full = tail_full + NST;
  uint64_t* s_full = q_full + 1;  // [2]
  uint64_t* p_full = s_full + 2;  // [2]
  uint64_t* o_full = p_full + 2;  // [2]
  uint64_t* drain = o_full + 2;
  uint64_t* v_clean = drain + 1;  // [kMaxTails]
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(v_clean + kMaxTails);  // [4 kMaxTails]
  uint32_t* tslot = s_bad + 4 * kMaxTails;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      ptx::mbar_init(&full[i], 1);
      ptx::mbar_init(&empty[i], 1);
      ptx::mbar_init(&tail_full[i], 1);
    }
    ptx::mbar_init(q_full, (kThreads - 64) / 32);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&s_full[i], 1);
      ptx::mbar_init(&p_full[i], 4);
      ptx::mbar_init(&o_full[i], 1);
    }
    ptx::mbar_init(drain, 1);
    for (int i = 0; i < kMaxTails; ++i) ptx::mbar_init(&v_clean[i], 64);
    ptx::fence_mbar_init();
  }
  if (tid >= 64 && tid < 64 + 4 * kMaxTails) s_bad[tid - 64] = 0;
  if (warp == 1) ptx::tmem_alloc(tslot, 512);
  if (warp == 0 && lane == 0) {
    ptx::prefetch_tmap(&tmK);
    ptx::prefetch_tmap(&tmV);
  }
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  // the item
  int lo = 0, hi = a.rm.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (items.first[mid] <= (int)blockIdx.x)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int b = items.request[lo], r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0;
  const int G = a.nq / a.nkv, queries = rows * G;
  const int in = blockIdx.x - items.first[lo], pairs = (queries + 255) / 256;
  const int g = in % a.nkv, pair = pairs - 1 - in / a.nkv;
  const int q0 = pair * 256, nq = min(256, queries - q0);
  const int i_min = q0 / G, h0 = q0 - i_min * G;  // row and head of the first query
  const int i_max = i_min + divide_group(a, h0 + nq - 1);
  const int len = a.len[b];
  const bool fits = rows_fit(len, rows, a.cap);
  const int L = fits ? len : 0;
  if (!fits && tid == 0 && a.err) atomicOr(a.err, kErrCapacity);
  const int end = L + i_max + 1;                // entries that some row sees
  const int cnt = fits ? (end + 127) / 128 : 0;  // key tiles
  const int from = L + i_min + 1;               // entries that not every row sees
  const int tail0 = from / 128;                 // the first tile that holds some
  const bool two = nq > 128;
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tslot;
  if (warp >= 2 && cnt > 0) {
    // the queries, every copy on its way at once
    constexpr int C = D / 8;
    const bf16* from_q = (const bf16*)a.q + (r0 + i_min) * a.q_stride + (int64_t)g * G * D;
#pragma unroll 4
    for (int x = tid - 64; x < nq * C; x += kThreads - 64) {
      const int r = x / C, cc = x % C, i = divide_group(a, h0 + r), h = h0 + r - i * G;
      ptx::cp_async16(qimg + (r >> 7) * S::STAGE + chunk_off(r & 127, cc), from_q + i * a.q_stride + h * D + 8 * cc);
    }
    ptx::cp_async_wait_all();
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(q_full);
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

  if (warp == 0) {
    if (lane == 0) {
      const uint64_t pol = ptx::policy_evict_last();
      const int z = b * a.nkv + g;
      uint32_t n = 0, tail = 0;  // slots whose last tile is on tail_full
      for (int t = 0; t < cnt && ok; ++t)
        for (int kv = 0; kv < 2; ++kv, ++n) {
          const uint32_t s = n % NST, bit = 1u << s;
          if (n >= NST && !wait(&empty[s], (n / NST - 1) & 1)) break;
          uint64_t* bar = &full[s];
          tail &= ~bit;
          if (kv && t >= tail0) {
            ptx::mbar_arrive(bar);  // (this tile's phase of it)
            bar = &tail_full[s];
            tail |= bit;
          }
          ptx::mbar_arrive_expect_tx(bar, S::STAGE);
#pragma unroll
          for (int h = 0; h < NR; ++h)
            ptx::tma_load_3d(ring + s * S::STAGE + h * kRegion, kv ? &tmV : &tmK, bar, 64 * h, t * 128, z, pol);
        }
      // no copy is in flight when the CTA ends
      for (uint32_t i = n > NST ? n - NST : 0; i < n; ++i) {
        const uint32_t s = i % NST;
        if ((tail >> s) & 1)
          ptx::mbar_wait(&tail_full[s], 0, ptx::kDrainNs);
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
    Stage at;
    auto scores = [&](int t, uint32_t k) {
      const uint32_t kt = ptx::desc_lo(ptx::smem_u32(ring + Stage::slot(k) * S::STAGE), 16u);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint32_t to = ((kk >> 2) * kRegion + 32u * (kk & 3)) >> 4;
        ptx::mma_bf16_lo(lead, tm + 128 * t, q_lo + t * (S::STAGE >> 4) + to, kt + to, IDESC1, kk > 0 ? 1u : 0u);
      }
      ptx::mma_commit_if(lead, &s_full[t]);
    };
    if (cnt > 0 && whole(wait(q_full, 0))) {
      uint32_t k = at.next<NST>(), v = at.next<NST>();
      if (whole(wait(&full[Stage::slot(k)], Stage::parity(k)))) {
        ptx::tc_fence_after();
        scores(0, k);
        if (two) scores(1, k);
        ptx::mma_commit_if(lead, &empty[Stage::slot(k)]);
      }
      for (int j = 0; j < cnt && ok; ++j) {
        const int tail = j - tail0;
        if (!whole(tail < 0 ? wait(&full[Stage::slot(v)], Stage::parity(v)) : wait(&v_clean[tail], 0))) break;
        const uint32_t vt = ptx::desc_lo(ptx::smem_u32(ring + Stage::slot(v) * S::STAGE), kRegion);
        const uint32_t v_now = v;
        k = at.next<NST>();
        v = at.next<NST>();
#pragma unroll 1
        for (int t = 0; t < (two ? 2 : 1); ++t) {
          if (!whole(wait(&p_full[t], j & 1))) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            ptx::mma_bf16_ta_lo(lead, tm + 256 + 128 * t, tm + 128 * t + 8u * kk, vt + 128u * kk, IDESC2,
                                j > 0 || kk > 0 ? 1u : 0u);
          if (t == (two ? 1 : 0)) ptx::mma_commit_if(lead, &empty[Stage::slot(v_now)]);
          if (j + 1 == cnt) {
            ptx::mma_commit_if(lead, &o_full[t]);
          } else {
            // (products run in the order of their issue: these scores come after the
            // product that reads the weights in their place)
            if (t == 0 && !whole(wait(&full[Stage::slot(k)], Stage::parity(k)))) break;
            ptx::tc_fence_after();
            scores(t, k);
            if (t == (two ? 1 : 0)) ptx::mma_commit_if(lead, &empty[Stage::slot(k)]);
          }
        }
      }
    }
    // no product is running when TMEM is freed
    ptx::mma_commit_if(lead, drain);
    ptx::mbar_wait(drain, 0, ptx::kDrainNs);
  } else if (warp < 4) {
    for (int t = tail0; t < cnt; ++t) {
      const uint32_t s = (2 * t + 1) % NST;
      if (!wait(&tail_full[s], 0)) break;
      clean_tile<D>(ring + s * S::STAGE, t * 128, from, end, from, tid - 64, s_bad);
      ptx::fence_proxy_async_smem();
      ptx::mbar_arrive(&v_clean[t - tail0]);
    }
  } else if (cnt > 0 && (two || warp < 8)) {
    const int t = (warp - 4) >> 2, quad = warp & 3, row = 32 * quad + lane;
    const uint32_t tl = tmem + ((uint32_t)(32 * quad) << 16);
    const uint32_t ts = tl + 128 * t, to = tl + 256 + 128 * t;
    const bool live = 128 * t + row < nq;
    const int q = h0 + min(128 * t + row, nq - 1), of = divide_group(a, q), i = i_min + of, h = g * G + (q - of * G);
    const float c = a.scale_log2;
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int j = 0; j < cnt; ++j) {
      wait(&s_full[t], j & 1);
      ok = __all_sync(~0u, ok);
      ptx::tc_fence_after();
      uint32_t v[128];
#pragma unroll
      for (int x = 0; x < 128; x += 32) ptx::tmem_ld32(ts + x, v + x);
      ptx::tmem_ld_wait();
      const int seen = L + i + 1 - j * 128;  // entries of the tile that the row sees
      if (j >= tail0) {
#pragma unroll
        for (int e = 0; e < 128; ++e)
          if (e >= seen) v[e] = 0xFF800000u;  // -inf
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < 128; e += 8)
#pragma unroll
        for (int f = 0; f < 4; ++f)
          mx[f] = max3(mx[f], __uint_as_float(v[e + 2 * f]), __uint_as_float(v[e + 2 * f + 1]));
      const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
      // (NaN scores pass the maximum by, and reach the sums)
      const bool grow = mt > m + kLazy;
      if (__any_sync(~0u, grow)) {
        const float m_new = grow ? mt : m;
        const float f = m == -INFINITY ? 0.f : ex2(m - m_new);
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
      }
      const float ref = m == -INFINITY ? 0.f : m;
      const uint64_t c2 = as2d::two(c, c), ref2 = as2d::two(-ref, -ref);
      uint64_t ls[2] = {0, 0};
#pragma unroll
      for (int x = 0; x < 128; x += 32) {
        uint32_t p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 y = of_two(fma2(as2d::two(__uint_as_float(v[x + 2 * e]), __uint_as_float(v[x + 2 * e + 1])), c2, ref2));
          const uint64_t w = as2d::two(ex2(y.x), ex2(y.y));
          ls[e & 1] = add2(ls[e & 1], w);
          const float2 f = of_two(w);
          p[e] = pack2(f.x, f.y);
        }
        ptx::tmem_st16(ts + x / 2, p);
      }
      const float2 sums = of_two(add2(ls[0], ls[1]));
      l += sums.x + sums.y;
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&p_full[t]);
    }
    wait(&o_full[t], 0);
    for (int x = 0; x < cnt - tail0; ++x) wait(&v_clean[x], 0);
    ok = __all_sync(~0u, ok);
    ptx::tc_fence_after();
    if (ok) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* out = (bf16*)a.out + ((size_t)(r0 + i) * a.nq + h) * D;
      uint32_t any = 0;
      for (int x = 0; x < 4 * kMaxTails; ++x) any |= s_bad[x];
#pragma unroll 1
      for (int d0 = 0; d0 < D; d0 += 16) {
        uint32_t o[16];
        ptx::tmem_ld16(to + d0, o);
        ptx::tmem_ld_wait();
        if (any) {
          // values that are not finite in entries that not every row sees: added where they are seen
          for (int x = 0; x < 4 * kMaxTails; ++x)
            for (uint32_t left = s_bad[x]; left; left &= left - 1) {
              const int e = from + 32 * x + __ffs(left) - 1;
              if (e > L + i) continue;
              const bf16* v = a.v + (((size_t)b * a.nkv + g) * a.cap + e) * D + d0;
#pragma unroll
              for (int y = 0; y < 16; ++y) {
                const float z = __bfloat162float(v[y]);
                if (!(fabsf(z) <= 3.4e38f)) o[y] = __float_as_uint(__uint_as_float(o[y]) + z);
              }
            }
          __syncwarp();
        }
        if (live) {
          uint32_t p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = pack2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
          reinterpret_cast<uint4*>(out + d0)[0] = make_uint4(p[0], p[1], p[2], p[3]);
          reinterpret_cast<uint4*>(out + d0)[1] = make_uint4(p[4], p[5], p[6], p[7]);
        }
        __syncwarp();
      }
      if (live && a.lse) a.lse[(size_t)(r0 + i) * a.nq + h] = row_lse(m, l);
    }
    ptx::tc_fence_before();
  }
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int D>
cudaError_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const TreeArgs& a, const Items& items, int64_t n,
                   cudaStream_t st) {
  static PerDevice opted;
  const cudaError_t e = opt_in(opted, prompt_kernel<D>, Shape<D>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_pdl(prompt_kernel<D>, dim3((unsigned)n), dim3(kThreads), Shape<D>::SMEM, st, 1, tk, tv, a, items);
}

}  // namespace

size_t prompt_attention_workspace(int) { return 256; }

cudaError_t launch_prompt_attention(const TreeArgs& a, int head_dim, int64_t max_keys, void* workspace,
                                    cudaStream_t st) {
  Items items = {};
  const int G = a.nq / a.nkv, batch = a.rm.batch;
  auto rows = [&](int b) { return a.rm.start[b + 1] - a.rm.start[b]; };
  for (int b = 0; b < batch; ++b) items.request[b] = (uint8_t)b;
  std::stable_sort(items.request, items.request + batch, [&](uint8_t x, uint8_t y) { return rows(x) > rows(y); });
  int64_t n = 0;
  for (int k = 0; k < batch; ++k) {
    items.first[k] = (int)n;
    n += ((int64_t)rows(items.request[k]) * G + 255) / 256 * a.nkv;
  }
  items.first[batch] = (int)n;
  CUtensorMap tk, tv;
  if (!encode_cache_map(&tk, a.k, head_dim, a.cap, (int64_t)batch * a.nkv) ||
      !encode_cache_map(&tv, a.v, head_dim, a.cap, (int64_t)batch * a.nkv))
    return cudaErrorInvalidValue;
  return head_dim == 128 ? launch<128>(tk, tv, a, items, n, st) : launch<64>(tk, tv, a, items, n, st);
}

}  // namespace as2d
