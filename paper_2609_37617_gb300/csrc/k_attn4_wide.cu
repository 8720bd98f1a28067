// k_attn4_wide.cu -- attention of a tree of drafted tokens over a cache in 4 bits, for
// requests of many queries to a kv head (as2d_cache4_attention; k_attn4.cu has few).
//
// With s_t = scale q k_t over the entries that a row sees: m = max s_t, l = sum e^(s_t - m),
// out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// The units (query tile of 128, 128-key tile) are spread over one CTA per SM and joined as
// those of k_tree_attn.cu.  Codes become 16-bit floats, exactly, on their way into shared
// memory, and the products run on tcgen05 with 16-bit floats: a query with a power of two of its own
// (two parts of 32-bit ones), weights up to 2^15 (two parts beside 32-bit queries).
//
// Per CTA (16 warps, TMEM full: two score buffers, two accumulators):
//   warps 0-7   two sets of four that take the item's key tiles in turn, a query a thread: S from
//               TMEM, mask, running maximum, P = 2^(S - m + 7) back into TMEM over S; each
//               set has its own accumulator, maximum and sum;
//   warps 8-14  codes and scales from memory, a quarter of a tile ahead in registers, into the operand images;
//   warp 15     issues the products.
// Every value that codes stand for is finite, so that what a row does not see needs no care
// beyond a weight of 0.
//
// Bound by the tiles' coming: a tile (128 keys and values, 18 KB) takes an SM 1.5 us beside bf16 queries, 1.8 beside 32-bit
// ones, whose products alone are 1.1; memory would bring one in 0.4.  448 queries of 28 / 4 heads of 128 over 60000
// entries, us on the device with 5 / 6 / 7 loading warps: bf16 97.6 / 86.6 / 84.3, 32-bit 109 / 100.5 / 99.1 (four, each
// with a quarter of every tile and the next tile's in registers: 85.6 / 105.8).  A sixteenth of a tile at a time, with
// a fence each: 133 / 145.  16 requests of 3 to 17 rows over 376 .. 7495, 32-bit: 37.9.
#include <algorithm>

#include "cache4.cuh"
#include "ptx_sm100.cuh"
#include "tree_dev.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 512, kLoaders = 7, kIssuer = 15;  // warps 8 .. 14 load, kIssuer issues
constexpr float kLazy = 8.f, kUp = 7.f;
// References from here on (base 2) are rounded by a half and more (exponent_of), as they are less kUp; below, weights
// stay within 2^15.75.
constexpr float kFar = 8388608.f;
// What turning to another item costs a CTA, in tiles.  us on the device with 2 / 3 / 4 / 5: 16 requests of 126 32-bit queries
// over 500 entries 18.6 / 20.1 / 20.6 / 23.7, over 4000 43.2 / 41.2 / 42.7 / 43.0, the ragged ones 41.4 / 37.9 / 38.3 / 39.4.
constexpr int kTurn = 3;

template <int D, bool F32>
struct Shape {
  static constexpr uint32_t STAGE = 128 * D * 2;
  static constexpr uint32_t Q = (F32 ? 2 : 1) * STAGE;
  static constexpr int NST = 4;
  static_assert(128u * D * (F32 ? 4 : 2) <= NST * STAGE, "queries in the ring");
  static constexpr uint32_t SMEM = 1024 + Q + NST * STAGE + 128 * 4 + 2 * 128 * 8 + (2 * NST + 6) * 8 + 16;
  static_assert(SMEM + sizeof(UnitPlan) + sizeof(First) + sizeof(Unit) <= 232448, "shared memory of one CTA");
};

// f16 A and B, fp32 accumulator.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn_major = false) {
  return ptx::idesc_bf16_f32(M, N, b_mn_major) & ~((1u << 7) | (1u << 10));
}

__device__ __forceinline__ uint32_t halves(float a, float b) {
  const __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ float2 floats_of(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// A piece of 32 dims of a key or value: its codes and two scales.
struct Piece {
  uint4 w;
  uint32_t s;
};
// Pieces of a tile of keys (or values): D / 32 a row.
template <int D>
__device__ __forceinline__ void load_piece(const uint8_t* codes, const uint8_t* scales, size_t row, int part, Piece& p) {
  p.w = __ldcs(reinterpret_cast<const uint4*>(codes + row * (D / 2)) + part);
  p.s = __ldcs(reinterpret_cast<const uint16_t*>(scales + row * (D / 16)) + part);
}
// Into the operand image of a tile: 128-byte-swizzled rows of halves.
template <int D>
__device__ __forceinline__ void put_piece(uint8_t* img, int row, int part, const Piece& p) {
  const uint32_t w[4] = {p.w.x, p.w.y, p.w.z, p.w.w};
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const __half2 s = scale_pair(__byte_perm(p.s, 0, b ? 0x4141 : 0x4040)), sh = scale_shift(s);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      __half2 v[4];
      decode_word(w[2 * b + c], s, sh, v);
      *reinterpret_cast<uint4*>(img + chunk_off(row, 4 * part + 2 * b + c)) = *reinterpret_cast<const uint4*>(v);
    }
  }
}

// Query n of warp w: four and four.
__device__ __forceinline__ int query_of(int w, int n) { return kThreads / 8 * (n >> 2) + 4 * w + (n & 3); }

// A warp's queries of an item as they are in memory, into shared memory.
template <int D, bool F32>
__device__ __forceinline__ void stage_queries(const TreeArgs& a, const Unit& it, int w, int end, int lane, uint8_t* to) {
  constexpr int ROW = D * (F32 ? 4 : 2), PIECES = ROW / 16;
  const int G = a.nq / a.nkv;
#pragma unroll 1
  for (int x = lane, row; (row = query_of(w, x / PIECES)) < end; x += 32) {
    const int q = it.qt * 128 + row, i = divide_group(a, q), h = it.g * G + (q - i * G);
    const int64_t at = (it.r0 + i) * a.q_stride + (int64_t)h * D;
    ptx::cp_async16(to + row * ROW + x % PIECES * 16, (const uint8_t*)a.q + at * (F32 ? 4 : 2) + x % PIECES * 16);
  }
  ptx::cp_async_wait_all();
  __syncwarp();
}

// Four queries (of which those below `end` are there) into the operand image(s), by a warp, eight
// lanes to a query: halves times a power of two that brings the largest dim to 2^14 .. 2^15, and
// what its scores are to be multiplied by.
template <int D, bool F32>
__device__ __forceinline__ void put_queries(const TreeArgs& a, const uint8_t* staged, int row, int end, int lane, uint8_t* img, float* back) {
  constexpr int N = F32 ? 4 : 8, PIECES = D / N / 8;  // dims of a piece of 16 bytes, a lane's pieces
  const int c = lane & 7;
  float x[PIECES][N];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const uint4 v = reinterpret_cast<const uint4*>(staged + row * D * (F32 ? 4 : 2))[c + 8 * p];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < N; ++e)
      x[p][e] = __uint_as_float(F32 ? w[e % 4] : e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  float most = 0.f, zero = 0.f;  // 0 times every dim: NaN if one is not finite
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      most = fmaxf(most, fabsf(x[p][e]));
      zero = fmaf(x[p][e], 0.f, zero);
    }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
  if ((__ballot_sync(~0u, zero != zero) >> (lane & 24)) & 0xFFu) zero = __uint_as_float(0x7FFFFFFFu);
  if (row >= end) return;
  // 2^up in two factors, as up may be 163
  const int up = most > 0.f && zero == 0.f ? 14 - ilogbf(most) : 0;
  const int u0 = up / 2, u1 = up - u0;
  const float f0 = __uint_as_float((uint32_t)(127 + u0) << 23), f1 = __uint_as_float((uint32_t)(127 + u1) << 23);
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    uint32_t hi[N / 2], lo[N / 2];
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const float y0 = x[p][2 * e] * f0 * f1 + zero, y1 = x[p][2 * e + 1] * f0 * f1 + zero;
      hi[e] = halves(y0, y1);
      const float2 r = floats_of(hi[e]);
      lo[e] = halves(y0 - r.x, y1 - r.y);
    }
    const int dim = (c + 8 * p) * N;
    uint8_t* to = img + chunk_off(row, dim / 8) + dim % 8 * 2;
    if constexpr (F32) {
      *reinterpret_cast<uint2*>(to) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint2*>(to + 128 * D * 2) = make_uint2(lo[0], lo[1]);
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    }
  }
  const float b = a.scale_log2 * __uint_as_float((uint32_t)(127 - u0) << 23) * __uint_as_float((uint32_t)(127 - u1) << 23);
  if (c == 0) back[row] = fminf(fmaxf(b, 1e-37f), 3.4e38f);  // (0 or infinity times a score of none: NaN)
}

template <bool F32>
__device__ __forceinline__ void write16(const TreeArgs& a, const float (&x)[16], float inv, size_t at) {
  if constexpr (F32) {
    float* out = (float*)a.out + at;
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<float4*>(out + e) = make_float4(x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = pack2(x[2 * e] * inv, x[2 * e + 1] * inv);
    uint4* out = reinterpret_cast<uint4*>((bf16*)a.out + at);
    out[0] = make_uint4(w[0], w[1], w[2], w[3]);
    out[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

template <int D, bool F32>
__global__ void __launch_bounds__(kThreads, 1)
    wide4_kernel(const __grid_constant__ Tree4Args a4, TreeWork ws, int turn) {
  using S = Shape<D, F32>;
  constexpr int NST = S::NST, PARTS = D / 32, MINE = PARTS;  // pieces of a row; a lane's of a quarter of a tile (of keys or values)
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* qimg = sm;
  uint8_t* ring = sm + S::Q;
  float2* s_ml = reinterpret_cast<float2*>(ring + NST * S::STAGE);  // [2 sets][128]
  float* s_back = reinterpret_cast<float*>(s_ml + 2 * 128);         // [128]
  uint64_t* full = reinterpret_cast<uint64_t*>(s_back + 128);
  uint64_t* empty = full + NST;
  uint64_t* s_full = empty + NST;  // [2]
  uint64_t* p_full = s_full + 2;   // [2]
  uint64_t* o_full = p_full + 2;
  uint64_t* drain = o_full + 1;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(drain + 1);
  __shared__ UnitPlan s_plan;
  __shared__ First s_first;
  __shared__ Unit s_next;
  const TreeArgs& a = a4.t;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      ptx::mbar_init(&full[i], 4);
      ptx::mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&s_full[i], 1);
      ptx::mbar_init(&p_full[i], 4);
    }
    ptx::mbar_init(o_full, 1);
    ptx::mbar_init(drain, 1);
    ptx::fence_mbar_init();
  }
  if (warp == kIssuer) ptx::tmem_alloc(tslot, 512);
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  if (warp == 0) {
    make_plan(a, 128, turn, lane, s_plan, blockIdx.x == 0);
    first_item(s_plan, a, blockIdx.x, gridDim.x, lane, s_first);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tslot;
  Unit it = s_first.it;
  const int u1 = s_first.u1, G = a.nq / a.nkv;
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
  uint32_t n = 0;                        // tiles (of keys or values) of the ring so far
  uint32_t turns = 0, p_turn = 0, items = 0;  // a set's key tiles so far, p_full's parities, items
  bool more = it.rows > 0;
  while (more) {
    const int cnt = it.t1 - it.t0, end = it.L + it.rows, queries = it.rows * G - it.qt * 128;
    const size_t head = ((size_t)it.b * a.nkv + it.g) * a.cap;
    // Quarters of the item's tiles, of keys and of values in turn, go round the loaders.  (Seven to four: a warp's next
    // quarter is at most two tiles of the ring on, so that the wait for the stage's last use is never for a phase
    // before the one that runs.)
    const int quarters = 8 * cnt;
    Piece next[MINE];
    auto fetch = [&](int g) {
      const uint8_t *codes = g & 4 ? a4.v : a4.k, *scales = g & 4 ? a4.vs : a4.ks;
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        const int piece = (g & 3) * 32 * MINE + x * 32 + lane, row = min((it.t0 + g / 8) * 128 + piece / PARTS, end - 1);
        load_piece<D>(codes, scales, head + row, piece % PARTS, next[x]);
      }
    };
    if (warp >= 8 && warp < kIssuer && warp - 8 < quarters) fetch(warp - 8);
    // (all of a warp's queries on their way together, by the ring, which is empty)
    const int last = min(queries, 128);
    stage_queries<D, F32>(a, it, warp, last, lane, ring);
#pragma unroll 1
    for (int k = 0; query_of(warp, k) < last; k += 4) put_queries<D, F32>(a, ring, query_of(warp, k + lane / 8), last, lane, qimg, s_back);
    ptx::fence_proxy_async_smem();
    if (warp == kIssuer && lane == 0) {  // the item after this one
      Unit then;
      int u = it.next;
      if (!next_item(s_plan, a, u, u1, then)) then.rows = 0;
      s_next = then;
    }
    __syncthreads();
    if (warp == kIssuer) {
      // the whole warp, for operands in uniform registers; one thread issues
      const uint32_t lead = ptx::elect_one(), tm = __shfl_sync(~0u, tmem, 0);
      auto whole = [&](bool) { return ok = __all_sync(~0u, ok); };
      constexpr uint32_t IDESC1 = idesc_f16(128, 128), IDESC2 = idesc_f16(128, D, true);
      const uint32_t q_lo = ptx::desc_lo(ptx::smem_u32(qimg), 16u);
      for (int j = 0; j <= cnt && ok; ++j) {
        if (j < cnt) {
          const uint32_t m = n + 2 * j, s = m % NST;
          if (!whole(wait(&full[s], (m / NST) & 1))) break;
          ptx::tc_fence_after();
          const uint32_t kt = ptx::desc_lo(ptx::smem_u32(ring + s * S::STAGE), 16u), ds = tm + 128 * (j & 1);
          // (products run in the order of their issue: these scores come after the
          // product that reads the weights in their place)
          // (the small parts first: the products' sums are cut off, not rounded, so that each addition to a
          // large one costs up to 2^-23 of it; 32-bit queries' results over 7500 entries were off by 2.0e-6, 1.6e-6 so)
#pragma unroll
          for (int part = F32 ? 1 : 0; part >= 0; --part)
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t to = ((kk >> 2) * kRegion + 32u * (kk & 3)) >> 4;
              ptx::mma_bf16_lo(lead, ds, q_lo + to + part * (128u * D * 2 >> 4), kt + to, IDESC1,
                               kk > 0 || (F32 && part == 0) ? 1u : 0u);
            }
          ptx::mma_commit_if(lead, &s_full[j & 1]);
          ptx::mma_commit_if(lead, &empty[s]);
        }
        if (j > 0) {
          const uint32_t m = n + 2 * j - 1, s = m % NST, i = (j - 1) & 1;
          if (!whole(wait(&full[s], (m / NST) & 1)) || !whole(wait(&p_full[i], (p_turn >> i) & 1))) break;
          p_turn ^= 1u << i;
          ptx::tc_fence_after();
          const uint32_t vt = ptx::desc_lo(ptx::smem_u32(ring + s * S::STAGE), kRegion);
          const uint32_t ds = tm + 256 + 128 * i, ps = tm + 128 * i;
#pragma unroll
          for (int part = F32 ? 1 : 0; part >= 0; --part)
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              ptx::mma_bf16_ta_lo(lead, ds, ps + (F32 ? 16u : 8u) * kk + 8u * part, vt + 128u * kk, IDESC2,
                                  j > 2 || kk > 0 || (F32 && part == 0) ? 1u : 0u);
          ptx::mma_commit_if(lead, &empty[s]);
          if (j == cnt) ptx::mma_commit_if(lead, o_full);
        }
      }
    } else if (warp >= 8) {
#pragma unroll 1
      for (int g = warp - 8; g < quarters; g += kLoaders) {
        const uint32_t m = n + g / 4, s = m % NST;
        if (m >= NST) wait(&empty[s], (m / NST - 1) & 1);
        ok = __all_sync(~0u, ok);
        if (ok) {
#pragma unroll
          for (int x = 0; x < MINE; ++x) {
            const int piece = (g & 3) * 32 * MINE + x * 32 + lane;
            put_piece<D>(ring + s * S::STAGE, piece / PARTS, piece % PARTS, next[x]);
          }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[s]);
        if (g + kLoaders < quarters) fetch(g + kLoaders);
      }
    } else {
      const int set = warp >> 2, quad = warp & 3, row = 32 * quad + lane;  // query of the tile, TMEM lane
      const uint32_t tl = tmem + ((uint32_t)(32 * quad) << 16);
      const uint32_t ts = tl + 128 * set, to = tl + 256 + 128 * set;
      const bool live = row < queries, warp_live = 32 * quad < queries;
      const float c = live ? s_back[row] : 1.f;
      const int q = it.qt * 128 + row, i = divide_group(a, q), h = it.g * G + (q - i * G);
      uint64_t vis = 0;
      if (live && it.t1 > it.L / 128) vis = visible_rows(a, it.r0 + i, i, it.rows);
      float ref = -INFINITY, l = 0.f;  // the reference, a score
#pragma unroll 1
      for (int j = set; j < cnt; j += 2, ++turns) {
        wait(&s_full[set], turns & 1);
        ok = __all_sync(~0u, ok);
        // (a warp without a query leaves what it has in the place of P: it reaches
        // the accumulators of rows that are not read)
        if (warp_live) {
          ptx::tc_fence_after();
          const int p0 = (it.t0 + j) * 128;
          const bool tail = p0 + 128 > it.L;
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
          for (int x = 0; x < 128; x += 32) {
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
          const float top = fmaxf(mx[0], mx[1]), mt = __fmul_rn(top, c);
          float m = __fmul_rn(ref, c);
          // (NaN scores pass the maximum by, and reach the sums; beside a far reference nothing greater is left)
          const bool grow = mt > m + kLazy || (fmaxf(fabsf(m), fabsf(mt)) >= kFar && mt > -INFINITY && top > ref);
          if (__any_sync(~0u, grow)) {
            const float m_new = grow ? mt : m, f = m == -INFINITY ? 0.f : ex2(m - m_new);
            l = grow ? l * f : l;
            if (j >= 2) {
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
          }
          const Exponent x2 = exponent_of([&] { return ref; }, m, c, kFar);
          const float at = x2.at - kUp;
          const uint64_t c2 = two(x2.by, x2.by), ref2 = two(-at, -at);
          uint64_t ls[2] = {0, 0};
          // P: of each 16 keys the weights' first parts, then the second ones
#pragma unroll 1
          for (int x = 0; x < 128; x += 32) {
            uint32_t v[32], p[F32 ? 32 : 16];
            ptx::tmem_ld32(ts + x, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 y = of_two(fma2(two(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), c2, ref2));
              const uint64_t w = two(ex2(y.x), ex2(y.y));
              ls[e & 1] = add2(ls[e & 1], w);
              const float2 f = of_two(w);
              const uint32_t hi = halves(f.x, f.y);
              if constexpr (F32) {
                const float2 r = floats_of(hi);
                p[(e & 8) * 2 + (e & 7)] = hi;
                p[(e & 8) * 2 + (e & 7) + 8] = halves(f.x - r.x, f.y - r.y);
              } else {
                p[e] = hi;
              }
            }
            if constexpr (F32) {
              ptx::tmem_st16(ts + x, p);
              ptx::tmem_st16(ts + x + 16, p + 16);
            } else {
              ptx::tmem_st16(ts + x / 2, p);
            }
          }
          const float2 sums = of_two(add2(ls[0], ls[1]));
          l += sums.x + sums.y;
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[set]);
      }
      // ---- the item's end: the two sets' parts, each set half of the dims ----
      wait(o_full, items & 1);
      ok = __all_sync(~0u, ok);
      ptx::tc_fence_after();
      s_ml[set * 128 + row] = make_float2(__fmul_rn(ref, c) - kUp, l);  // (what the sum is relative to)
      ptx::named_bar_sync(1, 256);
      const float m0 = s_ml[row].x, m1 = s_ml[128 + row].x;
      const float M = fmaxf(m0, m1), w0 = part_weight(m0, M), w1 = part_weight(m1, M);
      const float lt = fmaf(s_ml[row].y, w0, s_ml[128 + row].y * w1);  // (a NaN stays)
      const bool done = it.t0 == 0 && it.t1 == it.tiles;
      const size_t part = (size_t)blockIdx.x * 2 + (it.t0 > 0 ? 0 : 1);
      const float inv = lt == 0.f ? 0.f : 1.f / lt;
      if (ok && warp_live) {
#pragma unroll 1
        for (int d0 = set * (D / 2); d0 < (set + 1) * (D / 2); d0 += 16) {
          uint32_t o0[16], o1[16];
          ptx::tmem_ld16(tl + 256 + d0, o0);
          if (cnt > 1) ptx::tmem_ld16(tl + 384 + d0, o1);
          ptx::tmem_ld_wait();
          float o[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            o[e] = __uint_as_float(o0[e]) * w0;
            if (cnt > 1) o[e] = fmaf(__uint_as_float(o1[e]), w1, o[e]);
          }
          if (live && !done) {
            float4* dst = ws.o + (part * (D / 4) + d0 / 4) * 128 + row;
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[e * 128] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          } else if (live) {
            write16<F32>(a, o, inv, ((size_t)(it.r0 + i) * a.nq + h) * D + d0);
          }
          __syncwarp();
        }
        if (live && set == 0) {
          if (!done)
            ws.ml[part * 128 + row] = make_float2(M, lt);
          else if (a.lse)
            a.lse[(size_t)(it.r0 + i) * a.nq + h] = row_lse(M, lt);
        }
      }
      ptx::tc_fence_before();
    }
    n += 2 * cnt;
    ++items;
    const Unit then = s_next;
    __syncthreads();
    ptx::tc_fence_after();
    it = then;
    more = it.rows > 0;
  }
  if (warp == kIssuer) {
    // no product is running when TMEM is freed
    ptx::mma_commit_if(ptx::elect_one(), drain);
    ptx::mbar_wait(drain, 0, ptx::kDrainNs);
  }
  __syncthreads();
  if (warp == kIssuer) ptx::tmem_dealloc(tmem, 512);
}

template <int D, bool F32>
cudaError_t launch(const Tree4Args& a4, const TreeWork& ws, int64_t max_keys, cudaStream_t st) {
  using S = Shape<D, F32>;
  static PerDevice opted;
  cudaError_t e = opt_in(opted, wide4_kernel<D, F32>, S::SMEM);
  if (e != cudaSuccess) return e;
  const int64_t items = tree_items(a4.t), tiles = (max_keys + 127) / 128, units = items * tiles;
  const int sms = device_sms();
  // no more CTAs to an item than pay for the joining of their parts
  const int ctas = (int)std::min(std::min<int64_t>(units, sms), items * (16 + tiles / 8));
  const int turn = units > sms ? kTurn : 0;
  e = launch_pdl(wide4_kernel<D, F32>, dim3(ctas), dim3(kThreads), S::SMEM, st, 1, a4, ws, turn);
  if (e != cudaSuccess) return e;
  return launch_tree_join(a4.t, D, ws, ctas, turn, st);
}

}  // namespace

cudaError_t launch_attention4_wide(const Tree4Args& a, int head_dim, int64_t max_keys, void* workspace, cudaStream_t st) {
  const TreeWork ws = tree_work(workspace, head_dim);
  if (head_dim == 128) return a.t.q_f32 ? launch<128, true>(a, ws, max_keys, st) : launch<128, false>(a, ws, max_keys, st);
  return a.t.q_f32 ? launch<64, true>(a, ws, max_keys, st) : launch<64, false>(a, ws, max_keys, st);
}

}  // namespace as2d
