// k_attn4.cu -- attention of a tree of drafted tokens over a cache in 4 bits
// (as2d_cache4_attention).
//
// With s_t = scale q k_t over the entries that a row sees (as k_tree_attn.cu):
//   m = max s_t, l = sum e^(s_t - m), out = sum e^(s_t - m) v_t / l, lse = m + ln l.
//
// The G = n_q / n_kv query heads of a kv head, for all rows of a request, form one query matrix,
// cut into tiles of 8 or 16; a unit is such a tile and 128 keys.  Units are spread over
// one or two CTAs per SM in even shares, or one request's items over the same number of CTAs each, and the
// parts joined by join4_kernel.  (Many queries: k_attn4_wide.cu.)
//
// Per CTA: eight warps, 16 keys of a tile each, with a ring of copies of their own and no barrier between
// them until the item's end.  The keys are the rows of the product (S^T = K Q^T, out^T = V^T P^T), so
// that 8 queries fill its columns: on tcgen05 a tile of 128 rows would be 7 of one token's queries, and codes
// would go through shared memory twice.  Codes become 16-bit floats in registers, exactly, on their way into
// mma.sync.  Queries are 16-bit floats times a power of two of their own: bf16 ones exactly (but for dims below 2^-31 of
// the largest), 32-bit ones in two parts, to 2^-22.  Weights beside bf16 queries are one 16-bit
// float, off by at most 2^-11 where the result's own rounding is off by 2^-8, beside 32-bit ones two.
//
// Bound, one row of 28 / 4 heads of 128 (floor: the cache's 4.5 bits a value, read once): over 15128 entries (1.3 us)
// by latency, 9.1 us on the device, of which one over 200 takes 5.1.  Over 60000 (5.1) 17.1, and 16 requests over
// 376 .. 7495 (5.2) 20.2: 0.75 us a tile on an SM whether it has one CTA or two.  Of the issue slots 52 % are used
// while it runs, of the pipe for whole numbers some 45 %: the 90 operations on bits and 96 on pairs of halves that decode a
// warp's 16 keys and values.  (Addresses kept in registers from tile to tile: 1 % less.)
#include <algorithm>

#include "cache4.cuh"
#include "ptx_sm100.cuh"
#include "tree_dev.cuh"

namespace as2d {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
// P may grow to less than 2^kLazy of its reference before sums are rescaled; a reference stands for 2^kUp
// (the weights, less than 2^(kLazy + kUp), use the range of 16-bit floats; where a score's last place is 2 or 4
// that is 2^14 or less beside a reference for 2^8, as scores of 2^kLazy more do not stay).
constexpr float kLazy = 8.f, kUp = 7.f;

// Queries of the partial results of an SM's CTAs: two of 8, or one of 16, two parts each.
constexpr int kParts = 2 * 16;

// What turning to another item costs a CTA, in tiles: its queries, the joining of its warps. us on the device with
// 3 / 4 / 5 / 8: 16 requests of one row over 376 .. 7495 entries 19.2 / 20.2 / 20.5 / 21.4, over 4000 19.3 / 19.9 /
// 19.7 / 20.0, 64 over 2000 30.3 / 30.4 / 30.4 / 30.5; with none the first 26 where 3 gave 21.
constexpr int kTurn = 4;

// How the items go over the CTAs: even shares of all units, or the same number of CTAs to each item.
enum Mode : int { kShares = 0, kDirect = 1 };

struct Work {
  float2* o;   // [2 CTAs][pairs of dims][32 lanes]
  float2* ml;  // [2 CTAs][queries] (reference base 2, sum)
};

// A query tile's operands: as halves times a power of two of the query's own, which brings its
// largest dim to 2^14 .. 2^15, in the order of the product's fragments (lane 4 g + t has dims D / 4
// t .. of query 8 nt + g); back: what scores are to be multiplied by.
template <int D, int NT, bool F32>
struct QueryTile {
  uint4 hi[NT][D / 32][32], lo[F32 ? NT : 1][F32 ? D / 32 : 1][32];
  float back[8 * NT];
};

template <int D, int NT, bool F32>
struct Shape {
  static constexpr int Q = 8 * NT;                         // queries of a tile
  static constexpr int CODES = 16 * D / 2, SCALES = D;     // bytes of a warp's 16 keys (or values)
  static constexpr int STAGE = 2 * (CODES + SCALES);
  static constexpr int CTAS = NT == 1 ? 2 : 1;             // of an SM
  static constexpr int NST = CTAS == 2 ? 5 : 10;
  static constexpr int RING = kWarps * NST * STAGE;
  static constexpr int PAIRS = D / 16 * NT * 2;            // of dims, a lane
  static constexpr int PARTS = kWarps * PAIRS * 32 * 8;
  static constexpr int AREA = RING > PARTS ? RING : PARTS;
  static constexpr int SMEM = AREA + sizeof(QueryTile<D, NT, F32>);
};

__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // 8 x 8 of 16 bits
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t halves(float a, float b) {
  const __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ uint32_t as_u32(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }

template <int N>
__device__ __forceinline__ void cp_async(void* dst, const void* src) {
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(__cvta_generic_to_global(src)) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(ptx::smem_u32(dst)), "l"(__cvta_generic_to_global(src)), "n"(N) : "memory");
}

// A value's 16-byte pieces: those that lanes of one g read together (rows 4t) lie in other banks.
__device__ __forceinline__ int value_off(int off, int row) { return off ^ (((row >> 2) & 3) << 5); }

// A warp's 16 keys and values from entry p on into a stage; entries from `end` on are
// copies of the last one (and masked).
template <int D>
__device__ __forceinline__ void load_slice(const Tree4Args& a, size_t head, int p, int end, int lane, uint8_t* to) {
  constexpr int ROW = D / 2, PIECES = ROW / 16, CODES = 16 * ROW, S = D / 16;
  const int last = end - 1 - p;  // of the slice
  const size_t at = head + p;
  const uint8_t *k = a.k + at * ROW, *v = a.v + at * ROW;
#pragma unroll
  for (int i = 0; i < PIECES / 2; ++i) {
    const int x = lane + 32 * i, row = x / PIECES, off = x % PIECES * 16;
    const int from = min(row, last) * ROW + off;
    cp_async<16>(to + row * ROW + off, k + from);
    cp_async<16>(to + CODES + value_off(row * ROW + off, row), v + from);
  }
  cp_async<S>(to + 2 * CODES + lane * S, (lane < 16 ? a.ks : a.vs) + at * S + min(lane & 15, last) * S);
}

// By the whole block.
template <int D, int NT, bool F32>
__device__ __forceinline__ void load_queries4(const TreeArgs& a, const Unit& it, int warp, int lane,
                                              QueryTile<D, NT, F32>& to) {
  constexpr int N = D / 32;  // dims of a lane
  const int G = a.nq / a.nkv;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int q = it.qt * 8 * NT + 8 * nt + warp;
    float x[N] = {};
    if (q < it.rows * G) {
      const int i = divide_group(a, q), h = it.g * G + (q - i * G);
      const int64_t at = (it.r0 + i) * a.q_stride + (int64_t)h * D + N * lane;
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const float2 v = *reinterpret_cast<const float2*>((const float*)a.q + at + e);
          x[e] = v.x, x[e + 1] = v.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>((const bf16*)a.q + at + e);
          x[e] = __uint_as_float(w << 16);
          x[e + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
      }
    }
    float most = 0.f, zero = 0.f;  // 0 times every dim: NaN if one is not finite
#pragma unroll
    for (int e = 0; e < N; ++e) {
      most = fmaxf(most, fabsf(x[e]));
      zero = fmaf(x[e], 0.f, zero);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    if (__any_sync(~0u, zero != zero)) zero = __uint_as_float(0x7FFFFFFFu);
    // 2^up in two factors, as up may be 163
    const int up = most > 0.f && zero == 0.f ? 14 - ilogbf(most) : 0;
    const int u0 = up / 2, u1 = up - u0;
    const float f0 = __uint_as_float((uint32_t)(127 + u0) << 23), f1 = __uint_as_float((uint32_t)(127 + u1) << 23);
    const int t = lane >> 3, e0 = lane * N % (D / 4) / 2;  // of the lane that has these dims, its pair
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const float y0 = x[2 * e] * f0 * f1 + zero, y1 = x[2 * e + 1] * f0 * f1 + zero;
      const uint32_t h = halves(y0, y1);
      reinterpret_cast<uint32_t*>(&to.hi[nt][(e0 + e) / 4][4 * warp + t])[(e0 + e) % 4] = h;
      if constexpr (F32) {
        const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&h));
        reinterpret_cast<uint32_t*>(&to.lo[nt][(e0 + e) / 4][4 * warp + t])[(e0 + e) % 4] = halves(y0 - r.x, y1 - r.y);
      }
    }
    if (lane == 0)
      to.back[8 * nt + warp] = fminf(a.scale_log2 * __uint_as_float((uint32_t)(127 - u0) << 23) *
                                         __uint_as_float((uint32_t)(127 - u1) << 23), 3.4e38f);
  }
}

// What a warp has of its queries: maxima (references, base 2) and sums of queries 8 nt + 2 t and + 1 (a
// lane's keys), and its dims of the accumulator.
template <int D, int NT>
struct Sums {
  float m[NT][2], l[NT][2];
  float o[NT][D / 16][4];
};

// Scores of 16 keys of a stage: s[nt][2 r + e] of key k0 + 2 r and query 8 nt + 2 t + e.
template <int D, int NT, bool F32>
__device__ __forceinline__ void scores(const uint8_t* st, int lane, const uint32_t (&qh)[NT][D / 8],
                                       const uint32_t (&ql)[F32 ? NT : 1][D / 8], const float (&back)[NT][2],
                                       float (&s)[NT][4]) {
  constexpr int ROW = D / 2, CODES = 16 * ROW, S = D / 16;
  const int g = lane >> 2, t = lane & 3;
  // the rows g and g + 8 of the product are keys k0 and k0 + 2 of the 16
  const int k0 = 4 * (g >> 1) + (g & 1);
  float s2[NT][4];  // (two chains of products)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[nt][e] = s2[nt][e] = 0.f;
  uint32_t w[2][D / 32], sb[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const uint8_t* row = st + (k0 + 2 * r) * ROW + t * (ROW / 4);
    const uint8_t* sc = st + 2 * CODES + (k0 + 2 * r) * S;
    if constexpr (D == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(row);
      w[r][0] = v.x, w[r][1] = v.y, w[r][2] = v.z, w[r][3] = v.w;
      sb[r] = *reinterpret_cast<const uint16_t*>(sc + 2 * t);
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(row);
      w[r][0] = v.x, w[r][1] = v.y;
      sb[r] = sc[t];
    }
  }
#pragma unroll
  for (int b = 0; b < D / 64; ++b) {  // 16 dims of a lane, a scale
    __half2 sc[2], sh[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      sc[r] = scale_pair(__byte_perm(sb[r], 0, b ? 0x4141 : 0x4040));
      sh[r] = scale_shift(sc[r]);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      __half2 v0[4], v1[4];
      decode_word(w[0][2 * b + c], sc[0], sh[0], v0);
      decode_word(w[1][2 * b + c], sc[1], sh[1], v1);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t f[4] = {as_u32(v0[2 * k]), as_u32(v1[2 * k]), as_u32(v0[2 * k + 1]), as_u32(v1[2 * k + 1])};
        const int at = 8 * b + 4 * c + 2 * k;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma16(k ? s2[nt] : s[nt], f, qh[nt][at], qh[nt][at + 1]);
          if constexpr (F32) mma16(k ? s[nt] : s2[nt], f, ql[nt][at], ql[nt][at + 1]);
        }
      }
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[nt][e] = (s[nt][e] + s2[nt][e]) * back[nt][e & 1];
}

// What is not seen of 16 keys from entry p on (`stop`: the request's end) gets a score of -inf.
template <int NT>
__device__ __forceinline__ void mask_slice(const TreeArgs& a, const Unit& it, int p, int stop, int lane, float (&s)[NT][4]) {
  const int g = lane >> 2, t = lane & 3, k0 = 4 * (g >> 1) + (g & 1);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int q = it.qt * 8 * NT + 8 * nt + 2 * t + e, i = min(divide_group(a, q), it.rows - 1);
      const uint64_t vis = visible_rows(a, it.r0 + i, i, it.rows);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int at = p + k0 + 2 * r, rel = at - it.L;
        if (at >= stop || (rel >= 0 && !((vis >> rel) & 1))) s[nt][2 * r + e] = -INFINITY;
      }
    }
}

// The weights of a slice's scores, as operands of its second product, and their sums.
template <int D, int NT, bool F32>
__device__ __forceinline__ void weights_of(const float (&s)[NT][4], Sums<D, NT>& x, uint32_t (&ph)[NT][2],
                                           uint32_t (&pl)[F32 ? NT : 1][2]) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float w4[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float m = x.m[nt][e & 1];
      w4[e] = ex2(s[nt][e] - ((m == -INFINITY ? 0.f : m) - kUp));
    }
    x.l[nt][0] += w4[0] + w4[2];
    x.l[nt][1] += w4[1] + w4[3];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint32_t h = halves(w4[2 * r], w4[2 * r + 1]);
      ph[nt][r] = transposed(h);
      if constexpr (F32) {
        const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&h));
        pl[nt][r] = transposed(halves(w4[2 * r] - y.x, w4[2 * r + 1] - y.y));
      }
    }
  }
}

// A slice's values into the accumulators: rows g and g + 8 of the products are dims D / 8 g + 2 mt and + 1.
template <int D, int NT, bool F32>
__device__ __forceinline__ void add_values(const uint8_t* st, int lane, const uint32_t (&ph)[NT][2],
                                           const uint32_t (&pl)[F32 ? NT : 1][2], Sums<D, NT>& x) {
  constexpr int ROW = D / 2, CODES = 16 * ROW, S = D / 16;
  const int g = lane >> 2, t = lane & 3;
  uint32_t vw[4][D / 64], vb[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = 4 * t + r;
    const uint8_t* at = st + CODES + value_off(row * ROW + g * (D / 16), row);
    if constexpr (D == 128) {
      const uint2 v = *reinterpret_cast<const uint2*>(at);
      vw[r][0] = v.x, vw[r][1] = v.y;
    } else {
      vw[r][0] = *reinterpret_cast<const uint32_t*>(at);
    }
    vb[r] = st[2 * CODES + 16 * S + row * S + (D == 128 ? g : g >> 1)];
  }
  const __half2 s0 = scale_pair(vb[0] | vb[1] << 16), s1 = scale_pair(vb[2] | vb[3] << 16);
  const __half2 h0 = scale_shift(s0), h1 = scale_shift(s1);
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    __half2 v[4][4];  // keys 0 and 1: even dims, odd dims; keys 2 and 3
    decode_word(__byte_perm(vw[0][c], vw[1][c], 0x5410), s0, h0, v[0]);
    decode_word(__byte_perm(vw[0][c], vw[1][c], 0x7632), s0, h0, v[1]);
    decode_word(__byte_perm(vw[2][c], vw[3][c], 0x5410), s1, h1, v[2]);
    decode_word(__byte_perm(vw[2][c], vw[3][c], 0x7632), s1, h1, v[3]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t f[4] = {as_u32(v[0][e]), as_u32(v[1][e]), as_u32(v[2][e]), as_u32(v[3][e])};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma16(x.o[nt][4 * c + e], f, ph[nt][0], ph[nt][1]);
        if constexpr (F32) mma16(x.o[nt][4 * c + e], f, pl[nt][0], pl[nt][1]);
      }
    }
  }
}

// 16 keys of a stage: entries p .. of the item.
template <int D, int NT, bool F32>
__device__ __forceinline__ void attend(const TreeArgs& a, const Unit& it, const uint8_t* st, int p, int stop, int lane, const uint32_t (&qh)[NT][D / 8],
                                       const uint32_t (&ql)[F32 ? NT : 1][D / 8], const float (&back)[NT][2],
                                       Sums<D, NT>& x) {
  float s[NT][4];
  scores<D, NT, F32>(st, lane, qh, ql, back, s);
  if (p + 16 > it.L) mask_slice<NT>(a, it, p, stop, lane, s);
  float most[NT][2];
  bool grow = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      most[nt][e] = fmaxf(s[nt][e], s[nt][2 + e]);
      grow = grow || most[nt][e] - x.m[nt][e] >= kLazy;
    }
  if (__any_sync(~0u, grow)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float now = most[nt][e];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) now = fmaxf(now, __shfl_xor_sync(~0u, now, o));
        const float m = x.m[nt][e];
        if (now - m >= kLazy) {
          const float f = m == -INFINITY ? 0.f : ex2(m - now);
          x.m[nt][e] = now;
          x.l[nt][e] *= f;
#pragma unroll
          for (int mt = 0; mt < D / 16; ++mt) {
            x.o[nt][mt][e] *= f;
            x.o[nt][mt][2 + e] *= f;
          }
        }
      }
  }
  uint32_t ph[NT][2], pl[F32 ? NT : 1][2];
  weights_of<D, NT, F32>(s, x, ph, pl);
  add_values<D, NT, F32>(st, lane, ph, pl, x);
}

// Two dims of a query: 32-bit or bf16.
template <bool F32>
__device__ __forceinline__ void write_pair(const TreeArgs& a, float2 x, size_t at) {
  if constexpr (F32)
    *reinterpret_cast<float2*>((float*)a.out + at) = x;
  else
    *reinterpret_cast<uint32_t*>((bf16*)a.out + at) = pack2(x.x, x.y);
}

// Result of a lane's pair of dims (as Sums): its query of the tile and first dim.
template <int D>
__device__ __forceinline__ void place_of(int pair, int lane, int& query, int& dim) {
  const int e = pair & 1, mt = (pair >> 1) % (D / 16), nt = (pair >> 1) / (D / 16);
  query = 8 * nt + 2 * (lane & 3) + e;
  dim = (lane >> 2) * (D / 8) + 2 * mt;
}

template <int D, int NT, bool F32>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1)
    attn4_kernel(const __grid_constant__ Tree4Args a4, Work ws, int mode, int turn) {  // (kDirect: turn CTAs to an item)
  using S = Shape<D, NT, F32>;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ UnitPlan s_plan;
  __shared__ First s_first;
  const TreeArgs& a = a4.t;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* ring = smem + warp * S::NST * S::STAGE;
  float2* s_o = reinterpret_cast<float2*>(smem);                                  // [warp][pair][lane]
  auto& s_q = *reinterpret_cast<QueryTile<D, NT, F32>*>(smem + S::AREA);
  __shared__ float s_m[kWarps][S::Q], s_l[kWarps][S::Q];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  Unit it;
  int u1 = 0;
  const size_t block = ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
  if (mode == kDirect) {
    const int p = blockIdx.x % turn;
    it.b = blockIdx.z, it.g = blockIdx.y, it.qt = blockIdx.x / turn;
    it.r0 = a.rm.start[it.b];
    it.rows = a.rm.start[it.b + 1] - it.r0;
    it.L = a.len[it.b];
    const bool some = it.qt * S::Q < it.rows * (a.nq / a.nkv), fits = rows_fit(it.L, it.rows, a.cap);
    if (some && !fits && tid == 0 && a.err) atomicOr(a.err, kErrCapacity);
    it.tiles = some && fits ? (it.L + it.rows + 127) / 128 : 0;
    it.t0 = it.tiles * p / turn;
    it.t1 = it.tiles * (p + 1) / turn;
    if (it.t0 == it.t1) {  // (a part of fewer tiles than parts)
      if (turn > 1 && tid < S::Q) ws.ml[block * S::Q + tid] = make_float2(-INFINITY, 0.f);
      return;
    }
  } else {
    if (warp == 0) {
      make_plan(a, S::Q, turn, lane, s_plan, blockIdx.x == 0);
      first_item(s_plan, a, blockIdx.x, gridDim.x, lane, s_first);
    }
    __syncthreads();
    it = s_first.it, u1 = s_first.u1;
    if (it.rows == 0) return;
  }
  const int G = a.nq / a.nkv;
  for (bool more = true; more;) {
    const int end = it.L + it.rows, n = it.t1 - it.t0;
    const size_t head = ((size_t)it.b * a.nkv + it.g) * a.cap;
    auto load = [&](int k) {
      if (k < n) load_slice<D>(a4, head, (it.t0 + k) * 128 + 16 * warp, end, lane, ring + k % S::NST * S::STAGE);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int k = 0; k < S::NST - 1; ++k) load(k);
    load_queries4<D, NT, F32>(a, it, warp, lane, s_q);
    __syncthreads();
    uint32_t qh[NT][D / 8], ql[F32 ? NT : 1][D / 8];
    float back[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const uint4 h = s_q.hi[nt][e][lane];
        qh[nt][4 * e] = h.x, qh[nt][4 * e + 1] = h.y, qh[nt][4 * e + 2] = h.z, qh[nt][4 * e + 3] = h.w;
        if constexpr (F32) {
          const uint4 l = s_q.lo[nt][e][lane];
          ql[nt][4 * e] = l.x, ql[nt][4 * e + 1] = l.y, ql[nt][4 * e + 2] = l.z, ql[nt][4 * e + 3] = l.w;
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) back[nt][e] = s_q.back[8 * nt + 2 * (lane & 3) + e];
    }
    Sums<D, NT> x;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      x.m[nt][0] = x.m[nt][1] = -INFINITY;
      x.l[nt][0] = x.l[nt][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) x.o[nt][mt][e] = 0.f;
    }
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S::NST - 2) : "memory");
      __syncwarp();
      const int p = (it.t0 + k) * 128 + 16 * warp;
      if (p < end) attend<D, NT, F32>(a, it, ring + k % S::NST * S::STAGE, p, end, lane, qh, ql, back, x);
      __syncwarp();
      load(k + S::NST - 1);
    }
    // ---- the warps' parts, brought to one reference, over the rings ----
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (lane < 4)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) s_m[warp][8 * nt + 2 * lane + e] = x.m[nt][e];
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int query = 8 * nt + 2 * (lane & 3) + e;
        float M = -INFINITY, l = x.l[nt][e];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w][query]);
        const float f = part_weight(x.m[nt][e], M);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(~0u, l, o);
        if (lane < 4) s_l[warp][query] = l * f;  // (a NaN stays)
#pragma unroll
        for (int mt = 0; mt < D / 16; ++mt)
          s_o[(warp * S::PAIRS + (nt * (D / 16) + mt) * 2 + e) * 32 + lane] =
              make_float2(x.o[nt][mt][e] * f, x.o[nt][mt][2 + e] * f);
      }
    __syncthreads();
    const bool done = mode == kDirect ? turn == 1 : it.t0 == 0 && it.t1 == it.tiles;
    const size_t part = mode == kDirect ? block : (size_t)blockIdx.x * 2 + (it.t0 > 0 ? 0 : 1);
    for (int j = tid; j < S::PAIRS * 32; j += kThreads) {
      int query, dim;
      place_of<D>(j / 32, lane, query, dim);
      const int q = it.qt * S::Q + query;
      if (q >= it.rows * G) continue;
      float l = 0.f;
      float2 o = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 v = s_o[w * S::PAIRS * 32 + j];
        l += s_l[w][query];
        o.x += v.x;
        o.y += v.y;
      }
      float M = -INFINITY;
      if (!done || dim == 0)
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w][query]);
      if (done) {
        const int i = divide_group(a, q), h = it.g * G + (q - i * G);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        write_pair<F32>(a, make_float2(o.x * inv, o.y * inv), ((size_t)(it.r0 + i) * a.nq + h) * D + dim);
        if (dim == 0 && a.lse) a.lse[(size_t)(it.r0 + i) * a.nq + h] = row_lse(M - kUp, l);
      } else {
        ws.o[part * S::PAIRS * 32 + j] = o;
        if (dim == 0) ws.ml[part * S::Q + query] = make_float2(M, l);
      }
    }
    more = false;
    if (mode == kShares) {
      int u = it.next;
      more = next_item(s_plan, a, u, u1, it);
    }
    __syncthreads();
  }
}

// The parts of items cut between CTAs, joined in CTA order.  A lane has two dims of a query,
// `split` warps of a block share an item's parts of 32 such, a block has 8 / split times 32.
template <int D, int NT, bool F32>
__global__ void __launch_bounds__(kThreads) join4_kernel(const __grid_constant__ TreeArgs a, Work ws, int mode, int ctas, int turn, int split) {
  using S = Shape<D, NT, F32>;
  __shared__ UnitPlan plan;
  __shared__ float2 s_o[kWarps][32], s_ml[kWarps][32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, each = S::PAIRS * split / kWarps;
  const int b = blockIdx.z, g = blockIdx.y, qt = blockIdx.x / each;
  const int pair = blockIdx.x % each * (kWarps / split) + warp / split, first_part = warp % split;
  const int r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0, G = a.nq / a.nkv;
  ptx::griddep_launch_dependents();
  const bool some = qt * S::Q < rows * G;
  int n = 0;  // parts
  size_t first_slot = 0;
  if (mode == kDirect) {
    n = some && rows_fit(a.len[b], rows, a.cap) ? turn : 0;
    first_slot = (((size_t)b * gridDim.y + g) * (gridDim.x / each) + qt) * turn;
  } else {
    if (some && tid < 32) make_plan(a, S::Q, turn, lane, plan, false);
    __syncthreads();
    const int tiles = some ? plan.tiles[b] : 0;
    if (tiles > 0) {
      const int first = plan.unit[b] + (g * plan.qts[b] + qt) * (tiles + turn) + turn;
      const int c0 = unit_owner(plan, first, ctas);
      n = unit_owner(plan, first + tiles - 1, ctas) - c0 + 1;
      first_slot = (size_t)c0 * 2;
    }
  }
  ptx::griddep_wait();
  if (n <= 1) return;  // skipped, or written by its CTA
  auto part = [&](int k) { return mode == kDirect ? first_slot + k : first_slot + 2 * k + (k == 0 ? 1 : 0); };
  int query, dim;
  place_of<D>(pair, lane, query, dim);
  const int q = qt * S::Q + query;
  float M = -INFINITY, l = 0.f;
  float2 o = make_float2(0.f, 0.f);
  constexpr int U = 5;  // parts in flight
  for (int k0 = first_part; k0 < n; k0 += U * split) {
    float2 ml[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * split;
      ml[u] = make_float2(-INFINITY, 0.f);
      v[u] = make_float2(0.f, 0.f);
      if (k < n && q < rows * G) {
        ml[u] = __ldcg(&ws.ml[part(k) * S::Q + query]);
        v[u] = __ldcg(&ws.o[(part(k) * S::PAIRS + pair) * 32 + lane]);
      }
    }
    const float before = M;
#pragma unroll
    for (int u = 0; u < U; ++u) M = fmaxf(M, ml[u].x);
    const float w = part_weight(before, M);
    l *= w, o.x *= w, o.y *= w;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = part_weight(ml[u].x, M);
      l = fmaf(ml[u].y, f, l);
      if (ml[u].x != -INFINITY) {  // (a part without tiles has written no more)
        o.x = fmaf(v[u].x, f, o.x);
        o.y = fmaf(v[u].y, f, o.y);
      }
    }
  }
  if (split > 1) {
    s_o[warp][lane] = o;
    s_ml[warp][lane] = make_float2(M, l);
    __syncthreads();
    if (first_part > 0) return;
    for (int w = 1; w < split; ++w) M = fmaxf(M, s_ml[warp + w][lane].x);
    l = 0.f, o = make_float2(0.f, 0.f);
    for (int w = 0; w < split; ++w) {
      const float2 ml = s_ml[warp + w][lane], v = s_o[warp + w][lane];
      const float f = part_weight(ml.x, M);
      l = fmaf(ml.y, f, l);
      o.x = fmaf(v.x, f, o.x);
      o.y = fmaf(v.y, f, o.y);
    }
  }
  if (q >= rows * G) return;
  const int i = divide_group(a, q), h = g * G + (q - i * G);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  write_pair<F32>(a, make_float2(o.x * inv, o.y * inv), ((size_t)(r0 + i) * a.nq + h) * D + dim);
  if (dim == 0 && a.lse) a.lse[(size_t)(r0 + i) * a.nq + h] = row_lse(M - kUp, l);
}

// Items of at most this many tiles are each done by one CTA (us, one row of 28 / 4 heads over 200 entries, with 1 / 2: 5.7 / 5.1;
// over 300, three tiles by three CTAs and joined: 5.6).
constexpr int kWholeTiles = 2;

template <int D, int NT, bool F32>
cudaError_t launch(const Tree4Args& a4, const Work& ws, int64_t max_keys, int sms, cudaStream_t st) {
  using S = Shape<D, NT, F32>;
  static PerDevice opted;
  const cudaError_t e = opt_in(opted, attn4_kernel<D, NT, F32>, S::SMEM);
  if (e != cudaSuccess) return e;
  const TreeArgs& a = a4.t;
  const int G = a.nq / a.nkv;
  int64_t items = 0;
  int most = 0;
  for (int b = 0; b < a.rm.batch; ++b) {
    const int rows = a.rm.start[b + 1] - a.rm.start[b];
    most = std::max(most, rows);
    items += (int64_t)(rows * G + S::Q - 1) / S::Q * a.nkv;
  }
  const int64_t tiles = (max_keys + 127) / 128, units = items * tiles;
  const dim3 each((most * G + S::Q - 1) / S::Q, a.nkv, a.rm.batch);
  if (tiles <= kWholeTiles)
    return launch_pdl(attn4_kernel<D, NT, F32>, each, dim3(kThreads), S::SMEM, st, 1, a4, ws, (int)kDirect, 1);
  int mode = kShares, ctas = (int)std::min<int64_t>(units, (int64_t)S::CTAS * sms);
  int turn = units > S::CTAS * sms ? kTurn : 0;
  int64_t parts = ctas / std::max<int64_t>(items, 1);
  // One request: the same number of CTAs to each of its items, without a plan: four fifths of the SMs, or
  // two to an SM where each would have more than eight tiles.  us, one row of 28 / 4 heads over 300 / 1564 / 8000 / 15128 / 60000 entries:
  // by even shares 6.5 / 7.0 / 9.5 / 12.8 / 17.5; 20 CTAs to an item 5.6 / 6.3 / 8.8 / 10.4 / 24.0,
  // 30 5.6 / 6.3 / 8.3 / 9.1 / 18.1, 38 (every SM has one, or some two and some none) 5.7 / 6.3 / 9.2 / 11.4 / -, 76 5.7 /
  // 6.3 / 8.9 / 10.4 / 17.2.
  if (a.rm.batch == 1 && 2 * items <= sms) {
    mode = kDirect;
    parts = std::max<int64_t>(1, 4 * sms / 5 / items);
    if (tiles > 8 * parts) parts = S::CTAS * sms / items;
    parts = std::min(parts, tiles);
    turn = (int)parts;
  }
  const cudaError_t f = launch_pdl(attn4_kernel<D, NT, F32>, mode == kDirect ? dim3(each.x * turn, each.y, each.z) : dim3(ctas),
                                   dim3(kThreads), S::SMEM, st, 1, a4, ws, mode, turn);
  if (f != cudaSuccess) return f;
  const int split = parts > 20 ? 8 : parts > 10 ? 4 : parts > 5 ? 2 : 1;
  const dim3 joins(each.x * (S::PAIRS * split / kWarps), each.y, each.z);
  return launch_pdl(join4_kernel<D, NT, F32>, joins, dim3(kThreads), 0, st, 1, a, ws, mode, ctas, turn, split);
}

// Calls of more queries to a kv head than kMostNarrow and of more units (16 queries, 128 keys) than so many to an SM
// go to k_attn4_wide.cu, which takes 128 queries for the reading of 16 but starts later: kOwn if it is one request, whose items
// have CTAs of their own; kWhole if items are done whole; else kUnits.  us on the device here / there (units to
// an SM), 28 / 4 heads of 128, queries in bf16:
//   one request  14 queries over 1564 / 15128   (0.3) 8.0 / 10.1   (3.1) 11.7 / 18.6
//                63 over 100 / 1500 / 8000      (0.1) 6.6 / 8.1    (1.3) 9.8 / 10.0    (6.6) 15.1 / 14.8
//                252 over 100 / 1500 / 4000     (0.8) 7.4 / 10.8   (5.1) 13.3 / 11.9   (13) 22.0 / 16.0
//                21 over 4000 / 15128           (1.7) 10.6 / 12.9  (6.3) 15.1 / 18.9
//   items whole  2 requests of 252, 16 of 21 over 200   (1.7) 7.5 / 11.6   (1.7) 7.7 / 11.1
//   others       4 of 28 / 63 over 300          (0.6) 8.8 / 9.8    (1.3) 11.2 / 10.6
//                4 of 84 over 600 / 2000        (3.2) 13.2 / 11.1  (10) 21.6 / 12.5
// Up to kMostNarrow queries a key tile is read once here too: 16 requests of 14 over 376 .. 7426 23.7 / 32.5.
constexpr int kMostNarrow = 16, kOwn = 8, kWhole = 2, kUnits = 1;

template <int D>
cudaError_t launch_d(const Tree4Args& a, void* workspace, int64_t max_keys, cudaStream_t st) {
  const int sms = device_sms(), G = a.t.nq / a.t.nkv;
  Work ws;
  ws.o = (float2*)workspace;
  ws.ml = ws.o + (size_t)sms * kParts * D / 2;
  int64_t queries = 0, items = 0;
  for (int b = 0; b < a.t.rm.batch; ++b) {
    const int64_t n = (int64_t)(a.t.rm.start[b + 1] - a.t.rm.start[b]) * G;
    queries = std::max(queries, n);
    items += (n + 15) / 16 * a.t.nkv;
  }
  const int64_t tiles = (max_keys + 127) / 128;
  const int most = a.t.rm.batch == 1 && 2 * items <= sms ? kOwn : tiles <= kWholeTiles ? kWhole : kUnits;
  if (queries > kMostNarrow && items * tiles > (int64_t)most * sms)
    return launch_attention4_wide(a, D, max_keys, workspace, st);
  if (queries <= 8)
    return a.t.q_f32 ? launch<D, 1, true>(a, ws, max_keys, sms, st) : launch<D, 1, false>(a, ws, max_keys, sms, st);
  return a.t.q_f32 ? launch<D, 2, true>(a, ws, max_keys, sms, st) : launch<D, 2, false>(a, ws, max_keys, sms, st);
}

}  // namespace

size_t attention4_workspace(int head_dim) {
  return std::max((size_t)device_sms() * kParts * (head_dim * 4 + 8), tree_attention_workspace(head_dim));
}

cudaError_t launch_attention4(const Tree4Args& a, int head_dim, int64_t max_keys, void* workspace, cudaStream_t st) {
  return head_dim == 128 ? launch_d<128>(a, workspace, max_keys, st) : launch_d<64>(a, workspace, max_keys, st);
}

}  // namespace as2d
