// k_append.cu -- rows of a projection finished and appended to a cache
// (as2d_cache_append, as2d_cache4_append).
//
// Of each head x of a row: y = x g / sqrt(mean x^2 + eps) (queries and keys that have gains),
// then y_j, y_{j + h} turned by the angle position theta^(-j / h), h half of the rotated dims.
// Queries go out, keys and values into the cache at the request's length, in bf16 or in 4
// bits.
//
// A thread has 8 dims of a head, D / 8 threads a head: four and those that they are paired with
// in the rotation, so that only sums of squares, and the largest magnitudes of 16 dims, go through
// shuffles.  Angles: a position times 2^64 turns of its frequency, modulo 2^64, is the angle in
// turns whatever the position, to 2^-64 of a turn and the frequency's own rounding.
//
// Codes are those of the exact values: keys that go into 4 bits are computed in pairs of floats (a
// number and what it is off by, Knuth's and Dekker's sums and products), to some 2^-38, and each
// code and scale is compared with the border that it is next to, which is exact in 32 bits.  (Values
// near a border computed again in 64 bits instead: the first call of that code on an SM took 11 us.)
//
// Each value is read and written once.  7564 rows of 28 / 4 heads of 128, us (floor): bf16 30.7 (20.5), 32-bit 50 (39), into
// 4 bits 51 (19) and 75 (37).  That is 4.5 and 5.3 TB/s, not what memory has: a batch of heads is loaded when the one before
// is stored, so that a load's time shows four times a row; in 4 bits it is the keys' arithmetic.  Few rows: a chain of
// norm, turn and codes.  145 rows (0.4) 4.2 on the device, into 4 bits 9.3: a fourth of a row's groups do its keys and values,
// the others go through the same code with nothing to write.
#include <algorithm>
#include <type_traits>

#include "cache4.cuh"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 3;  // heads of a thread whose loads are on their way together
// Four dims as they are in memory.
template <bool F32>
struct Raw {
  uint32_t w[F32 ? 4 : 2];
};
template <bool F32>
__device__ __forceinline__ void load4(const void* base, int64_t at, Raw<F32>& x) {
  if constexpr (F32) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>((const float*)base + at));
    x.w[0] = v.x, x.w[1] = v.y, x.w[2] = v.z, x.w[3] = v.w;
  } else {
    const uint2 v = __ldcs(reinterpret_cast<const uint2*>((const bf16*)base + at));
    x.w[0] = v.x, x.w[1] = v.y;
  }
}
template <bool F32>
__device__ __forceinline__ void floats(const Raw<F32>& r, float* x) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    x[e] = __uint_as_float(F32 ? r.w[F32 ? e : 0] : e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
}
__device__ __forceinline__ void store4(bf16* to, const float* y) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(y[0], y[1]), b = __floats2bfloat162_rn(y[2], y[3]);
  *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store4(float* to, const float* y) {
  *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
}

// The two fours of dims that thread c of a head has: 4 c of the rotated dims' first half and those they
// are paired with; behind the rotated dims eight side by side.
struct Dims {
  int a, b;
  bool pair;
};
__device__ __forceinline__ Dims dims_of(int c, int half) {
  if (4 * c < half) return {4 * c, half + 4 * c, true};
  const int d = 8 * c;  // (2 half + 8 (c - half / 4))
  return {d, d + 4, false};
}

// ---- pairs of floats ------------------------------------------------------------

struct Two {
  float h, l;
};
__device__ __forceinline__ Two product(float a, float b) {
  const float h = __fmul_rn(a, b);
  return {h, fmaf(a, b, -h)};
}
__device__ __forceinline__ Two sum(float a, float b) {
  const float h = __fadd_rn(a, b), t = __fsub_rn(h, a);
  return {h, __fadd_rn(__fsub_rn(a, __fsub_rn(h, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two sum(Two a, Two b) {
  const Two s = sum(a.h, b.h);
  return {s.h, s.l + (a.l + b.l)};
}
__device__ __forceinline__ Two product(Two a, Two b) {
  const Two p = product(a.h, b.h);
  return {p.h, p.l + fmaf(a.h, b.l, a.l * b.h)};
}

// cos(k pi / 32)
__constant__ float2 kCosines[17] = {
    {1.0f, 0.0f}, {0.9951847195625305f, 7.109666189109021e-09f}, {0.9807852506637573f, 2.9739473106360492e-08f},
    {0.9569403529167175f, -1.7184508038781132e-08f}, {0.9238795042037964f, 2.830748968563057e-08f}, {0.8819212913513184f, -2.7002963420841297e-08f},
    {0.8314695954322815f, 1.687026340846387e-08f}, {0.7730104327201843f, 2.0642552556182636e-08f}, {0.7071067690849304f, 1.2101617485882343e-08f},
    {0.6343932747840881f, 9.37955757507325e-09f}, {0.5555702447891235f, -1.1769521357507529e-08f}, {0.4713967442512512f, -7.425253745196869e-09f},
    {0.3826834261417389f, 6.2233507236442165e-09f}, {0.290284663438797f, 1.3815665056426951e-08f}, {0.19509032368659973f, -1.670471427850373e-09f},
    {0.0980171412229538f, -8.933931927579408e-10f}, {0.0f, 0.0f}};

// Sine and cosine of an angle given in 2^-64 turns: the nearest of 64 parts of a turn, from the table,
// and the Taylor series of what is left (at most pi / 64; its next terms are below 2^-42).
__device__ __forceinline__ void turn_exactly(uint64_t turns, Two& sn, Two& cs) {
  const uint32_t k = (uint32_t)((turns + (1ull << 57)) >> 58) & 63u;
  const int64_t left = (int64_t)(turns - ((uint64_t)k << 58));
  const float a = (float)(int32_t)(left >> 34) * 0x1p-30f, b = (float)(uint32_t)((left >> 10) & 0xFFFFFF) * 0x1p-54f;
  Two x = product(a, 6.28318548f);  // 2 pi, and what that is off by
  x.l += fmaf(a, -1.74845553e-7f, b * 6.28318548f);
  Two z = product(x.h, x.h);
  z.l = fmaf(2.f * x.h, x.l, z.l);
  const Two s = {x.h, fmaf(x.h * z.h, fmaf(z.h, fmaf(z.h, -1.f / 5040.f, 1.f / 120.f), -1.f / 6.f), x.l)};
  const Two w = {-0.5f * z.h, fmaf(z.h * z.h, fmaf(z.h, -1.f / 720.f, 1.f / 24.f), -0.5f * z.l)};  // cos - 1
  const float2 u = kCosines[k & 15], v = kCosines[16 - (k & 15)];
  Two C = {u.x, u.y}, S = {v.x, v.y};
  if (k & 16) {
    const Two t = C;
    C = {-S.h, -S.l};
    S = t;
  }
  if (k & 32) C = {-C.h, -C.l}, S = {-S.h, -S.l};
  const Two Ss = product(S, s), Cs = product(C, s);
  const Two c = sum(C, sum(product(C, w), Two{-Ss.h, -Ss.l})), t = sum(S, sum(product(S, w), Cs));
  cs = sum(c.h, c.l);  // (the first parts the nearest)
  sn = sum(t.h, t.l);
}

// What 8 dims (two fours) become in 4 bits.
struct Coded {
  float s[2];
  uint32_t c[8];  // code_bits
};

// The larger of a head's two fours' numbers with the other fours of their 16 dims.
__device__ __forceinline__ void over_blocks(float& u, float& v, bool pair) {
  u = fmaxf(u, __shfl_xor_sync(~0u, u, 1)), v = fmaxf(v, __shfl_xor_sync(~0u, v, 1));
  const float u2 = __shfl_xor_sync(~0u, u, 2), v2 = __shfl_xor_sync(~0u, v, 2);
  if (pair)
    u = fmaxf(u, u2), v = fmaxf(v, v2);
  else
    u = v = fmaxf(u, v);
}

// Exact values of bf16.
__device__ __forceinline__ void code8(const float (&y)[8], bool pair, Coded& to) {
  float most[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 8; ++e) most[e / 4] = fmaxf(most[e / 4], fabsf(y[e]));
  over_blocks(most[0], most[1], pair);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    to.s[k] = exact_scale(most[k]);
    const float inv = reciprocal(to.s[k]);
#pragma unroll
    for (int e = 4 * k; e < 4 * k + 4; ++e) to.c[e] = code_bits_clamped(y[e], inv);
  }
}

// A whole number n next to (x.h + x.l) / s, 0 if s is, made the nearest one (ties to even).
__device__ __forceinline__ float nearest(float n, Two x, float s) {
  // (n s, its difference from x.h and that one's from the border, where it is near, are exact)
  const float d = fmaf(-n, s, x.h), past = (fabsf(d) - 0.5f * s) + (d < 0.f ? -x.l : x.l);
  const bool other = past > 0.f || (past == 0.f && ((int)n & 1));
  return other && s > 0.f ? n + copysignf(1.f, d) : n;
}

// Values as pairs of floats (their first parts the nearest to them).
__device__ __forceinline__ void code8(const Two (&y)[8], bool pair, Coded& to) {
  float most[2] = {0.f, 0.f}, rest[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int e = 0; e < 8; ++e) most[e / 4] = fmaxf(most[e / 4], fabsf(y[e].h));
  over_blocks(most[0], most[1], pair);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (fabsf(y[e].h) == most[e / 4]) rest[e / 4] = fmaxf(rest[e / 4], y[e].h < 0.f ? -y[e].l : y[e].l);
  over_blocks(rest[0], rest[1], pair);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    // the scale: a seventh in steps of those around it
    const int e = min(max((int)(__float_as_uint(most[k] * (1.f / 7.f)) >> 23), 127 - 14), 127 + 9);
    const float step = __uint_as_float((uint32_t)(e - 3) << 23), big = fminf(most[k], 7168.f);
    const float n = rintf(big * (1.f / 7.f) * __uint_as_float((uint32_t)(2 * 127 + 3 - e) << 23));
    const float s = fminf(fminf(nearest(n, {big, most[k] < 7168.f ? rest[k] : 0.f}, 7.f * step), 16.f) * step, kMaxScale4);
    to.s[k] = s;
    const float inv = reciprocal(s);
#pragma unroll
    for (int f = 4 * k; f < 4 * k + 4; ++f) {
      const float c = rintf(fminf(fmaxf(y[f].h * inv, -7.f), 7.f));
      to.c[f] = code_bits_near(nearest(c, y[f], s));
    }
  }
}

// Four codes, as the even four of a word.
__device__ __forceinline__ uint32_t half_word(const uint32_t* c) {
  return __byte_perm(c[0], c[1], 0x5410) | __byte_perm(c[2], c[3], 0x5410) << 4;
}

// `per` groups of C threads to a row, each its heads in turn (a row's sines and cosines, and the
// gains, stay in registers).
template <int D, bool F32, bool FOUR>
__global__ void __launch_bounds__(kThreads, 4) append_kernel(const __grid_constant__ AppendArgs a, int per) {
  constexpr int C = D / 8, G = kThreads / C;  // threads of a head, groups of them
  const int tid = threadIdx.x, c = tid % C, group = tid / C;
  const int r = blockIdx.x * (G / per) + group / per, h0 = group % per;
  const Dims d = dims_of(c, a.half);
  const bool row_live = r < a.rm.rows;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  // a row's queries, keys and values, and the first of this group's heads of each
  const int64_t row = row_live ? r : 0;
  const int heads[3] = {a.nq, a.nkv, a.nkv};
  const int64_t from[3] = {row * a.q_stride, row * a.k_stride, row * a.v_stride};
  const void* const base[3] = {a.q, a.k, a.v};
  auto load = [&](auto kind, int head, Raw<F32>(&raw)[2]) {
    constexpr int K = decltype(kind)::value;
    const int h = min(head, heads[K] - 1);  // (one that is no head's is not used)
    load4(base[K], from[K] + h * D + d.a, raw[0]);
    load4(base[K], from[K] + h * D + d.b, raw[1]);
  };
  using Q = std::integral_constant<int, 0>;
  using Key = std::integral_constant<int, 1>;
  using Value = std::integral_constant<int, 2>;
  Raw<F32> raw_k[2], raw_v[2], raw_q[kAtOnce][2];
  load(Key(), h0, raw_k);
  load(Value(), h0, raw_v);
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) load(Q(), h0 + k * per, raw_q[k]);
  // the gains of these dims, queries' and keys'
  float gain[2][8];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float* g = k ? a.k_norm : a.q_norm;
#pragma unroll
    for (int e = 0; e < 8; ++e) gain[k][e] = 1.f;
    if (g) {
      const float4 u = *reinterpret_cast<const float4*>(g + d.a), v = *reinterpret_cast<const float4*>(g + d.b);
      gain[k][0] = u.x, gain[k][1] = u.y, gain[k][2] = u.z, gain[k][3] = u.w;
      gain[k][4] = v.x, gain[k][5] = v.y, gain[k][6] = v.z, gain[k][7] = v.w;
    }
  }
  int b = 0, at = -1, position = 0;
  if (row_live) {
    b = row_request(a.rm, r);
    const int L = a.len[b], i = r - a.rm.start[b];
    const bool fits = rows_fit(L, a.rm.start[b + 1] - a.rm.start[b], a.cap);
    if (!fits && i == 0 && h0 == 0 && c == 0 && a.err) atomicOr(a.err, kErrCapacity);
    at = fits ? L + i : -1;
    position = a.positions ? a.positions[r] : fits ? L + i : 0;
  }
  float sn[4], cs[4], sn_l[4], cs_l[4];  // (the second parts for keys in 4 bits)
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sn[e] = sn_l[e] = cs_l[e] = 0.f, cs[e] = 1.f;
    if (!d.pair) continue;
    const uint64_t turns = (uint64_t)(int64_t)position * a.turn[d.a + e];
    if constexpr (FOUR) {
      Two s, c;
      turn_exactly(turns, s, c);
      sn[e] = s.h, sn_l[e] = s.l, cs[e] = c.h, cs_l[e] = c.l;
    } else {
      sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &sn[e], &cs[e]);
    }
  }
  bool odd = false;
  // One head of a row (threads whose head there is not take part in the shuffles).
  auto finish = [&](auto kind, const Raw<F32>(&raw)[2], int head) {
    constexpr int K = decltype(kind)::value;
    const bool live = at >= 0 && head < heads[K];
    const float* norm = K == 0 ? a.q_norm : K == 1 ? a.k_norm : nullptr;
    float x[8], y[8];
    Two z[8];  // (keys in 4 bits)
    floats<F32>(raw[0], x);
    floats<F32>(raw[1], x + 4);
    if constexpr (FOUR && K == 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = {x[e], 0.f};
      if (norm) {
        Two ss = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = sum(ss, product(x[e], x[e]));
#pragma unroll
        for (int o = C / 2; o > 0; o >>= 1) ss = sum(ss, Two{__shfl_xor_sync(~0u, ss.h, o), __shfl_xor_sync(~0u, ss.l, o)});
        // f = 1 / sqrt(v): r (1 + e / 2 + 3 e^2 / 8), e = 1 - v r^2 of the approximate root r
        const Two v = sum(Two{ss.h * (1.f / D), ss.l * (1.f / D)}, Two{a.eps, 0.f});
        const float r = rsqrtf(v.h);
        const Two p = product(v, product(r, r));
        const float err = (1.f - p.h) - p.l;
        const Two f = {r, r * err * fmaf(0.375f, err, 0.5f)};
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = product(product(x[e], gain[1][e]), f);
      }
      if (d.pair)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Two u = z[e], v = z[4 + e], s = {sn[e], sn_l[e]}, c = {cs[e], cs_l[e]}, ns = {-sn[e], -sn_l[e]};
          z[e] = sum(product(u, c), product(v, ns));
          z[4 + e] = sum(product(v, c), product(u, s));
        }
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = sum(z[e].h, z[e].l);
    } else {
      if (K < 2 && norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = C / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
        const float f = rsqrtf(fmaf(ss, 1.f / D, a.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * f * gain[K & 1][e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e];
      }
      if (K < 2 && d.pair)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = y[e], v = y[4 + e];
          y[e] = u * cs[e] - v * sn[e];
          y[4 + e] = v * cs[e] + u * sn[e];
        }
    }
    if (K == 0) {
      if (live) {
        const size_t to = ((size_t)r * a.nq + head) * D;
        if constexpr (F32) {
          store4((float*)a.q_out + to + d.a, y);
          store4((float*)a.q_out + to + d.b, y + 4);
        } else {
          store4((bf16*)a.q_out + to + d.a, y);
          store4((bf16*)a.q_out + to + d.b, y + 4);
        }
      }
    } else if (FOUR) {
      // (NaN counts as 0, an infinity as more than the largest scale)
      Coded to;
      bool strange = false;
      if constexpr (K == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          strange = strange || !(fabsf(y[e]) <= 3.4028235e38f);
          if (!(y[e] == y[e])) y[e] = 0.f;
          z[e] = {y[e], 0.f};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(fabsf(z[e].h) <= 3.4028235e38f)) strange = true, z[e] = {z[e].h == z[e].h ? z[e].h : 0.f, 0.f};
      }
      if constexpr (K == 2 && !F32)
        code8(y, d.pair, to);
      else
        code8(z, d.pair, to);
      // the words of codes: of paired fours a thread writes the one of its even or odd neighbours
      const uint32_t wa = half_word(to.c), wb = half_word(to.c + 4);
      const uint32_t there = __shfl_xor_sync(~0u, c & 1 ? wa : wb, 1);
      const uint32_t word = !d.pair ? wa | wb << 8 : c & 1 ? there | wb << 8 : wa | there << 8;
      const int word_at = !d.pair ? d.a / 8 : c & 1 ? (d.b - 4) / 8 : d.a / 8;
      if (live) {
        odd = odd || strange;
        const size_t entry = ((size_t)b * a.nkv + head) * a.cap + at;
        reinterpret_cast<uint32_t*>(K == 2 ? a.cv4 : a.ck4)[entry * C + word_at] = word;
        uint8_t* scales = (K == 2 ? a.cvs : a.cks) + entry * (D / 16);
        if (d.pair) {
          if (c % 4 < 2) scales[(c % 4 ? d.b : d.a) / 16] = scale_byte(to.s[c % 4]);
        } else if (c % 2 == 0) {
          scales[d.a / 16] = scale_byte(to.s[0]);
        }
      }
    } else if (live) {
      bf16* to = (K == 2 ? a.cv : a.ck) + (((size_t)b * a.nkv + head) * a.cap + at) * D;
      store4(to + d.a, y);
      store4(to + d.b, y + 4);
    }
  };
  // (the rounds are those of a whole block)
#pragma unroll 1
  for (int t0 = 0; t0 < a.nkv; t0 += per) {
    if (t0 > 0) load(Key(), t0 + h0, raw_k), load(Value(), t0 + h0, raw_v);
    finish(Key(), raw_k, t0 + h0);
    finish(Value(), raw_v, t0 + h0);
  }
#pragma unroll 1
  for (int t0 = 0; t0 < a.nq; t0 += kAtOnce * per) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int t = t0 + k * per;
      if (t0 > 0) load(Q(), t + h0, raw_q[k]);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (t0 + k * per < a.nq) finish(Q(), raw_q[k], t0 + k * per + h0);
  }
  if (FOUR && __any_sync(~0u, odd) && (tid & 31) == 0 && a.err) atomicOr(a.err, kErrNotFinite);
}

template <int D, bool F32>
cudaError_t launch(const AppendArgs& a, cudaStream_t st) {
  constexpr int G = kThreads / (D / 8);
  // few rows: as many threads to one as there are heads; many: two groups, whose sines, cosines and
  // gains serve all their heads (7564 rows, us with 2 / 4 / 8: 30.7 / 31.7 / 41)
  int per = 2;
  while (per < G && per < a.nq && (int64_t)a.rm.rows * per / G < 2 * device_sms()) per *= 2;
  return launch_pdl(a.ck4 ? append_kernel<D, F32, true> : append_kernel<D, F32, false>,
                    dim3((a.rm.rows + G / per - 1) / (G / per)), dim3(kThreads), 0, st, 1, a, per);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int head_dim, bool f32, cudaStream_t st) {
  if (head_dim == 128) return f32 ? launch<128, true>(a, st) : launch<128, false>(a, st);
  return f32 ? launch<64, true>(a, st) : launch<64, false>(a, st);
}

}  // namespace as2d
