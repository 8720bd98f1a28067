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
// Codes are those of the exact values: a value or a scale that 32-bit arithmetic finds nearer to
// the border of two codes than its error (some 2e-6 of them) has its head computed once more in
// 64 bits.
//
// Bound by memory: each value is read and written once.
#include <algorithm>
#include <type_traits>

#include "cache4.cuh"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 3;  // heads of a thread whose loads are on their way together
// How far a finished value may be from its exact one, over |y_j| + |y_j'| of its pair: the mean square
// adds 6 roundings of 2^-24 to its root, rsqrtf 4, two products 2, sine and cosine (one step, and an
// angle rounded to 2^-25 of a half turn) 4, the rotation 2.
constexpr float kOff = 1.5e-6f;

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

__device__ __forceinline__ uint64_t turns_of(const AppendArgs& a, int position, int j) {
  return (uint64_t)(int64_t)position * a.turn[j];
}

// Sine and cosine of an angle given in 2^-64 turns, to some 2^-50: the nearest eighth of a turn, and
// the Taylor series of what is left (at most pi / 8; its next terms are below 2^-55).  64-bit operations are
// slow here (one warp's take some 64 cycles), and the library's sincospi has several times as many.
__device__ __forceinline__ void turn_exactly(uint64_t turns, double& sn, double& cs) {
  const uint64_t eighth = (turns + (1ull << 60)) >> 61;
  const double t = (double)(int64_t)(turns - (eighth << 61)) * (6.283185307179586477 * 0x1p-64), t2 = t * t;
  double s = 1. / 6227020800., c = 1. / 479001600.;
  s = fma(s, t2, -1. / 39916800.);
  c = fma(c, t2, -1. / 3628800.);
  s = fma(s, t2, 1. / 362880.);
  c = fma(c, t2, 1. / 40320.);
  s = fma(s, t2, -1. / 5040.);
  c = fma(c, t2, -1. / 720.);
  s = fma(s, t2, 1. / 120.);
  c = fma(c, t2, 1. / 24.);
  s = fma(s, t2, -1. / 6.);
  c = fma(c, t2, -0.5);
  s = fma(s * t2, t, t);
  c = fma(c, t2, 1.);
  if (eighth & 1) {  // by an eighth of a turn
    const double u = (c - s) * 0.70710678118654752440;
    s = (c + s) * 0.70710678118654752440;
    c = u;
  }
  const uint32_t quarter = (uint32_t)(eighth >> 1) & 3u;
  sn = quarter & 1 ? c : s;
  cs = quarter & 1 ? -s : c;
  if (quarter & 2) sn = -sn, cs = -cs;
}

// Those of a head's dims (y[0 .. 3] at d.a, y[4 .. 7] at d.b) that `which` has bits for, in 64
// bits.  By whole warps, whose heads may be keys and values: every thread takes part in the shuffles.
template <int D>
__device__ __noinline__ void finish_exactly(const AppendArgs& a, const float (&x)[8], const float* gain, bool turn,
                                            int position, Dims d, uint32_t which, double (&y)[8]) {
  double f = 1.0;
  if (__any_sync(~0u, gain != nullptr)) {
    double ss = 0.0;
    for (int e = 0; e < 8; ++e) ss = fma((double)x[e], (double)x[e], ss);
    for (int o = D / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
    // 1 / sqrt(v): r (1 + e / 2 + 3 e^2 / 8), e = 1 - v r^2 of the 32-bit root, off by e^3
    const double v = fma(ss, 1.0 / D, (double)a.eps), r = (double)rsqrtf((float)v), e = fma(-v * r, r, 1.0);
    f = v > 0.0 && (float)v < INFINITY && (float)v > 1e-37f ? fma(r * e, fma(0.375, e, 0.5), r) : 1.0 / sqrt(v);
  }
  for (int e = 0; e < 4; ++e) {
    if (!((which >> e | which >> (4 + e)) & 1)) continue;
    double u = x[e], v = x[4 + e];
    if (gain) u *= f * (double)gain[d.a + e], v *= f * (double)gain[d.b + e];
    if (turn && d.pair) {
      double sn, cs;
      turn_exactly(turns_of(a, position, d.a + e), sn, cs);
      const double w = u * cs - v * sn;
      v = v * cs + u * sn;
      u = w;
    }
    y[e] = u, y[4 + e] = v;
  }
}

// What 8 dims (two fours) become in 4 bits.
struct Coded {
  float s[2];
  uint32_t c[8];  // code_bits
};

// The larger of a head's two fours' numbers with the other fours of their 16 dims.
template <typename T>
__device__ __forceinline__ void over_blocks(T& u, T& v, bool pair) {
  const T u1 = __shfl_xor_sync(~0u, u, 1), v1 = __shfl_xor_sync(~0u, v, 1);
  u = u1 > u ? u1 : u, v = v1 > v ? v1 : v;
  const T u2 = __shfl_xor_sync(~0u, u, 2), v2 = __shfl_xor_sync(~0u, v, 2);
  if (pair)
    u = u2 > u ? u2 : u, v = v2 > v ? v2 : v;
  else
    u = v = v > u ? v : u;
}

// off: how far each of the values may be from its exact one (0: it is exact, of bf16).  Returns
// bits of the dims whose code, and 2^8 if a scale, is that near to a border.
__device__ __forceinline__ uint32_t code8(const float (&y)[8], const float (&off)[8], bool pair, Coded& to, bool& odd) {
  float most[2] = {0.f, 0.f}, far[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    most[e / 4] = fmaxf(most[e / 4], fabsf(y[e]));
    odd = odd || !(fabsf(y[e]) <= 3.4028235e38f);
    far[e / 4] = fmaxf(far[e / 4], off[e]);
  }
  over_blocks(most[0], most[1], pair);
  over_blocks(far[0], far[1], pair);
  uint32_t near = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float t = most[k] * (1.f / 7.f);
    float steps;
    const float s = scale_of(t, steps), exact = exact_scale(most[k]), inv_step = steps > 0.f ? __fdividef(steps, t) : 0.f;
    if (far[k] > 0.f && fabsf(fabsf(steps - rintf(steps)) - 0.5f) <= (far[k] + 2.5e-7f * t) * inv_step * 1.001f) near |= 256u;
    to.s[k] = far[k] > 0.f ? s : exact;
    const float inv = reciprocal(to.s[k]);
#pragma unroll
    for (int e = 4 * k; e < 4 * k + 4; ++e) {
      const float q = y[e] * inv;
      if (off[e] > 0.f && fabsf(fabsf(q - rintf(q)) - 0.5f) <= fmaf(off[e], inv, 4e-6f)) near |= 1u << e;
      to.c[e] = off[e] > 0.f ? code_bits_near(q) : code_bits_clamped(y[e], inv);
    }
  }
  if (odd)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (y[e] != y[e]) to.c[e] = code_bits_near(0.f);
  return near;
}

// The same of exact values: with bit 2^8 of `which` all of it, else those codes that it has bits for.
__device__ __noinline__ void code8_exactly(const double (&y)[8], uint32_t which, bool pair, Coded& to) {
  if (which & 256u) {
    double most[2] = {0.0, 0.0}, steps;
    for (int e = 0; e < 8; ++e) most[e / 4] = fmax(most[e / 4], fabs(y[e]));
    over_blocks(most[0], most[1], pair);
    for (int k = 0; k < 2; ++k) to.s[k] = scale_of(most[k] / 7.0, steps);
  }
  for (int e = 0; e < 8; ++e)
    if ((which >> e) & 1) {
      // which of the two whole numbers around it is nearer: their border times s is exact, and the
      // quotient in 32 bits is within 1e-4 of the right one
      const double s = to.s[e / 4], m = fabs(y[e]);
      if (!(m <= 3.4e38)) {
        to.c[e] = code_bits_near(m == m ? copysignf(7.f, (float)y[e]) : 0.f);
      } else if (s == 0.0) {
        to.c[e] = code_bits_near(0.f);
      } else {
        const float low = fminf(floorf((float)m * reciprocal((float)s) - 1e-4f), 7.f);
        const double over = m - ((double)low + 0.5) * s;
        const float up = low + (over > 0.0 || (over == 0.0 && ((int)low & 1)) ? 1.f : 0.f);
        const double more = m - ((double)up + 0.5) * s;  // (low may have been one too low)
        const float c = up + (more > 0.0 || (more == 0.0 && ((int)up & 1)) ? 1.f : 0.f);
        to.c[e] = code_bits_near(copysignf(c, (float)y[e]));
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
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs a, int per) {
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
  float sn[4], cs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sn[e] = 0.f, cs[e] = 1.f;
    if (d.pair) sincospif((float)(int32_t)(turns_of(a, position, d.a + e) >> 32) * 0x1p-31f, &sn[e], &cs[e]);
  }
  bool odd = false;
  // One head of a row (threads whose head there is not take part in the shuffles).
  auto finish = [&](auto kind, const Raw<F32>(&raw)[2], int head) {
    constexpr int K = decltype(kind)::value;
    const bool live = at >= 0 && head < heads[K];
    const float* norm = K == 0 ? a.q_norm : K == 1 ? a.k_norm : nullptr;
    float x[8], y[8], off[8];  // off: how far a value is from the exact one, at most (4 bits)
    floats<F32>(raw[0], x);
    floats<F32>(raw[1], x + 4);
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
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = y[e], v = y[4 + e];
      if (FOUR && K > 0) {
        off[e] = norm || F32 ? kOff * fabsf(u) : 0.f;
        off[4 + e] = norm || F32 ? kOff * fabsf(v) : 0.f;
        if (K == 1 && d.pair) off[e] = off[4 + e] = kOff * (fabsf(u) + fabsf(v));
      }
      if (K < 2 && d.pair) {
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
      Coded to;
      bool strange = false;
      const uint32_t near = code8(y, off, d.pair, to, strange);
      uint32_t which = __reduce_or_sync(~0u, live ? near : 0u);
      if (which) {
        if (which & 256u) which = 511u;
        double z[8];
        finish_exactly<D>(a, x, norm, K == 1, position, d, which, z);
        code8_exactly(z, which, d.pair, to);
      }
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
  // few rows: as many threads to one as there are heads; many: four groups, whose sines, cosines and
  // gains serve all their heads
  int per = 4;
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
