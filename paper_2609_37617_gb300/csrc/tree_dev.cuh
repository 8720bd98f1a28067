// tree_dev.cuh -- device code shared by the kernels that multiply a call's query
// rows with a cache's keys on the tensor cores (k_tree_attn.cu,
// k_attn_weights.cu).
#pragma once

#include <cfloat>

#include "ptx_sm100.cuh"
#include "tree_plan.cuh"

namespace as2d {

constexpr uint32_t kRegion = 128 * 128;  // 64 columns of 128 rows, bytes

// Byte offset of the 16-byte chunk j (of a row's D / 8) of row r in a 128-row
// operand image of 128-byte-swizzled K-major bf16.
__device__ __forceinline__ uint32_t chunk_off(int r, int j) {
  return (uint32_t)(j >> 3) * kRegion + (uint32_t)r * 128u + (uint32_t)(((j & 7) ^ (r & 7)) << 4);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two floats side by side, and arithmetic on both at once.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 of_two(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// The larger of three (NaN is passed by).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// hi = bf16(x), lo = bf16(x - hi) of two numbers.
__device__ __forceinline__ void hi_lo(float a, float b, uint32_t& h, uint32_t& l) {
  h = pack2(a, b);
  l = pack2(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xFFFF0000u));
}

// Whether a key holds infinities and no NaN, by a whole warp.
template <int D>
__device__ __forceinline__ bool infinite_key(const bf16* k, int lane) {
  bool inf = false, none = true;
#pragma unroll
  for (int d = 0; d < D; d += 32) {
    const float y = fabsf(__bfloat162float(k[d + lane]));
    inf = inf || y == INFINITY;
    none = none && y == y;
  }
  return __any_sync(~0u, inf) && __all_sync(~0u, none);
}

// A 32-bit query's product with a key, in 32-bit arithmetic.
template <int D>
__device__ __forceinline__ float exact_product(const float* q, const bf16* k) {
  float s = 0.f;
#pragma unroll 1
  for (int d = 0; d < D && s == s; d += 8) {  // (NaN stays)
    const uint4 y = *reinterpret_cast<const uint4*>(k + d);
    const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s = fmaf(q[d + 2 * e], __uint_as_float(w[e] << 16), s);
      s = fmaf(q[d + 2 * e + 1], __uint_as_float(w[e] & 0xFFFF0000u), s);
    }
  }
  return s;
}

// The visible rows of row r of a request, as a mask of its `rows` rows.
__device__ __forceinline__ uint64_t visible_rows(const TreeArgs& a, int r, int i, int rows) {
  const uint64_t all = ~0ull >> (64 - rows);
  return (a.visible ? a.visible[r] : ~0ull >> (63 - i)) & all;
}

// Which of keys [p0, p0 + 32) a row sees.
__device__ __forceinline__ uint32_t key_bits(int p0, int L, uint64_t vis) {
  const int off = L - p0;  // prefix entries in the word
  if (off >= 32) return ~0u;
  if (off >= 0) return ((1u << off) - 1) | (uint32_t)(vis << off);
  return off > -64 ? (uint32_t)(vis >> -off) : 0u;
}

__device__ __forceinline__ void mask_scores(uint32_t (&v)[32], uint32_t bits) {
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!((bits >> e) & 1)) v[e] = 0xFF800000u;  // -inf
}

// The weight of a part (maximum m) beside a maximum M: 0 where the part holds
// nothing that the row sees.
__device__ __forceinline__ float part_weight(float m, float M) {
  return m == -INFINITY ? 0.f : (m == M ? 1.f : ex2(m - M));
}

// What a score s of a row becomes a weight by, 2^(s by - at): by = c (the scale, base 2) and at = m, the
// rounded product of c and the reference r (a score; m -inf: none), as long as m is off by little.  From
// `far` on its rounding would be a factor of 2 and more of every weight, up to infinity, so r is multiplied by
// c's power of two, exactly: there scores next to each other in 32 bits are as far apart as a row's largest and
// nothing.  NaN for m = +inf, a score of more than 32 bits.  (r(): called where it is needed.)
struct Exponent {
  float by, at;
};
template <typename R>
__device__ __forceinline__ Exponent exponent_of(R r, float m, float c, float far) {
  Exponent x = {c, m == -INFINITY ? 0.f : m};
  if (fabsf(x.at) >= far) {
    x.by = __uint_as_float(__float_as_uint(c) & 0x7F800000u);
    x.at = m == INFINITY ? NAN : __fmul_rn(r(), x.by);
  }
  return x;
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= FLT_MAX; }

// The ring's next stage and its parity, as slot | parity << 8.
struct Stage {
  uint32_t x = 0;
  template <int NST>
  __device__ __forceinline__ uint32_t next() {
    const uint32_t now = x;
    x = (now & 255u) + 1 == NST ? (now & 256u) ^ 256u : now + 1;
    return now;
  }
  static __device__ __forceinline__ uint32_t slot(uint32_t x) { return x & 255u; }
  static __device__ __forceinline__ uint32_t parity(uint32_t x) { return x >> 8; }
};

// The queries of an item into the operand image(s), by N threads (a multiple of a
// row's chunks of 16 bytes), B chunks of a thread in flight (32-bit queries); rows
// past the item's queries are left as they are (what they hold reaches no other row).
// LATER: the image is written only after ready() (its last readers), called by every
// thread once its first loads, and the others' into L2, are on their way.
template <int D, bool F32, int N, int B, bool LATER, typename F>
__device__ __forceinline__ void load_queries(const TreeArgs& a, const Unit& it, int tid, uint8_t* img, F ready) {
  constexpr int C = D / 8, R = N / C;  // chunks of a row, rows of a step
  static_assert(N % C == 0, "a thread keeps its chunk");
  const int G = a.nq / a.nkv, n0 = it.qt * 128, n = min(128, it.rows * G - n0), c = tid % C;
  auto at = [&](int r) {
    const int i = divide_group(a, n0 + r), h = it.g * G + (n0 + r - i * G);
    return (it.r0 + i) * a.q_stride + (int64_t)h * D + 8 * c;
  };
  // (chunks of 16 bytes of bf16 or 32 of floats, lines of 128)
  auto to_l2 = [&](int r) {
    if (LATER && c % (F32 ? 4 : 8) == 0)
      for (; r < n; r += R) ptx::prefetch_l2((const uint8_t*)a.q + at(r) * (F32 ? 4 : 2));
  };
  if constexpr (!F32) {
    // straight into shared memory, every copy on its way at once
    to_l2(tid / C);
    ready();
#pragma unroll 1
    for (int r = tid / C; r < n; r += R) ptx::cp_async16(img + chunk_off(r, c), (const bf16*)a.q + at(r));
    ptx::cp_async_wait_all();
  } else {
    int r0 = tid / C;
    bool first = true;
    do {
      uint4 v[B][2];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const int r = r0 + R * u;
        if (r < n) {
          const uint4* s = reinterpret_cast<const uint4*>((const float*)a.q + at(r));
          v[u][0] = s[0];
          v[u][1] = s[1];
        }
      }
      if (first) {
        if (R * B < 128) to_l2(r0 + R * B);
        ready();
        first = false;
      }
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const int r = r0 + R * u;
        if (r < n) {
          uint8_t* to = img + chunk_off(r, c);
          const float* x = reinterpret_cast<const float*>(&v[u][0]);
          uint32_t h[4], l[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) hi_lo(x[2 * e], x[2 * e + 1], h[e], l[e]);
          *reinterpret_cast<uint4*>(to) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(to + 128 * D * 2) = make_uint4(l[0], l[1], l[2], l[3]);
        }
      }
      r0 += R * B;
    } while (r0 < n);
  }
}

}  // namespace as2d
