// tree_dev.cuh -- device code shared by the kernels that multiply a call's query
// rows with a cache's keys on the tensor cores (k_tree_attn.cu,
// k_attn_weights.cu).
#pragma once

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

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// hi = bf16(x), lo = bf16(x - hi) of two numbers.
__device__ __forceinline__ void hi_lo(float a, float b, uint32_t& h, uint32_t& l) {
  h = pack2(a, b);
  l = pack2(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xFFFF0000u));
}

// The visible rows of row r of a request, as a mask of its `rows` rows.
__device__ __forceinline__ uint64_t visible_rows(const TreeArgs& a, int r, int i, int rows) {
  const uint64_t all = ~0ull >> (64 - rows);
  return (a.visible ? a.visible[r] : ~0ull >> (63 - i)) & all;
}

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

// The queries of an item into the operand image(s), by N threads; rows past the
// item's queries are left as they are (what they hold reaches no other row).
template <int D, bool F32, int N, int B>
__device__ __forceinline__ void load_queries(const TreeArgs& a, const Unit& it, int tid, uint8_t* img) {
  constexpr int C = D / 8;  // chunks of a row (B: of a thread, loads in flight)
  const int G = a.nq / a.nkv, n0 = it.qt * 128;
  const int n = min(128, it.rows * G - n0) * C;
  for (int c0 = tid; c0 < n; c0 += N * B) {
    uint4 v[B][F32 ? 2 : 1];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int c = c0 + N * u;
      if (c < n) {
        const int q = n0 + c / C, i = q / G, h = it.g * G + (q - i * G);
        const int64_t at = (it.r0 + i) * a.q_stride + (int64_t)h * D + 8 * (c % C);
        if (F32) {
          const uint4* s = reinterpret_cast<const uint4*>((const float*)a.q + at);
          v[u][0] = s[0];
          v[u][F32 ? 1 : 0] = s[1];
        } else {
          v[u][0] = *reinterpret_cast<const uint4*>((const bf16*)a.q + at);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int c = c0 + N * u;
      if (c < n) {
        uint8_t* to = img + chunk_off(c / C, c % C);
        if (F32) {
          const float* x = reinterpret_cast<const float*>(&v[u][0]);
          uint32_t h[4], l[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) hi_lo(x[2 * e], x[2 * e + 1], h[e], l[e]);
          *reinterpret_cast<uint4*>(to) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(to + 128 * D * 2) = make_uint4(l[0], l[1], l[2], l[3]);
        } else {
          *reinterpret_cast<uint4*>(to) = v[u][0];
        }
      }
    }
  }
}

}  // namespace as2d
