// k_append.cu -- rows of a projection finished and appended to a cache
// (as2d_cache_append, as2d_cache4_append).
//
// Of each head x of a row: y = x g / sqrt(mean x^2 + eps) (queries and keys that have gains),
// then y_j, y_{j + h} turned by the angle position theta^(-j / h), h half of the rotated dims.
// Queries go out, keys and values into the cache at the request's length, in bf16 or in 4
// bits.
//
// A thread has 8 dims of a head (16 bytes of bf16; a word of codes), D / 8 threads a head;
// sums of squares and the other halves of the rotation go through shuffles.  Angles: a
// position times 2^64 turns of its frequency, modulo 2^64, is the angle in turns whatever the
// position, to 2^-64 of a turn and the frequency's own rounding; a row's sines and
// cosines are computed once, in shared memory.
//
// Codes are those of the exact values: a value or a scale that 32-bit arithmetic finds nearer to
// the border of two codes than its error (some 2e-6 of them) has its head computed once more in
// 64 bits.
//
// Bound by memory: each value is read and written once.
#include <cmath>

#include "cache4.cuh"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

constexpr int kThreads = 256, kMostRows = 4;
// How far a finished value may be from its exact one, over |y_j| + |y_j'| of its pair: the mean
// square, its root, the division and two products add 11 roundings of 2^-24, sine and cosine (one
// step, and an angle rounded to 2^-25 of a half turn) 4, the rotation 2.
constexpr float kOff = 1.5e-6f;

// 8 dims as they are in memory.
template <bool F32>
struct Raw {
  uint4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t at, Raw<F32>& x) {
  const uint4* p = reinterpret_cast<const uint4*>((const char*)base + at * (F32 ? 4 : 2));
  x.w[0] = __ldcs(p);
  if constexpr (F32) x.w[1] = __ldcs(p + 1);
}
template <bool F32>
__device__ __forceinline__ void floats(const Raw<F32>& r, float (&x)[8]) {
  const uint4 a = r.w[0];
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  if constexpr (F32) {
    const uint4 b = r.w[1];
    const uint32_t v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]), x[4 + e] = __uint_as_float(v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
}

__device__ __forceinline__ void store8(bf16* to, const float (&y)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* to, const float (&y)[8]) {
  reinterpret_cast<float4*>(to)[0] = make_float4(y[0], y[1], y[2], y[3]);
  reinterpret_cast<float4*>(to)[1] = make_float4(y[4], y[5], y[6], y[7]);
}

// Those of 8 dims of a head that `which` has bits for, in 64 bits.  By whole warps, whose heads
// may be keys and values: every thread takes part in the shuffles.
template <int D>
__device__ __noinline__ void finish_exactly(const AppendArgs& a, const float (&x)[8], const float* gain, bool turn,
                                            int position, int c, uint32_t which, double (&y)[8]) {
  constexpr int C = D / 8;
  double ss = 0.0;
  for (int e = 0; e < 8; ++e) ss = fma((double)x[e], (double)x[e], ss);
  for (int o = C / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
  const double f = 1.0 / sqrt(ss / D + (double)a.eps);
  const int h = a.half, d0 = 8 * c, other = d0 < h ? c + h / 8 : c - h / 8;
  const int from = (threadIdx.x & 31 & ~(C - 1)) | (other & (C - 1));
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (!((which >> e) & 1)) continue;  // (the same in every thread)
    double v = gain ? (double)x[e] * f * (double)gain[8 * c + e] : (double)x[e];
    const double z = __shfl_sync(~0u, v, from);
    if (turn && d0 < 2 * h) {
      const int j = (d0 < h ? d0 : d0 - h) + e;
      double sn, cs;
      sincospi((double)(int64_t)((uint64_t)(int64_t)position * a.turn[j]) * 0x1p-63, &sn, &cs);
      v = d0 < h ? v * cs - z * sn : v * cs + z * sn;
    }
    __syncwarp();
    y[e] = v;
  }
}

// What 8 dims become in 4 bits.
struct Coded {
  float s;
  uint32_t c[8];  // code_bits
};

// off: how far each of the values may be from its exact one (0: it is exact, of bf16).  Returns
// bits of the dims whose code, and 2^8 if the scale, is that near to a border.
__device__ __forceinline__ uint32_t code8(const float (&y)[8], const float (&off)[8], Coded& to, bool& odd) {
  float most = 0.f, far = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    most = fmaxf(most, fabsf(y[e]));
    odd = odd || !(fabsf(y[e]) <= 3.4028235e38f);
    far = fmaxf(far, off[e]);
  }
  most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
  far = fmaxf(far, __shfl_xor_sync(~0u, far, 1));
  const float t = most * (1.f / 7.f);
  float steps;
  const float s = scale_of(t, steps), exact = exact_scale(most), inv_step = steps > 0.f ? steps / t : 0.f;
  uint32_t near = far > 0.f && fabsf(fabsf(steps - rintf(steps)) - 0.5f) <= (far + 2.5e-7f * t) * inv_step ? 256u : 0u;
  to.s = far > 0.f ? s : exact;
  const float inv = reciprocal(to.s);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = y[e] * inv;
    if (off[e] > 0.f && fabsf(fabsf(q - rintf(q)) - 0.5f) <= fmaf(off[e], inv, 4e-6f)) near |= 1u << e;
    to.c[e] = code_bits(off[e] > 0.f ? q : on_grid(y[e], inv));
  }
  if (odd)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (y[e] != y[e]) to.c[e] = code_bits(0.f);
  return near;
}

// The same of exact values: with bit 2^8 of `which` all of it, else those codes that it has bits for.
__device__ __noinline__ void code8_exactly(const double (&y)[8], uint32_t which, Coded& to) {
  if (which & 256u) {
    double most = 0.0, steps;
    for (int e = 0; e < 8; ++e) most = fmax(most, fabs(y[e]));
    most = fmax(most, __shfl_xor_sync(~0u, most, 1));
    to.s = scale_of(most / 7.0, steps);
  }
  for (int e = 0; e < 8; ++e)
    if ((which >> e) & 1) {
      const double q = to.s > 0.f ? y[e] / (double)to.s : 0.0;
      to.c[e] = code_bits(y[e] == y[e] ? (float)rint(fmin(fmax(q, -7.0), 7.0)) : 0.f);
    }
}

// What a thread has of one head of a row of a block.
struct Place {
  int i, head;   // row of the block, head of the row: queries, keys, values
  bool live;     // there is such a head
  bool isq, isv;
  int hh;        // head among its kind
};

// A block: R rows, U heads at once a thread.
template <int D, bool F32, bool FOUR, int U>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs a, int R) {
  constexpr int C = D / 8, G = kThreads / C;  // threads of a head, heads at once
  __shared__ float2 s_turn[kMostRows][64];
  __shared__ int s_req[kMostRows], s_at[kMostRows], s_pos[kMostRows];
  const int tid = threadIdx.x, c = tid % C, H = a.nq + 2 * a.nkv;
  const int r0 = blockIdx.x * R, n = min(R, a.rm.rows - r0), units = n * H;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  auto place = [&](int u) {
    Place p;
    p.live = u < units;
    p.i = p.live ? u / H : 0;
    p.head = p.live ? u - p.i * H : 0;
    p.isq = p.head < a.nq, p.isv = p.head >= a.nq + a.nkv;
    p.hh = p.isq ? p.head : p.head - a.nq - (p.isv ? a.nkv : 0);
    return p;
  };
  Raw<F32> raw[U];
  auto load = [&](int u0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const Place p = place(u0 + k * G + tid / C);
      const int64_t stride = p.isq ? a.q_stride : p.isv ? a.v_stride : a.k_stride;
      if (p.live) load8(p.isq ? a.q : p.isv ? a.v : a.k, (r0 + p.i) * stride + p.hh * D + 8 * c, raw[k]);
    }
  };
  load(0);
  if (tid < n) {
    const int r = r0 + tid, b = row_request(a.rm, r), L = a.len[b], rows = a.rm.start[b + 1] - a.rm.start[b];
    const int i = r - a.rm.start[b];
    const bool fits = rows_fit(L, rows, a.cap);
    if (!fits && i == 0 && a.err) atomicOr(a.err, kErrCapacity);
    s_req[tid] = b;
    s_at[tid] = fits ? L + i : -1;
    s_pos[tid] = a.positions ? a.positions[r] : fits ? L + i : 0;
  }
  __syncthreads();
  for (int t = tid; t < n * a.half; t += kThreads) {
    const int i = t / a.half, j = t - i * a.half;
    const uint64_t turns = (uint64_t)(int64_t)s_pos[i] * a.turn[j];
    float2 v;
    sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &v.y, &v.x);
    s_turn[i][j] = v;
  }
  __syncthreads();
  bool odd = false;
  const int h = a.half, d0 = 8 * c, other = d0 < h ? c + h / 8 : c - h / 8;
  const int from = (tid & 31 & ~(C - 1)) | (other & (C - 1));
  for (int u0 = 0; u0 < units; u0 += U * G) {
    if (u0 > 0) load(u0);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (u0 + k * G >= units) break;
      // (threads past the last unit take part in the shuffles)
      const Place p = place(u0 + k * G + tid / C);
      const bool live = p.live && s_at[p.i] >= 0;
      const float* gain = p.isq ? a.q_norm : p.isv ? nullptr : a.k_norm;
      float y[8], off[8];  // off: how far a value is from the exact one, at most (4 bits)
      float ss = 0.f, x[8];
      floats<F32>(raw[k], x);
      if (!p.live)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int o = C / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
      if (gain) {
        const float f = 1.f / sqrtf(ss * (1.f / D) + a.eps);
        const float4 g0 = reinterpret_cast<const float4*>(gain)[2 * c], g1 = reinterpret_cast<const float4*>(gain)[2 * c + 1];
        const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * f * g[e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) off[e] = gain || F32 ? kOff * fabsf(y[e]) : 0.f;
      if (h > 0) {
        const bool turned = !p.isv && d0 < 2 * h;
        const float2* turn = s_turn[p.i] + (d0 < h ? d0 : d0 - h);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = __shfl_sync(~0u, y[e], from);
          if (turned) {
            const float2 t = turn[e];
            if (FOUR) off[e] = kOff * (fabsf(y[e]) + fabsf(z));
            y[e] = d0 < h ? y[e] * t.x - z * t.y : y[e] * t.x + z * t.y;
          }
        }
      }
      if (FOUR) {
        Coded to;
        bool strange = false;
        const bool mine = live && !p.isq;
        const uint32_t near = code8(y, off, to, strange);
        uint32_t which = __reduce_or_sync(~0u, mine ? near : 0u);
        if (which) {
          if (which & 256u) which = 511u;
          double z[8];
          finish_exactly<D>(a, x, gain, !p.isv, s_pos[p.i], c, which, z);
          code8_exactly(z, which, to);
        }
        if (mine) {
          odd = odd || strange;
          const size_t at = (((size_t)s_req[p.i] * a.nkv + p.hh) * a.cap + s_at[p.i]) * C + c;
          reinterpret_cast<uint32_t*>(p.isv ? a.cv4 : a.ck4)[at] = code_word(to.c);
          if (c % 2 == 0) (p.isv ? a.cvs : a.cks)[at / 2] = scale_byte(to.s);
        }
      } else if (live && !p.isq) {
        store8((p.isv ? a.cv : a.ck) + (((size_t)s_req[p.i] * a.nkv + p.hh) * a.cap + s_at[p.i]) * D + 8 * c, y);
      }
      if (live && p.isq) {
        const size_t at = ((size_t)(r0 + p.i) * a.nq + p.hh) * D + 8 * c;
        if constexpr (F32)
          store8((float*)a.q_out + at, y);
        else
          store8((bf16*)a.q_out + at, y);
      }
    }
  }
  if (FOUR && __any_sync(~0u, odd) && (tid & 31) == 0 && a.err) atomicOr(a.err, kErrNotFinite);
}

template <int D, bool F32>
cudaError_t launch(const AppendArgs& a, cudaStream_t st) {
  constexpr int U = F32 ? 2 : 3;
  const int R = a.rm.rows <= 4 * device_sms() ? 1 : kMostRows;
  return launch_pdl(a.ck4 ? append_kernel<D, F32, true, U> : append_kernel<D, F32, false, U>,
                    dim3((a.rm.rows + R - 1) / R), dim3(kThreads), 0, st, 1, a, R);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int head_dim, bool f32, cudaStream_t st) {
  if (head_dim == 128) return f32 ? launch<128, true>(a, st) : launch<128, false>(a, st);
  return f32 ? launch<64, true>(a, st) : launch<64, false>(a, st);
}

}  // namespace as2d
