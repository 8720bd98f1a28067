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

constexpr int kThreads = 256;

template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  if constexpr (F32) {
    const float4* p = reinterpret_cast<const float4*>((const float*)base + at);
    const float4 a = __ldcs(p), b = __ldcs(p + 1);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>((const bf16*)base + at));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
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

// 8 dims of a head in 64 bits, as the 32-bit code below.
template <int D>
__device__ __noinline__ void finish_exactly(const AppendArgs& a, const float (&x)[8], const float* gain, int position,
                                            int c, double (&y)[8]) {
  constexpr int C = D / 8;
  // (heads with gains and heads without share a warp: every thread takes part in the shuffles)
  double ss = 0.0;
  for (int e = 0; e < 8; ++e) ss = fma((double)x[e], (double)x[e], ss);
  for (int o = C / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
  const double f = 1.0 / sqrt(ss / D + (double)a.eps);
  for (int e = 0; e < 8; ++e) y[e] = gain ? (double)x[e] * f * (double)gain[8 * c + e] : (double)x[e];
  const int h = a.half, d0 = 8 * c, other = d0 < h ? c + h / 8 : c - h / 8;
  const int from = (threadIdx.x & 31 & ~(C - 1)) | (other & (C - 1));
  for (int e = 0; e < 8; ++e) {
    const double z = __shfl_sync(~0u, y[e], from);
    if (d0 < 2 * h) {
      const int j = (d0 < h ? d0 : d0 - h) + e;
      double sn, cs;
      sincospi((double)(int64_t)((uint64_t)(int64_t)position * a.turn[j]) * 0x1p-63, &sn, &cs);
      y[e] = d0 < h ? y[e] * cs - z * sn : y[e] * cs + z * sn;
    }
    __syncwarp();
  }
}

// 8 dims into 4 bits.  off: how far each may be from its exact value (0: it is exact);
// returns whether a code or the scale is that near to a border.
template <typename T>
__device__ __forceinline__ bool quantise(const T (&y)[8], const float (&off)[8], uint32_t& codes, uint8_t& scale,
                                         bool& odd) {
  T most = 0;
  float far = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T m = fabs(y[e]);
    most = m > most ? m : most;  // (NaN is passed by)
    odd = odd || !(m <= (T)3.4028235e38f);
    far = fmaxf(far, off[e]);
  }
  const T there = __shfl_xor_sync(~0u, most, 1);
  most = there > most ? there : most;
  far = fmaxf(far, __shfl_xor_sync(~0u, far, 1));
  T units;
  const T seventh = most / (T)7;
  const float s = scale_of(seventh, units);
  bool near = far > 0.f && fabs(fabs(units - rint(units)) - (T)0.5) * (seventh / (units > 0 ? units : (T)1)) <=
                               (T)(far + 2e-7f * (float)seventh);
  int c[8];
  const float inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(T) == 4) {
      const float q = s > 0.f ? __fdiv_rn(y[e], s) : 0.f;
      near = near || (off[e] > 0.f && fabsf(fabsf(q - rintf(q)) - 0.5f) <= off[e] * inv + 2e-6f);
      c[e] = (int)rintf(fminf(fmaxf(q, -7.f), 7.f));
    } else {
      const double q = s > 0.f ? y[e] / (double)s : 0.0;
      c[e] = (int)rint(fmin(fmax(q, -7.0), 7.0));
    }
    if (y[e] != y[e]) c[e] = 0;
  }
  codes = code_word(c);
  scale = scale_byte(s);
  return near;
}

// A block: R rows (grid-stride).  A unit is a head of a row, 8 dims a thread.
template <int D, bool F32, bool FOUR>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs a, int R) {
  constexpr int C = D / 8, G = kThreads / C;  // threads of a head, heads at once
  __shared__ float2 s_turn[8][64];
  __shared__ int s_req[8], s_at[8], s_pos[8];
  const int tid = threadIdx.x, c = tid % C, H = a.nq + 2 * a.nkv;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  bool odd = false;
  for (int r0 = blockIdx.x * R; r0 < a.rm.rows; r0 += gridDim.x * R) {
    const int n = min(R, a.rm.rows - r0);
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
    const int units = n * H;
    for (int u0 = 0; u0 < units; u0 += G) {
      const int u = u0 + tid / C, i = u / H, head = u - i * H;
      // (threads past the last unit take part in the shuffles)
      const bool live = u < units && s_at[min(i, n - 1)] >= 0;
      const bool isq = head < a.nq, isv = head >= a.nq + a.nkv;
      const int hh = isq ? head : head - a.nq - (isv ? a.nkv : 0), r = r0 + i;
      float x[8] = {};
      if (live)
        load8<F32>(isq ? a.q : isv ? a.v : a.k, r * (isq ? a.q_stride : isv ? a.v_stride : a.k_stride) + hh * D + 8 * c, x);
      const float* gain = isq ? a.q_norm : isv ? nullptr : a.k_norm;
      float y[8];
      float ss = 0.f;
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
      // how far a value is from the exact one, at most (4 bits)
      float off[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) off[e] = gain || F32 ? 1e-6f * fabsf(y[e]) : 0.f;
      const int h = a.half, d0 = 8 * c, other = d0 < h ? c + h / 8 : c - h / 8;
      const int from = (tid & 31 & ~(C - 1)) | (other & (C - 1));
      const bool turned = !isv && d0 < 2 * h;
      if (h > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = __shfl_sync(~0u, y[e], from);
          if (turned) {
            const float2 t = s_turn[min(i, n - 1)][(d0 < h ? d0 : d0 - h) + e];
            if (FOUR) off[e] = 1e-6f * (fabsf(y[e]) + fabsf(z));
            y[e] = d0 < h ? y[e] * t.x - z * t.y : y[e] * t.x + z * t.y;
          }
        }
      }
      if (FOUR) {
        uint32_t codes;
        uint8_t scale;
        bool strange = false;
        bool near = quantise(y, off, codes, scale, strange);
        if (__any_sync(~0u, near && live && !isq)) {
          double z[8];
          finish_exactly<D>(a, x, gain, s_pos[min(i, n - 1)], c, z);
          if (isv)
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = x[e];
          bool ignore = false;
          quantise(z, off, codes, scale, ignore);
        }
        if (live && !isq) {
          odd = odd || strange;
          const size_t at = (((size_t)s_req[i] * a.nkv + hh) * a.cap + s_at[i]) * C + c;
          reinterpret_cast<uint32_t*>(isv ? a.cv4 : a.ck4)[at] = codes;
          if (c % 2 == 0) (isv ? a.cvs : a.cks)[at / 2] = scale;
        }
      } else if (live && !isq) {
        store8((isv ? a.cv : a.ck) + (((size_t)s_req[i] * a.nkv + hh) * a.cap + s_at[i]) * D + 8 * c, y);
      }
      if (live && isq) {
        const size_t at = ((size_t)r * a.nq + hh) * D + 8 * c;
        if constexpr (F32)
          store8((float*)a.q_out + at, y);
        else
          store8((bf16*)a.q_out + at, y);
      }
    }
    __syncthreads();
  }
  if (FOUR && __any_sync(~0u, odd) && (tid & 31) == 0 && a.err) atomicOr(a.err, kErrNotFinite);
}

template <int D, bool F32>
cudaError_t launch(const AppendArgs& a, cudaStream_t st) {
  const int sms = device_sms();
  const int R = a.rm.rows <= 4 * sms ? 1 : 4;
  const int64_t blocks = std::min<int64_t>((a.rm.rows + R - 1) / R, 64 * sms);
  return launch_pdl(a.ck4 ? append_kernel<D, F32, true> : append_kernel<D, F32, false>, dim3((unsigned)blocks),
                    dim3(kThreads), 0, st, 1, a, R);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int head_dim, bool f32, cudaStream_t st) {
  if (head_dim == 128) return f32 ? launch<128, true>(a, st) : launch<128, false>(a, st);
  return f32 ? launch<64, true>(a, st) : launch<64, false>(a, st);
}

}  // namespace as2d
