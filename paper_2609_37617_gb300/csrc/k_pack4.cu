// k_pack4.cu -- entries of a cache in bf16 written into one in 4 bits and read back
// (as2d_cache4_write, as2d_cache4_read).
//
// A thread has 8 dims: 16 bytes of bf16, a word of codes; two threads share a scale.
// Bound by memory: 2 + 0.5625 bytes a value.  28 layers of 15128 entries, written and read back (4 kv heads of 128:
// floor 327 us): 356, 6.2 TB/s.
#include <algorithm>

#include "cache4.cuh"
#include "ptx_sm100.cuh"

namespace as2d {
namespace {

// Pieces of a thread on their way together, and blocks to an SM in all, at most: us, the 15128 entries, with 2 / 4 / 8
// pieces 366 / 358 / 377, with 16 / 64 / 256 blocks 364 / 358 / 385.
constexpr int kThreads = 256, kAtOnce = 4;
constexpr int64_t kBlocks = 64;

// The largest magnitude of the 16 is found on pairs of bf16 as whole numbers, of which NaN and
// infinities are the largest.
__device__ __forceinline__ void write8(uint4 v, uint32_t& codes, uint8_t& scale, bool& odd) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = __vmaxu2(top, w[e] & 0x7FFF7FFFu);
  top = __vmaxu2(top, __shfl_xor_sync(~0u, top, 1));
  const uint32_t most = max(top & 0xFFFFu, top >> 16);
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
  const float s = exact_scale(__uint_as_float(most << 16)), inv = reciprocal(s);
  uint32_t c[8];
  if (s >= 6.103515625e-5f && s < kMaxScale4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = code_bits(x[e], inv);
  } else if (most < 0x7F80u) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = code_bits_clamped(x[e], inv);
  } else {
    // (the largest number is not the largest magnitude where there is NaN; an infinity has the largest scale)
    odd = true;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));
    const uint32_t pair = 3u << (threadIdx.x & 30);
    m = fmaxf(m, __shfl_xor_sync(pair, m, 1));
    const float t = exact_scale(m), f = reciprocal(t);
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = code_bits_clamped(x[e] == x[e] ? x[e] : 0.f, f);
    codes = code_word(c);
    scale = scale_byte(t);
    return;
  }
  codes = code_word(c);
  scale = scale_byte(s);
}

__device__ __forceinline__ uint4 read8(uint32_t codes, uint8_t scale) {
  const __half2 s = scale_pair((uint32_t)scale * 0x10001u);
  __half2 v[4];
  decode_word(codes, s, scale_shift(s), v);
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(v[e]);
    w[e] = __float_as_uint(f.x) >> 16 | (__float_as_uint(f.y) & 0xFFFF0000u);  // (exact)
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// grid: (pieces of a unit's entries, units, keys or values)
template <int D, bool WRITE>
__global__ void __launch_bounds__(kThreads) pack4_kernel(const __grid_constant__ Pack4Args a) {
  constexpr int C = D / 8;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  bf16* const x = blockIdx.z ? a.v : a.k;
  uint8_t* const codes = blockIdx.z ? a.v4 : a.k4;
  uint8_t* const scales = blockIdx.z ? a.vs : a.ks;
  bool odd = false;
  for (int64_t unit = blockIdx.y; unit < a.units; unit += gridDim.y) {
    const int b = (int)(unit / a.nkv % a.batch);
    const int from = a.start ? a.start[b] : 0, to = a.end[b];
    if (from >= to) continue;
    if (from < 0 || to > min(a.cap, a.cap4)) {
      if (threadIdx.x == 0 && a.err) atomicOr(a.err, kErrCapacity);
      continue;
    }
    const size_t at_x = ((size_t)unit * a.cap + from) * D, at_c = ((size_t)unit * a.cap4 + from) * C;
    const int n = (to - from) * C;  // pieces of 8 dims
    for (int p0 = blockIdx.x * kThreads * kAtOnce; p0 < n; p0 += gridDim.x * kThreads * kAtOnce) {
      if constexpr (WRITE) {
        uint4 v[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int p = p0 + u * kThreads + threadIdx.x;
          v[u] = p < n ? __ldcs(reinterpret_cast<const uint4*>(x + at_x) + p) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int p = p0 + u * kThreads + threadIdx.x;
          uint32_t w;
          uint8_t s;
          write8(v[u], w, s, odd);
          if (p >= n) continue;
          reinterpret_cast<uint32_t*>(codes)[at_c + p] = w;
          if (p % 2 == 0) scales[(at_c + p) / 2] = s;
        }
      } else {
        uint32_t w[kAtOnce];
        uint8_t s[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int p = min(p0 + u * kThreads + (int)threadIdx.x, n - 1);
          w[u] = __ldcs(reinterpret_cast<const uint32_t*>(codes) + at_c + p);
          s[u] = __ldcs(scales + (at_c + p) / 2);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int p = p0 + u * kThreads + threadIdx.x;
          if (p < n) __stcs(reinterpret_cast<uint4*>(x + at_x) + p, read8(w[u], s[u]));
        }
      }
    }
  }
  if (WRITE && __any_sync(~0u, odd) && threadIdx.x % 32 == 0 && a.err) atomicOr(a.err, kErrNotFinite);
}

}  // namespace

cudaError_t launch_pack4(const Pack4Args& a, int head_dim, bool write, int max_entries, cudaStream_t st) {
  const int64_t pieces = (int64_t)max_entries * (head_dim / 8), each = kThreads * kAtOnce;
  const int64_t units = std::min<int64_t>(a.units, 65535);
  const int64_t x = std::max<int64_t>(1, std::min<int64_t>((pieces + each - 1) / each, (kBlocks * device_sms() + units - 1) / units));
  auto* kernel = head_dim == 128 ? (write ? pack4_kernel<128, true> : pack4_kernel<128, false>)
                                 : (write ? pack4_kernel<64, true> : pack4_kernel<64, false>);
  return launch_pdl(kernel, dim3((unsigned)x, (unsigned)units, 2), dim3(kThreads), 0, st, 1, a);
}

}  // namespace as2d
