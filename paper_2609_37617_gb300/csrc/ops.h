// ops.h -- launchers of the operators on caches and logits (include/as2d.h,
// "Operators on caches and logits"), shared by their entry points (ops_api.cu)
// and the state's calls (as2d_api.cu).
#pragma once

#include <atomic>

#include "as2d_internal.h"

namespace as2d {

// What is found out or set once per device (a kernel's attributes, how many of its
// clusters run at once): `ask` gives a value >= 0, asked again until it does.
struct PerDevice {
  std::atomic<int> value[64] = {};  // + 1; 0: not asked yet
  template <typename F>
  int get(F ask) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return -1;
    if (dev < 64)
      if (const int v = value[dev].load(std::memory_order_acquire)) return v - 1;
    const int v = ask();
    if (v >= 0 && dev < 64) value[dev].store(v + 1, std::memory_order_release);
    return v;
  }
};

// Opts a kernel into `smem` bytes of dynamic shared memory on the current device
// (and, with `big`, into clusters of more than eight).
template <typename K>
cudaError_t opt_in(PerDevice& done, K* kernel, int smem, bool big = false) {
  cudaError_t e = cudaSuccess;
  done.get([&] {
    if (smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && big) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e == cudaSuccess ? 0 : -1;
  });
  return e;
}

// Clusters of `ranks` CTAs of a kernel that run at once on the current device (0:
// not found out).
template <typename K>
int resident_clusters(PerDevice& known, K* kernel, int threads, int smem, int ranks) {
  const int n = known.get([&] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ranks * 256);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int most = 0;
    if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) == cudaSuccess) return most;
    (void)cudaGetLastError();
    return 0;
  });
  return n > 0 ? n : 0;
}

constexpr int kMaxTree = AS2D_MAX_TREE;

// The rows of a call (as2d_tree_rows) over one layer of a cache.
struct TreeArgs {
  RowMap rm;                // rows of each request; may be none
  const int32_t* len;       // device [batch]
  int cap, nq, nkv;
  uint32_t group_inv;       // 2^32 / (nq / nkv), rounded up (divide_group)
  const void* q;            // [rows][nq][d], rows q_stride elements apart
  int q_f32;
  int64_t q_stride;
  const uint64_t* visible;  // device [rows], or null: a chain
  float scale_log2;         // scale log2(e)
  const bf16* k;            // the layer's [batch][nkv][cap][d]
  const bf16* v;
  void* out;                // [rows][nq][d] of the queries' type
  bf16* out_lo;             // not null (32-bit queries): out takes bf16 hi parts, this the lo parts
  float* lse;               // [rows][nq], nullable
  int32_t* err;             // error bits, nullable
  unsigned long long timeout_ns = 2000000000ull;  // limit of the kernel's waits
};

inline uint32_t group_inverse(int nq, int nkv) {
  const uint32_t g = (uint32_t)(nq / nkv);
  return (uint32_t)(((1ull << 32) + g - 1) / g);  // (0 for 1)
}

struct WeightArgs {
  TreeArgs t;               // out and v unused; lse is read
  const int32_t* skip;      // device [batch], nullable: requests (not 0) whose rows add nothing
  float* w;                 // the layer's [batch][nkv][cap]
};

struct EvictArgs {
  bf16 *k, *v;              // [units][cap][d], unit = (layer batch + b) nkv + g
  float* w;                 // [units][cap]
  int32_t* len;             // device [batch]
  int n_layers, batch, nkv, cap, recent;
  int32_t keep[kMaxBatch];
  uint16_t* at;             // [units][cap] old position of each entry that stays
  int32_t* first;           // [units] entries before it stay where they are; -1: nothing moves
};

struct SampledArgs {
  const float *probs, *draft, *u;
  const int32_t* cand;
  int batch, vocab;
  int32_t start[kMaxBatch + 1];  // rows before request b (k + 1 each)
  int32_t *n_out, *token_out;
};

// Partial results of items of 128 queries that are cut between CTAs.
struct TreeWork {
  float4* o;   // [2 CTAs][D / 4][128] partial accumulators, four dims of a query
               // together: slot 0 an item that began in an earlier CTA, slot 1 one
               // that began in this
  float2* ml;  // [2 CTAs][128] (maximum base 2, sum)
};

// Rows of a projection for one layer of a cache, in bf16 or in 4 bits (as2d_new_rows).
struct AppendArgs {
  RowMap rm;
  const int32_t* len;       // device [batch]
  const int32_t* positions; // device [rows], or null: len + i
  int cap, nq, nkv;
  const void *q, *k, *v;    // [rows][heads][d], rows strides apart
  int64_t q_stride, k_stride, v_stride;
  void* q_out;              // [rows][nq][d]
  const float *q_norm, *k_norm;  // [d], nullable
  float eps;
  int half;                 // half of the rotated dims
  uint64_t turn[64];        // 2^64 times the turns a position makes, by dim of the first half
  bf16 *ck, *cv;            // the layer's [batch][nkv][cap][d]
  uint8_t *ck4, *cks, *cv4, *cvs;  // or, in 4 bits, codes and scales
  int32_t* err;             // error bits, nullable
};

struct Pack4Args {
  bf16 *k, *v;              // [units][cap][d]
  uint8_t *k4, *ks, *v4, *vs;  // [units][cap4][..]
  const int32_t *start, *end;  // device [batch]; start nullable
  int batch, nkv, cap, cap4;
  int64_t units;            // (layers batch nkv)
  int32_t* err;
};

// As TreeArgs of an attention over a cache in 4 bits (k and v unused).
struct Tree4Args {
  TreeArgs t;
  const uint8_t *k, *ks, *v, *vs;  // the layer's
};

// SMs of the current device; (request, kv head, tile of 128 queries) items of a call.
int device_sms();
int64_t tree_items(const TreeArgs& a);
// (launches, nullable: counts the kernels enqueued)
cudaError_t launch_tree_attention(const TreeArgs& a, int head_dim, int64_t max_keys, void* workspace,
                                  cudaStream_t st, int64_t* launches = nullptr);
size_t tree_attention_workspace(int head_dim);
TreeWork tree_work(void* workspace, int head_dim);
// The parts of items that `ctas` CTAs left by even shares of their units (make_plan), joined.
cudaError_t launch_tree_join(const TreeArgs& a, int head_dim, const TreeWork& ws, int ctas, int turn, cudaStream_t st);
cudaError_t launch_attention_weights(const WeightArgs& a, int head_dim, int64_t max_keys, cudaStream_t st);
cudaError_t launch_cache_evict(const EvictArgs& a, int head_dim, cudaStream_t st);
size_t cache_evict_workspace(int64_t units, int cap);
void cache_evict_carve(EvictArgs& a, int64_t units, void* workspace);
cudaError_t launch_token_probs(const float* logits, int rows, int vocab, float temperature, float* probs,
                               cudaStream_t st);
cudaError_t launch_accept_sampled(const SampledArgs& a, cudaStream_t st);
cudaError_t launch_append(const AppendArgs& a, int head_dim, bool f32, cudaStream_t st);
cudaError_t launch_pack4(const Pack4Args& a, int head_dim, bool write, int max_entries, cudaStream_t st);
cudaError_t launch_attention4(const Tree4Args& a, int head_dim, int64_t max_keys, void* workspace, cudaStream_t st);
cudaError_t launch_attention4_wide(const Tree4Args& a, int head_dim, int64_t max_keys, void* workspace, cudaStream_t st);
size_t attention4_workspace(int head_dim);
cudaError_t launch_prompt_attention(const TreeArgs& a, int head_dim, int64_t max_keys, void* workspace,
                                    cudaStream_t st);
size_t prompt_attention_workspace(int head_dim);

}  // namespace as2d
