// ops_api.cu -- entry points of the operators on caches and logits: argument
// checks and launches (include/as2d.h, "Operators on caches and logits").
#include <cmath>

#include "ops.h"

using namespace as2d;

namespace {

as2d_status invalid(const char* msg) { return report_error(AS2D_ERR_INVALID_ARG, msg); }

constexpr int kMaxOpVocab = 1 << 24;

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

as2d_status launched(cudaError_t e, const char* what) {
  return e == cudaSuccess ? AS2D_OK : report_error(AS2D_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

as2d_status check_cache(const as2d_cache* c, bool data) {
  if (!c) return invalid("cache is NULL");
  if (c->n_layers < 1 || c->batch < 1 || c->n_kv < 1 || c->capacity < 1)
    return invalid("the cache's sizes must be positive");
  if (c->batch > kMaxBatch) return invalid("batch must be in [1, AS2D_MAX_BATCH]");
  if (c->head_dim != 64 && c->head_dim != 128)
    return report_error(AS2D_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (c->capacity > 65536)
    return report_error(AS2D_ERR_UNSUPPORTED, "capacity above 65536 positions is not supported");
  if ((int64_t)c->n_layers * c->batch * c->n_kv > (1 << 30) || c->n_kv > 65535)
    return report_error(AS2D_ERR_UNSUPPORTED, "too many heads");
  if (data && (!c->k || !c->v)) return invalid("a cache pointer is NULL");
  if (data && (!aligned(c->k, 16) || !aligned(c->v, 16))) return invalid("the caches must be 16-byte aligned");
  return AS2D_OK;
}

// Checks of the rows of a call, and its arguments but for outputs.  max_keys:
// the most entries a request can have by the host's bound.
as2d_status check_rows(const as2d_cache* c, int32_t layer, const as2d_tree_rows* r, TreeArgs& a,
                       int64_t& max_keys) {
  as2d_status st = check_cache(c, true);
  if (st != AS2D_OK) return st;
  if (layer < 0 || layer >= c->n_layers) return invalid("layer outside [0, n_layers)");
  if (!r || !r->kv_len || !r->rows) return invalid("rows, its kv_len and its rows are required");
  if (r->q_type != AS2D_TYPE_BF16 && r->q_type != AS2D_TYPE_F32) return invalid("q_type is no AS2D_TYPE_*");
  if (r->n_q < 1 || r->n_q % c->n_kv != 0) return invalid("n_q must be a positive multiple of n_kv");
  if (r->n_q / c->n_kv > 1024 || r->n_q > 65535) return report_error(AS2D_ERR_UNSUPPORTED, "too many query heads");
  if (!(r->scale > 0.f) || !std::isfinite(r->scale * 1.4426950408889634f))
    return invalid("scale must be > 0 and scale log2(e) finite");
  if (r->max_len < 0 || r->max_len > c->capacity) return invalid("max_len outside [0, capacity]");
  a.rm.batch = c->batch;
  a.rm.start[0] = 0;
  int most = 0;
  for (int b = 0; b < c->batch; ++b) {
    if (r->rows[b] < 0 || r->rows[b] > kMaxTree) return invalid("rows must be in [0, AS2D_MAX_TREE]");
    if (r->rows[b] > c->capacity) return report_error(AS2D_ERR_CAPACITY, "more rows than the capacity");
    a.rm.start[b + 1] = a.rm.start[b] + r->rows[b];
    if (r->rows[b] > most) most = r->rows[b];
  }
  a.rm.rows = a.rm.start[c->batch];
  const int64_t size = r->q_type == AS2D_TYPE_F32 ? 4 : 2;
  if (a.rm.rows > 0 && !r->q) return invalid("q is NULL");
  if (r->q_stride < (int64_t)r->n_q * c->head_dim) return invalid("q_stride is less than n_q head_dim");
  if (!aligned(r->q, 16) || r->q_stride * size % 16 != 0)
    return invalid("q and q_stride in bytes must be multiples of 16");
  if (!aligned(r->visible, 8)) return invalid("visible must be 8-byte aligned");
  if (!aligned(r->kv_len, 4)) return invalid("kv_len must be 4-byte aligned");
  a.len = r->kv_len;
  a.cap = c->capacity;
  a.nq = r->n_q;
  a.nkv = c->n_kv;
  a.group_inv = group_inverse(a.nq, a.nkv);
  a.q = r->q;
  a.q_f32 = r->q_type == AS2D_TYPE_F32;
  a.q_stride = r->q_stride;
  a.visible = r->visible;
  a.scale_log2 = r->scale * 1.4426950408889634f;
  const size_t at = (size_t)layer * c->batch * c->n_kv * c->capacity * c->head_dim;
  a.k = (const bf16*)c->k + at;
  a.v = (const bf16*)c->v + at;
  max_keys = (r->max_len > 0 ? r->max_len : c->capacity) + most;
  if (max_keys > c->capacity) max_keys = c->capacity;
  // units of work (tiles, and up to eight for each turn), counted in 32 bits on the device
  const int64_t tiles = (c->capacity + 127) / 128 + 8, G = r->n_q / c->n_kv;
  if ((a.rm.rows * G / 64 + c->batch) * c->n_kv * tiles > 0x7fffffff)
    return report_error(AS2D_ERR_UNSUPPORTED, "too many heads, rows and positions");
  return AS2D_OK;
}

as2d_status check_workspace(const void* workspace, int64_t bytes, size_t need) {
  if (!workspace || !aligned(workspace, 256)) return invalid("the workspace must be 256-byte aligned");
  if (bytes < 0 || (uint64_t)bytes < need) return invalid("the workspace is too small");
  return AS2D_OK;
}

}  // namespace

extern "C" as2d_status as2d_tree_attention_workspace(const as2d_cache* cache, int64_t* bytes) {
  clear_error();
  const as2d_status st = check_cache(cache, false);
  if (st != AS2D_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = (int64_t)tree_attention_workspace(cache->head_dim);
  return AS2D_OK;
}

extern "C" as2d_status as2d_tree_attention(const as2d_cache* cache, int32_t layer,
                                           const as2d_tree_rows* rows, void* out, float* lse,
                                           void* workspace, int64_t workspace_bytes,
                                           int32_t* error_bits, void* stream) {
  clear_error();
  TreeArgs a{};
  int64_t max_keys = 0;
  as2d_status st = check_rows(cache, layer, rows, a, max_keys);
  if (st != AS2D_OK) return st;
  st = check_workspace(workspace, workspace_bytes, tree_attention_workspace(cache->head_dim));
  if (st != AS2D_OK) return st;
  if (a.rm.rows == 0) return AS2D_OK;
  if (!out || !aligned(out, 16)) return invalid("out must be 16-byte aligned");
  if (!aligned(lse, 4) || !aligned(error_bits, 4)) return invalid("lse and error_bits must be 4-byte aligned");
  a.out = out;
  a.lse = lse;
  a.err = error_bits;
  return launched(launch_tree_attention(a, cache->head_dim, max_keys, workspace, (cudaStream_t)stream),
                  "as2d_tree_attention");
}

extern "C" as2d_status as2d_attention_weights(const as2d_cache* cache, int32_t layer,
                                              const as2d_tree_rows* rows, const float* lse,
                                              float* weights, int32_t* error_bits, void* stream) {
  clear_error();
  WeightArgs a{};
  int64_t max_keys = 0;
  const as2d_status st = check_rows(cache, layer, rows, a.t, max_keys);
  if (st != AS2D_OK) return st;
  if (a.t.rm.rows == 0) return AS2D_OK;
  if (!lse || !weights) return invalid("lse and weights are required");
  if (!aligned(lse, 4) || !aligned(weights, 4) || !aligned(error_bits, 4))
    return invalid("lse, weights and error_bits must be 4-byte aligned");
  a.t.lse = const_cast<float*>(lse);
  a.t.err = error_bits;
  a.w = weights + (size_t)layer * cache->batch * cache->n_kv * cache->capacity;
  return launched(launch_attention_weights(a, cache->head_dim, max_keys, (cudaStream_t)stream),
                  "as2d_attention_weights");
}

extern "C" as2d_status as2d_cache_evict_workspace(const as2d_cache* cache, int64_t* bytes) {
  clear_error();
  const as2d_status st = check_cache(cache, false);
  if (st != AS2D_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = (int64_t)cache_evict_workspace((int64_t)cache->n_layers * cache->batch * cache->n_kv, cache->capacity);
  return AS2D_OK;
}

extern "C" as2d_status as2d_cache_evict(const as2d_cache* cache, float* weights, int32_t* kv_len,
                                        const int32_t* keep, int32_t recent, void* workspace,
                                        int64_t workspace_bytes, void* stream) {
  clear_error();
  as2d_status st = check_cache(cache, true);
  if (st != AS2D_OK) return st;
  if (!weights || !kv_len || !keep) return invalid("weights, kv_len and keep are required");
  if (!aligned(weights, 4) || !aligned(kv_len, 4)) return invalid("weights and kv_len must be 4-byte aligned");
  if (recent < 0) return invalid("recent must be >= 0");
  const int64_t units = (int64_t)cache->n_layers * cache->batch * cache->n_kv;
  st = check_workspace(workspace, workspace_bytes, cache_evict_workspace(units, cache->capacity));
  if (st != AS2D_OK) return st;
  EvictArgs a{};
  a.k = (bf16*)cache->k;
  a.v = (bf16*)cache->v;
  a.w = weights;
  a.len = kv_len;
  a.n_layers = cache->n_layers;
  a.batch = cache->batch;
  a.nkv = cache->n_kv;
  a.cap = cache->capacity;
  a.recent = recent;
  for (int b = 0; b < cache->batch; ++b) {
    if (keep[b] < 0) return invalid("keep must be >= 0");
    a.keep[b] = keep[b];
  }
  cache_evict_carve(a, units, workspace);
  return launched(launch_cache_evict(a, cache->head_dim, (cudaStream_t)stream), "as2d_cache_evict");
}

extern "C" as2d_status as2d_token_probs(const float* logits, int32_t n_rows, int32_t vocab,
                                        float temperature, float* probs, void* stream) {
  clear_error();
  if (n_rows < 0 || vocab < 1) return invalid("n_rows must be >= 0 and vocab >= 1");
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return invalid("temperature must be finite and > 0");
  if (vocab > kMaxOpVocab) return report_error(AS2D_ERR_UNSUPPORTED, "vocab above 2^24 is not supported");
  if (n_rows == 0) return AS2D_OK;
  if (!logits || !probs) return invalid("logits and probs are required");
  if (!aligned(logits, 4) || !aligned(probs, 4)) return invalid("logits and probs must be 4-byte aligned");
  return launched(launch_token_probs(logits, n_rows, vocab, temperature, probs, (cudaStream_t)stream),
                  "as2d_token_probs");
}

extern "C" as2d_status as2d_accept_sampled(const float* probs, const float* draft_probs,
                                           const int32_t* candidates, const int32_t* k, int32_t batch,
                                           int32_t vocab, const float* u, int32_t* n_accepted,
                                           int32_t* token, void* stream) {
  clear_error();
  if (!probs || !k || !u || !n_accepted || !token)
    return invalid("probs, k, u, n_accepted and token are required");
  for (const void* p : {(const void*)probs, (const void*)draft_probs, (const void*)candidates, (const void*)u,
                        (const void*)n_accepted, (const void*)token})
    if (!aligned(p, 4)) return invalid("the tensors of an acceptance must be 4-byte aligned");
  if (batch < 1 || batch > kMaxBatch) return invalid("batch must be in [1, AS2D_MAX_BATCH]");
  if (vocab < 1) return invalid("vocab must be >= 1");
  if (vocab > kMaxOpVocab) return report_error(AS2D_ERR_UNSUPPORTED, "vocab above 2^24 is not supported");
  SampledArgs a{};
  a.start[0] = 0;
  for (int b = 0; b < batch; ++b) {
    if (k[b] < 0 || k[b] > kMaxK) return invalid("k must be in [0, AS2D_MAX_K]");
    a.start[b + 1] = a.start[b] + k[b] + 1;
  }
  if (a.start[batch] > batch && !candidates) return invalid("candidates is NULL");
  a.probs = probs;
  a.draft = draft_probs;
  a.u = u;
  a.cand = candidates;
  a.batch = batch;
  a.vocab = vocab;
  a.n_out = n_accepted;
  a.token_out = token;
  return launched(launch_accept_sampled(a, (cudaStream_t)stream), "as2d_accept_sampled");
}
