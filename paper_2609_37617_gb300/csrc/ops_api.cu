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
// the most entries a request can have by the host's bound; limit: the most rows of
// a request; tile: the fewest queries of an item.
as2d_status check_rows(const as2d_cache* c, int32_t layer, const as2d_tree_rows* r, TreeArgs& a,
                       int64_t& max_keys, int32_t limit = kMaxTree, int tile = 64) {
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
    if (r->rows[b] < 0 || r->rows[b] > limit)
      return invalid(limit == kMaxTree ? "rows must be in [0, AS2D_MAX_TREE]" : "rows must be >= 0");
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
  if ((a.rm.rows * G / tile + c->batch) * c->n_kv * tiles > 0x7fffffff)
    return report_error(AS2D_ERR_UNSUPPORTED, "too many heads, rows and positions");
  return AS2D_OK;
}

// A cache in 4 bits, as one in bf16 of the same sizes.
as2d_status check_cache4(const as2d_cache4* c, bool data, as2d_cache& sizes) {
  if (!c) return invalid("cache is NULL");
  sizes = {c->k, c->v, c->n_layers, c->batch, c->n_kv, c->capacity, c->head_dim};
  const as2d_status st = check_cache(&sizes, data);
  if (st != AS2D_OK) return st;
  if (data && (!c->k_scale || !c->v_scale)) return invalid("a scale pointer is NULL");
  if (data && (!aligned(c->k_scale, 8) || !aligned(c->v_scale, 8))) return invalid("scales must be 8-byte aligned");
  return AS2D_OK;
}

// Checks of the rows of a projection and q_out, for a cache of these sizes.
as2d_status check_new_rows(const as2d_cache* c, int32_t layer, const as2d_new_rows* r, const void* q_out,
                           const int32_t* error_bits, AppendArgs& a) {
  if (layer < 0 || layer >= c->n_layers) return invalid("layer outside [0, n_layers)");
  if (!r || !r->kv_len || !r->rows) return invalid("rows, its kv_len and its rows are required");
  if (r->type != AS2D_TYPE_BF16 && r->type != AS2D_TYPE_F32) return invalid("type is no AS2D_TYPE_*");
  if (r->n_q < 1) return invalid("n_q must be positive");
  if (r->n_q > 65535) return report_error(AS2D_ERR_UNSUPPORTED, "too many query heads");
  const int d = c->head_dim;
  if (r->rotary < 0 || r->rotary > d || r->rotary % 32 != 0)
    return invalid("rotary must be a multiple of 32 in [0, head_dim]");
  if (r->rotary > 0 && (!(r->theta > 0.f) || !std::isfinite(r->theta))) return invalid("theta must be finite and > 0");
  if ((r->q_norm || r->k_norm) && (!(r->eps >= 0.f) || !std::isfinite(r->eps)))
    return invalid("eps must be finite and >= 0");
  a.rm.batch = c->batch;
  a.rm.start[0] = 0;
  int64_t total = 0;
  for (int b = 0; b < c->batch; ++b) {
    if (r->rows[b] < 0) return invalid("rows must be >= 0");
    if (r->rows[b] > c->capacity) return report_error(AS2D_ERR_CAPACITY, "more rows than the capacity");
    total += r->rows[b];
    a.rm.start[b + 1] = (int32_t)total;
  }
  a.rm.rows = (int32_t)total;
  if (total > (1 << 24)) return report_error(AS2D_ERR_UNSUPPORTED, "more than 2^24 rows");
  if (total > 0 && (!r->q || !r->k || !r->v || !q_out)) return invalid("q, k, v and q_out are required");
  const int64_t size = r->type == AS2D_TYPE_F32 ? 4 : 2;
  if (r->q_stride < (int64_t)r->n_q * d || r->k_stride < (int64_t)c->n_kv * d || r->v_stride < (int64_t)c->n_kv * d)
    return invalid("a row's stride is less than its heads");
  for (int64_t stride : {r->q_stride, r->k_stride, r->v_stride})
    if (stride > INT64_MAX / (8 << 24) || stride * size % 16 != 0)
      return invalid("strides in bytes must be multiples of 16");
  for (const void* p : {r->q, r->k, r->v, q_out, (const void*)r->q_norm, (const void*)r->k_norm})
    if (!aligned(p, 16)) return invalid("q, k, v, q_out and gains must be 16-byte aligned");
  for (const void* p : {(const void*)r->kv_len, (const void*)r->positions, (const void*)error_bits})
    if (!aligned(p, 4)) return invalid("kv_len, positions and error_bits must be 4-byte aligned");
  a.len = r->kv_len;
  a.positions = r->positions;
  a.cap = c->capacity;
  a.nq = r->n_q;
  a.nkv = c->n_kv;
  a.q = r->q;
  a.k = r->k;
  a.v = r->v;
  a.q_stride = r->q_stride;
  a.k_stride = r->k_stride;
  a.v_stride = r->v_stride;
  a.q_out = const_cast<void*>(q_out);
  a.q_norm = r->q_norm;
  a.k_norm = r->k_norm;
  a.eps = r->eps;
  a.half = r->rotary / 2;
  a.err = const_cast<int32_t*>(error_bits);
  // theta^(-2j / rotary) / 2 pi of a turn modulo 1, in 2^-64 of one: a product of the powers
  // for the bits of j, each rounded once
  double power[6], f[64];
  for (int i = 0; (1 << i) < a.half; ++i) power[i] = std::pow((double)r->theta, -(double)(1 << i) / a.half);
  for (int j = 0; j < a.half; ++j) {
    f[j] = j == 0 ? 1.0 : f[j & (j - 1)] * power[__builtin_ctz(j)];
    const double turns = f[j] * 0.15915494309189533577;
    a.turn[j] = (uint64_t)std::ldexp(turns - std::floor(turns), 64);
  }
  return AS2D_OK;
}

// What as2d_cache4_write and as2d_cache4_read are given.
as2d_status pack4(const as2d_cache4* c4, const as2d_cache* c, int32_t layer, const int32_t* start, const int32_t* end,
                  int32_t max_entries, int32_t* error_bits, bool write, void* stream, const char* what) {
  as2d_cache sizes;
  as2d_status st = check_cache4(c4, true, sizes);
  if (st == AS2D_OK) st = check_cache(c, true);
  if (st != AS2D_OK) return st;
  if (c->n_layers != c4->n_layers || c->batch != c4->batch || c->n_kv != c4->n_kv || c->head_dim != c4->head_dim)
    return invalid("the caches' sizes differ in more than the capacity");
  if (layer < -1 || layer >= c->n_layers) return invalid("layer outside [-1, n_layers)");
  if (!end) return invalid("end is required");
  if (!aligned(start, 4) || !aligned(end, 4) || !aligned(error_bits, 4))
    return invalid("start, end and error_bits must be 4-byte aligned");
  const int32_t most = c->capacity < c4->capacity ? c->capacity : c4->capacity;
  if (max_entries < 0 || max_entries > most) return invalid("max_entries outside [0, capacity]");
  const int64_t of_layer = (int64_t)c->batch * c->n_kv, first = layer > 0 ? layer * of_layer : 0;
  const int d = c->head_dim;
  Pack4Args a{};
  a.k = (bf16*)c->k + first * c->capacity * d;
  a.v = (bf16*)c->v + first * c->capacity * d;
  a.k4 = c4->k + first * c4->capacity * (d / 2);
  a.v4 = c4->v + first * c4->capacity * (d / 2);
  a.ks = c4->k_scale + first * c4->capacity * (d / 16);
  a.vs = c4->v_scale + first * c4->capacity * (d / 16);
  a.start = start;
  a.end = end;
  a.batch = c->batch;
  a.nkv = c->n_kv;
  a.cap = c->capacity;
  a.cap4 = c4->capacity;
  a.units = layer >= 0 ? of_layer : of_layer * c->n_layers;
  a.err = error_bits;
  return launched(launch_pack4(a, d, write, max_entries > 0 ? max_entries : most, (cudaStream_t)stream), what);
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

extern "C" as2d_status as2d_cache_append(const as2d_cache* cache, int32_t layer, const as2d_new_rows* rows,
                                         void* q_out, int32_t* error_bits, void* stream) {
  clear_error();
  as2d_status st = check_cache(cache, true);
  if (st != AS2D_OK) return st;
  AppendArgs a{};
  st = check_new_rows(cache, layer, rows, q_out, error_bits, a);
  if (st != AS2D_OK || a.rm.rows == 0) return st;
  const size_t at = (size_t)layer * cache->batch * cache->n_kv * cache->capacity * cache->head_dim;
  a.ck = (bf16*)cache->k + at;
  a.cv = (bf16*)cache->v + at;
  return launched(launch_append(a, cache->head_dim, rows->type == AS2D_TYPE_F32, (cudaStream_t)stream),
                  "as2d_cache_append");
}

extern "C" as2d_status as2d_cache4_append(const as2d_cache4* cache, int32_t layer, const as2d_new_rows* rows,
                                          void* q_out, int32_t* error_bits, void* stream) {
  clear_error();
  as2d_cache sizes;
  as2d_status st = check_cache4(cache, true, sizes);
  if (st != AS2D_OK) return st;
  AppendArgs a{};
  st = check_new_rows(&sizes, layer, rows, q_out, error_bits, a);
  if (st != AS2D_OK || a.rm.rows == 0) return st;
  const size_t at = (size_t)layer * cache->batch * cache->n_kv * cache->capacity;
  a.ck4 = cache->k + at * (cache->head_dim / 2);
  a.cv4 = cache->v + at * (cache->head_dim / 2);
  a.cks = cache->k_scale + at * (cache->head_dim / 16);
  a.cvs = cache->v_scale + at * (cache->head_dim / 16);
  return launched(launch_append(a, cache->head_dim, rows->type == AS2D_TYPE_F32, (cudaStream_t)stream),
                  "as2d_cache4_append");
}

extern "C" as2d_status as2d_cache4_write(const as2d_cache4* to, const as2d_cache* from, int32_t layer,
                                         const int32_t* start, const int32_t* end, int32_t max_entries,
                                         int32_t* error_bits, void* stream) {
  clear_error();
  return pack4(to, from, layer, start, end, max_entries, error_bits, true, stream, "as2d_cache4_write");
}

extern "C" as2d_status as2d_cache4_read(const as2d_cache4* from, const as2d_cache* to, int32_t layer,
                                        const int32_t* start, const int32_t* end, int32_t max_entries,
                                        int32_t* error_bits, void* stream) {
  clear_error();
  return pack4(from, to, layer, start, end, max_entries, error_bits, false, stream, "as2d_cache4_read");
}

extern "C" as2d_status as2d_cache4_attention_workspace(const as2d_cache4* cache, int64_t* bytes) {
  clear_error();
  as2d_cache sizes;
  const as2d_status st = check_cache4(cache, false, sizes);
  if (st != AS2D_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = (int64_t)attention4_workspace(cache->head_dim);
  return AS2D_OK;
}

extern "C" as2d_status as2d_cache4_attention(const as2d_cache4* cache, int32_t layer, const as2d_tree_rows* rows,
                                             void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                             int32_t* error_bits, void* stream) {
  clear_error();
  as2d_cache sizes;
  as2d_status st = check_cache4(cache, true, sizes);
  if (st != AS2D_OK) return st;
  Tree4Args a{};
  int64_t max_keys = 0;
  st = check_rows(&sizes, layer, rows, a.t, max_keys, kMaxTree, 8);
  if (st != AS2D_OK) return st;
  st = check_workspace(workspace, workspace_bytes, attention4_workspace(cache->head_dim));
  if (st != AS2D_OK) return st;
  if (a.t.rm.rows == 0) return AS2D_OK;
  if (!out || !aligned(out, 16)) return invalid("out must be 16-byte aligned");
  if (!aligned(lse, 4) || !aligned(error_bits, 4)) return invalid("lse and error_bits must be 4-byte aligned");
  const size_t at = (size_t)layer * cache->batch * cache->n_kv * cache->capacity;
  a.k = cache->k + at * (cache->head_dim / 2);
  a.v = cache->v + at * (cache->head_dim / 2);
  a.ks = cache->k_scale + at * (cache->head_dim / 16);
  a.vs = cache->v_scale + at * (cache->head_dim / 16);
  a.t.k = a.t.v = nullptr;
  a.t.out = out;
  a.t.lse = lse;
  a.t.err = error_bits;
  return launched(launch_attention4(a, cache->head_dim, max_keys, workspace, (cudaStream_t)stream),
                  "as2d_cache4_attention");
}

extern "C" as2d_status as2d_prompt_attention_workspace(const as2d_cache* cache, int64_t* bytes) {
  clear_error();
  const as2d_status st = check_cache(cache, false);
  if (st != AS2D_OK) return st;
  if (!bytes) return invalid("bytes is NULL");
  *bytes = (int64_t)prompt_attention_workspace(cache->head_dim);
  return AS2D_OK;
}

extern "C" as2d_status as2d_prompt_attention(const as2d_cache* cache, int32_t layer, const as2d_tree_rows* rows,
                                             void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                             int32_t* error_bits, void* stream) {
  clear_error();
  as2d_status st = check_cache(cache, true);
  if (st != AS2D_OK) return st;
  TreeArgs a{};
  int64_t max_keys = 0;
  st = check_rows(cache, layer, rows, a, max_keys, INT32_MAX, 256);
  if (st != AS2D_OK) return st;
  if (a.q_f32) return report_error(AS2D_ERR_UNSUPPORTED, "prompt attention takes bf16 queries");
  if (a.visible) return invalid("visible must be NULL: prompts are causal");
  if (a.rm.rows > (1 << 24)) return report_error(AS2D_ERR_UNSUPPORTED, "more than 2^24 rows");
  st = check_workspace(workspace, workspace_bytes, prompt_attention_workspace(cache->head_dim));
  if (st != AS2D_OK) return st;
  if (a.rm.rows == 0) return AS2D_OK;
  if (!out || !aligned(out, 32)) return invalid("out must be 32-byte aligned");
  if (!aligned(lse, 4) || !aligned(error_bits, 4)) return invalid("lse and error_bits must be 4-byte aligned");
  a.out = out;
  a.lse = lse;
  a.err = error_bits;
  return launched(launch_prompt_attention(a, cache->head_dim, max_keys, workspace, (cudaStream_t)stream),
                  "as2d_prompt_attention");
}
