// k_basic.cu -- the verification pass's small kernels: embedding gather (with
// the rotary table and the first projection's operand), the accept scan with
// the on-device state update, rollback, and a load-time conversion.
//
// Every reduction below runs in an order fixed by the reduced dimension alone
// (never by the number of rows in the call), so each row's result is bitwise
// the same whether it is the only row (a k = 0 decode step) or one of the
// k + 1 rows of a block: batched and sequential execution agree exactly, which
// is the pathwise-equivalence requirement of App. C.4 held bit for bit.
#include "as2d_internal.h"
#include "ptx_sm100.cuh"
#include "small_dev.cuh"

namespace as2d {
namespace {

// ---- embedding gather --------------------------------------------------------

// (cos, sin) of pos * theta^(-2e/d), e < d/2: angle and trigonometry in
// double, rounded once to float.
__device__ __forceinline__ float2 rope_angle(int pos, int e, int d, double theta) {
  const double ang = (double)pos * pow(theta, -2.0 * (double)e / (double)d);
  double sn, cs;
  sincos(ang, &sn, &cs);
  return make_float2((float)cs, (float)sn);
}

// The rotary table of every position of a state, built once at set-up.
__global__ void rope_table_kernel(float2* __restrict__ out, int d, double theta) {
  const int pos = blockIdx.x, e = threadIdx.x;
  out[(size_t)pos * (d / 2) + e] = rope_angle(pos, e, d, theta);
}

// Also writes the row's rotary table -- gathered from the state's table of
// every position when there is one (rope_full), else computed.
__global__ void __launch_bounds__(128) embed_kernel(
    RowMap m, const int32_t* __restrict__ cand, const int32_t* __restrict__ root,
    const int32_t* __restrict__ root_override, const bf16* __restrict__ E, int H, int V, float* __restrict__ h, int32_t* err, int32_t* bad,
    const int32_t* __restrict__ len, int cap, float2* __restrict__ rope,
    const float2* __restrict__ rope_full, int d, double theta, const float* __restrict__ g0,
    bf16* __restrict__ xn, float* __restrict__ ss, int ss_ld, const int32_t* __restrict__ depth,
    const int32_t* __restrict__ off) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  __shared__ float part[4];
  const int r = blockIdx.x;
  const int b = row_request(m, r);
  const int i = r - m.start[b];
  // the token and the length first: the table row's load waits for the token,
  // and nothing may stand between them
  int tok = (i == 0) ? (root_override ? root_override[b] : root[b]) : cand[m.start[b] - b + i - 1];
  const int L = len[b];
  // a row's place past the prefix (its depth in a tree), and the entries evicted
  // before it
  const int ahead = (depth ? depth[r] : i) + (off ? off[b] : 0);
  const bool bad_tok = tok < 0 || tok >= V;
  // a request whose length leaves no room for its rows is flagged and skipped
  // downstream (rows_fit); its rows take position 0's rotary entries
  const bool fits = rows_fit(L, m.start[b + 1] - m.start[b], cap);
  float2 cs = make_float2(0.f, 0.f);
  if ((int)threadIdx.x < d / 2) {
    // (the table holds the positions of a cache that nothing was evicted from)
    const int e = threadIdx.x, pos = fits ? L + ahead : 0;
    cs = rope_full && pos < cap ? rope_full[(size_t)pos * (d / 2) + e] : rope_angle(pos, e, d, theta);
  }
  if (bad_tok) tok = 0;
  embed_row_body(E + (size_t)tok * H, g0, H, r, ss_ld, h, xn, ss, threadIdx.x, 128, part, 0);
  if ((int)threadIdx.x < d / 2) rope[(size_t)r * (d / 2) + threadIdx.x] = cs;
  if (threadIdx.x == 0 && (!fits || bad_tok)) {
    atomicOr(err, (fits ? 0 : kErrCapacity) | (bad_tok ? kErrBadToken : 0));
    bad[b] = 1;
  }
}

// ---- accept scan + state update ---------------------------------------------------

// One warp per request (App. C.2): g_i from the packed maxima, the number of
// leading candidates equal to the greedy tokens by ballot, the correction by
// shuffle, then L += n + 1 and root = correction, all on the device.
__global__ void accept_kernel(AcceptArgs a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  accept_request(a, blockIdx.x, threadIdx.x);
}

// A prefill of several passes runs the LM head over its last row alone.  If its
// last pass is flagged, the root is the greedy token after the last row that
// was kept: a pass before the last that is kept (kKeepFirst, kKeepNext) leaves
// the LM head's operand of its last row, and a flagged last pass (kKeepRestore)
// takes it up in the place of its own.
__global__ void __launch_bounds__(256) keep_row_kernel(int32_t op, const int32_t* bad, int32_t* kept,
                                                       bf16* xn, size_t lo, int H, float* ss, int ss_ld,
                                                       bf16* kept_x, float* kept_ss) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const bool flagged = *bad != 0, restore = op == kKeepRestore;
  if (threadIdx.x == 0 && !restore && (op == kKeepFirst || !flagged)) *kept = flagged ? 0 : 1;
  if (restore ? !(flagged && *kept) : flagged) return;
  for (int c = threadIdx.x; c < H; c += 256) {
    bf16 *x = xn + c, *k = kept_x + c;
    if (restore)
      x[0] = k[0], x[lo] = k[H];
    else
      k[0] = x[0], k[H] = x[lo];
  }
  for (int t = threadIdx.x; t < H / 128; t += 256) {
    if (restore)
      ss[(size_t)t * ss_ld] = kept_ss[t];
    else
      kept_ss[t] = ss[(size_t)t * ss_ld];
  }
}

// ---- trees -----------------------------------------------------------------------

// One warp per request, lane i its row i (row 0 the root): a row's depth and the
// rows it sees, itself and its ancestors, from its parent's.  A parent that is
// no earlier row flags the request; its rows are then taken as a chain.
__global__ void tree_plan_kernel(RowMap m, const int32_t* __restrict__ parents, uint64_t* __restrict__ visible,
                                 int32_t* __restrict__ depth, int32_t* err, int32_t* bad) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int b = blockIdx.x, lane = threadIdx.x, r0 = m.start[b], rows = m.start[b + 1] - r0;
  const bool node = lane > 0 && lane < rows;
  const int up = node ? parents[r0 - b + lane - 1] : 0;
  const bool wrong = __any_sync(0xFFFFFFFFu, node && (up < 0 || up >= lane));
  uint32_t sees = 1u << lane;
  int d = 0;
  for (int i = 1; i < rows; ++i) {  // (a parent's row is done before its children's)
    const int p = wrong ? i - 1 : __shfl_sync(0xFFFFFFFFu, up, i);
    const uint32_t of = __shfl_sync(0xFFFFFFFFu, sees, p);
    const int dp = __shfl_sync(0xFFFFFFFFu, d, p);
    if (lane == i) sees |= of, d = dp + 1;
  }
  if (lane < rows) {
    visible[r0 + lane] = sees;
    depth[r0 + lane] = d;
  }
  if (wrong && lane == 0) {
    atomicOr(err, kErrBadTree);
    bad[b] = 1;
  }
}

struct AcceptTreeArgs {
  RowMap rm;
  const int32_t *cand, *parents;
  unsigned long long* best;
  int32_t *len, *root, *bad;
  int32_t *n_out, *corr_out, *greedy_out;
  int32_t *path, *path_out, *from;
};

// One warp per request: from the root down, the candidate below the last one
// accepted that equals the greedy token there (the first, if several do).
__global__ void accept_tree_kernel(AcceptTreeArgs a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int b = blockIdx.x, lane = threadIdx.x, r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0;
  const unsigned long long v = lane < rows ? a.best[r0 + lane] : 0ull;
  const bool node = lane > 0 && lane < rows;
  const int cand = node ? a.cand[r0 - b + lane - 1] : -1, up = node ? a.parents[r0 - b + lane - 1] : -1;
  const int bad = a.bad[b], len = a.len[b];
  const int g = (int)(0xFFFFFFFFu - (uint32_t)(v & 0xFFFFFFFFull));
  if (lane < rows) {
    a.best[r0 + lane] = 0ull;
    if (a.greedy_out) a.greedy_out[r0 + lane] = g;
  }
  int at = 0, n = 0, mine = -1;  // mine: the (lane + 1)th accepted
  if (!bad)
    for (;; ++n) {
      const int want = __shfl_sync(0xFFFFFFFFu, g, at);
      const unsigned m = __ballot_sync(0xFFFFFFFFu, node && up == at && cand == want);
      if (!m) break;
      at = __ffs(m) - 1;
      if (lane == n) mine = at;
    }
  const int corr = __shfl_sync(0xFFFFFFFFu, g, at);
  const bool moves = __any_sync(0xFFFFFFFFu, mine >= 0 && mine != lane + 1);
  if (lane < kMaxK) {
    a.path[b * kMaxK + lane] = mine;
    if (a.path_out) a.path_out[b * kMaxK + lane] = mine;
  }
  if (lane == 0) {
    a.from[b] = moves ? len : -1;
    a.n_out[b] = bad ? -1 : n;
    a.corr_out[b] = bad ? -1 : corr;
    if (bad) {
      a.bad[b] = 0;
    } else {
      a.len[b] = len + n + 1;
      a.root[b] = corr;
    }
  }
}

// The accepted candidates' entries, at from + path[j], to from + 1 + j, where a chain
// would have put them; a thread per 16 bytes of (layer, request, kv head, cache),
// and one for the tracked weights of a head.  path ascends, so every entry is
// read before its place is written.
template <int D>
__global__ void __launch_bounds__(128) keep_path_kernel(const int32_t* __restrict__ path, const int32_t* __restrict__ from,
                                                        int batch, int nkv, int cap, int units, bf16* kc, bf16* vc,
                                                        float* weights) {
  constexpr int C = D / 8, P = 2 * C, U = 128 / P;  // pieces of an entry, of both caches, units of a CTA
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int unit = blockIdx.x * U + threadIdx.x / P, c = threadIdx.x % P;
  if (unit >= units) return;
  const int b = (unit / nkv) % batch, L = from[b];
  if (L < 0) return;
  const int32_t* rows = path + b * kMaxK;
  uint4* x = reinterpret_cast<uint4*>((c < C ? kc : vc) + ((size_t)unit * cap + L) * D) + c % C;
  float* w = weights && c == 0 ? weights + (size_t)unit * cap + L : nullptr;
  for (int j = 0; j < kMaxK; ++j) {
    const int r = rows[j];
    if (r < 0) break;
    x[(size_t)(1 + j) * C] = x[(size_t)r * C];
    if (w) w[1 + j] = w[r];
  }
}

// ---- sampled acceptance: the state update ------------------------------------------

struct CommitArgs {
  RowMap rm;
  unsigned long long* best;
  int32_t *len, *root, *bad, *err;
  int32_t *n_out, *corr_out, *greedy_out;
};

__global__ void commit_sampled_kernel(CommitArgs a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int b = blockIdx.x, lane = threadIdx.x, r0 = a.rm.start[b], rows = a.rm.start[b + 1] - r0;
  if (lane < rows) {
    const unsigned long long v = a.best[r0 + lane];
    a.best[r0 + lane] = 0ull;
    if (a.greedy_out) a.greedy_out[r0 + lane] = (int)(0xFFFFFFFFu - (uint32_t)(v & 0xFFFFFFFFull));
  }
  if (lane != 0) return;
  const int n = a.n_out[b], token = a.corr_out[b], bad = a.bad[b];
  if (bad || token < 0) {
    if (!bad) atomicOr(a.err, kErrNoToken);
    a.n_out[b] = -1;
    a.corr_out[b] = -1;
    a.bad[b] = 0;
  } else {
    a.len[b] += n + 1;
    a.root[b] = token;
  }
}

struct KeepArgs {
  int32_t batch, cap;
  int32_t keep[kMaxBatch];
};

__global__ void note_evict_kernel(KeepArgs a, const int32_t* len, int32_t* off, int32_t* floor) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int b = threadIdx.x;
  if (b >= a.batch) return;
  const int L = len[b];
  if (L > a.keep[b] && L <= a.cap) {
    off[b] += L - a.keep[b];
    floor[b] = a.keep[b];
  }
}

struct RollbackArgs {
  int32_t batch;
  int32_t len[kMaxBatch];
  int32_t root[kMaxBatch];
};

__global__ void rollback_kernel(RollbackArgs a, int32_t* len, int32_t* root,
                                int32_t* err, const int32_t* floor) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  int b = threadIdx.x;
  if (b >= a.batch) return;
  if (a.len[b] <= len[b] && a.len[b] >= floor[b]) {
    len[b] = a.len[b];
    root[b] = a.root[b];
  } else {
    atomicOr(err, kErrRollback);
  }
}

__global__ void f32_from_bf16_kernel(float* dst, const bf16* src, int64_t n) {
  int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) dst[i] = __bfloat162float(src[i]);
}

}  // namespace

// ---- launchers ------------------------------------------------------------------------

cudaError_t launch_embed(const RowMap& m, const Model& md, KvState& kv,
                         const int32_t* cand, cudaStream_t st, const int32_t* root_override,
                         const int32_t* depth) {
  ++kv.launches;
  return launch_pdl(embed_kernel, dim3(m.rows), dim3(128), 0, st, 1, m, cand,
                    (const int32_t*)kv.d_root, root_override, (const bf16*)md.embed, md.cfg.hidden,
                    md.cfg.vocab, kv.h, kv.d_err, kv.d_err + 1, (const int32_t*)kv.d_len,
                    kv.capacity, kv.rope, (const float2*)kv.rope_full, md.cfg.head_dim,
                    (double)md.cfg.rope_theta, md.attn_norm[0], kv.xn, kv.ss, kv.rows_alloc, depth,
                    (const int32_t*)kv.d_off);
}

cudaError_t launch_rope_table(const Model& md, KvState& kv, cudaStream_t st) {
  rope_table_kernel<<<kv.capacity, md.cfg.head_dim / 2, 0, st>>>(
      kv.rope_full, md.cfg.head_dim, (double)md.cfg.rope_theta);
  return cudaGetLastError();
}

cudaError_t launch_accept(const RowMap& m, const Model& md, KvState& kv,
                          const int32_t* cand, const as2d_verify_out& out,
                          cudaStream_t st, AcceptMode mode, bool kept_root) {
  (void)md;
  ++kv.launches;
  AcceptArgs a{m, cand, kv.best, kv.d_len, kv.d_root, kv.d_err + 1, out.n_accepted,
               out.correction_token, out.greedy, mode, kept_root ? kv.kept : nullptr};
  return launch_pdl(accept_kernel, dim3(m.batch), dim3(32), 0, st, 1, a);
}

cudaError_t launch_tree_plan(const RowMap& m, const Model& md, KvState& kv, const int32_t* parents,
                             cudaStream_t st) {
  (void)md;
  ++kv.launches;
  return launch_pdl(tree_plan_kernel, dim3(m.batch), dim3(32), 0, st, 1, m, parents, kv.tree_visible, kv.tree_depth,
                    kv.d_err, kv.d_err + 1);
}

cudaError_t launch_accept_tree(const RowMap& m, const Model& md, KvState& kv, const int32_t* cand, const TreeCall& t,
                               const as2d_verify_out& out, cudaStream_t st) {
  kv.launches += 2;
  AcceptTreeArgs a{m, cand, t.parents, kv.best, kv.d_len, kv.d_root, kv.d_err + 1, out.n_accepted,
                   out.correction_token, out.greedy, kv.tree_path, t.path, kv.tree_from};
  const cudaError_t e = launch_pdl(accept_tree_kernel, dim3(m.batch), dim3(32), 0, st, 1, a);
  if (e != cudaSuccess) return e;
  const int units = md.cfg.n_layers * kv.batch * md.cfg.n_kv_heads, per = 128 / (md.cfg.head_dim / 4);
  const dim3 grid((units + per - 1) / per);
  auto kernel = md.cfg.head_dim == 128 ? keep_path_kernel<128> : keep_path_kernel<64>;
  return launch_pdl(kernel, grid, dim3(128), 0, st, 1, (const int32_t*)kv.tree_path, (const int32_t*)kv.tree_from,
                    kv.batch, md.cfg.n_kv_heads, kv.capacity, units, kv.k_cache, kv.v_cache, kv.track);
}

cudaError_t launch_commit_sampled(const RowMap& m, KvState& kv, const as2d_verify_out& out, cudaStream_t st) {
  ++kv.launches;
  CommitArgs a{m, kv.best, kv.d_len, kv.d_root, kv.d_err + 1, kv.d_err, out.n_accepted, out.correction_token,
               out.greedy};
  return launch_pdl(commit_sampled_kernel, dim3(m.batch), dim3(32), 0, st, 1, a);
}

cudaError_t launch_note_evict(KvState& kv, const int32_t* keep, cudaStream_t st) {
  KeepArgs a{kv.batch, kv.capacity, {}};
  for (int b = 0; b < kv.batch; ++b) a.keep[b] = keep[b];
  return launch_pdl(note_evict_kernel, dim3(1), dim3(kMaxBatch), 0, st, 1, a, (const int32_t*)kv.d_len, kv.d_off,
                    kv.d_floor);
}

cudaError_t launch_keep_row(const Model& md, KvState& kv, KeepRow op, int row, cudaStream_t st) {
  ++kv.launches;
  const int H = md.cfg.hidden;
  return launch_pdl(keep_row_kernel, dim3(1), dim3(256), 0, st, 1, (int32_t)op,
                    (const int32_t*)(kv.d_err + 1), kv.kept, kv.xn + (size_t)row * H,
                    (size_t)kv.rows_alloc * H, H, kv.ss + row, kv.rows_alloc, kv.kept_x, kv.kept_ss);
}

cudaError_t launch_rollback(KvState& kv, const int32_t* new_len,
                            const int32_t* new_root, cudaStream_t st) {
  RollbackArgs a;
  a.batch = kv.batch;
  for (int b = 0; b < kv.batch; ++b) {
    a.len[b] = new_len[b];
    a.root[b] = new_root[b];
  }
  return launch_pdl(rollback_kernel, dim3(1), dim3(kMaxBatch), 0, st, 1, a, kv.d_len, kv.d_root,
                    kv.d_err, (const int32_t*)kv.d_floor);
}

cudaError_t launch_f32_from_bf16(float* dst, const void* src, int64_t n,
                                 cudaStream_t st) {
  f32_from_bf16_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(
      dst, (const bf16*)src, n);
  return cudaGetLastError();
}

}  // namespace as2d
