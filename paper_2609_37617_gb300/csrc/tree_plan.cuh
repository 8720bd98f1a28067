// tree_plan.cuh -- how the rows of a call over a cache are cut into items and
// units and spread over CTAs, from the lengths on the device (k_tree_attn.cu,
// k_attn_weights.cu).
//
// An item is one (request, kv head, query tile), a unit one tile of 128 keys of
// an item or, at its head, one of `extra` units that stand for what a CTA spends on
// turning to another item (its queries, its epilogue): a CTA that ends one item
// and begins another gets fewer tiles.  Items and their units are numbered request
// by request, kv head by kv head, query tile by query tile (the query tiles of a
// head read its keys one after another, from L2).
#pragma once

#include "ops.h"

namespace as2d {

struct alignas(16) UnitPlan {
  int extra;                      // units of an item that are no tiles
  int unit[kMaxBatch + 1];  // units before each request (the host refuses calls of 2^31)
  int len[kMaxBatch];
  int tiles[kMaxBatch];           // key tiles of a request's items
  int qts[kMaxBatch];             // query tiles of a request
};

// q / G for the G query heads of a kv head: exact for q < 2^16, G <= 2^10 (the
// inverse is off by less than 1, q times that by less than 2^32 / G).
__device__ __forceinline__ int divide_group(const TreeArgs& a, int q) {
  return a.group_inv == 0 ? q : (int)__umulhi((uint32_t)q, a.group_inv);
}

// What a CTA does of one item: key tiles [t0, t1) of it.
struct Unit {
  int b, g, qt, tiles, t0, t1;
  int L, rows, r0;
  int next;
};

// Filled by one warp; requests without rows, or whose length leaves no room for
// theirs, or that skip (device [batch], nullable) names, have no units.
__device__ __forceinline__ void make_plan(const TreeArgs& a, int q_tile, int extra, int lane, UnitPlan& p, bool flag,
                                          const int32_t* skip = nullptr) {
  const int G = a.nq / a.nkv;
  int before = 0;
  bool over = false;
#pragma unroll
  for (int h = 0; h < kMaxBatch / 32; ++h) {
    const int b = 32 * h + lane;
    int L = 0, tiles = 0, qts = 0;
    if (b < a.rm.batch) {
      const int rows = a.rm.start[b + 1] - a.rm.start[b];
      L = a.len[b];
      qts = (rows * G + q_tile - 1) / q_tile;
      if (rows > 0 && rows_fit(L, rows, a.cap))
        tiles = skip && skip[b] ? 0 : (L + rows + 127) / 128;
      else
        over = over || rows > 0;
    }
    const int n = tiles > 0 ? a.nkv * qts * (tiles + extra) : 0;
    int at = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(~0u, at, o);
      if (lane >= o) at += t;
    }
    p.unit[b] = before + at - n;
    p.len[b] = L;
    p.tiles[b] = tiles;
    p.qts[b] = qts;
    before += __shfl_sync(~0u, at, 31);
  }
  if (lane == 0) p.unit[kMaxBatch] = before, p.extra = extra;
  if (flag && __any_sync(~0u, over) && lane == 0 && a.err) atomicOr(a.err, kErrCapacity);
}

// Units [u0, u1) of CTA c: even shares of all of them (one more for the first
// CTAs, and no more CTAs than units).
__device__ __forceinline__ void unit_range(const UnitPlan& p, int c, int ctas, int& u0, int& u1) {
  const int n = p.unit[kMaxBatch], of = min(ctas, n);
  u0 = u1 = 0;
  if (c >= of) return;
  const int each = n / of, more = n - each * of;
  u0 = c * each + min(c, more);
  u1 = u0 + each + (c < more ? 1 : 0);
}
// The CTA that does unit u.
__device__ __forceinline__ int unit_owner(const UnitPlan& p, int u, int ctas) {
  const int n = p.unit[kMaxBatch], of = min(ctas, n);
  const int each = n / of, more = n - each * of, wide = more * (each + 1);
  return u < wide ? u / (each + 1) : more + (u - wide) / each;
}

// What is done of unit u's item (of request lo) from u on, up to unit u1 at most;
// `next`: the first unit after that.  May hold no tile.
__device__ __forceinline__ Unit unit_of(const UnitPlan& p, const TreeArgs& a, int lo, int u, int u1) {
  Unit it;
  it.b = lo;
  it.tiles = p.tiles[lo];
  it.L = p.len[lo];
  it.r0 = a.rm.start[lo];
  it.rows = a.rm.start[lo + 1] - it.r0;
  const int per = it.tiles + p.extra, rel = u - p.unit[lo], item = rel / per, at = rel - item * per;
  it.g = item / p.qts[lo];
  it.qt = item - it.g * p.qts[lo];
  const int end = min(per, at + u1 - u);
  it.next = u + end - at;
  it.t0 = max(at - p.extra, 0);
  it.t1 = max(end - p.extra, 0);
  return it;
}

__device__ __forceinline__ Unit unit_at(const UnitPlan& p, const TreeArgs& a, int u, int u1) {
  int lo = 0, hi = kMaxBatch - 1;  // the last request whose first unit is at or before u
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.unit[mid] <= u)
      lo = mid;
    else
      hi = mid - 1;
  }
  return unit_of(p, a, lo, u, u1);
}

// The same of the first item from u on of which there is a tile to do; u: the first
// unit after it.  False past unit u1.  (Not inlined: the kernels' roles run it once
// an item each, and are short of instruction cache.)
static __device__ __noinline__ bool next_item(const UnitPlan& p, const TreeArgs& a, int& u, int u1, Unit& it) {
  while (u < u1) {
    it = unit_at(p, a, u, u1);
    u = it.next;
    if (it.t0 < it.t1) return true;
  }
  return false;
}

// By a whole warp: the last request whose first unit is at or before u.
__device__ __forceinline__ int request_of(const UnitPlan& p, int u, int lane) {
  int lo = -1;
#pragma unroll
  for (int h = 0; h < kMaxBatch / 32; ++h) lo += __popc(__ballot_sync(~0u, p.unit[32 * h + lane] <= u));
  return lo;
}
// A CTA's share and its first item (rows 0: none), found by the warp that made the
// plan for all of them: each on its own spent 1 us on it.
struct First {
  Unit it;
  int u1;
};
__device__ __forceinline__ void first_item(const UnitPlan& p, const TreeArgs& a, int c, int ctas, int lane, First& f) {
  __syncwarp();
  int u0, u1;
  unit_range(p, c, ctas, u0, u1);
  const int lo = request_of(p, u0, lane);
  Unit it;
  it.rows = 0;
  if (u0 < u1) {
    it = unit_of(p, a, lo, u0, u1);
    int u = it.next;
    if (it.t0 >= it.t1 && !next_item(p, a, u, u1, it)) it.rows = 0;
  }
  if (lane == 0) f.it = it, f.u1 = u1;
}

// ln of a sum l of powers of two relative to 2^M; -inf of nothing.
__device__ __forceinline__ float row_lse(float M, float l) {
  return l == 0.f ? -INFINITY : (M + log2f(l)) * 0.69314718055994531f;
}

}  // namespace as2d
