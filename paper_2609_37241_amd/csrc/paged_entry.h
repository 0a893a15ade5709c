// What the entry points of the paged KV cache share: checks of caches, tables and
// attention calls, and the run of a paged op's launches.
#pragma once
#include <math.h>

#include <utility>

#include "entry.h"

namespace tri {
namespace {

// A tensor of three dimensions d (stride, extent) whose items are `width` neighbouring
// elements: the strides, taken from the shortest up, must each leave room for
// what lies below (a dimension of one has no stride), so no two items
// overlap; the whole within kSpanMax bytes.
typedef std::pair<int64_t, int64_t> Dim;
inline bool view_ok(Dim x, Dim y, Dim z, int64_t width, uint64_t es) {
  Dim d[3] = {x, y, z};
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j)   // one without extent comes first
      if (d[i].second != 1 && (d[j].second == 1 || d[j].first < d[i].first)) std::swap(d[i], d[j]);
    if (d[i].second == 1) continue;
    if (d[i].first < width || !extent_ok(d[i].second, d[i].first, width, es)) return false;
    width = (d[i].second - 1) * d[i].first + width;
  }
  return true;
}

// The cache of a call: sizes, pointers and their alignment, strides.
inline int check_kv(const tri_kv_cache &c, uint64_t es) {
  if (c.n_pages < 1 || c.page < 1 || c.nk < 1 || c.hd < 1) return TRI_E_INVALID;
  if (c.page > TRI_MAX_PAGE || c.nk > kHeadsMax || c.hd > kAttnHdMax) return TRI_E_UNSUPPORTED;
  if (!c.k || !c.v || (addr(c.k) | addr(c.v)) % es) return TRI_E_INVALID;
  if (!view_ok({c.k_ps, c.n_pages}, {c.k_ss, c.page}, {c.k_hs, c.nk}, c.hd, es) ||
      !view_ok({c.v_ps, c.n_pages}, {c.v_ss, c.page}, {c.v_hs, c.nk}, c.hd, es))
    return TRI_E_INVALID;
  return kGo;
}

// Every slot of the cache starts at a multiple of 16 bytes (the stride of a
// dimension of one does not count).
inline uint64_t kv_bits(const tri_kv_cache &c, uint64_t es) {
  return addr(c.k) | addr(c.v) | (c.n_pages > 1 ? uint64_t(c.k_ps | c.v_ps) * es : 0) |
         (c.page > 1 ? uint64_t(c.k_ss | c.v_ss) * es : 0) |
         (c.nk > 1 ? uint64_t(c.k_hs | c.v_hs) * es : 0);
}

// A block table: width, row stride over R rows of `cols` entries, positions
// below 2^31.
inline int check_table(const void *table, int64_t rs, int32_t R, int32_t cols, int32_t page) {
  if (R < 1 || cols < 1 || page < 1) return TRI_E_INVALID;
  if (R > TRI_MAX_REQUESTS || page > TRI_MAX_PAGE || int64_t(cols) * page >= kPosLimit)
    return TRI_E_UNSUPPORTED;
  if (!table || addr(table) % 4) return TRI_E_INVALID;
  return rs < cols || !extent_ok(R, rs, cols, 4) ? int(TRI_E_INVALID) : int(kGo);
}

// Validation of an attention call: common, table, cache (elements of kv_es bytes),
// heads, q and out, lengths, scale, window and bound, workspace.
inline int attn_check(const tri_attention_args &a, bool pointers, uint64_t kv_es) {
  int st = check_common(a.dtype, a.T);
  if (st != kGo) return st;
  const uint64_t es = es_of(uint32_t(a.dtype));
  if (pointers) {
    st = check_table(a.table, a.table_rs, a.R, a.cols, a.kv.page);
    if (st != kGo) return st;
    st = check_kv(a.kv, kv_es);
    if (st != kGo) return st;
  } else if (a.R < 1 || a.cols < 1 || a.kv.page < 1 || a.kv.nk < 1 || a.kv.hd < 1 ||
             a.R > TRI_MAX_REQUESTS || a.kv.page > TRI_MAX_PAGE || a.kv.nk > kHeadsMax ||
             a.kv.hd > kAttnHdMax) {
    return TRI_E_INVALID;
  }
  if (int64_t(a.cols) * a.kv.page > kKeysMax) return TRI_E_UNSUPPORTED;
  if (a.nq < 1) return TRI_E_INVALID;
  if (a.nq > kHeadsMax || a.T * a.nq >= kPosLimit) return TRI_E_UNSUPPORTED;
  if (a.nq % a.kv.nk) return TRI_E_INVALID;
  const int64_t w = int64_t(a.nq) * a.kv.hd;
  if (pointers) {
    if (!a.q || !a.out || !a.kv_len || !a.q_start) return TRI_E_INVALID;
    if ((addr(a.q) | addr(a.out)) % es || (addr(a.kv_len) | addr(a.q_start)) % 4)
      return TRI_E_INVALID;
    if (a.q_ts < w || a.o_ts < w || !extent_ok(a.T, a.q_ts, w, es) ||
        !extent_ok(a.T, a.o_ts, w, es))
      return TRI_E_INVALID;
    if (!isfinite(a.scale)) return TRI_E_INVALID;
    if (a.workspace_bytes < 0 || addr(a.workspace) % 16 || (a.workspace_bytes && !a.workspace))
      return TRI_E_INVALID;
  }
  if (a.window < 0 || a.max_kv < 0) return TRI_E_INVALID;
  return kGo;
}

// The most keys a row can see.
inline int64_t attn_keys(const tri_attention_args &a) {
  int64_t n = int64_t(a.cols) * a.kv.page;
  if (a.max_kv && a.max_kv < n) n = a.max_kv;
  if (a.window && a.window < n) n = a.window;
  return n;
}

inline bool attn_aligned(const tri_attention_args &a, uint64_t kv_es) {
  const uint64_t es = es_of(uint32_t(a.dtype));
  return ((addr(a.q) | addr(a.out) | (a.T > 1 ? uint64_t(a.q_ts | a.o_ts) * es : 0) |
           kv_bits(a.kv, kv_es)) &
          15u) == 0;
}

// Whether one tile of each request reads all its keys, and these, in elements of kv_es
// bytes, outgrow the last-level cache.
inline bool attn_outgrows(const tri_attention_args &a, uint64_t kv_es) {
  const double bytes = 2.0 * double(a.R) * double(attn_keys(a)) * double(a.kv.nk) *
                       double(a.kv.hd) * double(kv_es);   // (up to 2^67)
  return bytes > double(kCacheBytes) && (a.T + a.R - 1) / a.R * (a.nq / a.kv.nk) <= 16;
}

// |scale| log2 e: the weights are 2^(c (q.k - maximum)); for 0 the least float32 above
// it: 2^128 of it is 2^-21, so all weights are 1 but for a masked score's, which
// stays -inf.
inline float weight_scale(float scale) {
  const float c2 = float(fabs(double(scale)) * 1.4426950408889634);
  if (!(c2 >= 0x1p-149f)) return 0x1p-149f;
  return !(c2 <= 3e38f) ? 3e38f : c2;
}

inline PagedArgs attn_args(const tri_attention_args &a, const AttnPlan &plan, float c2, bool stream) {
  const int32_t g = a.nq / a.kv.nk;
  float *part = static_cast<float *>(a.workspace);
  return {a.q, a.out, {a.kv.k, a.kv.k_ps, a.kv.k_ss, a.kv.k_hs},
          {a.kv.v, a.kv.v_ps, a.kv.v_ss, a.kv.v_hs}, a.table, a.kv_len, a.q_start,
          plan.splits > 1 ? part : nullptr,
          plan.splits > 1 ? part + a.T * a.nq * plan.splits * a.kv.hd : nullptr,
          a.q_ts, a.o_ts, a.table_rs, int32_t(a.T), a.R, a.cols, a.kv.n_pages,
          a.kv.page, a.nq, a.kv.nk, a.kv.hd, g, plan.splits, plan.tiles, a.window,
          c2, uint16_t(a.scale < 0.0f), uint16_t(stream), fast_div_of(uint32_t(a.kv.page)),
          fast_div_of(uint32_t(g))};
}

// The launches of a paged op (`block` work-items a workgroup the first, 256
// any other), in order, stopping at the first failure. On a miss, installed by
// the call itself or not, they are kept for tri_spec_install_last_miss.
inline tri_status run_paged(tri_cache *c, uint32_t op, const Key &k, int64_t T, const uint32_t *grid,
                     int n, uint32_t block, const void *args, uint32_t size, void *stream) {
  int32_t vi;
  bool auto_inst = false;
  const int st = lookup(c, op, k, T, &vi, &auto_inst);
  if (st != TRI_OK || auto_inst) {
    for (int i = 0; i < 2; ++i) c->miss_grid[i] = i < n ? grid[i] : 0;
    c->miss_block = block;
  }
  if (st != TRI_OK) return tri_status(st);
  Version &v = c->versions[vi];
  tri_launch_rec l[3];
  int rc = 0;
  for (int i = 0; i < v.plan.n_launches; ++i) {
    l[i] = {v.plan.kvariant[i], grid[i], i == 0 ? block : kBlock};
    if (rc == 0)
      rc = launch(c, v, i, key_dtype(k), grid[i], l[i].block_x, args, size, stream);
  }
  record(c, op, v, vi, k, v.plan.n_launches, l, rc ? TRI_E_LAUNCH : TRI_OK);
  return finish(c, v, auto_inst, rc);
}

}  // namespace
}  // namespace tri
