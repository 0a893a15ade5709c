// Entry points of the paged KV cache: the step's bookkeeping, the store of new
// K and V, attention over pages. Same path as the other ops: validate, pack
// the guard key, look the version up, launch.
#include <math.h>

#include <utility>

#include "entry.h"

using namespace tri;

namespace {

// One of K and V: its three strides, taken from the shortest up, must each
// leave room for what lies below (a dimension of one has no stride), so no two
// slots overlap; the whole within kSpanMax bytes.
bool view_ok(const tri_kv_cache &c, int64_t ps, int64_t ss, int64_t hs, uint64_t es) {
  std::pair<int64_t, int64_t> d[3] = {{ps, c.n_pages}, {ss, c.page}, {hs, c.nk}};
  int64_t width = c.hd;
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
int check_kv(const tri_kv_cache &c, uint64_t es) {
  if (c.n_pages < 1 || c.page < 1 || c.nk < 1 || c.hd < 1) return TRI_E_INVALID;
  if (c.page > TRI_MAX_PAGE || c.nk > kHeadsMax || c.hd > kAttnHdMax) return TRI_E_UNSUPPORTED;
  if (!c.k || !c.v || (addr(c.k) | addr(c.v)) % es) return TRI_E_INVALID;
  if (!view_ok(c, c.k_ps, c.k_ss, c.k_hs, es) || !view_ok(c, c.v_ps, c.v_ss, c.v_hs, es))
    return TRI_E_INVALID;
  return kGo;
}

// Every slot of the cache starts at a multiple of 16 bytes (the stride of a
// dimension of one does not count).
uint64_t kv_bits(const tri_kv_cache &c, uint64_t es) {
  return addr(c.k) | addr(c.v) | (c.n_pages > 1 ? uint64_t(c.k_ps | c.v_ps) * es : 0) |
         (c.page > 1 ? uint64_t(c.k_ss | c.v_ss) * es : 0) |
         (c.nk > 1 ? uint64_t(c.k_hs | c.v_hs) * es : 0);
}

// A block table: width, row stride over R rows of `cols` entries, positions
// below 2^31.
int check_table(const void *table, int64_t rs, int32_t R, int32_t cols, int32_t page) {
  if (R < 1 || cols < 1 || page < 1) return TRI_E_INVALID;
  if (R > TRI_MAX_REQUESTS || page > TRI_MAX_PAGE || int64_t(cols) * page >= kPosLimit)
    return TRI_E_UNSUPPORTED;
  if (!table || addr(table) % 4) return TRI_E_INVALID;
  return rs < cols || !extent_ok(R, rs, cols, 4) ? int(TRI_E_INVALID) : int(kGo);
}

// Validation of an attention call: common, table, cache, heads, q and out,
// lengths, scale, window and bound, workspace.
int attn_check(const tri_attention_args &a, bool pointers) {
  int st = check_common(a.dtype, a.T);
  if (st != kGo) return st;
  const uint64_t es = es_of(uint32_t(a.dtype));
  if (pointers) {
    st = check_table(a.table, a.table_rs, a.R, a.cols, a.kv.page);
    if (st != kGo) return st;
    st = check_kv(a.kv, es);
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
int64_t attn_keys(const tri_attention_args &a) {
  int64_t n = int64_t(a.cols) * a.kv.page;
  if (a.max_kv && a.max_kv < n) n = a.max_kv;
  if (a.window && a.window < n) n = a.window;
  return n;
}

bool attn_aligned(const tri_attention_args &a) {
  const uint64_t es = es_of(uint32_t(a.dtype));
  return ((addr(a.q) | addr(a.out) | (a.T > 1 ? uint64_t(a.q_ts | a.o_ts) * es : 0) |
           kv_bits(a.kv, es)) &
          15u) == 0;
}

AttnPlan plan_of(const tri_attention_args &a, uint64_t workspace) {
  return attn_plan(uint32_t(a.dtype), a.T, a.R, a.nq, a.kv.nk, a.kv.hd, attn_aligned(a),
                   attn_keys(a), workspace);
}

// The launches of a paged op (`block` work-items a workgroup the first, 256
// any other), in order, stopping at the first failure. On a miss, installed by
// the call itself or not, they are kept for tri_spec_install_last_miss.
tri_status run_paged(tri_cache *c, uint32_t op, const Key &k, int64_t T, const uint32_t *grid,
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

extern "C" {

tri_status tri_kv_slots(tri_cache *c, const tri_kv_slots_args *p, void *stream) {
  if (!c) return TRI_E_INVALID;
  const uint32_t op = TRI_OP_KV_SLOTS;
  c->stats.calls++;
  if (!p) return finish_early(c, op, TRI_E_INVALID);
  const tri_kv_slots_args &a = *p;
  // T is the room in slots and pos: without any, lengths and pages are done all
  // the same
  int st = check_common(TRI_F32, a.T);
  if (st != kGo && a.T != 0) return finish_early(c, op, st);
  st = check_table(a.table, a.table_rs, a.R, a.cols, a.page);
  if (st != kGo) return finish_early(c, op, st);
  if (int64_t(a.R) * a.cols >= kPosLimit) return finish_early(c, op, TRI_E_UNSUPPORTED);
  if (a.n_free < 0 || !a.kv_len || !a.new_len || !a.free_count || (a.n_free && !a.free_pages) ||
      (a.T && (!a.slots || !a.pos)) || !a.q_start || !a.kv_len_out || !a.free_out)
    return finish_early(c, op, TRI_E_INVALID);
  if ((addr(a.kv_len) | addr(a.new_len) | addr(a.free_count) | addr(a.free_pages) | addr(a.pos) |
       addr(a.q_start) | addr(a.kv_len_out) | addr(a.free_out)) % 4 || addr(a.slots) % 8)
    return finish_early(c, op, TRI_E_INVALID);
  // what is read while it is written elsewhere: lengths, counts, the stack
  struct Span {
    uint64_t b, e;
  };
  const auto span = [](const void *q, uint64_t bytes) { return Span{addr(q), addr(q) + bytes}; };
  const uint64_t n = uint64_t(a.R);
  const Span in[4] = {span(a.kv_len, 4 * n), span(a.new_len, 4 * n), span(a.free_count, 4),
                      span(a.free_pages, 4 * uint64_t(a.n_free))};
  const Span out[6] = {span(a.table, 4 * ((n - 1) * uint64_t(a.table_rs) + uint64_t(a.cols))),
                       span(a.slots, 8 * uint64_t(a.T)), span(a.pos, 4 * uint64_t(a.T)),
                       span(a.q_start, 4 * (n + 1)), span(a.kv_len_out, 4 * n),
                       span(a.free_out, 8)};
  const auto meet = [](const Span &x, const Span &y) { return x.b < y.e && y.b < x.e; };
  for (int i = 0; i < 6; ++i) {
    for (int j = i + 1; j < 6; ++j)
      if (meet(out[i], out[j])) return finish_early(c, op, TRI_E_INVALID);
    for (int j = 0; j < 4; ++j)
      if (meet(out[i], in[j])) return finish_early(c, op, TRI_E_INVALID);
  }
  const Key k = make_key(op, 0, a.T, 0, 0, 0, 0, 0, 0, 0);
  const KvSlotsArgs args{a.kv_len, a.new_len, a.table, a.free_pages, a.free_count, a.slots, a.pos,
                         a.q_start, a.kv_len_out, a.free_out, a.T, a.table_rs, a.R, a.page,
                         a.cols, a.n_free, fast_div_of(uint32_t(a.page))};
  const uint32_t grid = kv_slots_grid(a.T, a.R);
  return run_paged(c, op, k, a.T, &grid, 1, kBlock, &args, sizeof args, stream);
}

tri_status tri_kv_write(tri_cache *c, tri_dtype dtype, const void *k, int64_t k_ts, const void *v,
                        int64_t v_ts, const int64_t *slots, int64_t T, const tri_kv_cache *kv,
                        void *stream) {
  if (!c) return TRI_E_INVALID;
  const uint32_t op = TRI_OP_KV_WRITE;
  c->stats.calls++;
  int st = check_common(dtype, T);
  if (st != kGo) return finish_early(c, op, st);
  if (!kv) return finish_early(c, op, TRI_E_INVALID);
  const uint64_t es = es_of(dtype);
  st = check_kv(*kv, es);
  if (st != kGo) return finish_early(c, op, st);
  const int64_t w = int64_t(kv->nk) * kv->hd;
  if (!k || !v || !slots || (addr(k) | addr(v)) % es || addr(slots) % 8)
    return finish_early(c, op, TRI_E_INVALID);
  if (k_ts < w || v_ts < w || !extent_ok(T, k_ts, w, es) || !extent_ok(T, v_ts, w, es))
    return finish_early(c, op, TRI_E_INVALID);
  const uint64_t bits =
      addr(k) | addr(v) | (T > 1 ? uint64_t(k_ts | v_ts) * es : 0) | kv_bits(*kv, es);
  const Key key = make_key(op, dtype, T, bits & 15u ? 0u : kAlign, 0, 0, 0, uint64_t(kv->hd), 0,
                           uint64_t(kv->nk));
  const bool vec = !(bits & 15u) && kv->hd % vec_elems(dtype) == 0;
  const uint32_t items = uint32_t(2 * w / (vec ? vec_elems(dtype) : 1));
  const KvWriteArgs args{k, v, slots, {kv->k, kv->k_ps, kv->k_ss, kv->k_hs},
                         {kv->v, kv->v_ps, kv->v_ss, kv->v_hs}, k_ts, v_ts, T,
                         int64_t(kv->n_pages) * kv->page, kv->page, kv->nk, kv->hd,
                         fast_div_of(uint32_t(kv->page)), fast_div_of(items), items};
  const uint32_t grid = kv_write_grid(T, items);
  return run_paged(c, op, key, T, &grid, 1, kBlock, &args, sizeof args, stream);
}

tri_status tri_paged_attention(tri_cache *c, const tri_attention_args *p, void *stream) {
  if (!c) return TRI_E_INVALID;
  const uint32_t op = TRI_OP_PAGED_ATTENTION;
  c->stats.calls++;
  if (!p) return finish_early(c, op, TRI_E_INVALID);
  const tri_attention_args &a = *p;
  const int st = attn_check(a, true);
  if (st != kGo) return finish_early(c, op, st);
  const AttnPlan plan = plan_of(a, uint64_t(a.workspace_bytes));
  if (!plan.grid[0]) return finish_early(c, op, TRI_E_UNSUPPORTED);
  Key k = make_key(op, uint32_t(a.dtype), a.T, attn_aligned(a) ? kAlign : 0u, 0, 0, 0,
                   uint64_t(a.kv.hd), uint64_t(a.nq), uint64_t(a.kv.nk));
  k.k3 = (uint64_t(plan.form) << 16) | (uint64_t(plan.splits > 1) << 24);
  float *part = static_cast<float *>(a.workspace);
  // K and V that outgrow the last-level cache do not stay for the next call:
  // where one tile reads them they are streamed (PA_ROWS; 64 requests of up to
  // 8k tokens, 8 K heads of 128 in bf16, 1 GB: 214 -> 193 us; 262 MB: 52 -> 56;
  // three tiles over 1 GB in float32, 195 -> 223)
  const double bytes = 2.0 * double(a.R) * double(attn_keys(a)) * double(a.kv.nk) *
                       double(a.kv.hd) * double(es_of(uint32_t(a.dtype)));   // (up to 2^67)
  const bool large = bytes > double(kCacheBytes) && (a.T + a.R - 1) / a.R * (a.nq / a.kv.nk) <= 16;
  const int32_t g = a.nq / a.kv.nk;
  // the weights are 2^(c (q.k - maximum)), c = |scale| log2 e; for 0 the least
  // float32 above it: 2^128 of it is 2^-21, so all weights are 1 but for a masked
  // score's, which stays -inf
  float c2 = float(fabs(double(a.scale)) * 1.4426950408889634);
  if (!(c2 >= 0x1p-149f)) c2 = 0x1p-149f;
  if (!(c2 <= 3e38f)) c2 = 3e38f;
  const PagedArgs args{a.q, a.out, {a.kv.k, a.kv.k_ps, a.kv.k_ss, a.kv.k_hs},
                       {a.kv.v, a.kv.v_ps, a.kv.v_ss, a.kv.v_hs}, a.table, a.kv_len, a.q_start,
                       plan.splits > 1 ? part : nullptr,
                       plan.splits > 1 ? part + a.T * a.nq * plan.splits * a.kv.hd : nullptr,
                       a.q_ts, a.o_ts, a.table_rs, int32_t(a.T), a.R, a.cols, a.kv.n_pages,
                       a.kv.page, a.nq, a.kv.nk, a.kv.hd, g, plan.splits, plan.tiles, a.window,
                       c2, uint16_t(a.scale < 0.0f), uint16_t(large), fast_div_of(uint32_t(a.kv.page)),
                       fast_div_of(uint32_t(g))};
  return run_paged(c, op, k, a.T, plan.grid, plan.splits > 1 ? 2 : 1, plan.block, &args, sizeof args,
                   stream);
}

int64_t tri_paged_attention_workspace(const tri_attention_args *p) {
  if (!p || attn_check(*p, false) != kGo) return 0;
  const AttnPlan plan = plan_of(*p, ~uint64_t(0));
  return int64_t(attn_workspace(p->T, p->nq, p->kv.hd, plan.splits));
}

}  // extern "C"
