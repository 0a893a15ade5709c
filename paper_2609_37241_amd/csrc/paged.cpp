// Entry points of the paged KV cache: the step's bookkeeping, the store of new
// K and V, attention over pages. Same path as the other ops: validate, pack
// the guard key, look the version up, launch.
#include "paged_entry.h"

using namespace tri;

namespace {

AttnPlan plan_of(const tri_attention_args &a, uint64_t workspace) {
  return attn_plan(uint32_t(a.dtype), a.T, a.R, a.nq, a.kv.nk, a.kv.hd,
                   attn_aligned(a, es_of(uint32_t(a.dtype))), attn_keys(a), workspace);
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
  const int st = attn_check(a, true, es_of(uint32_t(a.dtype)));
  if (st != kGo) return finish_early(c, op, st);
  const uint64_t es = es_of(uint32_t(a.dtype));
  const AttnPlan plan = plan_of(a, uint64_t(a.workspace_bytes));
  if (!plan.grid[0]) return finish_early(c, op, TRI_E_UNSUPPORTED);
  Key k = make_key(op, uint32_t(a.dtype), a.T, attn_aligned(a, es) ? kAlign : 0u, 0, 0, 0,
                   uint64_t(a.kv.hd), uint64_t(a.nq), uint64_t(a.kv.nk));
  k.k3 = (uint64_t(plan.form) << 16) | (uint64_t(plan.splits > 1) << 24);
  // K and V that outgrow the last-level cache do not stay for the next call:
  // where one tile reads them they are streamed (PA_ROWS; 64 requests of up to
  // 8k tokens, 8 K heads of 128 in bf16, 1 GB: 214 -> 193 us; 262 MB: 52 -> 56;
  // three tiles over 1 GB in float32, 195 -> 223)
  const PagedArgs args = attn_args(a, plan, weight_scale(a.scale), attn_outgrows(a, es));
  return run_paged(c, op, k, a.T, plan.grid, plan.splits > 1 ? 2 : 1, plan.block, &args, sizeof args,
                   stream);
}

int64_t tri_paged_attention_workspace(const tri_attention_args *p) {
  if (!p || attn_check(*p, false, 0) != kGo) return 0;
  const AttnPlan plan = plan_of(*p, ~uint64_t(0));
  return int64_t(attn_workspace(p->T, p->nq, p->kv.hd, plan.splits));
}

}  // extern "C"
