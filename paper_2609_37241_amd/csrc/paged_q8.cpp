// Entry points of the paged KV cache in 8 bits: rows into it and out of it, attention
// over it. The same path as over the other caches.
#include "paged_entry.h"

using namespace tri;

namespace {

// The scales of a cache: code, block, pointers and their alignment, strides.
int check_q8(const tri_kv_q8 &q, const tri_kv_cache &c) {
  if ((q.code != TRI_INT8 && q.code != TRI_E4M3) || q.block < 1 || c.page % q.block)
    return TRI_E_INVALID;
  if (!q.k_scale || !q.v_scale || (addr(q.k_scale) | addr(q.v_scale)) % 4) return TRI_E_INVALID;
  const int64_t n = c.page / q.block;
  return view_ok({q.k_ps, c.n_pages}, {q.k_bs, n}, {q.k_hs, c.nk}, 1, 4) &&
                 view_ok({q.v_ps, c.n_pages}, {q.v_bs, n}, {q.v_hs, c.nk}, 1, 4)
             ? int(kGo)
             : int(TRI_E_INVALID);
}

uint64_t key_code(const tri_kv_q8 &q) { return uint64_t(uint32_t(q.code)) << 32; }

tri_status rows_q8(tri_cache *c, uint32_t op, const tri_kv_rows_args *p, void *stream) {
  if (!c) return TRI_E_INVALID;
  c->stats.calls++;
  if (!p) return finish_early(c, op, TRI_E_INVALID);
  const tri_kv_rows_args &a = *p;
  int st = check_common(a.dtype, a.T);
  if (st != kGo) return finish_early(c, op, st);
  const uint64_t es = es_of(uint32_t(a.dtype));
  st = check_table(a.table, a.table_rs, a.R, a.cols, a.kv.page);
  if (st == kGo) st = check_kv(a.kv, 1);
  if (st == kGo) st = check_q8(a.q8, a.kv);
  if (st != kGo) return finish_early(c, op, st);
  const int64_t w = int64_t(a.kv.nk) * a.kv.hd;
  if (!a.k || !a.v || !a.kv_len || !a.q_start || (addr(a.k) | addr(a.v)) % es ||
      (addr(a.kv_len) | addr(a.q_start)) % 4 || a.k_ts < w || a.v_ts < w ||
      !extent_ok(a.T, a.k_ts, w, es) || !extent_ok(a.T, a.v_ts, w, es))
    return finish_early(c, op, TRI_E_INVALID);
  const bool write = op == TRI_OP_KV_WRITE_Q8;
  // what is written for K and for V at one place: codes or scales that fit neither
  if (write ? a.kv.k == a.kv.v || a.q8.k_scale == a.q8.v_scale : a.k == a.v)
    return finish_early(c, op, TRI_E_INVALID);
  // rows in 16-byte vectors, their codes in 4 or 8 bytes
  const uint64_t rows = addr(a.k) | addr(a.v) | (a.T > 1 ? uint64_t(a.k_ts | a.v_ts) * es : 0);
  const bool aligned = !(rows & 15u) && !(kv_bits(a.kv, 1) & (16 / es - 1));
  Key k = make_key(op, uint32_t(a.dtype), a.T, aligned ? kAlign : 0u, 0, 0, 0, uint64_t(a.kv.hd), 0,
                   uint64_t(a.kv.nk));
  const tri_kv_q8 &q = a.q8;
  const bool vec = aligned && a.kv.hd % vec_elems(uint32_t(a.dtype)) == 0;
  const int32_t per = a.kv.hd / int32_t(vec ? vec_elems(uint32_t(a.dtype)) : 1);
  // blocks that the rows can touch, by the two ways to number them
  const int64_t by_block = a.T / q.block + 2 * int64_t(a.R);
  const bool by_row = a.T <= by_block;
  const int64_t units = by_row ? a.T : by_block;
  // the rows that a block gets, were the requests equal
  const int64_t rows_each = (a.T + a.R - 1) / a.R < q.block ? (a.T + a.R - 1) / a.R : q.block;
  const uint32_t team = write && vec ? q8_write_team(rows_each * per) : 1;
  const uint32_t inner = write && team == 0 ? q8_write_inner(units, a.kv.nk) : 1;
  k.k3 = key_code(q) | (write && vec ? uint64_t(team) << 16 : 0);
  const Q8RowsArgs args{a.k, a.v, {a.kv.k, a.kv.k_ps, a.kv.k_ss, a.kv.k_hs},
                        {a.kv.v, a.kv.v_ps, a.kv.v_ss, a.kv.v_hs},
                        {q.k_scale, q.k_ps, q.k_bs, q.k_hs}, {q.v_scale, q.v_ps, q.v_bs, q.v_hs},
                        a.table, a.kv_len, a.q_start, a.k_ts, a.v_ts, a.table_rs, int32_t(a.T), a.R,
                        a.cols, a.kv.n_pages, a.kv.page, a.kv.nk, a.kv.hd, q.block,
                        fast_div_of(uint32_t(a.kv.page)), fast_div_of(uint32_t(q.block)),
                        fast_div_of(uint32_t(per)), per,
                        int32_t(units), by_row, inner};
  const uint32_t grid = write ? q8_write_grid(units, a.kv.nk, team, inner) : q8_read_grid(a.T);
  return run_paged(c, op, k, a.T, &grid, 1, kBlock, &args, sizeof args, stream);
}

AttnPlan plan_of(const tri_attention_args &a, uint64_t workspace) {
  return attn_q8_plan(uint32_t(a.dtype), a.T, a.R, a.nq, a.kv.nk, a.kv.hd, attn_aligned(a, 1),
                      attn_keys(a), int64_t(a.cols) * a.kv.page, workspace);
}

}  // namespace

extern "C" {

tri_status tri_kv_write_quant(tri_cache *c, const tri_kv_rows_args *p, void *stream) {
  return rows_q8(c, TRI_OP_KV_WRITE_Q8, p, stream);
}

tri_status tri_kv_read_quant(tri_cache *c, const tri_kv_rows_args *p, void *stream) {
  return rows_q8(c, TRI_OP_KV_READ_Q8, p, stream);
}

tri_status tri_paged_attention_quant(tri_cache *c, const tri_attention_args *p, const tri_kv_q8 *q8,
                                  void *stream) {
  if (!c) return TRI_E_INVALID;
  const uint32_t op = TRI_OP_PAGED_ATTENTION_Q8;
  c->stats.calls++;
  if (!p) return finish_early(c, op, TRI_E_INVALID);
  const tri_attention_args &a = *p;
  int st = attn_check(a, true, 1);
  if (st == kGo) st = q8 ? check_q8(*q8, a.kv) : int(TRI_E_INVALID);
  if (st != kGo) return finish_early(c, op, st);
  const AttnPlan plan = plan_of(a, uint64_t(a.workspace_bytes));
  if (!plan.grid[0]) return finish_early(c, op, TRI_E_UNSUPPORTED);
  Key k = make_key(op, uint32_t(a.dtype), a.T, attn_aligned(a, 1) ? kAlign : 0u, 0, 0, 0,
                   uint64_t(a.kv.hd), uint64_t(a.nq), uint64_t(a.kv.nk));
  k.k3 = (uint64_t(plan.form) << 16) | (uint64_t(plan.splits > 1) << 24) |
         (uint64_t(plan.heads) << 25) | key_code(*q8);
  // (no `stream`: PA8_ROWS streams always, see there; the other forms never)
  const PagedQ8Args args{attn_args(a, plan, 1.0f, false),
                         {q8->k_scale, q8->k_ps, q8->k_bs, q8->k_hs},
                         {q8->v_scale, q8->v_ps, q8->v_bs, q8->v_hs},
                         weight_scale(a.scale), q8->block, fast_div_of(uint32_t(q8->block)),
                         int32_t(plan.grid[0]),
                         plan.step_shift, q8_join_four(a.T, a.nq),
                         int32_t(0x7FFFFFFF / (a.kv.nk >> plan.heads))};
  return run_paged(c, op, k, a.T, plan.grid, plan.splits > 1 ? 2 : 1, plan.block, &args, sizeof args,
                   stream);
}

int64_t tri_paged_attention_quant_workspace(const tri_attention_args *p) {
  if (!p || attn_check(*p, false, 1) != kGo) return 0;
  const AttnPlan plan = plan_of(*p, ~uint64_t(0));
  return int64_t(attn_workspace(p->T, p->nq, p->kv.hd, plan.splits));
}

}  // extern "C"
