// What the op entry points share: status and argument checks, the guard key,
// lookup (with the miss path), the launch of one kernel of a version and the
// bookkeeping around it. Inline: each entry point is one straight path.
#pragma once
#include <string.h>

#include "internal.h"
#include "kernargs.h"

namespace tri {
namespace {

enum { kGo = 2 };   // validation passed, continue (distinct from every status)

inline uint64_t es_of(uint32_t dtype) { return dtype == TRI_F32 ? 4u : 2u; }
inline uint64_t addr(const void *p) { return uint64_t(uintptr_t(p)); }

// Status of a call that ended before lookup: T == 0 (OK) or an error.
inline tri_status finish_early(tri_cache *c, uint32_t op, int st) {
  if (st == TRI_OK)
    c->stats.empty++;
  else
    c->stats.errors++;
  tri_selection &r = c->last;
  memset(&r, 0, sizeof r);
  r.op = int32_t(op);
  r.status = st;
  r.version = -1;
  return tri_status(st);
}

inline int check_common(int32_t dtype, int64_t T) {
  if (dtype != TRI_F32 && dtype != TRI_BF16) return TRI_E_INVALID;
  if (T < 0) return TRI_E_INVALID;
  if (T == 0) return TRI_OK;
  if (T > kTMax) return TRI_E_UNSUPPORTED;
  return kGo;
}

// `rows` rows of `width` elements, `stride` elements apart (stride >= width
// >= 1, rows >= 1): their span ((rows - 1) * stride + width) * es must not
// exceed kSpanMax bytes. No memory that large exists, and within it every
// offset a kernel forms stays far from int64 overflow.
inline bool extent_ok(int64_t rows, int64_t stride, int64_t width, uint64_t es) {
  const uint64_t lim = kSpanMax / es;
  if (uint64_t(width) > lim) return false;
  return rows <= 1 || uint64_t(stride) <= (lim - uint64_t(width)) / uint64_t(rows - 1);
}

// ---- guard flags --------------------------------------------------------------
inline unsigned flags_of(uint64_t or_bits, bool contig) {
  return ((or_bits & 15u) == 0 ? kAlign : 0u) | (contig ? kContig : 0u);
}

inline uint32_t f32_bits(float f) {
  uint32_t b;
  memcpy(&b, &f, sizeof b);
  return b;
}

inline Key make_key(uint32_t op, uint32_t dtype, int64_t T, unsigned flags, uint32_t base_bits,
                    uint64_t H, uint64_t I, uint64_t hd, uint64_t nq, uint64_t nk) {
  Key k;
  k.k0 = uint64_t(op) | (uint64_t(dtype) << 8) | (uint64_t(token_bucket(T)) << 16) |
         (uint64_t(flags) << 24) | (uint64_t(base_bits) << 32);
  k.k1 = H | (I << 32);
  k.k2 = hd | (nq << 16) | (nk << 32);
  k.k3 = k.k4 = k.k5 = 0;
  return k;
}

// ---- lookup and launch bookkeeping -----------------------------------------------------
// The bookkeeping of a miss: counter, recorded key, selection record.
inline tri_selection &note_miss(tri_cache *c, uint32_t op, const Key &k, int64_t T) {
  c->stats.misses++;
  c->has_miss = true;
  c->miss_key = k;
  c->miss_T = T;
  tri_selection &r = c->last;
  memset(&r, 0, sizeof r);
  r.op = int32_t(op);
  r.version = -1;
  key_words(k, r.key);
  r.status = TRI_MISS;
  return r;
}

// Finds the version for `k`. On a miss records it and, with auto-install,
// installs and returns the new version (*auto_inst = true).
inline int lookup(tri_cache *c, uint32_t op, const Key &k, int64_t T, int32_t *vi,
                  bool *auto_inst) {
  int32_t i = find_version(c, op, k);
  if (i >= 0) {
    *vi = i;
    return TRI_OK;
  }
  tri_selection &r = note_miss(c, op, k, T);
  if (!(c->flags & TRI_CACHE_AUTO_INSTALL)) return TRI_MISS;
  const tri_status st = install_key(c, k, -1, (c->flags & TRI_CACHE_GENERIC) != 0);
  if (st != TRI_OK) {
    r.status = st;
    return st;
  }
  *vi = find_version(c, op, k);
  *auto_inst = true;
  return TRI_OK;
}

inline void record(tri_cache *c, uint32_t op, const Version &v, int32_t vi, const Key &k,
                   int n, const tri_launch_rec *l, int st) {
  tri_selection &r = c->last;
  r.op = int32_t(op);
  r.status = st;
  r.version = vi;
  r.variant = v.plan.variant;
  r.n_launches = n;
  r.roles[0] = v.plan.roles[0];
  r.roles[1] = v.plan.roles[1];
  r.roles[2] = v.plan.roles[2];
  for (int i = 0; i < 3; ++i) r.launch[i] = i < n ? l[i] : tri_launch_rec{0, 0, 0};
  key_words(k, r.key);
}

inline tri_status finish(tri_cache *c, Version &v, bool auto_inst, int rc) {
  if (rc != 0) {
    if (!auto_inst) c->stats.errors++;
    return TRI_E_LAUNCH;
  }
  if (!auto_inst) {
    c->stats.hits++;
    v.hits++;
  }
  return TRI_OK;
}

// Launch i of version v of cache c with its argument block: from a
// resident block when the launch has an argument-free form and the cache
// holds (or can hold) the block in a slot the launch may take (any slot up
// to kResidentMaxGrid workgroups, else the first kResidentAnyGridSlots);
// otherwise with kernel arguments. 0 or the launch's failure code.
inline int launch(tri_cache *c, const Version &v, int i, uint32_t dtype, uint32_t grid,
                  uint32_t block, const void *args, uint32_t size, void *stream) {
  if (v.fn_res[i]) {
    const uint32_t limit = grid <= kResidentMaxGrid ? kResidentSlots : kResidentAnyGridSlots;
    const int32_t slot = resident_slot(c, resident_family(v.plan.kvariant[i]), dtype, args,
                                       size, grid, stream, limit);
    if (slot >= 0) {
      const int rc = be_launch_resident(v.fn_res[i], grid, block, uint32_t(slot), stream);
      if (rc == 0) c->resident_launches++;
      return rc;
    }
  }
  return be_launch(v.fn[i], grid, block, args, size, stream);
}

}  // namespace
}  // namespace tri
