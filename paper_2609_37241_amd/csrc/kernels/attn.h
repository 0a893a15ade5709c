// Attention over pages on the matrix cores (PA_ROWS, PA_TILE): rows of 16-byte
// aligned heads of up to 256 elements, held in HDP of them (64, 128 or 256).
//
// Both forms compute the transposed products, S^T = K Q^T and O^T = V^T P^T: a
// lane then holds scores of one query only, so the softmax needs no exchange
// but the maximum over the lanes that share the query, and the scores are the
// second product's operand where they lie. A matrix instruction sums over
// keys in any order as long as both operands have the same one, so the keys
// are taken in the order in which the first product leaves them:
//   16x16 (S^T: lane l holds query l % 16, keys 4 (l / 16) + i, i < 4), and
//   32x32 (query l % 32, keys 8 b + 4 (l / 32) + i, b < 4).
// V is needed with the keys along a lane's elements: bf16 rows in LDS are read
// by the transposing read (16 lanes exchange 4 rows of 16 elements), float32
// ones element by element.
//
// The weights are 2^(c (x - m)) with x = q.k, c = |scale| log2 e > 0 (a negative
// scale changes q's sign) and m the running maximum of x. Sums and products
// accumulate in float32. The matrix instruction takes both operands in one type,
// and V's exponents do not fit float16, so bf16 weights meet V in bf16; the sum
// they are divided by takes them unrounded. PA_ROWS, where HBM is what bounds,
// takes them in two parts, the rounded weight and what that leaves, with a product
// each: off by 2^-16, so that the result is the plain computation's (relative
// root mean square against 64 bits 0.0017, the rounding of the result itself; with
// one part 0.0018), at no cost in the tracked decode cases but 0.2 us at 500
// keys. PA_TILE and PA_PAIR take the rounded weight alone, off by at most half a
// step, 2^-8: 0.0019 to 0.0023. The second part would cost them 27 % (2048 tokens
// behind 6144, 282 -> 360 us; the windowed mixture 43.3 -> 49.6, heads of 256 29.6
// -> 32.3); see there for the maximum.
#pragma once
#include "paged.h"

namespace tri {
namespace dev {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// 4 rows of 16 bf16 elements, row l / 4 read by lane l of 16 (4 elements
// each): lane l gets element l of the four rows.
__device__ inline u32x2 lds_transpose(const void *p) {
  typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)p));
}

// x or -x: with `flip` the sign bits of a vector's elements change, so that
// the scale is positive and the largest product has the largest score.
template <int DT>
__device__ inline void flip_sign(u32x4 &v, uint32_t flip) {
  const uint32_t bits = flip ? (DT == kF32 ? 0x80000000u : 0x80008000u) : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] ^= bits;
}

// Over the lanes l, l ^ 16, l ^ 32, l ^ 48 (or l, l ^ 32), the same in all.
__device__ inline float max_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float max_16_32(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return max_32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float sum_16_32(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return sum_32(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Two weights as bf16, and what that leaves of them as bf16 too: the sum of the
// two is off by at most 2^-16 of a weight.
__device__ inline u32x2 split_weights(float x, float y) {
  const uint32_t w = Elt<kBF16>::pack2(x, y);
  return u32x2{w, Elt<kBF16>::pack2(x - __uint_as_float(w << 16),
                                    y - __uint_as_float(w & 0xFFFF0000u))};
}

// The bits of `seen` (bit i: key k0 + i) whose keys are in [lo, hi).
__device__ inline uint64_t in_range(uint64_t seen, int32_t k0, int32_t lo, int32_t hi) {
  const int32_t a = clamp_i32(lo - k0, 0, 64), b = clamp_i32(hi - k0, 0, 64);
  const uint64_t below_b = b == 64 ? ~uint64_t(0) : (uint64_t(1) << b) - 1;
  const uint64_t below_a = a == 64 ? ~uint64_t(0) : (uint64_t(1) << a) - 1;
  return seen & below_b & ~below_a;
}

// Clears the infinities and NaN of a vector; whether there were any.
template <int DT>
__device__ inline bool clear_not_finite(u32x4 &v) {
  u32x4 keep;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == kF32) {
      keep[i] = (v[i] & 0x7F800000u) == 0x7F800000u ? 0u : ~0u;
    } else {
      keep[i] = ((v[i] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) |
                ((v[i] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
    }
  }
  const bool bad = (keep[0] & keep[1] & keep[2] & keep[3]) != ~0u;
  v &= keep;
  return bad;
}

// V may hold infinities or NaN at a key that some rows of a tile see and others
// must not (a later token of the same chunk, an earlier one than the window): a
// product over all keys would make NaN of their weight of 0. So in the steps
// whose keys the rows see differently such elements go to LDS as zeros. In the
// other steps the products make an infinity or NaN of them, which of the two
// depends on whether float32 has the weight as 0. So where there were any in the
// end, an element of a row is formed again: the sum of those that it sees, from
// memory, whatever their weights (above 0, a weight has no say in it); a row's
// result then does not depend on the other rows of its tile. The look at the sums
// is within what boxes differ by; one at every step's V took 2 % of the 128-row
// tiles and 13 % of float32 heads of 256.

// Whether a row's sums, at weights that are finite, hold an infinity or NaN.
template <int N, class F>
__device__ inline bool holds_not_finite(const F *o, int n, float l) {
  float z[4] = {};
#pragma unroll
  for (int d = 0; d < N; ++d)
    for (int i = 0; i < n; ++i) z[i % 4] = fmaf(o[d][i], 0.0f, z[i % 4]);
  const float all = (z[0] + z[1]) + (z[2] + z[3]);
  return all != all && fabsf(l) < __builtin_inff();
}

// Whether the hdb bytes of a key's V hold one.
template <int DT>
__device__ inline bool row_not_finite(const char *v, int hdb) {
  bool odd = false;
  for (int c = 0; c < hdb; c += 16) {
    u32x4 x = *reinterpret_cast<const u32x4 *>(v + c);
    odd |= clear_not_finite<DT>(x);
  }
  return odd;
}

// Four elements of a row's sums, the first of them e, from the key's V at v where
// the row sees it: the first infinity or NaN (bit `at` of `had` is clear) takes the
// element's place. Without branches, whose masks would not fit the registers.
template <int DT>
__device__ inline void add_not_finite(const char *v, bool sees, int32_t e, int32_t hd, int at,
                                      uint32_t *had, float *o) {
  const bool inside = e < hd;
  float y[4];
  if constexpr (DT == kF32) {
    Elt<kF32>::unpack(*reinterpret_cast<const u32x4 *>(v + (inside ? e : 0) * 4), y);
  } else {
    const u32x2 x = *reinterpret_cast<const u32x2 *>(v + (inside ? e : 0) * 2);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      y[2 * i] = __uint_as_float(x[i] << 16);
      y[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool odd = inside & sees & !(fabsf(y[i]) < __builtin_inff());
    const uint32_t bit = 1u << ((at + i) & 31);
    const float z = *had & bit ? o[i] + y[i] : y[i];
    o[i] = odd ? z : o[i];
    *had |= odd ? bit : 0u;
  }
  __builtin_amdgcn_sched_barrier(0);   // (or all elements' masks live at once)
}

// The tile of queries that a workgroup computes: M rows of request r's n * g
// rows of one K head (row i: token i / g, head i % g). Tiles are numbered
// through the requests without knowing their lengths on the host: those of r
// start at floor(q_start[r] g / M) + r, which leaves each request room for
// ceil(n g / M) and the whole fewer than floor(T g / M) + R + 1.
struct Tile {
  int32_t r;        // request, -1: nothing to do
  int32_t row0, rows;
  Request rq;
  int32_t p0, p1;   // positions of the first and the last row
};

template <int M>
__device__ inline Tile find_tile(const PagedArgs &a, int32_t tile) {
  Tile t;
  const auto starts = [&](int32_t r, int32_t q0) {
    return int64_t(clamp_i32(q0, 0, a.T)) * a.g / M + r <= tile;
  };
  if (a.R <= 64) {   // all in one round of loads
    const int lane = threadIdx.x & 63, x = lane < a.R ? lane : 0;
    const int32_t q0 = a.q_start[x], q1 = a.q_start[x + 1], kv = a.kv_len[x];
    const uint64_t hit = __ballot(lane < a.R && starts(x, q0));
    t.r = hit ? 63 - __builtin_clzll(hit) : -1;
    if (t.r < 0) return t;
    t.rq = clamped(a, __builtin_amdgcn_readlane(q0, t.r), __builtin_amdgcn_readlane(q1, t.r),
                   __builtin_amdgcn_readlane(kv, t.r));
  } else {
    t.r = last_request(a.R, [&](int32_t x) { return starts(x, a.q_start[x]); });
    t.r = __builtin_amdgcn_readfirstlane(t.r);
    if (t.r < 0) return t;
    t.rq = request_of(a, t.r);
  }
  const int64_t all = int64_t(t.rq.q1 - t.rq.q0) * a.g;
  const int64_t at = (tile - (int64_t(t.rq.q0) * a.g / M + t.r)) * M;
  if (at < 0 || at >= all) {
    t.r = -1;
    return t;
  }
  t.row0 = int32_t(at);
  t.rows = int32_t(all - at < M ? all - at : M);
  const int32_t base = t.rq.kv - (t.rq.q1 - t.rq.q0);
  t.p0 = base + int32_t(fast_div(uint32_t(t.row0), a.g_div));
  t.p1 = base + int32_t(fast_div(uint32_t(t.row0 + t.rows - 1), a.g_div));
  return t;
}

// Token (row of q and out) and query head of row i of a tile of K head kh.
__device__ inline void row_of(const PagedArgs &a, const Tile &t, int32_t i, int32_t kh,
                              int32_t *token, int32_t *head) {
  const uint32_t x = uint32_t(t.row0 + i), tok = fast_div(x, a.g_div);
  *token = t.rq.q0 + int32_t(tok);
  *head = kh * a.g + int32_t(x - tok * uint32_t(a.g));
}

// Four neighbouring elements of the result (or of the partial sums).
template <int DT>
__device__ inline void store4(const PagedArgs &a, int32_t token, int32_t head, int32_t d,
                              const float *v) {
  char *o = static_cast<char *>(a.out) +
            (int64_t(token) * a.o_ts + int64_t(head) * a.hd + d) * Elt<DT>::ES;
  if constexpr (DT == kF32)
    *reinterpret_cast<u32x4 *>(o) = Elt<kF32>::pack(v);
  else
    *reinterpret_cast<u32x2 *>(o) =
        u32x2{Elt<kBF16>::pack2(v[0], v[1]), Elt<kBF16>::pack2(v[2], v[3])};
}

// ---- PA_ROWS ------------------------------------------------------------------------------------
// Few rows per request (decode): a tile is 16 rows, and the wavefronts (eight,
// or four of the widest heads, whose registers leave no room for more) share
// out its keys, KB at a time each with its own softmax, joined in LDS at
// the end. HBM-bound: K and V come in whole rows, a wavefront's loads covering
// 1 KiB of them, and pass through a part of LDS that is the wavefront's own (no
// barrier), first K, then V, on their way into the products. Each is in flight
// until its step begins, and the pages of the step after are looked up
// meanwhile. Read in the order of the first product's operand instead, 64
// bytes of 16 rows a load, 1 GiB came at 6.35 TB/s, in whole rows at 6.95
// (nontemporal; 6.1 and 6.2 without). 64 requests of 8192 keys, 8 K heads of 128
// in bf16 (2.1 GB), 342 us with the join, 6.3 TB/s; of up to 8192, 193 us, 5.55
// TB/s: the longest splits end last. Four wavefronts take as long (500 keys: 10.0
// -> 11.7 us); two steps in flight do not fit the registers (252 us).
template <int DT, int HDP>
struct RowsShape {
  static constexpr int ES = Elt<DT>::ES;
  static constexpr int NW = rows_waves(HDP);              // wavefronts
  static constexpr int KB = DT == kF32 ? 16 : 32;         // keys of a step
  static constexpr int MB = KB / 16;
  static constexpr int NS = HDP * ES / 64;                // 16-byte vectors of a lane's query
  static constexpr int CH = HDP * ES / 16;                // vectors of a row
  static constexpr int RP = 64 / CH;                      // rows of a load
  static constexpr int NP = KB / RP;
  // bytes of a row in LDS: 8 rows of K on different banks; 16 rows of the
  // transposing read of V (of a column of float32)
  static constexpr int KS = HDP * ES + 16;
  static constexpr int VS = HDP * ES + (DT == kF32 ? 16 : 32);
  static constexpr int ND = HDP / 16;
  static constexpr int OS = HDP + 4;                      // floats of a row of O in LDS
  static constexpr int WAVE_LDS = KB * VS > 16 * OS * 4 ? KB * VS : 16 * OS * 4;
};

template <int DT, int HDP>
__device__ void body_pa_rows(const PagedArgs &a) {
  typedef RowsShape<DT, HDP> S;
  constexpr int ES = S::ES, KB = S::KB, MB = S::MB, NS = S::NS, ND = S::ND, NW = S::NW;
  __shared__ __attribute__((aligned(16))) char lds[NW * S::WAVE_LDS];
  __shared__ float wave_m[NW][16], wave_l[NW][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, quarter = lane >> 4;
  const uint32_t kh = blockIdx.x % uint32_t(a.nk), rest = blockIdx.x / uint32_t(a.nk);
  const int32_t split = int32_t(rest % uint32_t(a.splits));
  const Tile t = find_tile<16>(a, int32_t(rest / uint32_t(a.splits)));
  if (t.r < 0) return;
  const int32_t lo = t.p0 < 0 ? 0 : first_key(t.p0, a.window), hi = t.p1 + 1;
  int32_t b, e;
  split_keys(lo, hi, a.splits, split, &b, &e);
  // what the lane's query sees; rows behind the tile's last do as that one
  int32_t token, head;
  row_of(a, t, n < t.rows ? n : t.rows - 1, int32_t(kh), &token, &head);
  const int32_t my_p = t.rq.kv - (t.rq.q1 - token);
  const int32_t my_lo = my_p < 0 ? 0 : first_key(my_p, a.window), my_hi = my_p + 1;
  // keys that all rows see
  const int32_t all_lo = t.p1 < 0 ? 0 : first_key(t.p1, a.window), all_hi = t.p0 + 1;

  const int hdb = a.hd * ES;
  u32x4 q[NS];
  {
    const char *p = static_cast<const char *>(a.q) +
                    (int64_t(token) * a.q_ts + int64_t(head) * a.hd) * ES + quarter * 16;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (quarter * 16 + 64 * s < hdb) q[s] = *reinterpret_cast<const u32x4 *>(p + 64 * s);
      flip_sign<DT>(q[s], a.flip);
    }
  }
  const int32_t *table = a.table + int64_t(t.r) * a.table_rs;
  const char *kp = static_cast<const char *>(a.k.p) + int64_t(kh) * a.k.hs * ES;
  const char *vp = static_cast<const char *>(a.v.p) + int64_t(kh) * a.v.hs * ES;
  char *vl = lds + wave * S::WAVE_LDS;

  f32x4 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x4{0, 0, 0, 0};
  float m = kNegInf, l = 0.0f;

  // the page of key k0 + lane % KB (beyond the end: the last key's)
  const auto look_up = [&](int32_t k0) {
    const int32_t key = k0 + (lane & (KB - 1));
    return table[fast_div(uint32_t(key < e ? key : e - 1), a.div)];
  };
  // where the lane's key lies (the pool's first page for one that is not
  // there), handed to the lanes that load its row
  const int srow = lane / S::CH, sbyte = (lane % S::CH) * 16;
  const bool one_layout = a.k.ps == a.v.ps && a.k.ss == a.v.ss;
  // behind the head's end a lane loads the first vector and clears it on the
  // way to LDS: loads under a mask measured 2-7 % more
  const bool padded = hdb < HDP * ES, inside = sbyte < hdb;
  const int lbyte = inside ? sbyte : 0;
  int64_t ko, vo;
  uint64_t seen = 0;      // bit i: key k0 + i is there
  const auto rows_of = [&](int32_t k0, int32_t page) {
    const int32_t mine = k0 + (lane & (KB - 1));
    const bool ok = mine < e && uint32_t(page) < uint32_t(a.n_pages);
    seen = __ballot(ok);
    const uint32_t key = uint32_t(mine < e ? mine : e - 1);
    const int64_t id = ok ? page : 0;
    const int64_t in = key - fast_div(key, a.div) * uint32_t(a.page);
    ko = (id * a.k.ps + in * a.k.ss) * ES;
    vo = ko;
    if (!one_layout) vo = (id * a.v.ps + in * a.v.ss) * ES;
  };
  u32x4 k[S::NP], v[S::NP];
  const auto load = [&](u32x4(&x)[S::NP], const char *p, int64_t at) {
    int64_t r[S::NP];
#pragma unroll
    for (int i = 0; i < S::NP; ++i) r[i] = __shfl(at, srow + S::RP * i);
    if (a.stream) {   // (the empty asm keeps the compiler from making one of the two)
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < S::NP; ++i)
        x[i] = ld16<true>(reinterpret_cast<const u32x4 *>(p + r[i] + lbyte));
      asm volatile("" ::: "memory");
    } else {
#pragma unroll
      for (int i = 0; i < S::NP; ++i)
        x[i] = ld16<false>(reinterpret_cast<const u32x4 *>(p + r[i] + lbyte));
    }
  };
  const auto to_lds = [&](u32x4(&x)[S::NP], int stride) {
    if (padded)
#pragma unroll
      for (int i = 0; i < S::NP; ++i)
        if (!inside) x[i] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < S::NP; ++i)
      *reinterpret_cast<u32x4 *>(vl + (srow + S::RP * i) * stride + sbyte) = x[i];
  };

  const auto sees = [&](int32_t key) { return key >= my_lo && key < my_hi; };
  int32_t odd_b = 0, odd_e = 0;   // from the first to the last step with infinities or NaN
  int32_t k0 = b + wave * KB, page = 0;
  if (k0 < e) {
    rows_of(k0, look_up(k0));
    load(k, kp, ko);
    load(v, vp, vo);
    if (k0 + NW * KB < e) page = look_up(k0 + NW * KB);
  }
  for (; k0 < e; k0 += NW * KB) {
    const bool more = k0 + NW * KB < e;
    const uint64_t there = seen;
    to_lds(k, S::KS);
    if (more) {
      rows_of(k0 + NW * KB, page);
      load(k, kp, ko);
    }
    // S^T
    f32x4 st[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      st[j] = f32x4{0, 0, 0, 0};
      // (float32: four sums side by side, whose rounding errors stay half those
      // of one sum four times as long. Two would leave heads of 64 another
      // wavefront a SIMD: six ragged requests 23.3 -> 21.5 us, but 64 of up to
      // 8192 keys 193 -> 207, and up to 1.24 times the plain form's error)
      f32x4 sum[4] = {};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(vl + (16 * j + n) * S::KS + quarter * 16 +
                                                         64 * s);
        if constexpr (DT == kF32) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[i]),
                                                          __uint_as_float(q[s][i]), sum[i], 0, 0, 0);
        } else {
          st[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x),
                                                          __builtin_bit_cast(bf16x8, q[s]), st[j],
                                                          0, 0, 0);
        }
      }
      if constexpr (DT == kF32) st[j] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    // V in K's place; rows that are not there are zero, so that no weight of 0
    // meets a NaN
    const int32_t k1 = k0 + KB < e ? k0 + KB : e;
    const bool mixed = k0 < all_lo || k1 > all_hi;   // some row sees not all of them
    const bool partial = mixed || there != ~uint64_t(0);
    if (partial) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < S::NP; ++i) {
        if (!((there >> (srow + S::RP * i)) & 1)) v[i] = u32x4{0, 0, 0, 0};
        if (mixed) odd |= clear_not_finite<DT>(v[i]);
      }
      if (__ballot(odd)) {
        if (odd_b == odd_e) odd_b = k0;
        odd_e = k1;
      }
    }
    to_lds(v, S::VS);
    if (more) {
      load(v, vp, vo);
      if (k0 + 2 * NW * KB < e) page = look_up(k0 + 2 * NW * KB);
    }
    // softmax: the lane's keys are k0 + 16 j + 4 quarter + i
    if (partial) {
      const uint32_t see = uint32_t(in_range(there, k0, my_lo, my_hi) >> (4 * quarter));
#pragma unroll
      for (int j = 0; j < MB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          st[j][i] = (see >> (16 * j + i)) & 1 ? st[j][i] : kNegInf;
    }
    float top = kNegInf;
#pragma unroll
    for (int j = 0; j < MB; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, st[j][i]);
    top = max_16_32(top);
    const float mn = fmaxf(m, top);
    const float ms = mn == kNegInf ? 0.0f : mn;
    const float alpha = weight_of(m, ms, a.scale);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int j = 0; j < MB; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st[j][i] = weight_of(st[j][i], ms, a.scale);
        l += st[j][i];
      }
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] *= alpha;
    u32x4 p = {0, 0, 0, 0}, rest = {0, 0, 0, 0};
    if constexpr (DT == kBF16) {
#pragma unroll
      for (int j = 0; j < MB; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x2 x = split_weights(st[j][2 * i], st[j][2 * i + 1]);
          p[2 * j + i] = x[0];
          rest[2 * j + i] = x[1];
        }
    }
    // O^T
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      if constexpr (DT == kF32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y =
              *reinterpret_cast<const float *>(vl + (4 * quarter + i) * S::VS + (16 * d + n) * 4);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(y, st[0][i], o[d], 0, 0, 0);
        }
      } else {
        const char *x = vl + (4 * quarter + (n >> 2)) * S::VS + (16 * d + 4 * (n & 3)) * 2;
        const u32x2 y0 = lds_transpose(x), y1 = lds_transpose(x + 16 * S::VS);
        const u32x4 y = {y0[0], y0[1], y1[0], y1[1]};
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y),
                                                       __builtin_bit_cast(bf16x8, p), o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y),
                                                       __builtin_bit_cast(bf16x8, rest), o[d], 0, 0,
                                                       0);
      }
    }
  }

  l = sum_16_32(l);
  if (__ballot(holds_not_finite<ND>(o, 4, l))) {
    odd_b = b + wave * KB;
    odd_e = e;
  }
  uint32_t had[(ND + 7) / 8] = {};
  for (int32_t x0 = odd_b; x0 < odd_e; x0 += NW * KB) {   // (the wavefront's own steps)
    int64_t mine = -1;
    if (lane < KB && x0 + lane < e) mine = slot_offset(table, uint32_t(x0 + lane), a, a.v);
    uint64_t keys = __ballot(mine >= 0 && row_not_finite<DT>(vp + mine * ES, hdb));
    for (; keys; keys &= keys - 1) {
      const int i = __builtin_ctzll(keys);
      const char *x = vp + __shfl(mine, i) * ES;
      const bool seen_here = sees(x0 + i);
      int32_t hd = a.hd;
      asm volatile("" : "+s"(hd));   // (else the masks of elements inside are shared with
                                     // the stores below and live all along)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        float z[4] = {o[d][0], o[d][1], o[d][2], o[d][3]};
        add_not_finite<DT>(x, seen_here, 16 * d + 4 * quarter, hd, 4 * d, &had[d / 8], z);
        o[d] = f32x4{z[0], z[1], z[2], z[3]};
      }
    }
  }

  // join the wavefronts
  if (quarter == 0) {
    wave_m[wave][n] = m;
    wave_l[wave][n] = l;
  }
  float *ol = reinterpret_cast<float *>(vl);
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<f32x4 *>(ol + n * S::OS + 16 * d + 4 * quarter) = o[d];
  __syncthreads();
  constexpr int PR = NW * 4;   // work-items of a row
  const int row = threadIdx.x / PR, part = threadIdx.x % PR;
  if (row >= t.rows) return;
  float top = kNegInf;
#pragma unroll
  for (int w = 0; w < NW; ++w)
    if (wave_l[w][row] != 0.0f) top = fmaxf(top, wave_m[w][row]);
  const float ts = top == kNegInf ? 0.0f : top;
  float f[NW], sum = 0.0f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    f[w] = 0.0f;
    if (wave_l[w][row] != 0.0f) {
      f[w] = weight_of(wave_m[w][row], ts, a.scale);
      sum += f[w] * wave_l[w][row];
    }
  }
  row_of(a, t, row, int32_t(kh), &token, &head);
  const int64_t at = (int64_t(token) * a.nq + head) * a.splits + split;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int c = 0; c < (HDP + 4 * PR - 1) / (4 * PR); ++c) {
    const int d = 4 * PR * c + 4 * part;
    if (d >= a.hd) break;
    f32x4 acc = {0, 0, 0, 0};
    const auto sum_of = [&](int w) {
      return *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds + w * S::WAVE_LDS) +
                                              row * S::OS + d);
    };
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const f32x4 x = sum_of(w);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(f[w], x[i], acc[i]);
    }
    if (holds_not_finite<1>(&acc, 4, sum)) {
      acc = f32x4{0, 0, 0, 0};
      for (int w = 0; w < NW; ++w) {
        const float fw = wave_l[w][row] != 0.0f ? weight_of(wave_m[w][row], ts, a.scale) : 0.0f;
        const f32x4 x = sum_of(w);
        for (int i = 0; i < 4; ++i) acc[i] = add_part(fw, x[i], acc[i]);
      }
    }
    if (a.splits > 1) {
      *reinterpret_cast<f32x4 *>(a.part + at * a.hd + d) = acc;
    } else {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = sum == 0.0f ? 0.0f : acc[i] * inv;
      store4<DT>(a, token, head, d, y);
    }
  }
  if (a.splits > 1 && part == 0) {
    a.ml[2 * at] = top;
    a.ml[2 * at + 1] = sum;
  }
}

// ---- PA_TILE ------------------------------------------------------------------------------------
// Many rows per request (chunks of a prompt): a tile is 128 rows, 32 of them a
// wavefront's, against KB keys at a time whose K and V the workgroup stages in
// LDS. MFMA-bound in principle; the 32 exponentials a lane takes per 32 matrix
// instructions and the 32 KiB of LDS that a wavefront reads for them each cost
// about as much, so two workgroups a compute unit fill each other's gaps. The
// next keys' loads are in flight during the products, and go to the other half
// of LDS between them (one barrier a step). 2048 rows behind 6144 keys, 32 + 8
// heads of 128 in bf16: 275 to 304 us, 792 to 875 TFLOP/s by box (a call back to
// back with others; alone after a pause, or under a profiler, 5 % more); the matrix
// pipes are busy for 40 % of it. Heads of 256 leave one workgroup a compute unit:
// four prompts of up to 1024 tokens, 16 heads, 29.5 us; 2048 tokens behind 2048,
// 194 us, 530 TFLOP/s (with steps of 32 keys 8 % more).
//
// With two groups of four wavefronts (PA_PAIR) each takes every other step, on
// tiles of its own, and the first adds up both: where the tiles are few, a
// compute unit has two wavefronts a SIMD all the same.
//
// The running maximum is the softmax's reference only; it is raised, and what
// was summed rescaled, when a weight would pass 2^8 (a branch that the first step
// takes and few others). Float32 loses nothing by that. In bf16 the largest weight
// of a row is then rounded like any other, where with the exact maximum it is 1:
// 0.0019 to 0.0023 against 0.0018 to 0.0020, for 289 instead of 282 us (2048 tokens
// behind 6144), 44.8 instead of 43.3 (the windowed mixture) and 33.3 instead of
// 29.6 (heads of 256).
template <int DT, int HDP>
struct TileShape {
  static constexpr int ES = Elt<DT>::ES;
  static constexpr int KB = DT == kF32 ? 32 : 64;
  static constexpr int NB = KB / 32;
  static constexpr int NQ = HDP * ES / 32;                // 16-byte vectors of a lane's query
  static constexpr int ND = HDP / 32;
  // bytes of a row in LDS. K: 8 rows of 16 bytes on different banks. V: the
  // transposing read's 4 rows of 64 bytes, or (float32) 32 elements of rows 4
  // apart
  static constexpr int KS = HDP * ES + 16;
  static constexpr int VS = HDP * ES + (DT == kF32 ? 32 : 64);
  static constexpr int BUF = KB * (KS + VS);
  static constexpr int CH = HDP * ES / 16;                // vectors of a row
  static constexpr int RP = 256 / CH;                     // rows that a pass stages
  static constexpr int NP = KB / RP;
};

constexpr int kAhead = 4;   // products between an operand's read from LDS and its use

template <int DT, int HDP, int KG>
__device__ void body_pa_tile(const PagedArgs &a) {
  typedef TileShape<DT, HDP> S;
  constexpr int ES = S::ES, KB = S::KB, NB = S::NB, NQ = S::NQ, ND = S::ND, NP = S::NP;
  constexpr int GROUP = 2 * S::BUF, STEP = KG * KB;
  __shared__ __attribute__((aligned(16))) char all_lds[KG * GROUP];
  __shared__ int32_t odd_b, odd_e;   // from the first to the last step with infinities or NaN
  // four wavefronts a group; group g takes the steps g, g + KG, ... of the keys
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int tid = threadIdx.x & 255, lane = tid & 63, wave = tid >> 6;
  char *lds = all_lds + group * GROUP;
  const int n = lane & 31, half = lane >> 5;
  const uint32_t kh = blockIdx.x % uint32_t(a.nk), rest = blockIdx.x / uint32_t(a.nk);
  const int32_t split = int32_t(rest % uint32_t(a.splits));
  // the last tiles, which see the most keys, first
  const Tile t = find_tile<128>(a, a.tiles - 1 - int32_t(rest / uint32_t(a.splits)));
  if (t.r < 0) return;
  if (threadIdx.x == 0) {
    odd_b = 0x7FFFFFFF;
    odd_e = 0;
  }
  const int32_t lo = t.p0 < 0 ? 0 : first_key(t.p0, a.window), hi = t.p1 + 1;
  int32_t b, e;
  split_keys(lo, hi, a.splits, split, &b, &e);
  const int32_t all_lo = t.p1 < 0 ? 0 : first_key(t.p1, a.window), all_hi = t.p0 + 1;
  // the lane's row (behind the last: as the last) and what it sees; what all
  // rows, and any row, of the wavefront see
  const int32_t row = 32 * wave + n;
  int32_t token, head;
  row_of(a, t, row < t.rows ? row : t.rows - 1, int32_t(kh), &token, &head);
  const int32_t base = t.rq.kv - t.rq.q1;
  const int32_t my_p = base + token;
  const int32_t my_lo = my_p < 0 ? 0 : first_key(my_p, a.window), my_hi = my_p + 1;
  const int32_t w0 = __builtin_amdgcn_readlane(my_p, 0), w1 = __builtin_amdgcn_readlane(my_p, 31);
  const int32_t w_lo = w0 < 0 ? 0 : first_key(w0, a.window), w_hi = w1 + 1;
  const int32_t w_all_lo = w1 < 0 ? 0 : first_key(w1, a.window), w_all_hi = w0 + 1;
  const bool idle = 32 * wave >= t.rows;
  const auto sees = [&](int32_t key) { return key >= my_lo && key < my_hi; };

  const int hdb = a.hd * ES;
  u32x4 q[NQ];
  {
    const char *p = static_cast<const char *>(a.q) +
                    (int64_t(token) * a.q_ts + int64_t(head) * a.hd) * ES + half * 16;
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (half * 16 + 32 * s < hdb) q[s] = *reinterpret_cast<const u32x4 *>(p + 32 * s);
      flip_sign<DT>(q[s], a.flip);
    }
  }
  const int32_t *table = a.table + int64_t(t.r) * a.table_rs;
  const char *kp = static_cast<const char *>(a.k.p) + int64_t(kh) * a.k.hs * ES;
  const char *vp = static_cast<const char *>(a.v.p) + int64_t(kh) * a.v.hs * ES;

  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = kNegInf, l = 0.0f;

  // staging: this work-item's vector of rows srow + RP i
  const int srow = tid / S::CH, sbyte = (tid % S::CH) * 16;
  // (behind the head's end as in PA_ROWS)
  const bool padded = hdb < HDP * ES, inside = sbyte < hdb;
  const int lbyte = inside ? sbyte : 0;
  // the page of key k0 + lane % KB (beyond the end: the last key's)
  const auto look_up = [&](int32_t k0) {
    const int32_t key = k0 + (lane & (KB - 1));
    return table[fast_div(uint32_t(key < e ? key : e - 1), a.div)];
  };
  u32x4 sk[NP], sv[NP];
  uint64_t seen = 0;     // bit i: key k0 + i of the staged step is there
  const bool one_layout = a.k.ps == a.v.ps && a.k.ss == a.v.ss;
  const auto load = [&](int32_t k0, int32_t page) {
    // where the lane's key lies (the pool's first page for one that is not
    // there), handed to the lanes that load its row
    const int32_t mine = k0 + (lane & (KB - 1));
    const bool ok = mine < e && uint32_t(page) < uint32_t(a.n_pages);
    seen = __ballot(ok);
    const uint32_t key = uint32_t(mine < e ? mine : e - 1);
    const int64_t id = ok ? page : 0;
    const int64_t in = key - fast_div(key, a.div) * uint32_t(a.page);
    const int64_t ko = (id * a.k.ps + in * a.k.ss) * ES;
    int64_t vo = ko;
    if (!one_layout) vo = (id * a.v.ps + in * a.v.ss) * ES;
    int64_t kr[NP], vr[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) kr[i] = vr[i] = __shfl(ko, srow + S::RP * i);
    if (!one_layout)
#pragma unroll
      for (int i = 0; i < NP; ++i) vr[i] = __shfl(vo, srow + S::RP * i);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      sk[i] = *reinterpret_cast<const u32x4 *>(kp + kr[i] + lbyte);
      sv[i] = *reinterpret_cast<const u32x4 *>(vp + vr[i] + lbyte);
    }
  };
  // rows of V that are not there are zero, so that no weight of 0 meets a NaN
  const auto store = [&](int32_t k0, int buf) {
    char *kl = lds + buf * S::BUF, *vl = kl + KB * S::KS;
    const int32_t k1 = k0 + KB < e ? k0 + KB : e;
    const bool mixed = k0 < all_lo || k1 > all_hi;
    const bool some = seen != ~uint64_t(0);   // (32 keys: their bits twice)
    bool odd = false;
    if (padded)
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (!inside) sk[i] = sv[i] = u32x4{0, 0, 0, 0};
    if (some)
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (!((seen >> (srow + S::RP * i)) & 1)) sv[i] = u32x4{0, 0, 0, 0};
    if (mixed)
#pragma unroll
      for (int i = 0; i < NP; ++i) odd |= clear_not_finite<DT>(sv[i]);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = srow + S::RP * i;
      *reinterpret_cast<u32x4 *>(kl + r * S::KS + sbyte) = sk[i];
      *reinterpret_cast<u32x4 *>(vl + r * S::VS + sbyte) = sv[i];
    }
    if (mixed && odd) {
      atomicMin(&odd_b, k0);
      atomicMax(&odd_e, k1);
    }
  };

  uint64_t there = 0;    // `seen` of the step being computed
  int32_t page = 0;
  const int32_t first = b + group * KB;
  if (b < e) {
    if (first < e) load(first, look_up(first));
    __syncthreads();     // odd_b, odd_e are set
    if (first < e) {
      store(first, 0);
      there = seen;
      if (first + STEP < e) {
        page = look_up(first + STEP);
        load(first + STEP, page);
        if (first + 2 * STEP < e) page = look_up(first + 2 * STEP);
      }
    }
    __syncthreads();
  }
  int buf = 0;
  for (int32_t k0 = first; k0 - group * KB < e; k0 += STEP) {
    const char *kl = lds + buf * S::BUF, *vl = kl + KB * S::KS;
    const bool work = !idle && k0 < e && k0 < w_hi && k0 + KB > w_lo;
    f32x16 st[NB];
    if (work) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[j][i] = 0.0f;
      // product i: vector i / NB of 32 keys i % NB; their reads kAhead products
      // before them (left to itself the scheduler makes each wait for its own)
      const auto read_k = [&](int i) {
        return *reinterpret_cast<const u32x4 *>(kl + (32 * (i % NB) + n) * S::KS + half * 16 +
                                                32 * (i / NB));
      };
      u32x4 k[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) k[i] = read_k(i);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < NB * NQ; ++i) {
        f32x16 &x = st[i % NB];
        const u32x4 y = k[i % kAhead];
        if constexpr (DT == kF32) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            x = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(y[c]),
                                                     __uint_as_float(q[i / NB][c]), x, 0, 0, 0);
        } else {
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, y),
                                                      __builtin_bit_cast(bf16x8, q[i / NB]), x, 0, 0,
                                                      0);
        }
        if (i + kAhead < NB * NQ) k[i % kAhead] = read_k(i + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    const uint64_t now = there;
    if (k0 + STEP < e) {
      store(k0 + STEP, buf ^ 1);
      there = seen;
      if (k0 + 2 * STEP < e) {
        load(k0 + 2 * STEP, page);
        if (k0 + 3 * STEP < e) page = look_up(k0 + 3 * STEP);
      }
    }
    if (work) {
      const auto read_v = [&](int i) {
        const int s = i / ND, d = i % ND;
        if constexpr (DT == kF32) {
          return u32x4{*reinterpret_cast<const uint32_t *>(
                           vl + (8 * (s / 4) + 4 * half + s % 4) * S::VS + (32 * d + n) * 4),
                       0, 0, 0};
        } else {
          // keys 16 s + 4 half + (0..3 and 8..11)
          const char *x = vl + (16 * s + 4 * half + ((lane & 15) >> 2)) * S::VS +
                          (32 * d + (lane & 16) + 4 * (lane & 3)) * 2;
          const u32x2 y0 = lds_transpose(x), y1 = lds_transpose(x + 8 * S::VS);
          return u32x4{y0[0], y0[1], y1[0], y1[1]};
        }
      };
      u32x4 y[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) y[i] = read_v(i);
      // the lane's keys are k0 + 32 j + 8 (i / 4) + 4 half + i % 4
      const int32_t k1 = k0 + KB < e ? k0 + KB : e;
      const bool mixed = k0 < w_all_lo || k1 > w_all_hi;
      if (mixed || now != ~uint64_t(0)) {
        const uint64_t see = in_range(now, k0, my_lo, my_hi) >> (4 * half);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            st[j][i] = (uint32_t(see >> (32 * j)) >> (8 * (i / 4) + i % 4)) & 1 ? st[j][i] : kNegInf;
      }
      float top = kNegInf;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, st[j][i]);
      top = max_32(top);
      if (__ballot((top - m) * a.scale > 8.0f)) {
        const float mn = fmaxf(m, top);
        const float alpha = weight_of(m, mn == kNegInf ? 0.0f : mn, a.scale);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          // (these sums live in accumulation registers; without this they
          // are copied at every step, before the branch)
          if constexpr (HDP > 128) asm volatile("" : "+a"(o[d]));
          o[d] *= alpha;
        }
      }
      const float ms = m == kNegInf ? 0.0f : m;
      // O^T, product i: elements 32 (i % ND) .. of V at keys 16 (i / ND) .. (bf16;
      // float32: at one key of each half). The reads of V run ahead as those
      // of K; the weights of the next keys are formed between the products.
      constexpr int NV = DT == kF32 ? 16 * ND : KB / 16 * ND;
      constexpr int WC = DT == kF32 ? 1 : 8;          // weights of a lane for ND products
      constexpr int WP = (WC + ND - 1) / ND;          // formed at each of them
      const auto weight = [&](int c) {
        const float x = weight_of(st[c / 16][c % 16], ms, a.scale);
        st[c / 16][c % 16] = x;
        l += x;
      };
#pragma unroll
      for (int c = 0; c < WC; ++c) weight(c);
      u32x4 p = {0, 0, 0, 0};
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = i / ND, d = i % ND;
        if constexpr (DT == kF32) {
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(y[i % kAhead][0]), st[0][s],
                                                      o[d], 0, 0, 0);
        } else {
          if (d == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              p[c] = Elt<kBF16>::pack2(st[s / 2][8 * (s % 2) + 2 * c],
                                       st[s / 2][8 * (s % 2) + 2 * c + 1]);
          }
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, y[i % kAhead]),
                                                         __builtin_bit_cast(bf16x8, p), o[d], 0, 0,
                                                         0);
        }
        if (i + kAhead < NV) y[i % kAhead] = read_v(i + kAhead);
#pragma unroll
        for (int c = WP * d; c < WP * (d + 1) && c < WC; ++c)
          if (WC * (s + 1) + c < 16 * NB) weight(WC * (s + 1) + c);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
    buf ^= 1;
  }

  l = sum_32(l);
  if constexpr (KG == 2) {
    // the second group's sums, lane by lane, through LDS (the last step's
    // barrier is behind all reads of the tiles)
    if (b < e) {
      f32x4 *x = reinterpret_cast<f32x4 *>(all_lds) + wave * (4 * ND * 64) + lane;
      float *y = reinterpret_cast<float *>(all_lds + 4 * (4 * ND * 64) * 16) + wave * 128 + lane;
      if (group == 1) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[(4 * d + i) * 64] = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        y[0] = m;
        y[64] = l;
      }
      __syncthreads();
      if (group == 0) {
        const float m1 = y[0], l1 = y[64];
        const float top = fmaxf(l != 0.0f ? m : kNegInf, l1 != 0.0f ? m1 : kNegInf);
        const float ts = top == kNegInf ? 0.0f : top;
        const float f0 = l != 0.0f ? weight_of(m, ts, a.scale) : 0.0f;
        const float f1 = l1 != 0.0f ? weight_of(m1, ts, a.scale) : 0.0f;
        m = top;
        l = f0 * l + f1 * l1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 z = x[(4 * d + i) * 64];
#pragma unroll
            for (int c = 0; c < 4; ++c)
              o[d][4 * i + c] = fmaf(f1, z[c], f0 * o[d][4 * i + c]);
          }
      }
    }
    if (group == 1) return;
  }
  // (the last step's barrier is behind what set odd_b and odd_e)
  int32_t x0 = b < e ? odd_b : 0, x1 = b < e ? odd_e : 0;
  if (__ballot(holds_not_finite<ND>(o, 16, l))) {
    x0 = b;
    x1 = e;
  }
  uint32_t had[(ND + 1) / 2] = {};
  for (; x0 < x1; x0 += 64) {
    int64_t mine = -1;
    if (x0 + lane < x1) mine = slot_offset(table, uint32_t(x0 + lane), a, a.v);
    uint64_t keys = __ballot(mine >= 0 && row_not_finite<DT>(vp + mine * ES, hdb));
    for (; keys; keys &= keys - 1) {
      const int i = __builtin_ctzll(keys);
      const char *x = vp + __shfl(mine, i) * ES;
      const bool seen_here = sees(x0 + i);
      int32_t hd = a.hd;
      asm volatile("" : "+s"(hd));   // (else the masks of elements inside are shared with
                                     // the stores below and live all along)
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float z[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) z[c] = o[d][4 * j + c];
          add_not_finite<DT>(x, seen_here, 32 * d + 8 * j + 4 * half, hd, 16 * d + 4 * j,
                             &had[d / 2], z);
#pragma unroll
          for (int c = 0; c < 4; ++c) o[d][4 * j + c] = z[c];
        }
    }
  }
  if (row >= t.rows) return;
  const int64_t at = (int64_t(token) * a.nq + head) * a.splits + split;
  const bool zero = a.splits == 1 && l == 0.0f;
  const float f = a.splits > 1 ? 1.0f : 1.0f / l;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e0 = 32 * d + 8 * i + 4 * half;
      if (e0 >= a.hd) continue;
      float y[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) y[x] = zero ? 0.0f : o[d][4 * i + x] * f;
      if (a.splits > 1)
        *reinterpret_cast<u32x4 *>(a.part + at * a.hd + e0) = Elt<kF32>::pack(y);
      else
        store4<DT>(a, token, head, e0, y);
    }
  if (a.splits > 1 && half == 0) {
    a.ml[2 * at] = m;
    a.ml[2 * at + 1] = l;
  }
}

}  // namespace dev
}  // namespace tri
