// Attention over pages of 8-bit codes on the matrix cores (PA8_ROWS, PA8_TILE): heads of
// a multiple of 16 elements up to 256, held in HDP of them (64, 128 or 256).
//
// The products are those of PA_ROWS and PA_TILE, S^T = K Q^T and O^T = V^T P^T, keys
// in the order in which the first leaves them. Every code is a bf16 number (8 bits of a whole
// number, 4 of e4m3), so codes meet queries and weights in bf16 as they are, and
// only those are ever rounded: bf16 queries are not; float32 ones are taken in three
// parts of 8 bits, cut off, not rounded, so that the parts' sum is the number
// itself, with a product each (three bf16 products for one of float32, whose
// instruction takes 16 times as long). Weights likewise: see the forms.
//
// A score is (q.k) (s c), s the key's scale and c = |scale| log2 e: powers of two,
// so that a weight is 2^(y - m). What a key's weight brings to the sums of V is the weight
// times the key's V scale, in float32 before it is cut into parts; the sum that
// divides takes the weight alone.
#pragma once
#include "attn.h"
#include "paged_q8.h"

#include <type_traits>

namespace tri {
namespace dev {

// Eight codes as bf16 (exact): v_cvt_scalef32_pk_bf16_fp8 of two, or a conversion to float32 of
// each, whose upper half it is.
template <int CT>
__device__ inline bf16x8 codes_bf16(u32x2 c) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (CT == kInt8) {
      float f[4];
      codes4<kInt8>(c[i], f);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        r[2 * i + j] = __builtin_amdgcn_perm(__float_as_uint(f[2 * j + 1]), __float_as_uint(f[2 * j]),
                                             0x07060302);
    } else {
      r[2 * i] = __builtin_bit_cast(uint32_t,
                                    __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, false));
      r[2 * i + 1] = __builtin_bit_cast(uint32_t,
                                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, true));
    }
  }
  return __builtin_bit_cast(bf16x8, r);
}

// 8 rows of 16 codes, lane l of 16 with the address of 8 of row l / 2: lane l gets code l of
// the eight rows.
__device__ inline u32x2 lds_transpose8(const void *p) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 *lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr)(uintptr_t)p));
}

// Two numbers as N pairs of bf16: N = 1 rounded; 2 rounded, and what that leaves (off by
// at most 2^-16); 3 cut off twice, and what is left: 24 bits, all of a float32 (its
// lowest ones aside where they are below bf16's least).
template <int N>
__device__ inline void bf16_parts(float x, float y, uint32_t *p) {
  if constexpr (N == 1) {
    p[0] = Elt<kBF16>::pack2(x, y);
  } else if constexpr (N == 2) {
    const u32x2 s = split_weights(x, y);
    p[0] = s[0];
    p[1] = s[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
      x -= __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
      y -= __uint_as_float(__float_as_uint(y) & 0xFFFF0000u);
    }
  }
}

// 8 neighbouring elements of a query (zeros where `inside` is false) in N parts, with `flip`
// negated. An infinity has no rest; a NaN whose first part is an infinity (its upper mantissa
// bits are zero) is one in its rest.
template <int DT, int N>
__device__ inline void load_query(const char *p, bool inside, uint32_t flip, u32x4 *q) {
  if constexpr (DT == kBF16) {
    static_assert(N == 1, "bf16 queries are one part");
    q[0] = u32x4{0, 0, 0, 0};
    if (inside) q[0] = *reinterpret_cast<const u32x4 *>(p);
    flip_sign<kBF16>(q[0], flip);
  } else {
    float f[8] = {};
    if (inside) {
      Elt<kF32>::unpack(*reinterpret_cast<const u32x4 *>(p), f);
      Elt<kF32>::unpack(*reinterpret_cast<const u32x4 *>(p + 16), f + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = flip ? -f[2 * i] : f[2 * i], y = flip ? -f[2 * i + 1] : f[2 * i + 1];
      uint32_t w[N];
      bf16_parts<N>(x, y, w);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (k > 0 && fabsf(x) == __builtin_inff()) w[k] &= 0xFFFF0000u;
        if (k > 0 && fabsf(y) == __builtin_inff()) w[k] &= 0x0000FFFFu;
        q[k][i] = w[k];
      }
    }
  }
}

// Clears the NaN codes of e4m3; whether there were any. (A code's low seven bits all
// set: adding 1 to them, apart from the sign, carries into its eighth.)
template <int CT>
__device__ inline bool clear_nan_codes(u32x4 &v) {
  if constexpr (CT == kInt8) return false;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t is = ((v[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    any |= is != 0;
    v[i] &= ~((is >> 7) * 0xFFu);
  }
  return any;
}

// Where key `key` of a request lies: page (-1: not in the pool), slot and block of it.
struct KeyPlace {
  int64_t id;
  uint32_t slot, block;
};
__device__ inline KeyPlace place_of(uint32_t key, int32_t page, const PagedQ8Args &a8) {
  const PagedArgs &a = a8.a;
  KeyPlace x;
  x.id = uint32_t(page) < uint32_t(a.n_pages) ? page : -1;
  x.slot = key - fast_div(key, a.div) * uint32_t(a.page);
  x.block = fast_div(x.slot, a8.block_div);
  return x;
}

// NaN in V at keys that some rows of a tile see and others must not (codes or scales): the
// steps whose keys the rows see differently take them as zeros, and note the keys' range.
// This makes NaN of the four elements from e on of a row that sees such a key.
template <int CT>
__device__ inline void add_nan(const char *v, bool sees, bool whole, int32_t e, int32_t hd, float *o) {
  const uint32_t c = *reinterpret_cast<const uint32_t *>(v + (e < hd ? e : 0));
  const uint32_t is = CT == kInt8 ? 0u : ((c & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (sees && (whole || (is >> (8 * i + 7)) & 1)) o[i] = __builtin_nanf("");
}

// Of 64 keys, one a lane (`inside`: the lane has one): which have NaN in V, in a code or
// everywhere, and where the lane's lies from vp.
struct NanKeys {
  int64_t at;
  uint64_t odd, whole;
};
template <int CT>
__device__ inline NanKeys nan_keys(int32_t key, bool inside, const int32_t *table, const char *vp,
                                   uint32_t kh, const PagedQ8Args &a8) {
  NanKeys k = {0, 0, 0};
  bool whole = false, odd = false;
  if (inside) {
    const KeyPlace x = place_of(uint32_t(key), table[fast_div(uint32_t(key), a8.a.div)], a8);
    if (x.id >= 0) {
      k.at = x.id * a8.a.v.ps + int64_t(x.slot) * a8.a.v.ss;
      const float s = *scale_at(a8.vs, x.id, x.block, kh);
      whole = s != s;
      odd = whole;
      for (int c = 0; CT == kE4M3 && c < a8.a.hd; c += 16) {
        u32x4 y = *reinterpret_cast<const u32x4 *>(vp + k.at + c);
        odd |= clear_nan_codes<CT>(y);
      }
    }
  }
  k.odd = __ballot(odd);
  k.whole = __ballot(whole);
  return k;
}

// ---- PA8_ROWS -----------------------------------------------------------------------------------
// Few rows per request (decode), as PA_ROWS: the wavefronts share out a tile's keys,
// each with its own softmax, joined in LDS at the end. HBM-bound: K and V come in whole rows,
// past the caches, always: through them 114 us for the 101 below, 40.8 for the 37.4 of 32 requests of 2000
// keys, whose codes the last-level cache would hold; only where several tiles of a call read the same keys
// are they 2-3 % faster (64 new tokens behind 3900, 16 and 4 heads, 22.2 for 22.6). They pass as
// codes through a part of LDS that is the wavefront's own, where a lane's 16 codes of K are two
// products' operands, and the transposing read of bytes gives it 8 keys of one element of V.
//
// Products of 16 rows would leave most of them empty where few query heads share a K head.
// So a tile is 16 / HG rows of each of HG neighbouring K heads, and a step of a wavefront 64 / HG
// keys of each: 64 rows of K, head by head, against all 16 columns. A column takes the
// scores of its own head's rows and gives the others' weights of 0, so the products are as many
// per byte as with one head, the exponentials 1 / HG, and what is read in a slot is HG
// heads long (64 requests of up to 8192 keys, 32 and 8 heads of 128, one / two / four a tile: 117
// / 111 / 101 us; all of 8192 213 / 205 / 188, 5.7 TB/s of codes; one of 131,072 68 / 62 / 62). float32
// queries, three products for one, over the ragged 64: 111 us (int8), 119 (e4m3, spills 17 registers a lane);
// 32 of them with 16 and 8 heads of 256 110, and 132 where e4m3 spills 70 (bf16, 98).
// A NaN code of V would meet other heads' weights of 0: a unit whose sums hold one where
// the weights are finite is done again with such codes cleared.
//
// A workgroup fills a compute unit (its registers), so what it does not overlap by itself
// nothing does: its start, the first loads and the join took 4.3 us of each of several
// workgroups a unit. So there is at most one a unit, and each takes as many steps: the
// steps of all tiles, numbered from the requests' lengths by every workgroup for itself, are
// cut into equal runs, which may end inside a tile; the parts of such a tile leave partial sums. A
// workgroup is a step ahead in loading K and V, two in looking up pages, also from
// one tile to the next.
template <int DT, int HDP, int HG>
struct Rows8Shape {
  static constexpr int ES = Elt<DT>::ES;
  static constexpr int NW = rows_waves(HDP);              // wavefronts
  static constexpr int TM = 16 / HG;                      // rows of a K head in a tile
  static constexpr int KB = 64;                           // rows of K of a step
  static constexpr int KH = KB / HG;                      // its keys
  static constexpr int MB = KB / 16, MH = MB / HG;        // 16 rows of K: all, a head's
  static constexpr int QP = DT == kF32 ? 3 : 1;           // parts of a query
  static constexpr int WP = DT == kF32 ? 3 : 2;           // and of a weight
  static constexpr int NS = HDP / 64;                     // 16-byte vectors of a lane's K
  static constexpr int CH = HDP / 16;                     // vectors of a row
  static constexpr int RP = 64 / CH;                      // rows of a load
  static constexpr int NP = KB / RP;
  // bytes of a row in LDS: 16 rows of 16 bytes on different banks
  static constexpr int LS = HDP + 16;
  static constexpr int ND = HDP / 16;
  static constexpr int OS = HDP + 4;                      // floats of a row of O in LDS
  static constexpr int WAVE_LDS = KB * LS > 16 * OS * 4 ? KB * LS : 16 * OS * 4;
};

// The steps that all tiles take, `step` keys each, numbered request by request, tile by
// tile, and that once for each HG heads: the host's choice of `step` keeps their number
// below 2^31. Requests whose rows overlap (starts that fall) could take more than the rows allow:
// sums stop at a8.most, and steps behind those that T rows and R requests can take are
// taken by nobody. Up to 64 requests are held by a lane each, more in LDS.
template <int TM>
struct Numbering {
  const PagedQ8Args &a8;
  int32_t *sums;              // [R] of LDS
  Request rq;                 // the lane's request
  int32_t first, all;         // steps before it, of all (for one HG heads)
  int32_t per;                // of a workgroup

  // Steps of each of a request's tiles, whose rows see at most 15 keys more than the window.
  __device__ int32_t steps_of(const Request &x) const {
    const int32_t w = a8.a.window, keys = w > 0 && w < 0x7FFFFF00 && w + 15 < x.kv ? w + 15 : x.kv;
    const int32_t n = int32_t((uint32_t(keys) + (1u << a8.step_shift) - 1) >> a8.step_shift);
    return n > 0 ? n : 1;
  }
  // Tiles of its n g rows of a K head.
  __device__ int32_t tiles_of(const Request &x) const {
    const int32_t n = x.q1 - x.q0;
    return n > 0 ? (n * a8.a.g + TM - 1) / TM : 0;
  }

  // The whole workgroup of NW wavefronts; `heads`: how often all steps are taken, `runs`:
  // workgroups to share them.
  template <int NW>
  __device__ void number(int32_t *wave_sums, int32_t heads, int32_t runs) {
    const PagedArgs &a = a8.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // over the first `lanes` lanes: sums with those of the lanes before, the largest
    const int lanes = a.R < 64 ? a.R : 64;
    const int32_t top = a8.most;
    const auto add = [&](int32_t x, int64_t y) { return y < top - x ? int32_t(x + y) : top; };
    const auto scan = [&](int32_t x) {
      for (int d = 1; d < lanes; d *= 2) {
        const int32_t y = __shfl_up(x, d);
        if (lane >= d) x = add(x, y);
      }
      return x;
    };
    const auto before_lane = [&](int32_t sum) {
      const int32_t x = __shfl_up(sum, 1);
      return lane > 0 ? x : 0;
    };
    const auto largest = [&](int32_t x) {
      for (int d = 1; d < lanes; d *= 2) {
        const int32_t y = __shfl_xor(x, d);
        x = y > x ? y : x;
      }
      return __builtin_amdgcn_readfirstlane(x);
    };
    int32_t most = 0;   // steps of the longest tile
    if (a.R <= 64) {
      rq = request_of(a, lane < a.R ? lane : 0);
      const int32_t steps = steps_of(rq);
      const int32_t sum = scan(lane < a.R ? add(0, int64_t(tiles_of(rq)) * steps) : 0);
      first = before_lane(sum);
      all = __builtin_amdgcn_readlane(sum, a.R - 1);
      most = largest(steps);
    } else {
      // consecutive requests a work-item, then the sums of what was before
      const int32_t each = (a.R + 64 * NW - 1) / (64 * NW), r0 = int32_t(threadIdx.x) * each;
      int32_t mine = 0;
      for (int32_t r = r0; r < r0 + each && r < a.R; ++r) {
        const Request x = request_of(a, r);
        const int32_t n = steps_of(x);
        most = n > most ? n : most;
        mine = add(mine, int64_t(tiles_of(x)) * n);
      }
      const int32_t sum = scan(mine);
      most = largest(most);
      if (lane == 63) {
        wave_sums[wave] = sum;
        wave_sums[NW + wave] = most;
      }
      __syncthreads();
      int32_t before = before_lane(sum);
      all = 0;
      for (int w = 0; w < NW; ++w) {
        before = add(before, w < wave ? wave_sums[w] : 0);
        all = add(all, wave_sums[w]);
        most = wave_sums[NW + w] > most ? wave_sums[NW + w] : most;
      }
      for (int32_t r = r0; r < r0 + each && r < a.R; ++r) {
        sums[r] = before;
        const Request x = request_of(a, r);
        before = add(before, int64_t(tiles_of(x)) * steps_of(x));
      }
      __syncthreads();
      all = __builtin_amdgcn_readfirstlane(all);
      most = __builtin_amdgcn_readfirstlane(most);
    }
    const int64_t room = (int64_t(a.T) * a.g / TM + a.R) * most;
    all = room < all ? int32_t(room) : all;
    per = int32_t((uint32_t(all) * uint32_t(heads) + uint32_t(runs) - 1) / uint32_t(runs));
    // a tile of n steps meets at most (n - 2) / per + 2 runs
    if (a.splits > 1) {
      const int32_t least = (most + a.splits - 2) / (a.splits - 1);
      per = per < least ? least : per;
    }
    if (per < 1) per = 1;
  }

  // The request of step `in` of all.
  __device__ int32_t find(int32_t in) const {
    if (a8.a.R > 64)
      return __builtin_amdgcn_readfirstlane(
          last_request(a8.a.R, [&](int32_t y) { return sums[y] <= in; }));
    const uint64_t hit = __ballot(int32_t(threadIdx.x & 63) < a8.a.R && first <= in);
    return 63 - __builtin_clzll(hit);
  }
  // Steps before request r.
  __device__ int32_t before(int32_t r) const {
    return a8.a.R > 64 ? __builtin_amdgcn_readfirstlane(sums[r]) : __builtin_amdgcn_readlane(first, r);
  }
  __device__ Request request(int32_t r) const {
    if (a8.a.R > 64) return request_of(a8.a, r);
    return {__builtin_amdgcn_readlane(rq.q0, r), __builtin_amdgcn_readlane(rq.q1, r),
            __builtin_amdgcn_readlane(rq.kv, r)};
  }
};

// What a workgroup does in one go: keys [b, e) of a tile's HG K heads from kh on, the tile's
// rows from row0 on of request r's.
struct Unit {
  int32_t r;                  // -1: none
  int32_t row0, b, e, steps;
  uint32_t kh;
  int32_t part;               // which part of the tile, -1: all of it
};

// The keys that a tile of `rows` rows sees some of, and the positions of its first and last row.
struct Span {
  int32_t rows, p0, p1, lo, hi;
};
template <int TM>
__device__ inline Span span_of(const PagedArgs &a, const Request &x, int32_t row0) {
  Span s;
  const int32_t all = (x.q1 - x.q0) * a.g, base = x.kv - (x.q1 - x.q0);
  s.rows = all - row0 < TM ? all - row0 : TM;
  s.p0 = base + int32_t(fast_div(uint32_t(row0), a.g_div));
  s.p1 = base + int32_t(fast_div(uint32_t(row0 + s.rows - 1), a.g_div));
  s.lo = s.p0 < 0 ? 0 : first_key(s.p0, a.window);
  s.hi = s.p1 + 1 > s.lo ? s.p1 + 1 : s.lo;
  return s;
}

// The unit at step *at of all, which ends at `end` (the workgroup's run) or with the tile; *at
// is behind it then. Without partial sums tiles are whole, and those that begin in the run are
// its workgroup's.
template <int HG>
__device__ inline Unit unit_at(const Numbering<16 / HG> &nb, int32_t *at, int32_t end, int32_t wave_keys) {
  constexpr int TM = 16 / HG;
  const PagedArgs &a = nb.a8.a;
  Unit u;
  u.r = -1;
  while (*at < end) {
    const uint32_t heads = uint32_t(*at) / uint32_t(nb.all);
    const int32_t in = *at - int32_t(heads) * nb.all, r = nb.find(in), before = nb.before(r);
    const Request x = nb.request(r);
    const int32_t steps = nb.steps_of(x);
    const int32_t tile = int32_t(uint32_t(in - before) / uint32_t(steps));
    const int32_t s0 = in - before - tile * steps, begin = *at - s0;
    int32_t to = begin + steps;
    if (a.splits < 2 && s0 > 0) {
      *at = to;
      continue;
    }
    u.part = -1;
    if (a.splits > 1) {
      if (s0 > 0 || to > end) u.part = int32_t(blockIdx.x) - int32_t(uint32_t(begin) / uint32_t(nb.per));
      to = to < end ? to : end;
    }
    u.r = r;
    u.kh = heads * HG;
    u.row0 = tile * TM;
    const Span s = span_of<TM>(a, x, u.row0);
    const int64_t from = s.lo + (int64_t(s0) << nb.a8.step_shift);
    const int64_t till = from + (int64_t(to - *at) << nb.a8.step_shift);
    u.b = int32_t(from < s.hi ? from : s.hi);
    u.e = int32_t(till < s.hi ? till : s.hi);
    u.steps = u.e > u.b ? (u.e - u.b + wave_keys - 1) / wave_keys : 1;
    *at = to;
    break;
  }
  return u;
}

template <int DT, int CT, int HDP, int HG>
__device__ void body_pa8_rows(const PagedQ8Args &a8) {
  typedef Rows8Shape<DT, HDP, HG> S;
  constexpr int ES = S::ES, KB = S::KB, KH = S::KH, MB = S::MB, MH = S::MH, NS = S::NS, ND = S::ND;
  constexpr int NW = S::NW, TM = S::TM, QP = S::QP, WP = S::WP;
  const PagedArgs &a = a8.a;
  __shared__ __attribute__((aligned(16))) char lds[NW * S::WAVE_LDS];
  __shared__ __attribute__((aligned(16))) float scales[NW][2][KB];   // s c of K, s of V
  __shared__ float wave_m[NW][16], wave_l[NW][16];
  __shared__ int32_t sums[TRI_MAX_REQUESTS], wave_sums[2 * NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, quarter = lane >> 4;
  const int hn = n / TM;                                   // the column's head
  const int lane_key = lane % KH, lane_head = lane / KH;   // the lane's row of K
  char *vl = lds + wave * S::WAVE_LDS;
  Numbering<TM> nb{a8, sums, {}, 0, 0, 0};
  nb.template number<NW>(wave_sums, a.nk / HG, int32_t(gridDim.x));
  const int64_t all = int64_t(nb.all) * (a.nk / HG), run = int64_t(blockIdx.x) * nb.per;
  const int32_t begin = int32_t(run < all ? run : all);
  const int32_t end = int32_t(run + nb.per < all ? run + nb.per : all);
  bool clean = false, again = false;   // NaN codes are cleared; there were some
start:
  int32_t at = begin;
  // what is computed, what is loaded (a step ahead), what is looked up (two)
  Unit now = unit_at<HG>(nb, &at, end, NW * KH);
  if (now.r < 0) return;
  Unit ahead = now, far = now;
  int32_t now_step = 0, ahead_step = 0, far_step = 0;
  // the step after: of the next unit after a unit's last (behind all units: the last's again)
  const auto advance = [&](Unit &x, int32_t &step) {
    if (++step < x.steps) return;
    const Unit y = unit_at<HG>(nb, &at, end, NW * KH);
    if (y.r >= 0) {
      x = y;
      step = 0;
    } else {
      x.r = -1;
    }
  };

  // the page of the lane's key in a step (beyond the end: the last key's)
  const auto look_up = [&](const Unit &x, int32_t step) {
    int32_t key = x.b + (step * NW + wave) * KH + lane_key;
    key = key < x.e ? key : x.e - 1;
    const int32_t r = x.r < 0 ? 0 : x.r;
    return a.table[r * a.table_rs + fast_div(uint32_t(key < 0 ? 0 : key), a.div)];
  };
  // where the lane's key lies (in the pool's first page for one that is not
  // there), handed to the lanes that load its row; behind the head's end a lane loads
  // the first vector and clears it on the way to LDS
  const int srow = lane / S::CH, sbyte = (lane % S::CH) * 16;
  const bool one_layout = a.k.ps == a.v.ps && a.k.ss == a.v.ss && a.k.hs == a.v.hs;
  const bool padded = a.hd < HDP, inside = sbyte < a.hd;
  const int lbyte = inside ? sbyte : 0;
  int64_t ko, vo;
  uint64_t seen = 0;      // bit i: row i of the step is there
  float ksc, vsc;         // the lane's row's scales
  const auto rows_of = [&](const Unit &x, int32_t step, int32_t page) {
    int32_t key = x.b + (step * NW + wave) * KH + lane_key;
    const bool in = key < x.e;
    key = in ? key : x.e - 1;
    const KeyPlace y = place_of(uint32_t(key < 0 ? 0 : key), page, a8);
    const bool ok = in && y.id >= 0;
    seen = __ballot(ok);
    const int64_t id = ok ? y.id : 0;
    const uint32_t h = x.kh + uint32_t(lane_head);
    ko = id * a.k.ps + int64_t(y.slot) * a.k.ss + int64_t(h) * a.k.hs;
    vo = ko;
    if (!one_layout) vo = id * a.v.ps + int64_t(y.slot) * a.v.ss + int64_t(h) * a.v.hs;
    ksc = *scale_at(a8.ks, id, y.block, h);
    vsc = *scale_at(a8.vs, id, y.block, h);   // (looked at in the next step only)
  };
  u32x4 k[S::NP], v[S::NP];
  const auto load = [&](u32x4(&x)[S::NP], const void *c, int64_t at) {
    const char *p = static_cast<const char *>(c) + lbyte;
    int64_t r[S::NP];
#pragma unroll
    for (int i = 0; i < S::NP; ++i) r[i] = __shfl(at, srow + S::RP * i);
#pragma unroll
    for (int i = 0; i < S::NP; ++i) x[i] = ld16<true>(reinterpret_cast<const u32x4 *>(p + r[i]));
  };
  const auto to_lds = [&](u32x4(&x)[S::NP]) {
    if (padded)
#pragma unroll
      for (int i = 0; i < S::NP; ++i)
        if (!inside) x[i] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < S::NP; ++i)
      *reinterpret_cast<u32x4 *>(vl + (srow + S::RP * i) * S::LS + sbyte) = x[i];
  };

  int32_t page = look_up(far, far_step);
  advance(far, far_step);
  rows_of(ahead, ahead_step, page);
  load(k, a.k.p, ko);
  // (loads return in order: before those of V, which need not be there for it)
  page = look_up(far, far_step);
  load(v, a.v.p, vo);
  ahead = far;
  ahead_step = far_step;
  if (far.r >= 0) advance(far, far_step);

  // product i of K takes elements 64 (i / 2) + 16 quarter + 8 (i % 2) .. of a row
  u32x4 q[2 * NS][QP];
  f32x4 o[ND];
  float m, l;
  int32_t my_lo, my_hi, all_lo, all_hi, odd_b, odd_e;
  // (behind the last unit loads are of keys that are not there: with a branch around
  // them the compiler waits for all loads at every step)
  for (;;) {
    if (now_step == 0) {
      // what the lane's query sees (rows behind the tile's last do as that one), and
      // what all rows see
      const Request rq = nb.request(now.r);
      const Span sp = span_of<TM>(a, rq, now.row0);
      const int c = n % TM;
      const uint32_t x = uint32_t(now.row0 + (c < sp.rows ? c : sp.rows - 1));
      const uint32_t tok = fast_div(x, a.g_div);
      const int32_t token = rq.q0 + int32_t(tok);
      const int32_t head = (int32_t(now.kh) + hn) * a.g + int32_t(x - tok * uint32_t(a.g));
      const int32_t my_p = rq.kv - (rq.q1 - token);
      my_lo = my_p < 0 ? 0 : first_key(my_p, a.window);
      my_hi = my_p + 1;
      all_lo = sp.p1 < 0 ? 0 : first_key(sp.p1, a.window);
      all_hi = sp.p0 + 1;
      const char *p = static_cast<const char *>(a.q) +
                      (int64_t(token) * a.q_ts + int64_t(head) * a.hd) * ES;
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) {
        const int d = 64 * (i / 2) + 16 * quarter + 8 * (i % 2);
        load_query<DT, QP>(p + d * ES, d < a.hd, a.flip, q[i]);
      }
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i] = f32x4{0, 0, 0, 0};
      m = kNegInf;
      l = 0.0f;
      odd_b = odd_e = 0;
    }
    const int32_t k0 = now.b + (now_step * NW + wave) * KH;
    const uint64_t there = seen;
    const int32_t k1 = k0 + KH < now.e ? k0 + KH : now.e;
    const bool mixed = clean || k0 < all_lo || k1 > all_hi;   // some row sees not all of them
    const bool partial = mixed || there != ~uint64_t(0);
    bool odd = false;
    float vs = (there >> lane) & 1 ? vsc : 0.0f;
    if (mixed && vs != vs) {
      odd = true;
      vs = 0.0f;
    }
    scales[wave][0][lane] = ksc * a8.scale;
    scales[wave][1][lane] = vs;
    to_lds(k);
    rows_of(ahead, ahead_step, page);
    load(k, a.k.p, ko);
    page = look_up(far, far_step);
    // S^T
    f32x4 st[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) {
      st[j] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(vl + (16 * j + n) * S::LS + quarter * 16 +
                                                         64 * s);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bf16x8 y = codes_bf16<CT>(u32x2{x[2 * i], x[2 * i + 1]});
#pragma unroll
          for (int c = QP - 1; c >= 0; --c)   // (the small parts first)
            st[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                y, __builtin_bit_cast(bf16x8, q[2 * s + i][c]), st[j], 0, 0, 0);
        }
      }
    }
    // V in K's place. Codes that are not there become zero, so that no weight of 0 meets a
    // NaN (in LDS: changed on their way they would take as many registers again)
    to_lds(v);
    if (CT == kE4M3 && partial) {
#pragma unroll 1
      for (int i = 0; i < S::NP; ++i) {
        u32x4 *p = reinterpret_cast<u32x4 *>(vl + (srow + S::RP * i) * S::LS + sbyte);
        u32x4 x = {0, 0, 0, 0};
        if ((there >> (srow + S::RP * i)) & 1) x = *p;
        if (mixed) odd |= clear_nan_codes<CT>(x);
        *p = x;
      }
    }
    if (mixed && __ballot(odd)) {
      if (odd_b == odd_e) odd_b = k0;
      odd_e = k1;
    }
    load(v, a.v.p, vo);
    // softmax over the column's own head: the lane's keys are k0 + 16 j + 4 quarter + i, j < MH
    f32x4 sc[MH];
#pragma unroll
    for (int j = 0; j < MH; ++j) {
      sc[j] = st[j];
#pragma unroll
      for (int h = 1; h < HG; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[j][i] = hn == h ? st[h * MH + j][i] : sc[j][i];
      sc[j] *= *reinterpret_cast<const f32x4 *>(&scales[wave][0][KH * hn + 16 * j + 4 * quarter]);
    }
    if (partial) {
      const uint64_t see = in_range(there >> (KH * hn), k0, my_lo, my_hi) >> (4 * quarter);
#pragma unroll
      for (int j = 0; j < MH; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sc[j][i] = (uint32_t(see >> (32 * (j / 2))) >> (16 * (j % 2) + i)) & 1 ? sc[j][i] : kNegInf;
    }
    float top = kNegInf;
#pragma unroll
    for (int j = 0; j < MH; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[j][i]);
    top = max_16_32(top);
    const float mn = fmaxf(m, top);
    const float ms = mn == kNegInf ? 0.0f : mn;
    const float alpha = exp2_hw(m - ms);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] *= alpha;
    uint32_t p[MH][2][WP];   // the weights' parts
#pragma unroll
    for (int j = 0; j < MH; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[j][i] = exp2_hw(sc[j][i] - ms);
        l += sc[j][i];
      }
      sc[j] *= *reinterpret_cast<const f32x4 *>(&scales[wave][1][KH * hn + 16 * j + 4 * quarter]);
#pragma unroll
      for (int i = 0; i < 2; ++i) bf16_parts<WP>(sc[j][2 * i], sc[j][2 * i + 1], p[j][i]);
    }
    // O^T, 32 rows of V at a time: 8 of a quarter's in the order of S^T
#pragma unroll
    for (int g = 0; g < KB / 32; ++g) {
      u32x4 w[WP];
#pragma unroll
      for (int c = 0; c < WP; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int y = 2 * g + j;
            w[c][2 * j + i] = HG == 1 || hn == y / MH ? p[y % MH][i][c] : 0u;
          }
      const int row = 32 * g + 4 * quarter + ((n >> 1) & 3) + 16 * (n >> 3);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const bf16x8 y = codes_bf16<CT>(lds_transpose8(vl + row * S::LS + 16 * d + 8 * (n & 1)));
#pragma unroll
        for (int c = WP - 1; c >= 0; --c)
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, __builtin_bit_cast(bf16x8, w[c]), o[d], 0, 0,
                                                         0);
      }
    }

    if (now_step + 1 == now.steps) {
      l = sum_16_32(l);
      if (CT == kE4M3 && HG > 1 && !clean && __ballot(holds_not_finite<ND>(o, 4, l))) again = true;
      for (int32_t x0 = odd_b; x0 < odd_e; x0 += NW * KH) {   // (the wavefront's own steps)
        const uint32_t h = now.kh + uint32_t(lane_head);
        const char *vp = static_cast<const char *>(a.v.p) + int64_t(h) * a.v.hs;
        const NanKeys x = nan_keys<CT>(x0 + lane_key, x0 + lane_key < now.e,
                                       a.table + now.r * a.table_rs, vp, h, a8);
        for (uint64_t keys = x.odd; keys; keys &= keys - 1) {
          const int i = __builtin_ctzll(keys);
          const int32_t key = x0 + i % KH;
          const char *c = static_cast<const char *>(a.v.p) +
                          int64_t(now.kh + uint32_t(i / KH)) * a.v.hs + __shfl(x.at, i);
          const bool sees = hn == i / KH && key >= my_lo && key < my_hi;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            float z[4] = {o[d][0], o[d][1], o[d][2], o[d][3]};
            add_nan<CT>(c, sees, (x.whole >> i) & 1, 16 * d + 4 * quarter, a.hd, z);
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
      const int row = threadIdx.x / PR, share = threadIdx.x % PR;
      const Request rq = nb.request(now.r);
      if (row % TM < span_of<TM>(a, rq, now.row0).rows) {
        // (all at once: with branches these reads took 2 us one after the other)
        float f[NW], wl[NW], top = kNegInf, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          wl[w] = wave_l[w][row];
          f[w] = wl[w] != 0.0f ? wave_m[w][row] : kNegInf;
          top = fmaxf(top, f[w]);
        }
        const float ts = top == kNegInf ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          f[w] = wl[w] != 0.0f ? exp2_hw(f[w] - ts) : 0.0f;
          sum += wl[w] != 0.0f ? f[w] * wl[w] : 0.0f;
        }
        const uint32_t x = uint32_t(now.row0 + row % TM), tok = fast_div(x, a.g_div);
        const int32_t to = rq.q0 + int32_t(tok);
        const int32_t oh = (int32_t(now.kh) + row / TM) * a.g + int32_t(x - tok * uint32_t(a.g));
        const int64_t slot = (int64_t(to) * a.nq + oh) * a.splits + now.part;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int c = 0; c < (HDP + 4 * PR - 1) / (4 * PR); ++c) {
          const int d = 4 * PR * c + 4 * share;
          if (d >= a.hd) break;
          f32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int w = 0; w < NW; ++w) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(
                reinterpret_cast<const float *>(lds + w * S::WAVE_LDS) + row * S::OS + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = fmaf(f[w], y[i], acc[i]);
          }
          if (now.part >= 0) {
            *reinterpret_cast<f32x4 *>(a.part + slot * a.hd + d) = acc;
          } else {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = sum == 0.0f ? 0.0f : acc[i] * inv;
            store4<DT>(a, to, oh, d, y);
          }
        }
        if (now.part >= 0 && share == 0) {
          a.ml[2 * slot] = top;
          a.ml[2 * slot + 1] = sum;
        }
      }
      // (the barrier: the sums are read)
      if (ahead.r < 0) {
        if (CT == kInt8 || HG == 1 || clean || !__syncthreads_or(again)) return;
        clean = true;
        goto start;
      }
      __syncthreads();
    }
    now = ahead;
    now_step = ahead_step;
    ahead = far;
    ahead_step = far_step;
    if (far.r >= 0) advance(far, far_step);
  }
}

// ---- PA8_TILE -----------------------------------------------------------------------------------
// Many rows per request (chunks of a prompt), as PA_TILE: a tile of 128 rows, 32 of them a
// wavefront's, against 64 keys at a time that the workgroup stages in LDS, here as the bf16
// numbers that their codes are: converted once, on the way to LDS, not by each of the
// four wavefronts. Two of these fetch the step's K and V scales, one a lane, which all
// read from LDS in fours (one of each four, where neighbouring keys share it, gained 1.5 %
// only: 2048 tokens behind 6144, 291 -> 287 us). The running maximum as in PA_TILE. bf16
// weights, times their V scales, are one part, rounded: that adds to the rounding of the result about as
// much again (0.0017 -> 0.0020 .. 0.0025 against 64 bits; in int8, where one key has nearly all of most rows'
// weight and its rounding is every element's, up to 0.0030), and a second part, as few rows have it, would
// take 362 us for the 288 of those tokens, 41.0 for 36.5 of the windowed mixture, 64.1 for 56.6 of the
// prompts. float32 ones are three parts, as are queries: those 2048 tokens 729 us, 330 TFLOP/s (990 of
// products in bf16); 1024 behind 3072, 16 and 8 heads of 256, whose registers spill, 268 (bf16 119).
// Bound, as there, by each wavefront's chain of products, exponentials and LDS reads: those 2048
// tokens, 32 and 8 heads of 128, 826 TFLOP/s in e4m3, 799 in int8 (from bf16 pages 845); a prompt's
// last tile alone, 1024 keys of heads of 256, takes the 57 us of four such prompts.
template <int DT, int HDP>
struct Tile8Shape {
  static constexpr int ES = Elt<DT>::ES;
  static constexpr int KB = 64;
  static constexpr int NB = KB / 32;
  static constexpr int QP = DT == kF32 ? 3 : 1;           // parts of a query, of a weight
  static constexpr int NQ = HDP / 16;                     // products of a lane's query
  static constexpr int ND = HDP / 32;
  // bytes of a row in LDS, as for bf16 in PA_TILE
  static constexpr int KS = HDP * 2 + 16;
  static constexpr int VS = HDP * 2 + 64;
  static constexpr int BUF = KB * (KS + VS);
  static constexpr int CH = HDP / 16;                     // vectors of a row of codes
  static constexpr int RP = 256 / CH;                     // rows that a pass stages
  static constexpr int NP = KB / RP;
};

template <int DT, int CT, int HDP, int KG>
__device__ void body_pa8_tile(const PagedQ8Args &a8) {
  typedef Tile8Shape<DT, HDP> S;
  constexpr int ES = S::ES, KB = S::KB, NB = S::NB, NQ = S::NQ, ND = S::ND, NP = S::NP, QP = S::QP;
  constexpr int GROUP = 2 * S::BUF, STEP = KG * KB;
  const PagedArgs &a = a8.a;
  __shared__ __attribute__((aligned(16))) char all_lds[KG * GROUP];
  __shared__ __attribute__((aligned(16))) float all_scales[KG][2][2][KB];   // s c of K, s of V
  __shared__ int32_t odd_b, odd_e;   // from the first to the last step with NaN that was cleared
  // four wavefronts a group; group g takes the steps g, g + KG, ... of the keys
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int tid = threadIdx.x & 255, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char *lds = all_lds + group * GROUP;
  float(*scales)[2][KB] = all_scales[group];
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

  u32x4 q[NQ][QP];
  {
    const char *p = static_cast<const char *>(a.q) +
                    (int64_t(token) * a.q_ts + int64_t(head) * a.hd) * ES;
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      const int d = 16 * s + 8 * half;
      load_query<DT, QP>(p + d * ES, d < a.hd, a.flip, q[s]);
    }
  }
  const int32_t *table = a.table + int64_t(t.r) * a.table_rs;
  const char *kp = static_cast<const char *>(a.k.p) + int64_t(kh) * a.k.hs;
  const char *vp = static_cast<const char *>(a.v.p) + int64_t(kh) * a.v.hs;

  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = kNegInf, l = 0.0f;

  // staging: this work-item's vector of rows srow + RP i
  const int srow = tid / S::CH, sbyte = (tid % S::CH) * 16;
  // (behind the head's end as in PA8_ROWS)
  const bool padded = a.hd < HDP, inside = sbyte < a.hd;
  const int lbyte = inside ? sbyte : 0;
  // the page of key k0 + lane (beyond the end: the last key's)
  const auto look_up = [&](int32_t k0) {
    const int32_t key = k0 + lane;
    return table[fast_div(uint32_t(key < e ? key : e - 1), a.div)];
  };
  u32x4 sk[NP], sv[NP];
  float sscale;          // K's (even wavefronts) or V's scale of the lane's key
  uint64_t seen = 0;     // bit i: key k0 + i of the staged step is there
  const bool one_layout = a.k.ps == a.v.ps && a.k.ss == a.v.ss;
  const ScaleView my_scale = wave & 1 ? a8.vs : a8.ks;
  const auto load = [&](int32_t k0, int32_t page) {
    // where the lane's key lies (the pool's first page for one that is not
    // there), handed to the lanes that load its row
    const int32_t mine = k0 + lane;
    const KeyPlace x = place_of(uint32_t(mine < e ? mine : e - 1), page, a8);
    const bool ok = mine < e && x.id >= 0;
    seen = __ballot(ok);
    const int64_t id = ok ? x.id : 0;
    sscale = *scale_at(my_scale, id, x.block, kh);
    const int64_t ko = id * a.k.ps + int64_t(x.slot) * a.k.ss;
    int64_t vo = ko;
    if (!one_layout) vo = id * a.v.ps + int64_t(x.slot) * a.v.ss;
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
  // codes of V that are not there are zero, and their scales, so that no weight of 0 meets
  // a NaN
  const auto store = [&](int32_t k0, int buf) {
    char *kl = lds + buf * S::BUF, *vl = kl + KB * S::KS;
    const int32_t k1 = k0 + KB < e ? k0 + KB : e;
    const bool mixed = k0 < all_lo || k1 > all_hi;
    const bool some = seen != ~uint64_t(0);
    bool odd = false;
    if (wave < 2) {
      float s = sscale;
      if (wave == 0) {
        s *= a8.scale;
      } else {
        if (some && !((seen >> lane) & 1)) s = 0.0f;
        if (mixed && s != s) {
          odd = true;
          s = 0.0f;
        }
      }
      scales[buf][wave][lane] = s;
    }
    if (padded)
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (!inside) sk[i] = sv[i] = u32x4{0, 0, 0, 0};
    if constexpr (CT == kE4M3) {
      if (some)
#pragma unroll
        for (int i = 0; i < NP; ++i)
          if (!((seen >> (srow + S::RP * i)) & 1)) sv[i] = u32x4{0, 0, 0, 0};
      if (mixed)
#pragma unroll
        for (int i = 0; i < NP; ++i) odd |= clear_nan_codes<CT>(sv[i]);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = srow + S::RP * i;
      bf16x8 *k = reinterpret_cast<bf16x8 *>(kl + r * S::KS + 2 * sbyte);
      bf16x8 *v = reinterpret_cast<bf16x8 *>(vl + r * S::VS + 2 * sbyte);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        k[c] = codes_bf16<CT>(u32x2{sk[i][2 * c], sk[i][2 * c + 1]});
        v[c] = codes_bf16<CT>(u32x2{sv[i][2 * c], sv[i][2 * c + 1]});
      }
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
      // before them
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
        const bf16x8 y = __builtin_bit_cast(bf16x8, k[i % kAhead]);
#pragma unroll
        for (int c = QP - 1; c >= 0; --c)
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, __builtin_bit_cast(bf16x8, q[i / NB][c]), x, 0,
                                                      0, 0);
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
        // keys 16 s + 4 half + (0..3 and 8..11)
        const int s = i / ND, d = i % ND;
        const char *x = vl + (16 * s + 4 * half + ((lane & 15) >> 2)) * S::VS +
                        (32 * d + (lane & 16) + 4 * (lane & 3)) * 2;
        const u32x2 y0 = lds_transpose(x), y1 = lds_transpose(x + 8 * S::VS);
        return u32x4{y0[0], y0[1], y1[0], y1[1]};
      };
      u32x4 y[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) y[i] = read_v(i);
      // the lane's keys are k0 + 32 j + 8 c + 4 half + i, element 4 c + i
      const auto scales_of = [&](int kind, int j, int c) {
        return *reinterpret_cast<const f32x4 *>(&scales[buf][kind][32 * j + 8 * c + 4 * half]);
      };
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x4 x = scales_of(0, j, c);
#pragma unroll
          for (int i = 0; i < 4; ++i) st[j][4 * c + i] *= x[i];
        }
      f32x4 vs[NB * 4];
#pragma unroll
      for (int c = 0; c < NB * 4; ++c) vs[c] = scales_of(1, c / 4, c % 4);
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
      if (__ballot(top - m > 8.0f)) {
        const float mn = fmaxf(m, top);
        const float alpha = exp2_hw(m - (mn == kNegInf ? 0.0f : mn));
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
      // O^T, product i: elements 32 (i % ND) .. of V at keys 16 (i / ND) ... The reads of V
      // run ahead as those of K; the weights of the next keys are formed between the products.
      constexpr int NV = KB / 16 * ND;
      constexpr int WC = 8;                           // weights of a lane for ND products
      constexpr int WP = (WC + ND - 1) / ND;          // formed at each of them
      const auto weight = [&](int c) {
        const float x = exp2_hw(st[c / 16][c % 16] - ms);
        l += x;
        st[c / 16][c % 16] = x * vs[c / 4][c % 4];
      };
#pragma unroll
      for (int c = 0; c < WC; ++c) weight(c);
      u32x4 p[QP];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = i / ND, d = i % ND;
        if (d == 0) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t x[QP];
            bf16_parts<QP>(st[s / 2][8 * (s % 2) + 2 * c], st[s / 2][8 * (s % 2) + 2 * c + 1], x);
#pragma unroll
            for (int f = 0; f < QP; ++f) p[f][c] = x[f];
          }
        }
#pragma unroll
        for (int c = QP - 1; c >= 0; --c)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, y[i % kAhead]),
                                                         __builtin_bit_cast(bf16x8, p[c]), o[d], 0, 0,
                                                         0);
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
        const float f0 = l != 0.0f ? exp2_hw(m - ts) : 0.0f;
        const float f1 = l1 != 0.0f ? exp2_hw(m1 - ts) : 0.0f;
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
  if (b < e && odd_b < odd_e) {
    for (int32_t x0 = odd_b; x0 < odd_e; x0 += 64) {
      const NanKeys k = nan_keys<CT>(x0 + lane, x0 + lane < odd_e, table, vp, kh, a8);
      for (uint64_t keys = k.odd; keys; keys &= keys - 1) {
        const int i = __builtin_ctzll(keys);
        const char *x = vp + __shfl(k.at, i);
        const bool sees = x0 + i >= my_lo && x0 + i < my_hi;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float z[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) z[c] = o[d][4 * j + c];
            add_nan<CT>(x, sees, (k.whole >> i) & 1, 32 * d + 8 * j + 4 * half, a.hd, z);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[d][4 * j + c] = z[c];
          }
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
