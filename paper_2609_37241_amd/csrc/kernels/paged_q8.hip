// The paged KV cache in 8 bits: rows into it (Q8W_*) and out of it (Q8R_*),
// attention at any alignment and head size (PA8_ANY).
#include "../internal.h"
#include "attn_q8.h"
#include "join.h"

namespace tri {
using namespace dev;

// ---- Q8W_* ------------------------------------------------------------------------------------
// A wavefront quantises the tokens that a call adds to one block, of one head of K or V:
// it takes the largest magnitude, makes the scale, and reads the rows again for their
// codes. Blocks are numbered through the requests without knowing their lengths on the
// host: those of r start at floor(q_start[r] / B) + 2 r, which leaves each request
// room for the floor((n - 2) / B) + 2 blocks that n tokens can touch. The
// wavefront has its block's scale to itself: no atomics, the same bits every time.
namespace {

// The block that wavefront `unit` of the numbering writes.
struct Touched {
  int64_t id;              // page, -1: nothing to do
  uint32_t block;          // of the page
  int32_t slot, held;      // first slot of the block; tokens that it holds already
  int32_t first, last;     // rows of k and v
};

__device__ inline Touched touched(const Q8RowsArgs &a, int64_t unit) {
  Touched t;
  t.id = -1;
  const int32_t r = __builtin_amdgcn_readfirstlane(last_request(a.R, [&](int32_t x) {
    return int64_t(fast_div(uint32_t(clamp_i32(a.q_start[x], 0, a.T)), a.block_div)) + 2 * int64_t(x) <=
           unit;
  }));
  if (r < 0) return t;
  const Request rq = request_of(a, r);
  const int32_t n = rq.q1 - rq.q0, base = rq.kv - n, lo = base < 0 ? 0 : base;
  if (n <= 0) return t;
  const int64_t j = unit - (int64_t(fast_div(uint32_t(rq.q0), a.block_div)) + 2 * int64_t(r));
  const int64_t begin = (int64_t(fast_div(uint32_t(lo), a.block_div)) + j) * a.block;
  if (begin >= rq.kv) return t;
  const uint32_t col = fast_div(uint32_t(begin), a.div);
  const int32_t id = a.table[r * a.table_rs + col];
  if (uint32_t(id) >= uint32_t(a.n_pages)) return t;
  t.slot = int32_t(uint32_t(begin) - col * uint32_t(a.page));
  t.block = fast_div(uint32_t(t.slot), a.block_div);
  const int32_t from = begin < lo ? lo : int32_t(begin);
  const int32_t to = rq.kv - begin > a.block ? int32_t(begin) + a.block : rq.kv;
  t.held = from - int32_t(begin);
  t.first = from - base + rq.q0;
  t.last = to - base + rq.q0;
  t.id = id;
  return t;
}

// Four elements of a row, or one.
template <int DT, bool VEC>
__device__ inline void load4(const char *p, float *x) {
  if constexpr (!VEC) {
    x[0] = Elt<DT>::ld(p, 0);
    x[1] = x[2] = x[3] = 0.0f;
  } else if constexpr (DT == kF32) {
    Elt<kF32>::unpack(*reinterpret_cast<const u32x4 *>(p), x);
  } else {
    const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
}

template <bool VEC>
__device__ inline uint32_t load_codes(const char *p) {
  if constexpr (VEC)
    return *reinterpret_cast<const uint32_t *>(p);
  else
    return *reinterpret_cast<const uint8_t *>(p);
}

template <bool VEC>
__device__ inline void store_codes(char *p, uint32_t c) {
  if constexpr (VEC)
    *reinterpret_cast<uint32_t *>(p) = c;
  else
    *reinterpret_cast<uint8_t *>(p) = uint8_t(c);
}

}  // namespace

template <int DT, int CT, bool VEC>
__global__ __launch_bounds__(256) void k_q8_write(Q8RowsArgs a) {
  constexpr int N = VEC ? 4 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t parts = 2 * uint32_t(a.nk);
  const int64_t items = (int64_t(fast_div(uint32_t(a.T), a.block_div)) + 2 * int64_t(a.R)) * parts;
  const int per = a.hd / N;   // work-items of a row
  for (int64_t it = int64_t(blockIdx.x) * 4 + wave; it < items; it += int64_t(gridDim.x) * 4) {
    const int64_t unit = it / parts;
    const uint32_t part = uint32_t(it - unit * parts);
    const bool is_v = part >= uint32_t(a.nk);
    const uint32_t h = is_v ? part - uint32_t(a.nk) : part;
    const Touched t = touched(a, unit);
    if (t.id < 0) continue;
    const int64_t ts = is_v ? a.v_ts : a.k_ts;
    const char *x = static_cast<const char *>(is_v ? a.v : a.k) +
                    (t.first * ts + int64_t(h) * a.hd) * Elt<DT>::ES;
    const PagedView &view = is_v ? a.cv : a.ck;
    char *c = static_cast<char *>(view.p) + t.id * view.ps + int64_t(t.slot) * view.ss +
              int64_t(h) * view.hs;
    float *scale = scale_at(is_v ? a.sv : a.sk, t.id, t.block, h);
    const float was = *scale;
    // the largest magnitude: as whole numbers, so that infinities and NaN are above all
    const int n = (t.last - t.first) * per;
    uint32_t most = 0;
    for (int i = lane; i < n; i += 64) {
      const int row = i / per, e = (i - row * per) * N;
      float f[4];
      load4<DT, VEC>(x + (row * ts + e) * Elt<DT>::ES, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t b = __float_as_uint(f[j]) & 0x7FFFFFFFu;
        most = b > most ? b : most;
      }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      const uint32_t b = __shfl_xor(most, d);
      most = b > most ? b : most;
    }
    const float need = scale_for<CT>(most);
    // (a scale of NaN stays one)
    const float now = t.held == 0 || need != need || need > was ? need : was;
    if (t.held > 0 && now > was) {
      for (int i = lane; i < t.held * per; i += 64) {
        const int row = i / per, e = (i - row * per) * N;
        char *p = c + row * view.ss + e;
        store_codes<VEC>(p, recode4<CT>(load_codes<VEC>(p), was, now));
      }
    }
    if (lane == 0) *scale = now;
    const Rounder r = rounder(now);
    for (int i = lane; i < n; i += 64) {
      const int row = i / per, e = (i - row * per) * N;
      float f[4];
      load4<DT, VEC>(x + (row * ts + e) * Elt<DT>::ES, f);
      store_codes<VEC>(c + (t.held + row) * view.ss + e, to_codes4<CT>(f, r));
    }
  }
}

// ---- Q8R_* ------------------------------------------------------------------------------------
// A wavefront gives one row of K and V back, four elements a work-item.
template <int DT, int CT, bool VEC>
__global__ __launch_bounds__(256) void k_q8_read(Q8RowsArgs a) {
  constexpr int N = VEC ? 4 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t row = int64_t(blockIdx.x) * 4 + wave; row < a.T; row += int64_t(gridDim.x) * 4) {
    const int32_t r = __builtin_amdgcn_readfirstlane(
        last_request(a.R, [&](int32_t x) { return a.q_start[x] <= row; }));
    if (r < 0) continue;
    const Request rq = request_of(a, r);
    if (row < rq.q0 || row >= rq.q1) continue;
    const int32_t p = rq.kv - (rq.q1 - int32_t(row));
    int64_t id = -1;
    uint32_t slot = 0;
    if (p >= 0) {
      const uint32_t col = fast_div(uint32_t(p), a.div);
      const int32_t x = a.table[r * a.table_rs + col];
      id = uint32_t(x) < uint32_t(a.n_pages) ? x : -1;
      slot = uint32_t(p) - col * uint32_t(a.page);
    }
    const uint32_t block = fast_div(slot, a.block_div);
    const int per = a.hd / N, half = a.nk * per;
    for (int i = lane; i < 2 * half; i += 64) {
      const bool is_v = i >= half;
      const int j = is_v ? i - half : i, h = j / per, e = (j - h * per) * N;
      const PagedView &view = is_v ? a.cv : a.ck;
      float f[4] = {};
      if (id >= 0) {
        const char *c = static_cast<const char *>(view.p) + id * view.ps + int64_t(slot) * view.ss +
                        int64_t(h) * view.hs + e;
        const float s = *scale_at(is_v ? a.sv : a.sk, id, block, uint32_t(h));
        if constexpr (VEC) {
          codes4<CT>(load_codes<VEC>(c), f);
#pragma unroll
          for (int k = 0; k < 4; ++k) f[k] *= s;
        } else {
          f[0] = code1<CT>(uint8_t(load_codes<VEC>(c))) * s;
        }
      }
      char *o = static_cast<char *>(is_v ? a.v : a.k) +
                (row * (is_v ? a.v_ts : a.k_ts) + int64_t(h) * a.hd + e) * Elt<DT>::ES;
      if constexpr (!VEC)
        Elt<DT>::st(o, 0, f[0]);
      else if constexpr (DT == kF32)
        *reinterpret_cast<u32x4 *>(o) = Elt<kF32>::pack(f);
      else
        *reinterpret_cast<u32x2 *>(o) =
            u32x2{Elt<kBF16>::pack2(f[0], f[1]), Elt<kBF16>::pack2(f[2], f[3])};
    }
  }
}

// ---- PA8_ANY ----------------------------------------------------------------------------------
// As PA_ANY: a wavefront per row, query head and split, a lane a key of 64 for the
// scores, and elements l, l + 64, ... of the head for the sums. A key that is not
// seen is never read. Scores are in powers of two from the start: (q.k s) c.
template <int DT, int CT>
__global__ __launch_bounds__(256) void k_pa8_any(PagedQ8Args a8) {
  constexpr int ES = Elt<DT>::ES;
  constexpr int NI = 8;   // 512 / 64
  const PagedArgs &a = a8.a;
  __shared__ float qs[4][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t items = int64_t(a.T) * a.nq * a.splits;
  for (int64_t it = int64_t(blockIdx.x) * 4 + wave; it < items; it += int64_t(gridDim.x) * 4) {
    const int64_t row = it / a.splits;
    const int32_t s = int32_t(it - row * a.splits);
    const int32_t t = int32_t(row / a.nq), h = int32_t(row - int64_t(t) * a.nq);
    const int32_t r = last_request(a.R, [&](int32_t x) { return a.q_start[x] <= t; });
    if (r < 0) continue;
    const Request rq = request_of(a, r);
    if (t < rq.q0 || t >= rq.q1) continue;
    const int32_t p = rq.kv - (rq.q1 - t);
    const int32_t lo = p < 0 ? 0 : first_key(p, a.window), hi = p + 1;
    int32_t b, e;
    split_keys(lo, hi, a.splits, s, &b, &e);
    const char *qp = static_cast<const char *>(a.q) + (int64_t(t) * a.q_ts + int64_t(h) * a.hd) * ES;
    for (int d = lane; d < a.hd; d += 64) {
      const float x = Elt<DT>::ld(qp, d);
      qs[wave][d] = a.flip ? -x : x;
    }
    const int32_t kh = int32_t(fast_div(uint32_t(h), a.g_div));
    const int32_t *table = a.table + r * a.table_rs;
    const uint8_t *kp = static_cast<const uint8_t *>(a.k.p) + int64_t(kh) * a.k.hs;
    const uint8_t *vp = static_cast<const uint8_t *>(a.v.p) + int64_t(kh) * a.v.hs;
    float m = kNegInf, l = 0.0f, acc[NI] = {};
    for (int32_t k0 = b; k0 < e; k0 += 64) {
      const int32_t key = k0 + lane;
      int64_t vo = -1;
      float sc = kNegInf, vs = 0.0f;
      if (key < e) {
        const uint32_t col = fast_div(uint32_t(key), a.div);
        const int32_t id = table[col];
        if (uint32_t(id) < uint32_t(a.n_pages)) {
          const uint32_t slot = uint32_t(key) - col * uint32_t(a.page);
          const uint32_t block = fast_div(slot, a8.block_div);
          const uint8_t *k = kp + id * a.k.ps + int64_t(slot) * a.k.ss;
          vo = id * a.v.ps + int64_t(slot) * a.v.ss;
          vs = *scale_at(a8.vs, id, block, uint32_t(kh));
          float x[4] = {};   // four sums: shorter chains, smaller errors
          int d = 0;
          for (; d + 4 <= a.hd; d += 4)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = fmaf(qs[wave][d + i], code1<CT>(k[d + i]), x[i]);
          for (; d < a.hd; ++d) x[0] = fmaf(qs[wave][d], code1<CT>(k[d]), x[0]);
          sc = (((x[0] + x[1]) + (x[2] + x[3])) * *scale_at(a8.ks, id, block, uint32_t(kh))) * a8.scale;
        }
      }
      const uint64_t seen = __ballot(vo >= 0);
      float top = sc;
#pragma unroll
      for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      const float mn = fmaxf(m, top);
      const float ms = mn == kNegInf ? 0.0f : mn;
      const float alpha = exp2_hw(m - ms);
      const float w = vo >= 0 ? exp2_hw(sc - ms) : 0.0f;
      float sum = w;
#pragma unroll
      for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
      l = l * alpha + sum;
      m = mn;
      const float wv = w * vs;
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i] *= alpha;
      for (int j = 0; j < 64; ++j) {
        if (!((seen >> j) & 1)) continue;
        const float wj = __shfl(wv, j);
        const uint8_t *v = vp + __shfl(vo, j);
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (lane + 64 * i < a.hd) acc[i] = fmaf(wj, code1<CT>(v[lane + 64 * i]), acc[i]);
      }
    }
    if (a.splits > 1) {
      const int64_t at = row * a.splits + s;
      if (lane == 0) {
        a.ml[2 * at] = m;
        a.ml[2 * at + 1] = l;
      }
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (lane + 64 * i < a.hd) a.part[at * a.hd + lane + 64 * i] = acc[i];
    } else {
      char *o = static_cast<char *>(a.out) + (int64_t(t) * a.o_ts + int64_t(h) * a.hd) * ES;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (lane + 64 * i < a.hd)
          Elt<DT>::st(o, lane + 64 * i, l == 0.0f ? 0.0f : acc[i] / l);
    }
  }
}

// ---- PA8_JOIN: the parts of the tiles that PA8_ROWS cut (join.h) -----------------------------
template <int DT, int HG>
__global__ __launch_bounds__(256) void k_pa8_join(PagedQ8Args a8) {
  constexpr int TM = 16 / HG;
  const PagedArgs &a = a8.a;
  __shared__ int32_t sums[TRI_MAX_REQUESTS], wave_sums[8];
  Numbering<TM> nb{a8, sums, {}, 0, 0, 0};
  nb.template number<4>(wave_sums, a.nk / HG, a8.runs);
  const auto parts_of = [&](int32_t t, int32_t h) {
    const int32_t r = __builtin_amdgcn_readfirstlane(
        last_request(a.R, [&](int32_t x) { return a.q_start[x] <= t; }));
    if (r < 0) return 0;
    const Request rq = nb.request(r);
    const int32_t kh = int32_t(fast_div(uint32_t(h), a.g_div));
    const int32_t tile = ((t - rq.q0) * a.g + h - kh * a.g) / TM, steps = nb.steps_of(rq);
    const uint32_t begin = uint32_t(nb.all * (kh / HG) + nb.before(r) + tile * steps);
    const uint32_t per = uint32_t(nb.per);
    return int32_t((begin + uint32_t(steps) - 1) / per - begin / per) + 1;
  };
  join_rows<DT, 4, kQ8Splits / 64>(a, a8.four != 0, parts_of);
}

namespace {
template <class F>
const void *sym(F *f) {
  return reinterpret_cast<const void *>(f);
}

template <int DT, int CT>
const void *rows_kernel(int32_t variant) {
  switch (variant) {
    case Q8W_ANY: return sym(&k_q8_write<DT, CT, false>);
    case Q8W_VEC: return sym(&k_q8_write<DT, CT, true>);
    case Q8R_ANY: return sym(&k_q8_read<DT, CT, false>);
    case Q8R_VEC: return sym(&k_q8_read<DT, CT, true>);
    case PA8_ANY: return sym(&k_pa8_any<DT, CT>);
    default: return nullptr;
  }
}
}  // namespace

const void *attn_q8_rows(uint32_t dtype, int32_t code, int32_t hdp, int32_t heads);
const void *attn_q8_tile_bf16(bool pair, int32_t code, int32_t hdp);
const void *attn_q8_tile_f32(int32_t code, int32_t hdp);

template <int DT>
static const void *join_kernel(int32_t heads) {
  return heads == 4 ? sym(&k_pa8_join<DT, 4>) : heads == 2 ? sym(&k_pa8_join<DT, 2>) : sym(&k_pa8_join<DT, 1>);
}

// sub: the code (tri_code) in bit 0; for the matrix forms the head size held from bit 6 on,
// for few rows the logarithm of the K heads of a tile in bits 1 and 2.
const void *paged_q8_kernel(int32_t variant, uint32_t dtype, int32_t sub) {
  const bool e4m3 = (sub & 1) == TRI_E4M3;
  const int32_t code = sub & 1, hdp = sub & ~63;
  const int32_t heads = 1 << ((sub >> 1) & 3);
  if (variant == PA8_JOIN)
    return dtype == TRI_F32 ? join_kernel<kF32>(heads) : join_kernel<kBF16>(heads);
  if (variant == PA8_ROWS) return attn_q8_rows(dtype, code, hdp, heads);
  if (variant == PA8_TILE && dtype == TRI_F32) return attn_q8_tile_f32(code, hdp);
  if (variant == PA8_TILE || variant == PA8_PAIR)
    return attn_q8_tile_bf16(variant == PA8_PAIR, code, hdp);
  if (dtype == TRI_F32)
    return e4m3 ? rows_kernel<kF32, kE4M3>(variant) : rows_kernel<kF32, kInt8>(variant);
  return e4m3 ? rows_kernel<kBF16, kE4M3>(variant) : rows_kernel<kBF16, kInt8>(variant);
}

}  // namespace tri
