// The paged KV cache in 8 bits: rows into it (Q8W_*) and out of it (Q8R_*),
// attention at any alignment and head size (PA8_ANY).
#include "../internal.h"
#include "attn_q8.h"
#include "join.h"

namespace tri {
using namespace dev;

namespace {

// The requests of a call: up to 64 held by a lane each, looked up all at once.
struct Requests {
  int32_t q0, q1, kv;
};
__device__ inline Requests requests(const Q8RowsArgs &a) {
  const int lane = threadIdx.x & 63, x = lane < a.R ? lane : 0;
  if (a.R > 64) return {0, 0, 0};
  return {a.q_start[x], a.q_start[x + 1], a.kv_len[x]};
}

// The last request r with first(r, q_start[r] in [0, T]) at or before what is looked for (first()
// tells), -1 if none.
template <class F>
__device__ inline int32_t find_request(const Q8RowsArgs &a, const Requests &h, Request *rq, F &&first) {
  const int lane = threadIdx.x & 63;
  if (a.R <= 64) {
    const uint64_t hit = __ballot(lane < a.R && first(lane, clamp_i32(h.q0, 0, a.T)));
    if (!hit) return -1;
    const int r = 63 - __builtin_clzll(hit);
    *rq = clamped(a, __builtin_amdgcn_readlane(h.q0, r), __builtin_amdgcn_readlane(h.q1, r),
                  __builtin_amdgcn_readlane(h.kv, r));
    return r;
  }
  const int32_t r = __builtin_amdgcn_readfirstlane(
      last_request(a.R, [&](int32_t x) { return first(x, clamp_i32(a.q_start[x], 0, a.T)); }));
  if (r >= 0) *rq = request_of(a, r);
  return r;
}

// A vector of a row (an element: in its first place, as float32), and its N elements.
template <int DT, int N>
__device__ inline u32x4 load_row(const char *p) {
  if constexpr (N == 1)
    return u32x4{__float_as_uint(Elt<DT>::ld(p, 0)), 0, 0, 0};
  else
    return *reinterpret_cast<const u32x4 *>(p);
}
template <int DT, int N>
__device__ inline void elements(const u32x4 &v, float *x) {
  if constexpr (N == 1)
    x[0] = __uint_as_float(v[0]);
  else
    Elt<DT>::unpack(v, x);
}

// N codes as they lie in a register (or two).
template <int N>
struct CodesOf {
  uint32_t w[(N + 3) / 4];
};
template <int N>
__device__ inline CodesOf<N> load_codes(const char *p) {
  CodesOf<N> c;
  if constexpr (N == 1) {
    c.w[0] = *reinterpret_cast<const uint8_t *>(p);
  } else if constexpr (N == 4) {
    c.w[0] = *reinterpret_cast<const uint32_t *>(p);
  } else {
    const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
    c.w[0] = v[0];
    c.w[1] = v[1];
  }
  return c;
}
template <int N>
__device__ inline void store_codes(char *p, const CodesOf<N> &c) {
  if constexpr (N == 1)
    *reinterpret_cast<uint8_t *>(p) = uint8_t(c.w[0]);
  else if constexpr (N == 4)
    *reinterpret_cast<uint32_t *>(p) = c.w[0];
  else
    *reinterpret_cast<u32x2 *>(p) = u32x2{c.w[0], c.w[1]};
}

}  // namespace

// ---- Q8W_* ------------------------------------------------------------------------------------
// A team of L lanes (16, a wavefront, or a workgroup) quantises the tokens that a call adds to one
// block, of one head of K or V: it holds them, 8 vectors a lane (an element a lane, Q8W_ANY),
// takes the largest magnitude, makes the scale and stores the codes; what it cannot hold
// it reads twice. A block belongs to one team alone: no atomics, the same bits every
// time. Bound by memory where there are many rows (8192 of 8 + 8 heads of 128, a scale for 16
// tokens: 14.4 us in e4m3, 7 TB/s, with the rows in the last-level cache; int8, whose exact quotient
// takes more work, 15.3; float32 rows 18.1 and 17.5, 4.7 TB/s), by a chain of four loads (starts, table and
// rows, scale, codes of a block that goes on) for single tokens (8 requests 6.2 us, KVW_VEC 2.4). At any
// alignment, an element a load, by its instructions: 8192 rows of 8 + 8 heads of 100 in bf16 36 us, of 128 an
// element off 44.
// Blocks are numbered through the requests without knowing their lengths on the
// host: n tokens touch at most floor((n - 2) / B) + 2 blocks, and at most n, so those of r
// start at floor(q_start[r] / B) + 2 r, or (a.by_row, the fewer) at q_start[r].
template <int DT, int CT, bool VEC, int L>
__global__ __launch_bounds__(256, L == 16 ? 4 : 5) void k_q8_write(Q8RowsArgs a) {
  constexpr int N = VEC ? Elt<DT>::V : 1, HOLD = 8;
  __shared__ uint32_t team_most[L == 256 ? 4 : 1];
  const int tid = threadIdx.x % L, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Requests held = requests(a);
  // teams of a wavefront take neighbouring heads of one block, a.inner times (what finds the
  // block costs as much as a few vectors)
  constexpr int TW = L < 64 ? 64 / L : 1;
  const uint32_t inner = L == 16 ? a.inner : 1;
  const uint32_t parts = 2 * uint32_t(a.nk), groups = (parts + TW * inner - 1) / (TW * inner);
  const int64_t items = int64_t(a.units) * groups;
  const int64_t first = L == 256 ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wave;
  const int64_t stride = int64_t(gridDim.x) * (L == 256 ? 1 : 4);
  for (int64_t it = first; it < items; it += stride) {
    const uint32_t unit = uint32_t(it / groups);
    const uint32_t part0 = uint32_t(it - int64_t(unit) * groups) * TW * inner;
    Request rq;
    const int32_t r = find_request(a, held, &rq, [&](int32_t x, int32_t q0) {
      return a.by_row ? uint32_t(q0) <= unit
                      : int64_t(fast_div(uint32_t(q0), a.block_div)) + 2 * int64_t(x) <= int64_t(unit);
    });
    if (r < 0) continue;
    const int32_t n = rq.q1 - rq.q0, base = rq.kv - n, lo = base < 0 ? 0 : base;
    if (n <= 0) continue;
    const int64_t j = a.by_row ? int64_t(unit) - rq.q0
                               : unit - (int64_t(fast_div(uint32_t(rq.q0), a.block_div)) + 2 * int64_t(r));
    const int64_t begin = (int64_t(fast_div(uint32_t(lo), a.block_div)) + j) * a.block;
    if (begin >= rq.kv) continue;
    const uint32_t col = fast_div(uint32_t(begin), a.div);
    const int32_t id = a.table[r * a.table_rs + col];
    // tokens that the block holds, and the rows that it gets
    const int32_t from = begin < lo ? lo : int32_t(begin);
    const int32_t to = rq.kv - begin > a.block ? int32_t(begin) + a.block : rq.kv;
    const int32_t old = from - int32_t(begin), row0 = from - base + rq.q0;
    const int32_t items_new = (to - from) * a.per;   // work-items
    const uint32_t slot = uint32_t(begin) - col * uint32_t(a.page);
    for (uint32_t in = 0; in < inner; ++in) {
      uint32_t part = part0 + in * TW;
      if (part >= parts) break;
      if constexpr (TW > 1) part += (threadIdx.x & 63) / L;
      const bool active = part < parts;
      const bool is_v = part >= uint32_t(a.nk);
      const uint32_t h = is_v ? part - uint32_t(a.nk) : part;
      const int64_t ts = is_v ? a.v_ts : a.k_ts;
      const char *x = static_cast<const char *>(is_v ? a.v : a.k) +
                      (row0 * ts + int64_t(h) * a.hd) * Elt<DT>::ES;
      const auto row_of = [&](int i, int *e) {
        asm volatile("" : "+v"(i));   // (or every place lives on from the load to the store)
        const int row = int(fast_div(uint32_t(i), a.per_div));
        *e = (i - row * a.per) * N;
        return row;
      };
      // the largest magnitude: as whole numbers, so that infinities and NaN are above all
      u32x4 f[HOLD];
      uint32_t most = 0;
      const auto take = [&](const u32x4 &v) {
        float y[N];
        elements<DT, N>(v, y);
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const uint32_t b = __float_as_uint(y[c]) & 0x7FFFFFFFu;
          most = b > most ? b : most;
        }
      };
      const auto load = [&](int i) {
        int e;
        const int row = row_of(i, &e);
        return load_row<DT, N>(x + (row * ts + e) * Elt<DT>::ES);
      };
#pragma unroll
      for (int k = 0; k < HOLD; ++k) {
        f[k] = u32x4{0, 0, 0, 0};
        if (L * k >= items_new) continue;   // (for all lanes)
        if (active && tid + L * k < items_new) f[k] = load(tid + L * k);
      }
      if (uint32_t(id) >= uint32_t(a.n_pages)) break;   // (only here: the rows' loads need no page)
      const PagedView &view = is_v ? a.cv : a.ck;
      char *c = static_cast<char *>(view.p) + id * view.ps + int64_t(slot) * view.ss +
                int64_t(h) * view.hs;
      float *scale = scale_at(is_v ? a.sv : a.sk, id, fast_div(slot, a.block_div), h);
      const float was = active ? *scale : 0.0f;
#pragma unroll
      for (int k = 0; k < HOLD; ++k)
        if (L * k < items_new) take(f[k]);
      for (int i = tid + L * HOLD; active && i < items_new; i += L) take(load(i));
#pragma unroll
      for (int d = (L < 64 ? L : 64) / 2; d; d >>= 1) {
        const uint32_t b = __shfl_xor(most, d);
        most = b > most ? b : most;
      }
      if constexpr (L == 256) {
        __syncthreads();   // (the last item's are read)
        if ((threadIdx.x & 63) == 0) team_most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) most = team_most[w] > most ? team_most[w] : most;
      }
      if (!active) continue;
      // (else the elements live on as float32, in twice the registers)
#pragma unroll
      for (int k = 0; k < HOLD; ++k) asm volatile("" : "+v"(f[k]));
      const float need = scale_for<CT>(most);
      // (a scale of NaN stays one)
      const float now = old == 0 || need != need || need > was ? need : was;
      if (old > 0 && now > was) {
        const int last = old * a.per;
#pragma unroll 1
        for (int i0 = tid; i0 < last; i0 += 2 * L) {
          char *p[2];
          CodesOf<N> y[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            int e;
            const int i = i0 + L * u < last ? i0 + L * u : i0, row = row_of(i, &e);
            p[u] = c + row * view.ss + e;
            y[u] = load_codes<N>(p[u]);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (i0 + L * u >= last) break;
#pragma unroll
            for (uint32_t &w : y[u].w) w = recode4<CT>(w, was, now);
            store_codes<N>(p[u], y[u]);
          }
        }
      }
      if (tid == 0) *scale = now;
      const Rounder rd = rounder(now);
      const auto put = [&](int i, const u32x4 &v) {
        int e;
        const int row = row_of(i, &e);
        float y[N];
        elements<DT, N>(v, y);
        CodesOf<N> z;
#pragma unroll
        for (int k = 0; k < (N + 3) / 4; ++k) {
          float four[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) four[m] = 4 * k + m < N ? y[4 * k + m] : 0.0f;
          z.w[k] = to_codes4<CT>(four, rd);
        }
        store_codes<N>(c + (old + row) * view.ss + e, z);
      };
#pragma unroll
      for (int k = 0; k < HOLD; ++k)
        if (L * k < items_new && tid + L * k < items_new) put(tid + L * k, f[k]);
      for (int i = tid + L * HOLD; i < items_new; i += L) put(i, load(i));
    }
  }
}

// ---- Q8R_* ------------------------------------------------------------------------------------
// A wavefront gives a row of K and V back, a vector a work-item (an element, Q8R_ANY), four of
// them in flight. Bound by memory: 32 ragged caches of up to 4000 tokens, 8 heads of 128, 83.6 us
// (4.9 TB/s, what a copy reaches); four rows a wavefront, one search for all, 86.9. 8192 rows of 8 + 8 heads of
// 128 into float32 18.6 (e4m3) and 20.8 (int8); at any alignment, an element a store, 49, of 100 43.
template <int DT, int CT, bool VEC>
__global__ __launch_bounds__(256) void k_q8_read(Q8RowsArgs a) {
  constexpr int N = VEC ? Elt<DT>::V : 1, U = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Requests held = requests(a);
  const int half = a.nk * a.per;
  for (int32_t row = int32_t(blockIdx.x) * 4 + wave; row < a.T; row += int32_t(gridDim.x) * 4) {
    Request rq;
    const int32_t r = find_request(a, held, &rq, [&](int32_t, int32_t q0) { return q0 <= row; });
    if (r < 0 || row < rq.q0 || row >= rq.q1) continue;
    const int32_t p = rq.kv - (rq.q1 - row);
    int64_t id = -1;
    uint32_t slot = 0;
    if (p >= 0) {
      const uint32_t col = fast_div(uint32_t(p), a.div);
      const int32_t x = a.table[r * a.table_rs + col];
      id = uint32_t(x) < uint32_t(a.n_pages) ? x : -1;
      slot = uint32_t(p) - col * uint32_t(a.page);
    }
    const uint32_t block = fast_div(slot, a.block_div);
    const int64_t at = id < 0 ? 0 : id;
    for (int i0 = lane; i0 < 2 * half; i0 += 64 * U) {
      CodesOf<N> c[U];
      float s[U];
      int64_t to[U];
      bool is_v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + 64 * u < 2 * half ? i0 + 64 * u : i0;
        is_v[u] = i >= half;
        const int j = is_v[u] ? i - half : i, h = int(fast_div(uint32_t(j), a.per_div));
        const int e = (j - h * a.per) * N;
        const PagedView &view = is_v[u] ? a.cv : a.ck;
        c[u] = load_codes<N>(static_cast<const char *>(view.p) + at * view.ps +
                             int64_t(slot) * view.ss + int64_t(h) * view.hs + e);
        s[u] = *scale_at(is_v[u] ? a.sv : a.sk, at, block, uint32_t(h));
        to[u] = row * (is_v[u] ? a.v_ts : a.k_ts) + int64_t(h) * a.hd + e;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + 64 * u >= 2 * half) break;
        float f[(N + 3) / 4 * 4];
#pragma unroll
        for (int k = 0; k < (N + 3) / 4; ++k) codes4<CT>(c[u].w[k], f + 4 * k);
#pragma unroll
        for (float &y : f) y = id < 0 ? 0.0f : y * s[u];
        char *o = static_cast<char *>(is_v[u] ? a.v : a.k) + to[u] * Elt<DT>::ES;
        if constexpr (VEC)
          *reinterpret_cast<u32x4 *>(o) = Elt<DT>::pack(f);
        else
          Elt<DT>::st(o, 0, f[0]);
      }
    }
  }
}

// ---- PA8_ANY ----------------------------------------------------------------------------------
// As PA_ANY: a wavefront per row, query head and split, a lane a key of 64 for the
// scores, and elements l, l + 64, ... of the head for the sums. A key that is not
// seen is never read. Scores are in powers of two from the start: (q.k s) c. Bound by its
// loads, a byte of V a lane, one or four of K (64 requests of up to 1000 keys, 32 and 8 heads of
// 100: 239 us; with a key's V at a time 594, bytes of K as well 612; PA_ANY over bf16 732).
template <int DT, int CT>
__global__ __launch_bounds__(256) void k_pa8_any(PagedQ8Args a8) {
  constexpr int ES = Elt<DT>::ES;
  constexpr int NI = 8;   // 512 / 64
  const PagedArgs &a = a8.a;
  __shared__ float qs[4][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t items = int64_t(a.T) * a.nq * a.splits;
  // whether four codes of K lie at a multiple of 4
  const bool words = ((uint64_t(a.hd) | uint64_t(a.k.p) | uint64_t(a.k.ps) | uint64_t(a.k.ss) |
                       uint64_t(a.k.hs)) & 3) == 0;
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
          if (words)
#pragma unroll 4
            for (; d < a.hd; d += 4) {
              float c[4];
              codes4<CT>(*reinterpret_cast<const uint32_t *>(k + d), c);
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = fmaf(qs[wave][d + i], c[i], x[i]);
            }
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
      // eight keys' loads in flight (of one that is not seen the pool's first slot, as 0)
      for (int j = 0; j < 64; j += 8) {
        if (!((seen >> j) & 0xFF)) continue;
        float wj[8];
        const uint8_t *v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          wj[u] = __shfl(wv, j + u);
          const int64_t at = __shfl(vo, j + u);
          v[u] = vp + (at < 0 ? 0 : at);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if (64 * i >= a.hd) break;
          const int d = lane + 64 * i < a.hd ? lane + 64 * i : 0;
          uint8_t c[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) c[u] = v[u][d];
#pragma unroll
          for (int u = 0; u < 8; ++u)
            acc[i] = fmaf(wj[u], (seen >> (j + u)) & 1 ? code1<CT>(c[u]) : 0.0f, acc[i]);
        }
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
// How many a row has follows from the same numbering; a tile that one workgroup had is there
// already. 32 rows of 90 parts 6.1 us, 2048 rows of one to eight 7.4: latency.
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
    const int32_t parts = int32_t((begin + uint32_t(steps) - 1) / per - begin / per) + 1;
    return parts < a.splits ? parts : a.splits;   // (a row in two requests: anything, but inside)
  };
  join_rows<DT, 4, kQ8Splits / 64>(a, a8.four != 0, parts_of);
}

namespace {
template <class F>
const void *sym(F *f) {
  return reinterpret_cast<const void *>(f);
}

template <int DT, int CT>
const void *rows_kernel(int32_t variant, int32_t team) {
  switch (variant) {
    case Q8W_ANY: return sym(&k_q8_write<DT, CT, false, 64>);
    case Q8W_VEC:
      return team == 2   ? sym(&k_q8_write<DT, CT, true, 256>)
             : team == 1 ? sym(&k_q8_write<DT, CT, true, 64>)
                         : sym(&k_q8_write<DT, CT, true, 16>);
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
// for few rows the logarithm of the K heads of a tile in bits 1 and 2; for the write there
// the lanes of a team, 16, 64 or 256.
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
    return e4m3 ? rows_kernel<kF32, kE4M3>(variant, sub >> 1) : rows_kernel<kF32, kInt8>(variant, sub >> 1);
  return e4m3 ? rows_kernel<kBF16, kE4M3>(variant, sub >> 1) : rows_kernel<kBF16, kInt8>(variant, sub >> 1);
}

}  // namespace tri
