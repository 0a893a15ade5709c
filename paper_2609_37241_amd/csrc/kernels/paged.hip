// The paged KV cache: the step's bookkeeping (KV_SLOTS), new K and V rows into
// their slots (KVW_*), attention at any alignment and head size (PA_ANY) and
// the sum of split results (PA_JOIN).
#include "../internal.h"
#include "paged.h"

namespace tri {
using namespace dev;

// ---- KV_SLOTS ------------------------------------------------------------------------------
// Every workgroup sums the lengths and the new pages of all requests for
// itself (at most 4096 of each: two loads and a scan, less than a second
// launch would cost), keeps both running sums in LDS and then places its share
// of the rows and of the new pages, each found by bisection. What bounds it is
// latency, three dependent rounds of memory and the scan: 8 requests of a token
// 2.9 us, 300 with 20000 rows 5.0.
namespace {
constexpr int kReqMax = TRI_MAX_REQUESTS;
constexpr int32_t kI32Max = 0x7FFFFFFF;

__device__ inline int32_t sat_i32(int64_t v) { return v > kI32Max ? kI32Max : int32_t(v); }

// The last r of [0, R) with sum[r] <= x; sum[0] = 0, x >= 0.
__device__ inline int32_t last_at_most(const int32_t *sum, int32_t R, int32_t x) {
  int32_t lo = 0, hi = R - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (sum[mid] <= x)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

struct SlotReq {
  int32_t held, have, want;   // tokens; pages held and new
  int64_t all;                // tokens afterwards
  int32_t more;
};

// Pages of n >= 0 tokens.
__device__ inline int32_t pages_of(int32_t n, const KvSlotsArgs &a) {
  const uint32_t full = fast_div(uint32_t(n), a.div);
  return int32_t(full + (uint32_t(n) != full * uint32_t(a.page)));
}

__device__ inline SlotReq slot_req(const KvSlotsArgs &a, int32_t r) {
  SlotReq q;
  q.held = clamp_i32(a.kv_len[r], 0, a.cols * a.page);
  const int32_t n = a.new_len[r];
  q.more = n > 0 ? n : 0;
  q.all = int64_t(q.held) + q.more;
  const int32_t need = pages_of(sat_i32(q.all), a);
  q.have = pages_of(q.held, a);
  q.want = (need > a.cols ? a.cols : need) - q.have;
  return q;
}
}  // namespace

__global__ __launch_bounds__(256) void k_kv_slots(KvSlotsArgs a) {
  __shared__ int32_t row0[kReqMax + 1], page0[kReqMax + 1], held[kReqMax];
  __shared__ int64_t wave_rows[4], wave_pages[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t R = a.R;
  const int32_t count = clamp_i32(a.free_count[0], 0, a.n_free);
  // each work-item takes `per` requests in a row
  const int per = (R + 255) / 256;
  const int r0 = tid * per, r1 = r0 + per < R ? r0 + per : R;
  int64_t rows = 0, pages = 0;
  SlotReq own{};
  for (int r = r0; r < r1; ++r) {
    const SlotReq q = slot_req(a, r);
    own = q;
    rows += q.more;
    pages += q.want;
  }
  int64_t sr = rows, sp = pages;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t ur = __shfl_up(sr, d), up = __shfl_up(sp, d);
    if (lane >= d) {
      sr += ur;
      sp += up;
    }
  }
  if (lane == 63) {
    wave_rows[wave] = sr;
    wave_pages[wave] = sp;
  }
  __syncthreads();
  sr -= rows;
  sp -= pages;
  int64_t all_pages = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) {
      sr += wave_rows[w];
      sp += wave_pages[w];
    }
    all_pages += wave_pages[w];
  }
  for (int r = r0; r < r1; ++r) {
    row0[r] = sat_i32(sr);
    page0[r] = sat_i32(sp);
    const SlotReq q = per == 1 ? own : slot_req(a, r);
    held[r] = q.held;
    sr += q.more;
    sp += q.want;
    if (r == R - 1) {
      row0[R] = sat_i32(sr);
      page0[R] = sat_i32(sp);
    }
  }
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * 256 + tid, step = int64_t(gridDim.x) * 256;
  for (int64_t t = first; t < a.T; t += step) {
    int64_t slot = -1;
    int32_t pos = 0;
    if (t < row0[R]) {
      const int32_t r = last_at_most(row0, R, int32_t(t));
      const int32_t have = pages_of(held[r], a);
      pos = sat_i32(int64_t(held[r]) + (t - row0[r]));
      const uint32_t col = fast_div(uint32_t(pos), a.div);
      if (col < uint32_t(a.cols)) {
        // a page held before is the table's, a new one the stack's: the entry
        // that this launch writes is not read
        int32_t id = -1;
        if (int32_t(col) < have) {
          id = a.table[r * a.table_rs + col];
        } else {
          const int64_t at = int64_t(count) - 1 - page0[r] - (int32_t(col) - have);
          if (at >= 0) id = a.free_pages[at];
        }
        if (id >= 0) slot = int64_t(id) * a.page + (uint32_t(pos) - col * uint32_t(a.page));
      }
    }
    a.slots[t] = slot;
    a.pos[t] = pos;
  }
  for (int64_t j = first; j < page0[R]; j += step) {
    const int32_t r = last_at_most(page0, R, int32_t(j));
    const int64_t at = int64_t(count) - 1 - j;
    a.table[r * a.table_rs + pages_of(held[r], a) + (j - page0[r])] = at >= 0 ? a.free_pages[at] : -1;
  }
  if (blockIdx.x == 0) {
    for (int r = tid; r < R; r += 256) {
      a.q_start[r] = row0[r];
      a.kv_len_out[r] = sat_i32(slot_req(a, r).all);
    }
    if (tid == 0) {
      a.q_start[R] = row0[R];
      a.free_out[0] = all_pages < count ? int32_t(count - all_pages) : 0;
      a.free_out[1] = all_pages > count ? sat_i32(all_pages - count) : 0;
    }
  }
}

// ---- KVW_* ------------------------------------------------------------------------------------
// A work-item moves one 16-byte vector (VEC) or one element of a row of K or
// V; a row's items are the K row's, then the V row's, so a workgroup writes
// whole heads. The load does not wait for the slot. HBM-bound from about a
// thousand rows on, latency below: 8192 rows of 8 + 8 heads of 128 in bf16 (67
// MB) 13.0 us, 5.2 TB/s; 8 rows 2.4 us. An element a work-item (KVW_ANY) is bound
// by the number of its loads and stores: 8192 rows of 8 + 8 heads of 36 in bf16 (19
// MB) 15 us, of 33 in float32 (35 MB) 16; of 40 by vectors 5.4.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void k_kv_write(KvWriteArgs a) {
  constexpr int N = VEC ? Elt<DT>::V : 1;
  const int64_t items = a.T * int64_t(a.row_items);
  const uint32_t half = a.row_items / 2;
  for (int64_t i0 = int64_t(blockIdx.x) * 256; i0 < items; i0 += int64_t(gridDim.x) * 256) {
    // rows of this workgroup: the first by a 64-bit division on the scalar
    // unit, the others from 32-bit remainders
    const int64_t t0 = i0 / a.row_items;
    const uint32_t off = uint32_t(i0 - t0 * a.row_items) + threadIdx.x;
    const uint32_t dt = fast_div(off, a.row_div);
    const int64_t t = t0 + dt;
    if (t >= a.T) continue;
    uint32_t c = off - dt * a.row_items;
    const bool is_v = c >= half;
    if (is_v) c -= half;
    const uint32_t e = c * N;
    const uint32_t h = e / uint32_t(a.hd), d = e - h * uint32_t(a.hd);
    const char *src = static_cast<const char *>(is_v ? a.v : a.k) +
                      (t * (is_v ? a.v_ts : a.k_ts) + e) * Elt<DT>::ES;
    const int64_t slot = a.slots[t];
    const PagedView &dst = is_v ? a.cv : a.ck;
    if (uint64_t(slot) >= uint64_t(a.n_slots)) continue;
    int64_t pg;
    if (slot >> 31)
      pg = slot / a.page;
    else
      pg = fast_div(uint32_t(slot), a.div);
    char *to = static_cast<char *>(dst.p) +
               (pg * dst.ps + (slot - pg * a.page) * dst.ss + int64_t(h) * dst.hs + d) *
                   Elt<DT>::ES;
    if constexpr (VEC)
      *reinterpret_cast<u32x4 *>(to) = *reinterpret_cast<const u32x4 *>(src);
    else if constexpr (DT == kF32)
      *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(src);
    else
      *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(src);
  }
}

// ---- PA_ANY ------------------------------------------------------------------------------------
// A wavefront per row, query head and split: 64 keys at a time, a lane forms
// one key's score from the query in LDS, the running maximum and sum of the
// softmax are the wavefront's, and for the sums of V lane l holds the elements
// l, l + 64, ... of the head. No alignment, any head size up to 512; a key that
// is not seen is never read. It serves what the matrix forms do not: rows at any
// alignment, heads of no whole number of vectors, and all heads of more than 256,
// also aligned ones. An element a load bounds it: 8 requests of 2000 keys, 32 + 8
// heads, bf16 of 36 125 us (aligned heads of 40 in PA_ROWS: 16) and of 512 920, float32
// of 33 130 and of 320 697.
template <int DT>
__global__ __launch_bounds__(256) void k_pa_any(PagedArgs a) {
  constexpr int ES = Elt<DT>::ES;
  constexpr int NI = 8;   // 512 / 64
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
    for (int d = lane; d < a.hd; d += 64) qs[wave][d] = Elt<DT>::ld(qp, d);
    const int32_t kh = int32_t(fast_div(uint32_t(h), a.g_div));
    const int32_t *table = a.table + r * a.table_rs;
    const char *kp = static_cast<const char *>(a.k.p) + int64_t(kh) * a.k.hs * ES;
    const char *vp = static_cast<const char *>(a.v.p) + int64_t(kh) * a.v.hs * ES;
    float m = kNegInf, l = 0.0f, acc[NI] = {};
    for (int32_t k0 = b; k0 < e; k0 += 64) {
      const int32_t key = k0 + lane;
      int64_t ko = -1, vo = -1;
      float sc = kNegInf;
      if (key < e) {
        ko = slot_offset(table, uint32_t(key), a, a.k);
        vo = slot_offset(table, uint32_t(key), a, a.v);
      }
      if (ko >= 0) {
        float x[4] = {};   // four sums: shorter chains, smaller errors
        int d = 0;
        for (; d + 4 <= a.hd; d += 4)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[i] = fmaf(qs[wave][d + i], Elt<DT>::ld(kp + ko * ES, d + i), x[i]);
        for (; d < a.hd; ++d) x[0] = fmaf(qs[wave][d], Elt<DT>::ld(kp + ko * ES, d), x[0]);
        const float dot = (x[0] + x[1]) + (x[2] + x[3]);
        sc = a.flip ? -dot : dot;
      }
      const uint64_t seen = __ballot(ko >= 0);
      float top = sc;
#pragma unroll
      for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      const float mn = fmaxf(m, top);
      const float ms = mn == kNegInf ? 0.0f : mn;
      const float alpha = weight_of(m, ms, a.scale);
      const float w = ko >= 0 ? weight_of(sc, ms, a.scale) : 0.0f;
      float sum = w;
#pragma unroll
      for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
      l = l * alpha + sum;
      m = mn;
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i] *= alpha;
      for (int j = 0; j < 64; ++j) {
        if (!((seen >> j) & 1)) continue;
        const float wj = __shfl(w, j);
        const char *v = vp + __shfl(vo, j) * ES;
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (lane + 64 * i < a.hd) acc[i] = fmaf(wj, Elt<DT>::ld(v, lane + 64 * i), acc[i]);
      }
    }
    // an infinity or NaN of V is in its element as it is, whatever its weight:
    // sums that are not finite, at weights that are, are formed again from those
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i) z = fmaf(acc[i], 0.0f, z);
    if (__ballot(z != z && fabsf(l) < __builtin_inff())) {
      uint32_t had = 0;   // bit i: acc[i] holds only those
#pragma unroll 1
      for (int32_t key = b; key < e; ++key) {
        const int64_t at = slot_offset(table, uint32_t(key), a, a.v);
        if (at < 0) continue;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int d = lane + 64 * i;
          const float y = d < a.hd ? Elt<DT>::ld(vp + at * ES, d) : 0.0f;
          const bool odd = !(fabsf(y) < __builtin_inff());
          const float sum = had & (1u << i) ? acc[i] + y : y;
          acc[i] = odd ? sum : acc[i];
          had |= odd ? 1u << i : 0u;
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

// ---- PA_JOIN -----------------------------------------------------------------------------------
// out = sum_s w_s part_s / sum_s w_s l_s, w_s = 2^(c (m_s - m)), over the splits of a
// row, m the largest m_s, always in the same order: the same bits every time.
// A split without a weight (l_s = 0) has no say in m. A
// wavefront per row, or four where there are many splits: what bounds it is
// the latency of the sums' loads, so as many lanes as a row leaves free take
// other splits, eight of them in flight. 32 rows of 64 splits, 4.7 us; 2048 of
// two, 4.8.
template <int DT, int VEC>
__device__ void join_rows(const PagedArgs &a) {
  __shared__ float sums[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t t0 = clamp_i32(a.q_start[0], 0, a.T), t1 = clamp_i32(a.q_start[a.R], 0, a.T);
  const bool four = a.splits > kJoinWave;
  // lanes across the elements (a power of two), groups across the splits
  int nl = 1;
  while (nl < 64 && nl * VEC < a.hd) nl *= 2;
  const int per_wave = 64 / nl, groups = four ? 4 * per_wave : per_wave;
  const int group = (four ? wave * per_wave : 0) + lane / nl;
  const int64_t rows = int64_t(a.T) * a.nq, step = int64_t(gridDim.x) * (four ? 1 : 4);
  for (int64_t row = four ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wave; row < rows;
       row += step) {
    const int32_t t = int32_t(row / a.nq), h = int32_t(row - int64_t(t) * a.nq);
    if (t < t0 || t >= t1) continue;
    const int64_t at = row * a.splits;
    // the sums, the first eight of a lane before what weighs them is known
    const auto read = [&](int s, int d, float *x) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[c] = 0.0f;
      if (s >= a.splits || d >= a.hd) return;
      const float *p = a.part + (at + s) * a.hd + d;
      if constexpr (VEC == 4)
        Elt<kF32>::unpack(*reinterpret_cast<const u32x4 *>(p), x);
      else
        x[0] = *p;
    };
    const int e = (lane % nl) * VEC;
    float x[8][VEC];
#pragma unroll
    for (int i = 0; i < 8; ++i) read(i * groups + group, e, x[i]);
    // at most 64 splits: one a lane
    const float m = lane < a.splits ? a.ml[2 * (at + lane)] : kNegInf;
    const float l = lane < a.splits ? a.ml[2 * (at + lane) + 1] : 0.0f;
    float top = l != 0.0f ? m : kNegInf;
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float w = l != 0.0f ? weight_of(m, top == kNegInf ? 0.0f : top, a.scale) : 0.0f;
    float sum = l != 0.0f ? w * l : 0.0f;
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const auto put = [&](int d, float *acc) {
      if (d >= a.hd || lane >= nl || (four && wave != 0)) return;
      char *o = static_cast<char *>(a.out) + (int64_t(t) * a.o_ts + int64_t(h) * a.hd) * Elt<DT>::ES;
#pragma unroll
      for (int c = 0; c < VEC; ++c) acc[c] = sum == 0.0f ? 0.0f : acc[c] / sum;
      if constexpr (VEC == 4 && DT == kF32)
        st_any<kF32, false>(o + d * 4, Elt<kF32>::pack(acc));
      else
#pragma unroll
        for (int c = 0; c < VEC; ++c) Elt<DT>::st(o, d + c, acc[c]);
    };
    bool odd = false;
    for (int d0 = 0; d0 < a.hd; d0 += nl * VEC) {   // (every lane stays: they exchange)
      const int d = d0 + e;
      float acc[VEC] = {};
      for (int s0 = 0; s0 < a.splits; s0 += 8 * groups) {
        if (d0 + s0 > 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) read(s0 + i * groups + group, d, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int s = s0 + i * groups + group;
          const float ws = __shfl(w, s & 63);
          if (s < a.splits) {
#pragma unroll
            for (int c = 0; c < VEC; ++c) acc[c] = fmaf(ws, x[i][c], acc[c]);
          }
        }
      }
      for (int y = nl; y < 64; y *= 2)
#pragma unroll
        for (int c = 0; c < VEC; ++c) acc[c] += __shfl_xor(acc[c], y);
      if (four) {
        __syncthreads();   // the sums of the elements before are read
#pragma unroll
        for (int c = 0; c < VEC; ++c) sums[wave][lane * VEC + c] = acc[c];
        __syncthreads();
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          acc[c] = (sums[0][lane * VEC + c] + sums[1][lane * VEC + c]) +
                   (sums[2][lane * VEC + c] + sums[3][lane * VEC + c]);
      }
#pragma unroll
      for (int c = 0; c < VEC; ++c) odd |= !(fabsf(acc[c]) < __builtin_inff());
      put(d, acc);
    }
    if (__ballot(odd)) {   // infinities or NaN of V, maybe where a weight is 0: once more
      for (int d0 = 0; d0 < a.hd; d0 += nl * VEC) {
        const int d = d0 + e;
        float acc[VEC] = {};
#pragma unroll 1
        for (int s = 0; s < a.splits; ++s) {
          const float ws = __shfl(w, s);
#pragma unroll
          for (int c = 0; c < VEC; ++c)
            if (d < a.hd) acc[c] = add_part(ws, a.part[(at + s) * a.hd + d + c], acc[c]);
        }
        put(d, acc);
      }
    }
  }
}

template <int DT>
__global__ __launch_bounds__(256) void k_pa_join(PagedArgs a) {
  if (a.hd % 4 == 0)
    join_rows<DT, 4>(a);
  else
    join_rows<DT, 1>(a);
}

namespace {
template <class F>
const void *sym(F *f) {
  return reinterpret_cast<const void *>(f);
}
}  // namespace

const void *attn_kernel_bf16(int32_t variant, int32_t hdp);
const void *attn_kernel_f32(int32_t variant, int32_t hdp);

const void *paged_kernel(int32_t variant, uint32_t dtype, int32_t sub) {
  const bool f32 = dtype == TRI_F32;
  switch (variant) {
    case PA_ROWS:
    case PA_TILE:
    case PA_PAIR: return f32 ? attn_kernel_f32(variant, sub) : attn_kernel_bf16(variant, sub);
    case KV_SLOTS: return sym(&k_kv_slots);
    case KVW_ANY: return f32 ? sym(&k_kv_write<kF32, false>) : sym(&k_kv_write<kBF16, false>);
    case KVW_VEC: return f32 ? sym(&k_kv_write<kF32, true>) : sym(&k_kv_write<kBF16, true>);
    case PA_ANY: return f32 ? sym(&k_pa_any<kF32>) : sym(&k_pa_any<kBF16>);
    case PA_JOIN: return f32 ? sym(&k_pa_join<kF32>) : sym(&k_pa_join<kBF16>);
    default: return nullptr;
  }
}

}  // namespace tri
