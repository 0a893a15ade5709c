// The sums of split attention joined: what PA_JOIN and PA8_JOIN share.
#pragma once
#include "paged.h"

namespace tri {
namespace dev {

// ---- joining splits -----------------------------------------------------------------------------------
// out = sum_s w_s part_s / sum_s w_s l_s, w_s = 2^(c (m_s - m)), over the splits of a
// row, m the largest m_s, always in the same order: the same bits every time.
// A split without a weight (l_s = 0) has no say in m. A
// wavefront per row, or four where there are many splits: what bounds it is
// the latency of the sums' loads, so as many lanes as a row leaves free take
// other splits, eight of them in flight. 32 rows of 64 splits, 4.7 us; 2048 of
// two, 4.8.
template <int DT, int VEC, int NM, class F>
__device__ void join_rows(const PagedArgs &a, bool four, F &&parts_of) {
  __shared__ float sums[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t t0 = clamp_i32(a.q_start[0], 0, a.T), t1 = clamp_i32(a.q_start[a.R], 0, a.T);
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
    const int32_t parts = parts_of(t, h);
    if (parts < 2) continue;   // the row is there already
    const int64_t at = row * a.splits;
    // the sums, the first eight of a lane before what weighs them is known
    const auto read = [&](int s, int d, float *x) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[c] = 0.0f;
      if (s >= parts || d >= a.hd) return;
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
    // at most 64 NM splits: NM a lane
    float m[NM], l[NM], w[NM], top = kNegInf, sum = 0.0f;
#pragma unroll
    for (int k = 0; k < NM; ++k) {
      const int i = lane + 64 * k;
      m[k] = i < parts ? a.ml[2 * (at + i)] : kNegInf;
      l[k] = i < parts ? a.ml[2 * (at + i) + 1] : 0.0f;
      top = fmaxf(top, l[k] != 0.0f ? m[k] : kNegInf);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll
    for (int k = 0; k < NM; ++k) {
      w[k] = l[k] != 0.0f ? weight_of(m[k], top == kNegInf ? 0.0f : top, a.scale) : 0.0f;
      sum += l[k] != 0.0f ? w[k] * l[k] : 0.0f;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const auto weight = [&](int s) {
      float x = __shfl(w[0], s & 63);
#pragma unroll
      for (int k = 1; k < NM; ++k) {
        const float y = __shfl(w[k], s & 63);
        x = s >= 64 * k ? y : x;
      }
      return x;
    };
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
      for (int s0 = 0; s0 < parts; s0 += 8 * groups) {
        if (d0 + s0 > 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) read(s0 + i * groups + group, d, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int s = s0 + i * groups + group;
          const float ws = weight(s);
          if (s < parts) {
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
        for (int s = 0; s < parts; ++s) {
          const float ws = weight(s);
#pragma unroll
          for (int c = 0; c < VEC; ++c)
            if (d < a.hd) acc[c] = add_part(ws, a.part[(at + s) * a.hd + d + c], acc[c]);
        }
        put(d, acc);
      }
    }
  }
}

}  // namespace dev
}  // namespace tri
