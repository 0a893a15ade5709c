// Device-side building blocks of the paged KV cache in 8 bits: codes, their
// scales, and the rounding of values to codes.
#pragma once
#include "paged.h"

namespace tri {
namespace dev {

constexpr int kInt8 = TRI_INT8, kE4M3 = TRI_E4M3;
constexpr float kLeastScale = 0x1p-100f;

// Four codes as float32 (exact).
template <int CT>
__device__ inline void codes4(uint32_t c, float *f) {
  if constexpr (CT == kInt8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = float(int32_t(c << (24 - 8 * i)) >> 24);
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), true);
    f[0] = lo[0];
    f[1] = lo[1];
    f[2] = hi[0];
    f[3] = hi[1];
  }
}

template <int CT>
__device__ inline float code1(uint8_t c) {
  if constexpr (CT == kInt8)
    return float(int8_t(c));
  else
    return __builtin_amdgcn_cvt_f32_fp8(int(c), 0);
}

// The scale that magnitudes of up to `most` (given in its bits; not a finite number:
// NaN) need. e4m3: 448 is 1.75 2^8, so the power of two at or above most / 448 goes by
// whether most's fraction is above 0.75.
template <int CT>
__device__ inline float scale_for(uint32_t most) {
  if (most >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  float s;
  if constexpr (CT == kInt8) {
    s = __uint_as_float(most) / 127.0f;
  } else {
    const int32_t e = int32_t(most >> 23) + ((most & 0x7FFFFFu) > 0x600000u) - 8;
    s = __uint_as_float(uint32_t(e > 1 ? e : 1) << 23);
  }
  return fmaxf(s, kLeastScale);
}

// What rounds values to the codes of one scale s.
struct Rounder {
  float s, inv;
  bool pow2;
};
__device__ inline Rounder rounder(float s) {
  return {s, 1.0f / s, (__float_as_uint(s) & 0x7FFFFFu) == 0};
}

// Four codes; all 0 with a scale of NaN. Whole numbers are the nearest to x / s, ties to even:
// 1.5 2^23 added, a float32's last place is 1, so the fused product is rounded to a whole
// number n, whose low byte is the sum's, off from the quotient's by one at most, where that is
// within 2^-16 of the middle of two. What n leaves of x, x - n s, is exact (a multiple of the
// smaller of both operands' last places, and no longer than s), so its distance to
// s / 2 says which of the two is nearer, and a tie is one; few are that near.
template <int CT>
__device__ inline uint32_t to_codes4(const float *x, const Rounder &r) {
  if (r.s != r.s) return 0;
  if constexpr (CT == kInt8) {
    constexpr float kMagic = 12582912.0f;
    float t[4], left[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t[i] = fmaf(x[i], r.inv, kMagic);
      left[i] = fmaf(-(t[i] - kMagic), r.s, x[i]);
    }
    const float h = 0.5f * r.s;
    if (fmaxf(fmaxf(fabsf(left[0]), fabsf(left[1])), fmaxf(fabsf(left[2]), fabsf(left[3]))) >= h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float far = fabsf(left[i]);
        if (far > h || (far == h && (__float_as_uint(t[i]) & 1u))) t[i] += left[i] > 0.0f ? 1.0f : -1.0f;
      }
    }
    return __builtin_amdgcn_perm(__float_as_uint(t[1]), __float_as_uint(t[0]), 0x0C0C0400) |
           __builtin_amdgcn_perm(__float_as_uint(t[3]), __float_as_uint(t[2]), 0x04000C0C);
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = r.pow2 ? x[i] * r.inv : x[i] / r.s;
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true));
  }
}

// A float32 from which any rounding to fewer bits, ties included, goes as from q itself: cut off, its last
// place 1 where that leaves something.
__device__ inline float to_odd(double q) {
  const float f = float(q);
  uint32_t b = __float_as_uint(f);
  if (double(f) != q) b = (b - uint32_t(fabs(double(f)) > fabs(q))) | 1u;
  return __uint_as_float(b);
}

// Codes of scale `was` as codes of `now` > was: the nearest to c was / now. A float32 product
// with the quotient is off by 2^-15 at most, so it tells which whole number is nearest, but within
// 2^-12 of the middle of two; e4m3's powers of two have exact products. Else 64 bits: c was is
// exact in them, and a quotient of 31 by 24 bits is a tie or more than 2^-56 of it off (e4m3's `now`
// is a power of two: the quotient is exact).
template <int CT>
__device__ inline uint32_t recode4(uint32_t c, float was, float now) {
  float f[4], y[4];
  codes4<CT>(c, f);
  const float ratio = was / now;
  bool plain = CT == kInt8 || ((__float_as_uint(was) | __float_as_uint(now)) & 0x7FFFFFu) == 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = f[i] * ratio;
    if constexpr (CT == kInt8) {
      const float n = rintf(y[i]);
      plain = plain && fabsf(y[i] - n) < 0.5f - 0x1p-12f;
      y[i] = n;
    }
  }
  if (!plain) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double q = double(f[i]) * double(was) / double(now);
      y[i] = CT == kInt8 ? float(rint(q)) : to_odd(q);
    }
  }
  if constexpr (CT == kInt8) {
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) out |= (uint32_t(int32_t(y[i])) & 0xFFu) << (8 * i);
    return out;
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true));
  }
}

// Where a block's scale lies: page, block of the page, head.
__device__ inline float *scale_at(const ScaleView &s, int64_t id, uint32_t block, uint32_t head) {
  return s.p + id * s.ps + int64_t(block) * s.bs + int64_t(head) * s.hs;
}

}  // namespace dev
}  // namespace tri
