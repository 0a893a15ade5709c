// Device-side building blocks of the paged KV cache's kernels: division by a
// launch constant, the request that a row belongs to, the slot of a key, and
// what the attention forms share.
#pragma once
#include "device.h"

namespace tri {
namespace dev {

__device__ inline uint32_t fast_div(uint32_t n, FastDiv d) {
  return d.mul ? __umulhi(n, d.mul) >> d.shift : n;
}

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kNegInf = -__builtin_inff();

// 2^(c (x - m)): the weight of a score x = q.k against a reference m, and what
// sums taken against a reference x become against m. The difference first: a
// float32 c m is off by up to half a step, which reaches 2^8 at |c m| = 2^32 and
// would leave the maximum itself a weight of 0 or infinity, where c x - c m is
// rounded but once (and c m alone may not be finite). It costs the 128-row tiles
// one operation a weight: 2048 tokens behind 6144, 274.5 -> 278.7 us.
__device__ inline float weight_of(float x, float m, float c) { return exp2_hw((x - m) * c); }

// acc + f x for a part x of a row's sum, taken against another reference; an
// infinity or NaN of V that the part holds stays what it is where f is 0.
__device__ inline float add_part(float f, float x, float acc) {
  return f == 0.0f && !(fabsf(x) < __builtin_inff()) ? acc + x : fmaf(f, x, acc);
}

// The keys that the rows of one request see. Lengths and starts are device
// data and may hold anything: clamped so that every row lies in [0, T) and
// every key in the table.
struct Request {
  int32_t q0, q1;   // rows
  int32_t kv;       // tokens in the cache
};

__device__ inline int32_t clamp_i32(int32_t v, int32_t lo, int32_t hi) {
  return v < lo ? lo : v > hi ? hi : v;
}

template <class A>
__device__ inline Request clamped(const A &a, int32_t q0, int32_t q1, int32_t kv) {
  return {clamp_i32(q0, 0, a.T), clamp_i32(q1, 0, a.T), clamp_i32(kv, 0, a.cols * a.page)};
}

template <class A>
__device__ inline Request request_of(const A &a, int32_t r) {
  return clamped(a, a.q_start[r], a.q_start[r + 1], a.kv_len[r]);
}

// First key that the row at position p (>= 0) sees.
__device__ inline int32_t first_key(int32_t p, int32_t window) {
  return window > 0 && p >= window ? p - window + 1 : 0;
}

// Elements from the start of K (or V) to a key's slot, or -1 where its page is
// not in the pool. `key` must be below cols * page.
__device__ inline int64_t slot_offset(const int32_t *row, uint32_t key, const PagedArgs &a,
                                      const PagedView &c) {
  const uint32_t col = fast_div(key, a.div);
  const int32_t id = row[col];
  if (uint32_t(id) >= uint32_t(a.n_pages)) return -1;
  return int64_t(id) * c.ps + int64_t(key - col * uint32_t(a.page)) * c.ss;
}

// The keys [lo, hi) of a tile cut into `splits` runs of whole 64s: run s, in
// [lo, hi] (hi < lo, rows before the first key: empty, at lo).
__device__ inline void split_keys(int32_t lo, int32_t hi, int32_t splits, int32_t s, int32_t *b,
                                  int32_t *e) {
  if (hi < lo) hi = lo;
  const int32_t n = hi - lo;
  const int64_t run = (int64_t(n) + int64_t(splits) * 64 - 1) / (int64_t(splits) * 64) * 64;
  const int64_t first = lo + s * run, last = first + run;
  *b = first < hi ? int32_t(first) : hi;
  *e = last < hi ? int32_t(last) : hi;
}

// The last r of [0, R) with first(r), -1 if none, for a first() that does not
// turn true again after it was false (else some r that it holds for, or -1):
// 64 requests probed at once, so two rounds of loads find any of 4096. The
// whole wavefront calls it and gets the same answer.
template <class F>
__device__ inline int32_t last_request(int32_t R, F &&first) {
  const int lane = threadIdx.x & 63;
  const int32_t step = (R + 63) >> 6;
  int32_t base = 0;
  if (step > 1) {
    const int32_t x = lane * step;
    const uint64_t hit = __ballot(x < R && first(x < R ? x : 0));
    if (!hit) return -1;
    base = (63 - __builtin_clzll(hit)) * step;
  }
  const int32_t x = base + lane;
  const int32_t m = step > 1 && R - base > step ? step : R - base;
  const uint64_t hit = __ballot(lane < m && first(lane < m ? x : base));
  return hit ? base + 63 - __builtin_clzll(hit) : -1;
}

}  // namespace dev
}  // namespace tri
