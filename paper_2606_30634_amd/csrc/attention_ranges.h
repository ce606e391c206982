// What the kernels of attention over key ranges share (attention_ranges.hip and attention_ranges_mfma.hip).
#pragma once
#include "common.h"
#include "kernels.h"

namespace {

__device__ __forceinline__ int64_t position(const RangeArgs& a, int b, int i) {
  return (int64_t)(a.q_start ? a.q_start[b] : a.Sk - a.Sq) + i;
}

// The keys that query i of sequence b sees; none is (0, 0)
__device__ __forceinline__ int2 seen_keys(const RangeArgs& a, int b, int i) {
  int lo = 0, hi;
  if (a.key_start) {
    lo = max(a.key_start[(int64_t)b * a.Sq + i], 0);
    hi = min(a.key_end[(int64_t)b * a.Sq + i], a.Sk);
  } else {
    hi = (int)min((int64_t)a.Sk, max((int64_t)0, position(a, b, i) + 1));
  }
  return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
}
__device__ __forceinline__ bool sees(const int2& s, int key) { return (uint32_t)(key - s.x) < (uint32_t)(s.y - s.x); }

// The same from the arrays that the backward lays out
__device__ __forceinline__ int2 seen_keys_kept(const RangeArgs& a, int64_t row) {
  const int lo = a.seen_lo[row];
  return make_int2(lo, lo + a.seen_len[row]);
}

// What a score is taken relative to in a row of this maximum or lse: a row of only -inf has weights of 0
__device__ __forceinline__ float weight_base(float m) { return m == -INFINITY ? 0.f : m; }

// tanh(y) and its derivative 1 - tanh(y)^2.  Up to |y| = 1/2 the odd polynomial y + y^3 P(y^2) with P the
// minimax fit of degree 3 (relative error 2^-26); beyond it 1 - u with u = 2 e / (1 + e), e = exp(-2 |y|),
// whose derivative u (2 - u) keeps its relative accuracy where tanh rounds to 1.
constexpr float TANH_SMALL = 0.5f;
__device__ __forceinline__ float tanh_excess(float z) {  // tanh(y) / y - 1, z = y^2
  float p = __builtin_fmaf(z, 0.0172414685f, -0.0530454814f);
  p = __builtin_fmaf(z, p, 0.1332587898f);
  return z * __builtin_fmaf(z, p, -0.3333314359f);
}
__device__ __forceinline__ float tanh_far(float y, float& slope) {
  const float e = __builtin_amdgcn_exp2f(fabsf(y) * -2.8853900817779268f);
  const float u = 2.0f * e * __builtin_amdgcn_rcpf(1.0f + e);
  slope = u * (2.0f - u);
  return copysignf(1.0f - u, y);
}
__device__ __forceinline__ float tanh_and_slope(float y, float& slope) {
  if (!(fabsf(y) < TANH_SMALL)) return tanh_far(y, slope);
  const float t = __builtin_fmaf(y, tanh_excess(y * y), y);
  slope = __builtin_fmaf(-t, t, 1.0f);
  return t;
}
// cap tanh(x / cap) and its derivative in x.  A score well below the cap is x and a small correction, so that x
// keeps its bits: through tanh and back it would lose two roundings of a score that is an exponent next.
__device__ __forceinline__ float capped(float x, float cap, float inv_cap, float& slope) {
  const float y = x * inv_cap;
  if (!(fabsf(y) < TANH_SMALL)) return cap * tanh_far(y, slope);
  const float r = tanh_excess(y * y), t = __builtin_fmaf(y, r, y);
  slope = __builtin_fmaf(-t, t, 1.0f);
  return __builtin_fmaf(x, r, x);
}

template <typename T>
__device__ __forceinline__ const T* rows_of(const HeadRows& r, int b, int h) {
  return (const T*)r.p + b * r.batch + h * r.head;
}
template <typename T>
__device__ __forceinline__ T* rows_out(const HeadRows& r, int b, int h) {
  return (T*)r.p + b * r.batch + h * r.head;
}

// Partial dq of share `split`, rows of Hq HD
template <int HD>
__device__ __forceinline__ float* dq_part(const RangeArgs& a, int split, int b, int h) {
  return a.part_q + ((int64_t)split * a.B + b) * a.Sq * a.Hq * HD + h * HD;
}

// A wave's minimum and maximum over all its lanes, by data-parallel moves (as wave_total)
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_same(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, ROWS, 0xf, false); }
template <typename F>
__device__ __forceinline__ int wave_fold(int v, F&& f) {
  v = f(v, dpp_or_same<0x111, 0xf>(v));
  v = f(v, dpp_or_same<0x112, 0xf>(v));
  v = f(v, dpp_or_same<0x114, 0xf>(v));
  v = f(v, dpp_or_same<0x118, 0xf>(v));
  v = f(v, dpp_or_same<0x142, 0xa>(v));
  v = f(v, dpp_or_same<0x143, 0xc>(v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_min_i(int v) { return wave_fold(v, [](int x, int y) { return min(x, y); }); }
__device__ __forceinline__ int wave_max_i(int v) { return wave_fold(v, [](int x, int y) { return max(x, y); }); }

// The keys [lo, hi) that some query of a wave sees (none: 0, 0), and those [all_lo, all_hi) that all of them see
// (none: all_lo > all_hi).  valid: the lane's query exists.
struct WaveKeys {
  int lo, hi, all_lo, all_hi;
  __device__ WaveKeys(const int2& s, bool valid) {
    const bool some = valid && s.x < s.y;
    hi = wave_max_i(some ? s.y : 0);
    lo = hi > 0 ? wave_min_i(some ? s.x : INT32_MAX) : 0;
    all_lo = wave_max_i(some ? s.x : valid ? INT32_MAX : 0);
    all_hi = wave_min_i(some ? s.y : valid ? 0 : INT32_MAX);
  }
  __device__ bool whole(int k0, int k1) const { return all_lo <= k0 && k1 <= all_hi; }  // all see [k0, k1)
};

}  // namespace
