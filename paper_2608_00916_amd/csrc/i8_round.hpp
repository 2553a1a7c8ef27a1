// Rows of values as int8 with one scale: a row's largest magnitude a maps to
// 127, q = rint(127 x / a), s = a / 127.
//
// The quotient is n / a with n = 127 x, which is exact for a bf16 x (8 + 7
// bits).  It is formed as t = n (1 / a) and one residual step
// t + (n - a t) (1 / a), whose result is the rounded quotient: an exact half
// (x = a / 2: 63.5) stays one, so q is the same as from a division at 3
// instead of about 10 instructions a value.
#pragma once

#include "common.hpp"

namespace moe {

constexpr uint32_t kInfBits = 0x7f800000u;

// One row's rounding: x -> q for the largest magnitude `top` (as fp32 bits).
// `pre` brings both into a range where 127 x and 1 / top are normal numbers.
struct Rounder {
  float pre, top, inv, scale;
  bool live;
  __device__ __forceinline__ explicit Rounder(uint32_t top_bits) {
    const float t = __uint_as_float(top_bits);
    live = top_bits < kInfBits && top_bits != 0u;
    pre = t < 1e-30f ? 0x1p100f : t > 1e30f ? 0x1p-100f : 1.0f;
    top = t * pre;
    inv = live ? 1.0f / top : 0.0f;
    scale = top_bits >= kInfBits ? __uint_as_float(0x7fc00000u) : t / 127.0f;
  }
  __device__ __forceinline__ int operator()(float x) const {
    const float n = x * pre * 127.0f;
    const float t = n * inv;
    const float r = __builtin_rintf(fmaf(fmaf(-top, t, n), inv, t));
    return live ? static_cast<int>(r) : 0;
  }
};

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = max(v, static_cast<uint32_t>(shfl_xor(static_cast<int>(v), m)));
  return v;
}

__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (a & 255) | ((b & 255) << 8) | ((c & 255) << 16) | (static_cast<uint32_t>(d) << 24);
}

// Largest magnitude of 8 bf16 as fp32 bits (NaN > infinity > finite).
__device__ __forceinline__ uint32_t top8(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fff0000u, (w[i] << 16) & 0x7fff0000u));
  return m;
}

__device__ __forceinline__ uint2 quant8(const uint4& v, const Rounder& r) {
  return make_uint2(pack4(r(lo_bf(v.x)), r(hi_bf(v.x)), r(lo_bf(v.y)), r(hi_bf(v.y))),
                    pack4(r(lo_bf(v.z)), r(hi_bf(v.z)), r(lo_bf(v.w)), r(hi_bf(v.w))));
}

}  // namespace moe
