// Values in e4m3 (four bits of exponent, three of mantissa; up to 448, NaN but no infinity), by the hardware's conversions.
#pragma once

#include "st_mfma.h"

namespace st {

template <int V>
struct Vec {
  float x[V];
};

// two e4m3 values of the low or high half of x
template <bool HIGH>
__device__ __forceinline__ float2 e4m3_pair(uint32_t x) {
  const auto y = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, HIGH);
  return make_float2(y[0], y[1]);
}
// four values, rounded to the nearest (|x| <= 448 or NaN)
__device__ __forceinline__ uint32_t e4m3_of(float a, float b, float c, float d) {
  int y = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, y, true);
}

// Times 2^(scale - 127) a code is beyond fp32, and bf16, from 2^(255 - scale) on: what to add to codes without their sign so that those, and
// NaN, reach the sign's place
__device__ __forceinline__ uint32_t e4m3_beyond(uint32_t scale) { return (0x80u - (uint32_t)min(0x7f, 8 * (262 - (int)scale))) * 0x01010101u; }

// V neighbouring values from their codes, and back
template <int V>
__device__ __forceinline__ Vec<V> load(const uint8_t* p) {
  Vec<V> y;
  uint32_t u[2] = {0, 0};
  if constexpr (V == 8) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    u[0] = w[0]; u[1] = w[1];
  } else if constexpr (V == 4) u[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (V == 2) u[0] = *reinterpret_cast<const uint16_t*>(p);
  else u[0] = *p;
#pragma unroll
  for (int e = 0; e < V; e += 2) {
    const float2 f = e % 4 ? e4m3_pair<true>(u[e / 4]) : e4m3_pair<false>(u[e / 4]);
    y.x[e] = f.x;
    if (e + 1 < V) y.x[e + 1] = f.y;
  }
  return y;
}
template <int V>
__device__ __forceinline__ void store(uint8_t* p, const Vec<V>& y) {
  auto at = [&](int e) { return e < V ? y.x[e] : 0.f; };
  const uint32_t u = e4m3_of(at(0), at(1), at(2), at(3));
  if constexpr (V == 8) *reinterpret_cast<u32x2*>(p) = u32x2{u, e4m3_of(at(4), at(5), at(6), at(7))};
  else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(p) = u;
  else if constexpr (V == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)u;
  else *p = (uint8_t)u;
}

}  // namespace st
