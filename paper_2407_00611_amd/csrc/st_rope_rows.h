// How norms and rotations hold a row (st_rope.hip, st_cache.hip): loads and stores, a lane's place in a row, sums over a row.
#pragma once

#include <type_traits>

#include "st_e4m3.h"
#include "st_rope.h"

namespace st {

// V neighbouring values, of bf16 or fp32
template <int V>
__device__ __forceinline__ Vec<V> load(const uint16_t* p) {
  Vec<V> y;
  if constexpr (V == 8) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) y.x[2 * j] = __uint_as_float(u[j] << 16), y.x[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
  } else if constexpr (V == 4) {
    const u32x2 u = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int j = 0; j < 2; ++j) y.x[2 * j] = __uint_as_float(u[j] << 16), y.x[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
  } else if constexpr (V == 2) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
    y.x[0] = __uint_as_float(u << 16);
    y.x[1] = __uint_as_float(u & 0xffff0000u);
  } else {
    y.x[0] = __uint_as_float((uint32_t)*p << 16);
  }
  return y;
}
template <int V>
__device__ __forceinline__ Vec<V> load(const float* p) {
  Vec<V> y;
  if constexpr (V >= 4) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + 4 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e) y.x[4 * j + e] = u[e];
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) y.x[j] = p[j];
  }
  return y;
}
// Results are said to be read by nobody soon: that leaves the caches to the inputs, 24 heads of 64 x 16384 tokens 45 us, 40.5 so, and an
// attention that reads them next is none the slower.  (Inputs loaded so: 52 us.)
template <int V>
__device__ __forceinline__ void store(uint16_t* p, const Vec<V>& y) {
  if constexpr (V == 8) __builtin_nontemporal_store(u32x4{pack_bf16(y.x[0], y.x[1]), pack_bf16(y.x[2], y.x[3]), pack_bf16(y.x[4], y.x[5]), pack_bf16(y.x[6], y.x[7])}, reinterpret_cast<u32x4*>(p));
  else if constexpr (V == 4) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(y.x[0], y.x[1]), pack_bf16(y.x[2], y.x[3])};
  else if constexpr (V == 2) *reinterpret_cast<uint32_t*>(p) = pack_bf16(y.x[0], y.x[1]);
  else *p = (uint16_t)pack_bf16(y.x[0], y.x[0]);
}
template <int V>
__device__ __forceinline__ void store(float* p, const Vec<V>& y) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) __builtin_nontemporal_store(f32x4{y.x[4 * j], y.x[4 * j + 1], y.x[4 * j + 2], y.x[4 * j + 3]}, reinterpret_cast<f32x4*>(p + 4 * j));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] = y.x[j];
  }
}

// Where a lane's V pairs of a row are.  pair >= D / 2: none.
template <int V, bool NEXT>
struct Place {
  int pair, a, b;            // first pair, first elements of the two vectors
  bool live;
};
template <int V, bool NEXT>
__device__ __forceinline__ Place<V, NEXT> place_of(const RopeArgs& g, int chunk) {
  Place<V, NEXT> p;
  p.pair = chunk * V;
  p.live = p.pair < g.D / 2;
  if (!p.live) p.pair = 0;
  const int rest = g.D - g.rot;
  if (NEXT) p.a = 2 * p.pair, p.b = p.a + V;
  else if (p.pair < g.rot / 2) p.a = p.pair, p.b = p.pair + g.rot / 2;
  else p.a = p.pair + g.rot / 2, p.b = p.a + rest / 2;
  return p;
}
// the V pairs (a, b) of a row that starts at `row`
template <int V, bool NEXT, typename T>
__device__ __forceinline__ void load_pairs(const T* row, const Place<V, NEXT>& p, Vec<V>& a, Vec<V>& b) {
  const Vec<V> x = load<V>(row + p.a), y = load<V>(row + p.b);
  if constexpr (NEXT) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      a.x[e] = 2 * e < V ? x.x[(2 * e) % V] : y.x[(2 * e) % V];
      b.x[e] = 2 * e + 1 < V ? x.x[(2 * e + 1) % V] : y.x[(2 * e + 1) % V];
    }
  } else {
    a = x;
    b = y;
  }
}
template <int V, bool NEXT, typename T>
__device__ __forceinline__ void store_pairs(T* row, const Place<V, NEXT>& p, const Vec<V>& a, const Vec<V>& b) {
  if constexpr (NEXT) {
    Vec<V> x, y;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x.x[e] = e % 2 == 0 ? a.x[e / 2] : b.x[e / 2];
      y.x[e] = (e + V) % 2 == 0 ? a.x[(e + V) / 2] : b.x[(e + V) / 2];
    }
    store<V>(row + p.a, x);
    store<V>(row + p.b, y);
  } else {
    store<V>(row + p.a, a);
    store<V>(row + p.b, b);
  }
}

// sum over the `lanes` (a power of two) neighbouring lanes of a row
__device__ __forceinline__ float row_sum(float x, int lanes) {
  // inside 16 lanes by data parallel primitives: neighbours, pairs, then mirrored halves, whose lanes agree by then
  if (lanes > 1) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xb1, 0xf, 0xf, false));    // quad_perm 1 0 3 2
  if (lanes > 2) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4e, 0xf, 0xf, false));    // quad_perm 2 3 0 1
  if (lanes > 4) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xf, 0xf, false));   // row_half_mirror
  if (lanes > 8) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xf, 0xf, false));   // row_mirror
  if (lanes > 16) x += __shfl_xor(x, 16);
  if (lanes > 32) x += __shfl_xor(x, 32);
  return x;
}

// ---- host side

// largest V with V | rot / 2 and V | (D - rot) / 2, of 8, 4, 2, 1
inline int pairs_per_lane(int D, int rot) {
  int v = 8;
  while (v > 1 && (rot / 2 % v || (D - rot) / 2 % v)) v /= 2;
  return v;
}
inline int lanes_of(int D, int v) {
  const int u = v == 1 ? 2 : 1, chunks = (D / 2 / v + u - 1) / u;
  int lanes = 1;
  while (lanes < chunks) lanes *= 2;
  return lanes;
}

// f(V, U, neighbouring)
template <typename F>
void with_pairs(const RopeArgs& g, F f) {
  using std::integral_constant;
  auto next = [&](auto v, auto u) {
    if (g.next) f(v, u, integral_constant<bool, true>());
    else f(v, u, integral_constant<bool, false>());
  };
  switch (pairs_per_lane(g.D, g.rot)) {
    case 8: return next(integral_constant<int, 8>(), integral_constant<int, 1>());
    case 4: return next(integral_constant<int, 4>(), integral_constant<int, 1>());
    case 2: return next(integral_constant<int, 2>(), integral_constant<int, 1>());
    default: return next(integral_constant<int, 1>(), integral_constant<int, 2>());
  }
}

}  // namespace st
