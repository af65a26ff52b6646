// Attention of packed rows against a cache of pages.
//
// A tile is 32 rows, packed over the heads of a KV head (row R is token R / G, head R % G of the group), so that a key is read once for all of
// them.  The four wavefronts of a workgroup share the tile's walk over the keys, 32 keys a step, and fold in LDS; walks are split over
// workgroups as st_cache_plan.h says, and their states joined by a second launch.
//
//   S^T = K Q^T and O^T += V^T P^T: a lane has one row (C layout column l % 32), its reference, sum and span in registers.
// Keys and values go from memory to the operand registers: the order of a contraction is free as long as both sides agree, so lane (r, g)
// takes 16-byte pieces of key r's row as they lie, and for the second product the values of DP / 32 neighbouring columns of the eight keys
// that its exponentials belong to.
#include <type_traits>

#include "st_cache_plan.h"
#include "st_score.h"

namespace st {
namespace {

constexpr int kKeys = kCacheKeys, kRows = kCacheRows;
constexpr float kUnset = -1e30f;                     // reference of a row that has met no key: whatever comes exceeds it
constexpr float kSumMost = 4096.f;                   // a lane's sum over sixteen keys beyond which a row's reference moves

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
// two values of a half of x, times a power of two: exact
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_of_e4m3(uint32_t x, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, HIGH));
}

// the parts of x (values of S side by side) that are an infinity or NaN become zero; whether there were any
template <typename S>
__device__ __forceinline__ bool drop_not_finite(uint32_t& x) {
  uint32_t mask;
  if constexpr (sizeof(S) == 1) {
    mask = (((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
    mask *= 0xffu;
  } else if constexpr (sizeof(S) == 2) {
    mask = (((x & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15;
    mask *= 0xffffu;
  } else {
    mask = (x & 0x7f800000u) == 0x7f800000u ? 0xffffffffu : 0u;
  }
  x &= ~mask;
  return mask != 0;
}

// One value of the pages
__device__ __forceinline__ float stored(const float* p, uint8_t) { return *p; }
__device__ __forceinline__ float stored(const uint16_t* p, uint8_t) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float stored(const uint8_t* p, uint8_t scale) { return e4m3_pair<false>(*p).x * scale_value(scale); }

// T: of the rows (bf16: on the bf16 matrix unit, D = DP; fp32: on the fp32 one, D <= DP); S: what the pages hold; MOD: scores may be capped, biased
template <typename T, typename S, int DP, bool MOD>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void cache_stream_kernel(const CacheAttnArgs a) {
  constexpr bool BF = std::is_same<T, uint16_t>::value, E4M3 = std::is_same<S, uint8_t>::value;
  constexpr int DB = DP / 32, EPC = 16 / (int)sizeof(S), NJ = DP / (2 * EPC);
  constexpr int VB = DB * (int)sizeof(S), VW = VB < 4 ? 1 : VB / 4;
  constexpr int PW = DB < 4 ? DB : 4, PASSES = DB / PW, FS = 32 * PW + 4;
  constexpr int QS = DP + 4;
  constexpr int kFold = 4 * kRows * FS * 4, kQ = BF ? 0 : kRows * QS * 4;
  __shared__ __attribute__((aligned(16))) char smem[kFold > kQ ? kFold : kQ];
  __shared__ float stat_m[4][kRows], stat_l[4][kRows];
  __shared__ PlanRoom room;
  __shared__ int any_bad;
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 5, r = lane & 31;
  const int G = a.Hq / c.Hkv, D = BF ? DP : c.D;
  const CacheItem t = find_item<kRows, kKeys>(a, &room);
  if (t.b < 0) return;
  const SeqSpan s = seq_span(a, t.b);
  const CacheWalk w = cache_walk<kRows, kKeys>(a, s, t, G);
  tell_rows<kRows>(a, s, t, G);
  const int M = s.r.n * G, live = min(M - t.tile * kRows, kRows);
  const int row = min(t.tile * kRows + r, M - 1), i = row / G, h = t.hk * G + row - i * G;
  const RowSpan see = row_span(a, s, i);
  const char* qrow = (const char*)a.q.ptr + ((int64_t)(s.r.first + i) * a.q.ss + (int64_t)h * a.q.sh) * (int)sizeof(T);

  bf16x8 qf[BF ? DP / 16 : 1];
  float* qs = (float*)smem;
  if constexpr (BF) {
#pragma unroll
    for (int x = 0; x < DP / 16; ++x) {                // (the order of the pieces of a key)
      const int d = E4M3 ? 32 * (x / 2) + 16 * g + 8 * (x % 2) : 16 * x + 8 * g;
      qf[x] = *reinterpret_cast<const bf16x8*>(qrow + d * 2);
    }
  } else {
    for (int x = tid; x < kRows * (QS / 4); x += 256) {   // (zeros behind D: they are multiplied by zeros)
      const int qr = x / (QS / 4), d = 4 * (x - qr * (QS / 4)), R = min(t.tile * kRows + qr, M - 1), qi = R / G;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      if (d < D) y = *reinterpret_cast<const f32x4*>((const float*)a.q.ptr + (int64_t)(s.r.first + qi) * a.q.ss + (int64_t)(t.hk * G + R - qi * G) * a.q.sh + d);
      *reinterpret_cast<f32x4*>(qs + qr * QS + d) = y;
    }
    __syncthreads();
  }

  // scores in log2 units; with a cap c2 is the exponent of its tanh
  const float slope = MOD && a.slopes ? a.slopes[h] : 0.f, slope2 = slope * kScoreLog2e;
  const bool cap = MOD && a.cap > 0.f;
  const float c2 = cap ? 2.f * kScoreLog2e * (a.scale / a.cap) : a.scale * kScoreLog2e, k1 = a.cap * kScoreLog2e;
  int near = 0;                                        // the nearest token that the row sees
  float besides = 0.f;                                 // what the bias of that one adds to lse
  if (MOD && see.lo < see.hi) {
    const int64_t p = s.pos + i;
    near = (int)min(max(p, (int64_t)see.lo), (int64_t)see.hi - 1);
    besides = -slope * (float)(p > near ? p - near : near - p);
  }

  // the pages of a block, one for its first 16 keys and one for the others
  const int32_t* table = c.table + (int64_t)t.b * c.width;
  auto table_at = [&](int n) { return table[min((n * kKeys + 16 * (lane & 1)) >> c.shift, c.width - 1)]; };
  const char* kbase = (const char*)c.k.ptr + (int64_t)t.hk * c.k.sh * (int)sizeof(S);
  const char* vbase = (const char*)c.v.ptr + (int64_t)t.hk * c.v.sh * (int)sizeof(S);
  const uint32_t k_off = (uint32_t)((r & 15) * c.k.ss * (int)sizeof(S)) + 16 * g;
  const uint32_t v_off = (uint32_t)(4 * g * c.v.ss * (int)sizeof(S)) + r * VB;
  const bool v_lane = BF || DB * r < D;

  struct Pages {
    int p[2];
    bool ok[2];
  };
  auto pages_of = [&](int entry) {
    Pages y;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int p = __builtin_amdgcn_readlane(entry, m);
      y.ok[m] = p >= 0 && p < c.n_pages;
      y.p[m] = y.ok[m] ? p : 0;
    }
    return y;
  };
  auto at = [&](const char* base, const View& v, const Pages& p, int n, int m) {
    return base + ((int64_t)p.p[m] * v.sb + (int64_t)((n * kKeys + 16 * m) & ((1 << c.shift) - 1)) * v.ss) * (int)sizeof(S);
  };
  u32x4 kr[NJ];
  uint32_t vr[16][VW];
  int k_sc = 0, v_sc = 0;                              // bytes of the scales: of the lane's key; of the halves in lanes 0 and 16
  auto load_k = [&](const Pages& p, int n) {
    const char* x0 = at(kbase, c.k, p, n, 0);
    const char* x1 = at(kbase, c.k, p, n, 1);
    const char* x = (r < 16 ? x0 : x1) + k_off;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (BF || (2 * j + g) * EPC < D) kr[j] = *reinterpret_cast<const u32x4*>(x + 32 * j);
      else kr[j] = u32x4{0, 0, 0, 0};
    }
    if constexpr (E4M3) k_sc = c.k_scale[(int64_t)(r < 16 ? p.p[0] : p.p[1]) * c.Hkv + t.hk];
  };
  auto load_v = [&](const Pages& p, int n) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const char* x = at(vbase, c.v, p, n, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const char* y = x + (8 * (e / 4) + e % 4) * c.v.ss * (int)sizeof(S) + v_off;
        uint32_t* to = vr[8 * m + e];
        if (!v_lane) {
#pragma unroll
          for (int d = 0; d < VW; ++d) to[d] = 0;
        } else if constexpr (VB == 2) to[0] = *reinterpret_cast<const uint16_t*>(y);
        else if constexpr (VB == 4) to[0] = *reinterpret_cast<const uint32_t*>(y);
        else if constexpr (VB == 8) {
          const u32x2 z = *reinterpret_cast<const u32x2*>(y);
          to[0] = z[0]; to[1] = z[1];
        } else {
#pragma unroll
          for (int d = 0; d < VW; d += 4) {
            const u32x4 z = *reinterpret_cast<const u32x4*>(y + 4 * d);
            to[d] = z[0]; to[d + 1] = z[1]; to[d + 2] = z[2]; to[d + 3] = z[3];
          }
        }
      }
    }
    if constexpr (E4M3) v_sc = c.v_scale[(int64_t)(r < 16 ? p.p[0] : p.p[1]) * c.Hkv + t.hk];
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  float m_run = kUnset, l_run = 0.f;
  bool bad = false;

  // wavefront w takes the blocks n1 - 1 - w, n1 - 5 - w, ...: the nearest keys, whose bias is least, first
  int n = w.n1 - 1 - wave;
  const bool some = n >= w.n0;
  Pages now{{0, 0}, {false, false}};
  int entry = 0;
  if (some) {
    now = pages_of(table_at(n));
    entry = table_at(max(n - 4, w.n0));
    load_k(now, n);
    load_v(now, n);
  }
  for (; n >= w.n0; n -= 4) {
    const int key0 = n * kKeys;
    f32x16 sc;
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = 0.f;
    const float ks = E4M3 ? __uint_as_float((uint32_t)k_sc << 23) : 1.f;
    if constexpr (BF) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if constexpr (E4M3) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const u32x4 f = {bf16_of_e4m3<false>(kr[j][2 * y], ks), bf16_of_e4m3<true>(kr[j][2 * y], ks), bf16_of_e4m3<false>(kr[j][2 * y + 1], ks),
                             bf16_of_e4m3<true>(kr[j][2 * y + 1], ks)};
            sc = mfma32(__builtin_bit_cast(bf16x8, f), qf[2 * j + y], sc);
          }
        } else {
          sc = mfma32(__builtin_bit_cast(bf16x8, kr[j]), qf[j], sc);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const float* q = qs + r * QS + (2 * j + g) * EPC;
        if (2 * EPC * j >= D) break;
#pragma unroll
        for (int x = 0; x < EPC; x += 4) {
          const f32x4 qv = *reinterpret_cast<const f32x4*>(q + x);
          float f[4];
          if constexpr (E4M3) {
            const float2 lo = e4m3_pair<false>(kr[j][x / 4]), hi = e4m3_pair<true>(kr[j][x / 4]);
            f[0] = lo.x * ks; f[1] = lo.y * ks; f[2] = hi.x * ks; f[3] = hi.y * ks;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(kr[j][e]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = mfma_f32(f[e], qv[e], sc);
        }
      }
    }
    // the keys' registers are free for the next block's
    const Pages next = pages_of(entry);
    const bool more = n - 4 >= w.n0;
    const bool whole = key0 >= w.all_lo && key0 + kKeys <= w.all_hi && now.ok[0] && now.ok[1];
    if (more) {
      load_k(next, n - 4);
      entry = table_at(max(n - 8, w.n0));
    }

    if constexpr (MOD) {
      const float x0 = (float)(near - key0 - 4 * g);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        if (cap) sc[v] = BF ? fmaf(-2.f * k1, cap_r(sc[v], c2), k1) : k1 * tanhf(sc[v] * (a.scale / a.cap));
        else sc[v] *= c2;
        sc[v] = fmaf(-slope2, fabsf(x0 - (float)(8 * (v / 4) + v % 4)), sc[v]);
      }
    }
    if (!whole) {
      const int l0 = see.lo - key0 - 4 * g, h0 = see.hi - key0 - 4 * g;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = 8 * (v / 4) + v % 4;
        sc[v] = key >= l0 && key < h0 && now.ok[v / 8] ? sc[v] : -INFINITY;
      }
    }
    // The reference of the exponents is lazy: it moves where a block's sum says that some exponent was large
    float p[16], sum;
    auto exponentials = [&]() {
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        p[v] = __builtin_amdgcn_exp2f(MOD ? sc[v] - m_run : fmaf(sc[v], c2, -m_run));
        sum += p[v];
      }
    };
    exponentials();
    if (__builtin_expect(__any(sum > kSumMost), 0)) {
      float top = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, sc[v]);
      const float m_new = fmaxf(m_run, xhalf_max(MOD ? top : top * c2));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
      exponentials();
    }
    l_run += sum;

    if (!whole) {                                      // nothing of what no row sees; of the rest, what is not finite is added at the end
      bool found = false;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int key = key0 + 8 * (x / 4) + 4 * g + x % 4;
        const bool in = key >= w.lo && key < w.hi && now.ok[x / 8];
#pragma unroll
        for (int d = 0; d < VW; ++d) {
          vr[x][d] = in ? vr[x][d] : 0;
          found = drop_not_finite<S>(vr[x][d]) || found;
        }
      }
      bad = bad || __any(found);
    }
    if constexpr (BF) {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        u32x4 hi, lo;                                  // probabilities as the sum of two bf16: 2^-16 of them is left out
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = p[8 * m + 2 * e], y = p[8 * m + 2 * e + 1];
          hi[e] = pack_bf16(x, y);
          lo[e] = pack_bf16(x - __uint_as_float(hi[e] << 16), y - __uint_as_float(hi[e] & 0xffff0000u));
        }
        u32x4 f[DB];
        const float vs = E4M3 ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_sc, 16 * m) << 23) : 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t* x = vr[8 * m + 2 * e];
          const uint32_t* y = vr[8 * m + 2 * e + 1];
          if constexpr (E4M3) {
#pragma unroll
            for (int d = 0; d < DB; d += 2) {
              const uint32_t z = __builtin_amdgcn_perm(y[0], x[0], d ? 0x07030602 : 0x05010400);
              f[d][e] = bf16_of_e4m3<false>(z, vs);
              f[d + 1][e] = bf16_of_e4m3<true>(z, vs);
            }
          } else {
#pragma unroll
            for (int d = 0; d < DB; ++d) f[d][e] = __builtin_amdgcn_perm(y[d / 2], x[d / 2], d % 2 ? 0x07060302 : 0x05040100);
          }
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          acc[d] = mfma32(__builtin_bit_cast(bf16x8, f[d]), __builtin_bit_cast(bf16x8, hi), acc[d]);
          acc[d] = mfma32(__builtin_bit_cast(bf16x8, f[d]), __builtin_bit_cast(bf16x8, lo), acc[d]);
        }
      }
    } else {
      const float vs[2] = {E4M3 ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_sc, 0) << 23) : 1.f,
                           E4M3 ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v_sc, 16) << 23) : 1.f};
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          float f;
          if constexpr (E4M3) {
            const float2 z = (d & 2) ? e4m3_pair<true>(vr[v][d / 4]) : e4m3_pair<false>(vr[v][d / 4]);
            f = ((d & 1) ? z.y : z.x) * vs[v / 8];
          } else {
            f = __uint_as_float(vr[v][d]);
          }
          acc[d] = mfma_f32(f, p[v], acc[d]);
        }
    }
    if (more) load_v(next, n - 4);
    now = next;
  }

  // ---- the four wavefronts' sums, against the highest of their references
  const float l = xhalf_sum(l_run);
  if (tid == 0) any_bad = 0;
  if (g == 0) {
    stat_m[wave][r] = m_run;
    stat_l[wave][r] = l;
  }
  __syncthreads();
  if (bad && lane == 0) any_bad = 1;
  const float m_all = fmaxf(fmaxf(stat_m[0][r], stat_m[1][r]), fmaxf(stat_m[2][r], stat_m[3][r]));
  const float weight = __builtin_amdgcn_exp2f(m_run - m_all);
  float* fold = (float*)smem;
  const bool part = t.shares > 1;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    if (pass > 0) __syncthreads();
    if (r < live)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int rho = 8 * (v / 4) + 4 * g + v % 4;
        float* to = fold + (wave * kRows + r) * FS + PW * rho;
#pragma unroll
        for (int d = 0; d < PW; ++d) to[d] = acc[PW * pass + d][v] * weight;
      }
    __syncthreads();
    for (int x = tid; x < live * 32; x += 256) {
      const int y = x >> 5, rho = x & 31, d0 = DB * rho + PW * pass;
      const int R = t.tile * kRows + y, yi = R / G, yh = t.hk * G + R - yi * G;
      if (!BF && d0 >= D) continue;
      const float top = fmaxf(fmaxf(stat_m[0][y], stat_m[1][y]), fmaxf(stat_m[2][y], stat_m[3][y]));
      float sum = 0.f, o[PW];
#pragma unroll
      for (int d = 0; d < PW; ++d) o[d] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sum += stat_l[k][y] * __builtin_amdgcn_exp2f(stat_m[k][y] - top);
#pragma unroll
        for (int d = 0; d < PW; ++d) o[d] += fold[(k * kRows + y) * FS + PW * rho + d];
      }
      if (__builtin_expect(any_bad, 0)) {              // what the blocks at the masks' edges left out, of the keys that this row sees
        const RowSpan ys = row_span(a, s, yi);
        for (int key = max(ys.lo, w.n0 * kKeys); key < min(ys.hi, w.n1 * kKeys); ++key) {
          const int page = page_of(c, t.b, key >> c.shift);
          const int b0 = key / kKeys * kKeys;
          if (page < 0) continue;
          const bool inner = b0 >= w.all_lo && b0 + kKeys <= w.all_hi && page_of(c, t.b, b0 >> c.shift) >= 0 && page_of(c, t.b, min((b0 + 16) >> c.shift, c.width - 1)) >= 0;
          if (inner) continue;
#pragma unroll
          for (int d = 0; d < PW; ++d) {
            const float z = stored((const S*)(vbase + ((int64_t)page * c.v.sb + (int64_t)(key & ((1 << c.shift) - 1)) * c.v.ss) * (int)sizeof(S)) + d0 + d,
                                   E4M3 ? c.v_scale[(int64_t)page * c.Hkv + t.hk] : (uint8_t)127);
            if (!(fabsf(z) <= 3.402823466e38f)) o[d] += z;
          }
        }
      }
      if (part) {
        float* to = a.part_o + ((int64_t)t.state * kRows + y) * D + d0;
#pragma unroll
        for (int d = 0; d < PW; ++d) to[d] = o[d];
        continue;
      }
      const float inv = sum != 0.f ? 1.f / sum : 0.f;
      const int64_t to = ((int64_t)(s.r.first + yi) * a.Hq + yh) * D + d0;
#pragma unroll
      for (int d = 0; d < PW; ++d) o[d] *= inv;
      if (a.o) {
#pragma unroll
        for (int d = 0; d < PW; ++d) a.o[to + d] = o[d];
      }
      if (a.o_lowp) {
        if constexpr (BF) {
#pragma unroll
          for (int d = 0; d < PW; d += 2) *reinterpret_cast<uint32_t*>((uint16_t*)a.o_lowp + to + d) = pack_bf16(o[d], o[d + 1]);
        } else {
#pragma unroll
          for (int d = 0; d < PW; ++d) ((float*)a.o_lowp)[to + d] = o[d];
        }
      }
    }
  }
  if (wave == 0 && g == 0 && r < live) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += stat_l[k][r] * __builtin_amdgcn_exp2f(stat_m[k][r] - m_all);
    if (part) a.part_row[(int64_t)t.state * kRows + r] = make_float4(m_all, sum, besides, 0.f);
    else a.lse[(int64_t)h * a.T + s.r.first + i] = sum != 0.f ? m_all * kScoreLn2 + logf(sum) + besides : -INFINITY;
  }
}

// Joins the states of rows whose walk was split: a row at a time, eight states side by side at 128 columns.  Rows that are whole cost a look.
__global__ __launch_bounds__(256) void cache_combine_kernel(const CacheAttnArgs a, int each, int bf16) {
  __shared__ f32x4 fold[256];
  __shared__ float weights[256], top_of[4], sum_of[4];
  const int tid = threadIdx.x, D = a.c.D, G = a.Hq / a.c.Hkv, vecs = D / 4, lanes = 256 / vecs, x = tid % vecs, y = tid / vecs;
  const int first = max(min(a.starts[0], a.T), 0), end = max(min(a.starts[a.c.B], a.T), 0);
  const int64_t row0 = (int64_t)blockIdx.x * each, rows = (int64_t)a.T * a.Hq;
  for (int64_t row = row0; row < min(row0 + each, rows); ++row) {
    const int t = (int)(row / a.Hq), h = (int)(row - (int64_t)t * a.Hq);
    if (t < first || t >= end) continue;
    const int4 at = a.info[t];                         // {first state, shares, row tiles, row of the sequence}
    if (at.y <= 1) {
      row += a.Hq - 1 - h;                             // nor are the token's other heads split
      continue;
    }
    const int hk = h / G, R = at.w * G + h - hk * G, tile = R / kRows;
    const int64_t s0 = at.x + (int64_t)(at.z - 1 - tile) * a.c.Hkv + hk, step = (int64_t)at.z * a.c.Hkv;
    if (at.x < 0 || at.w < 0 || at.z <= tile || s0 + (at.y - 1) * step >= a.plan.states) continue;
    float top = kUnset, sum = 0.f, besides = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < at.y; k0 += 256) {           // their weights, against the highest reference so far
      float4 st = make_float4(kUnset, 0.f, 0.f, 0.f);
      if (k0 + tid < at.y) st = a.part_row[(s0 + (k0 + tid) * step) * kRows + R % kRows];
      float m = st.x;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
      __syncthreads();
      if ((tid & 63) == 0) top_of[tid >> 6] = m;
      __syncthreads();
      m = fmaxf(fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3])), top);
      const float e = __builtin_amdgcn_exp2f(st.x - m), old = __builtin_amdgcn_exp2f(top - m);
      weights[tid] = e;
      float l = st.y * e;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
      if ((tid & 63) == 0) sum_of[tid >> 6] = l;
      if (tid == 0) besides = st.z;
      __syncthreads();
      top = m;
      sum = sum * old + ((sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]));
      o *= old;
      const int n = min(at.y - k0, 256);
      if (y < lanes)
        for (int k = y; k < n; k += 4 * lanes) {       // four loads in flight
          f32x4 z[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            z[u] = *reinterpret_cast<const f32x4*>(a.part_o + ((s0 + (int64_t)(k0 + min(k + u * lanes, n - 1)) * step) * kRows + R % kRows) * D + 4 * x);
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (k + u * lanes < n) o += z[u] * weights[k + u * lanes];
        }
    }
    fold[tid] = o;
    __syncthreads();
    if (y == 0) {
      for (int k = 1; k < lanes; ++k) o += fold[k * vecs + x];
      o *= sum != 0.f ? 1.f / sum : 0.f;
      const int64_t to = row * D + 4 * x;
      if (a.o) *reinterpret_cast<f32x4*>(a.o + to) = o;
      if (a.o_lowp && bf16) *reinterpret_cast<u32x2*>((uint16_t*)a.o_lowp + to) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
      else if (a.o_lowp) *reinterpret_cast<f32x4*>((float*)a.o_lowp + to) = o;
      if (x == 0) a.lse[(int64_t)h * a.T + t] = sum != 0.f ? top * kScoreLn2 + logf(sum) + besides : -INFINITY;
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnArgs& a, bool bf16, hipStream_t stream) {
  if (a.plan.grid <= 0 || a.plan.grid > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("cache_attn", stream);
  const dim3 grid((unsigned)a.plan.grid), block(256);
  const bool mod = a.cap > 0.f || a.slopes;
  auto go = [&](auto plain, auto modified) { hipLaunchKernelGGL(mod ? modified : plain, grid, block, 0, stream, a); };
#define ST_STREAM(T, S, DP) go(cache_stream_kernel<T, S, DP, false>, cache_stream_kernel<T, S, DP, true>)
  const int D = a.c.D;
  if (bf16 && a.c.dtype == ST_E4M3) D == 128 ? ST_STREAM(uint16_t, uint8_t, 128) : ST_STREAM(uint16_t, uint8_t, 64);
  else if (bf16) D == 128 ? ST_STREAM(uint16_t, uint16_t, 128) : ST_STREAM(uint16_t, uint16_t, 64);
  else if (a.c.dtype == ST_E4M3) D > 128 ? ST_STREAM(float, uint8_t, 256) : D > 64 ? ST_STREAM(float, uint8_t, 128) : ST_STREAM(float, uint8_t, 64);
  else D > 128 ? ST_STREAM(float, float, 256) : D > 64 ? ST_STREAM(float, float, 128) : ST_STREAM(float, float, 64);
#undef ST_STREAM
  return hipGetLastError();
}

hipError_t launch_cache_combine(const CacheAttnArgs& a, bool bf16, hipStream_t stream) {
  const int64_t rows = (int64_t)a.T * a.Hq, blocks = rows < 4096 ? rows : 4096;
  if (rows <= 0) return hipSuccess;
  if (rows > 0x7fffffff * (int64_t)64) return hipErrorInvalidValue;
  ProfScope prof("cache_combine", stream);
  const int each = (int)((rows + blocks - 1) / blocks);
  hipLaunchKernelGGL(cache_combine_kernel, dim3((unsigned)((rows + each - 1) / each)), dim3(256), 0, stream, a, each, bf16 ? 1 : 0);
  return hipGetLastError();
}

}  // namespace st
