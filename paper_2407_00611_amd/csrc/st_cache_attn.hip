// Attention of packed rows against a cache of pages.
//
// A tile is 16 or 32 rows, packed over the heads of a KV head (row R is token R / G, head R % G of the group), so that a key is read once for
// all of them.  The four wavefronts of a workgroup share the tile's walk over the keys, 32 keys a step, and fold in LDS; walks are split over
// workgroups as st_cache_plan.h says, and their states joined by a second launch.
//
//   S^T = K Q^T and O^T += V^T P^T: a lane has one row (C layout column), its reference, sum and span in registers.
// Keys and values go from memory to the operand registers: the order of a contraction is free as long as both sides agree, so a lane takes
// 16-byte pieces of its key's row as they lie, and for the second product the values of D / tile neighbouring columns of the eight (sixteen)
// keys that its exponentials belong to.
//
// Bound by memory where sequences are long: 64 sequences of 400 to 8192 tokens (32/8 heads of 128, pages of 16 in 8 bits, 561 MB) take
// 119 us, 4.7 TB/s, and 5 for the join; one of 131072 (269 MB) 50 us, 5.3 TB/s, and 7.5 for the join of its 256 shares.  The matrix unit
// is busy for a tenth of that, so a tile of 16 rows of which four are filled costs nothing.  Short walks are chains of latencies: one
// token against 700 takes 8 us (lengths and tables, keys, products, fold) and 3.7 for the join, in two launches.
//
// A step's keys and values are loaded a step ahead, into registers: a ring in LDS would read and write every byte once more, and what it
// saves, addresses, is a few instructions for 32 keys.  Probabilities meet the values as two bf16 parts (high and rest): the second product
// has time to spare, and of O 2^-16 is lost, 2^-8 with one part.
#include <type_traits>

#include "st_cache_plan.h"
#include "st_score.h"

namespace st {
namespace {

constexpr int kKeys = kCacheKeys;
constexpr int kManyWaves = 16, kManyRows = 512;      // wavefronts of a row whose states are many; up to so many rows
constexpr int kScan = 4;                             // tokens looked at together for values that are not finite: a part of a page
constexpr float kSumMost = 4096.f;                   // a lane's sum over its keys of a block beyond which a row's reference moves

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The matrix instructions of a tile of 32 or 16 rows: lane l holds row (column) l % ROWS of both operands, C rows as Tile::row says
template <int ROWS>
struct Tile;
template <>
struct Tile<32> {
  typedef f32x16 Acc;
  static __device__ __forceinline__ int row(int v, int g) { return 8 * (v / 4) + 4 * g + v % 4; }   // g = l / 32; also the key of score v
  static __device__ __forceinline__ Acc mul(bf16x8 a, bf16x8 b, Acc c) { return mfma32(a, b, c); }
  static __device__ __forceinline__ Acc mul(float a, float b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ float sum(float x) { return xhalf_sum(x); }
  static __device__ __forceinline__ float max(float x) { return xhalf_max(x); }
};
template <>
struct Tile<16> {
  typedef f32x4 Acc;
  static __device__ __forceinline__ int row(int v, int g) { return 16 * (v / 4) + 4 * g + v % 4; }  // g = l / 16; scores 4 .. 7 are a second tile's
  static __device__ __forceinline__ Acc mul(bf16x8 a, bf16x8 b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Acc mul(float a, float b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ float sum(float x) {
    x += __shfl_xor(x, 16);
    return xhalf_sum(x);
  }
  static __device__ __forceinline__ float max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return xhalf_max(x);
  }
};
// two values of a half of x, times a power of two: exact
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_of_e4m3(uint32_t x, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, HIGH));
}

// The parts of x (values of S side by side) that are an infinity or NaN become zero; which there were.  One more at the lowest place of such
// a value's exponent reaches its sign (e4m3, with a scale that makes infinities: e4m3_beyond).  (The empty statement keeps the compiler from putting the last step off
// until all words' masks are there, for which there are no registers; of whole words it keeps a bit each by itself.)
template <typename S>
__device__ __forceinline__ uint32_t drop_not_finite(uint32_t& x, uint32_t beyond) {
  uint32_t mask;
  if constexpr (sizeof(S) == 1) mask = ((((x & 0x7f7f7f7fu) + beyond) & 0x80808080u) >> 7) * 0xffu;
  else if constexpr (sizeof(S) == 2) mask = ((((x & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
  else mask = (x & 0x7f800000u) == 0x7f800000u ? 0xffffffffu : 0u;
  x &= ~mask;
  if constexpr (sizeof(S) < 4) asm volatile("" : "+v"(x));
  return mask;
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// One value of the pages
__device__ __forceinline__ float stored(const float* p, uint8_t) { return *p; }
__device__ __forceinline__ float stored(const uint16_t* p, uint8_t) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float stored(const uint8_t* p, uint8_t scale) { return e4m3_pair<false>(*p).x * scale_value(scale); }

// wavefronts on a SIMD that the registers leave room for
template <typename T, typename S, int ROWS, int DP>
constexpr int stream_waves() {
  return DP > 128 ? (sizeof(S) == 1 ? 2 : 1) : ROWS == 16 ? (DP <= 64 ? 4 : sizeof(S) == 1 ? 3 : 2) : 2;
}

// T: of the rows (bf16: on the bf16 matrix unit, D = DP; fp32: on the fp32 one, D <= DP); S: what the pages hold; MOD: scores may be capped, biased
template <typename T, typename S, int ROWS, int DP, bool MOD>
__global__ __launch_bounds__(256, (stream_waves<T, S, ROWS, DP>())) void cache_stream_kernel(const CacheAttnArgs a) {
  constexpr bool BF = std::is_same<T, uint16_t>::value, E4M3 = std::is_same<S, uint8_t>::value;
  typedef Tile<ROWS> M;
  typedef typename M::Acc Acc;
  constexpr int GROUPS = 64 / ROWS;                    // lanes of a row
  constexpr int NS = kKeys / GROUPS, NA = NS < 16 ? 4 : 16, TILES = NS / NA;   // scores of a lane, as TILES tiles of keys of NA registers
  constexpr int DB = DP / ROWS;                        // columns of O of a lane's matrix row
  constexpr int EPC = 16 / (int)sizeof(S), NJ = DP / (GROUPS * EPC);           // values of a piece, pieces of a key's row a lane
  constexpr int VB = DB * (int)sizeof(S), VW = VB < 4 ? 1 : VB / 4;            // bytes and words of a lane's columns
  constexpr int PW = DB < 4 ? DB : 4, PASSES = DB / PW, FS = ROWS * PW + 4;    // folding: columns at a time
  constexpr bool LATE = (int)sizeof(S) * DP > 512;     // no room for keys and values at once: values are loaded as they are needed
  constexpr int QS = DP + 4;
  constexpr int kFold = 4 * ROWS * FS * 4, kQ = BF ? 0 : ROWS * QS * 4;
  static_assert(NJ >= 1 && VB >= 2 && DB >= 2 && (ROWS == 16 || DP <= kTallCacheHead), "a lane takes part in every product");
  __shared__ __attribute__((aligned(16))) char smem[kFold > kQ ? kFold : kQ];
  __shared__ float stat_m[4][ROWS], stat_l[4][ROWS];
  __shared__ int any_bad;
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane / ROWS, r = lane % ROWS;
  const int G = a.Hq / c.Hkv, D = BF ? DP : c.D;
  SeqSpan s;
  const CacheItem t = find_item<ROWS, kKeys>(a, s);
  if (t.b < 0) return;
  const CacheWalk w = cache_walk<ROWS, kKeys>(a, s, t, G);
  tell_rows<ROWS>(a, s, t, G);
  const int all_rows = s.r.n * G, live = min(all_rows - t.tile * ROWS, ROWS);
  const int row = min(t.tile * ROWS + r, all_rows - 1), i = row / G, h = t.hk * G + row - i * G;
  const RowSpan see = row_span(a, s, i);
  const char* qrow = (const char*)a.q.ptr + ((int64_t)(s.r.first + i) * a.q.ss + (int64_t)h * a.q.sh) * (int)sizeof(T);

  // the pages of a block, one for its first 16 keys and one for the others
  const int32_t* table = c.table + (int64_t)t.b * c.width;
  auto table_at = [&](int n) { return table[min((n * kKeys + 16 * (lane & 1)) >> c.shift, c.width - 1)]; };
  // wavefront w takes the blocks n1 - 1 - w, n1 - 5 - w, ...: the nearest keys, whose bias is least, first
  int n = w.n1 - 1 - wave;
  const bool some = n >= w.n0;
  int entry = 0, entry0 = 0;
  if (some) {
    entry0 = table_at(n);
    entry = table_at(max(n - 4, w.n0));
  }

  bf16x8 qf[BF ? DP / (8 * GROUPS) : 1];
  float* qs = (float*)smem;
  if constexpr (BF) {
#pragma unroll
    for (int x = 0; x < DP / (8 * GROUPS); ++x) {      // (the order of the pieces of a key)
      const int d = E4M3 ? 16 * GROUPS * (x / 2) + 16 * g + 8 * (x % 2) : 8 * GROUPS * x + 8 * g;
      qf[x] = *reinterpret_cast<const bf16x8*>(qrow + d * 2);
    }
  } else {
    for (int x = tid; x < ROWS * (QS / 4); x += 256) {   // (zeros behind D: they are multiplied by zeros)
      const int qr = x / (QS / 4), d = 4 * (x - qr * (QS / 4)), R = min(t.tile * ROWS + qr, all_rows - 1), qi = R / G;
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

  const char* kbase = (const char*)c.k.ptr + (int64_t)t.hk * c.k.sh * (int)sizeof(S);
  const char* vbase = (const char*)c.v.ptr + (int64_t)t.hk * c.v.sh * (int)sizeof(S);
  const uint32_t k_off = (uint32_t)((r & 15) * c.k.ss * (int)sizeof(S)) + 16 * g;
  // columns behind a head's end are those of a matrix row that is not stored: others are read in their place, by eights
  const uint32_t v_off = (uint32_t)(4 * g * c.v.ss * (int)sizeof(S)) + (BF || DB * r < D ? r * VB : 0);
  const uint32_t v_up = DB > 8 && DB * r + 8 >= D ? 0 : 8 * sizeof(S);

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
  u32x4 kr[TILES][NJ];
  uint32_t vr[NS][VW];
  int k_sc = 0, v_sc = 0;                              // bytes of the scales of the halves, in lanes 0 and 32
  auto load_k = [&](const Pages& p, int n) {
    const char* half[2] = {at(kbase, c.k, p, n, 0), at(kbase, c.k, p, n, 1)};
#pragma unroll
    for (int y = 0; y < TILES; ++y) {
      const char* x = (ROWS == 32 ? (r < 16 ? half[0] : half[1]) : half[y]) + k_off;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (BF || (GROUPS * j + g) * EPC < D) kr[y][j] = *reinterpret_cast<const u32x4*>(x + 16 * GROUPS * j);
        else kr[y][j] = u32x4{0, 0, 0, 0};
      }
    }
    if constexpr (E4M3) k_sc = c.k_scale[(int64_t)(lane < 32 ? p.p[0] : p.p[1]) * c.Hkv + t.hk];
  };
  auto load_v = [&](const Pages& p, int n) {
    const char* half[2] = {at(vbase, c.v, p, n, 0), at(vbase, c.v, p, n, 1)};
#pragma unroll
    for (int v = 0; v < NS; ++v) {
      const int k0 = M::row(v, 0);
      const char* y = half[k0 / 16] + k0 % 16 * c.v.ss * (int)sizeof(S) + v_off;
      uint32_t* to = vr[v];
      if constexpr (VB == 2) to[0] = *reinterpret_cast<const uint16_t*>(y);
      else if constexpr (VB == 4) to[0] = *reinterpret_cast<const uint32_t*>(y);
      else if constexpr (VB == 8) {
        const u32x2 z = *reinterpret_cast<const u32x2*>(y);
        to[0] = z[0]; to[1] = z[1];
      } else {
#pragma unroll
        for (int d = 0; d < VW; d += 4) {
          constexpr int kEight = 8 * (int)sizeof(S) / 4;   // words of eight values
          const u32x4 z = *reinterpret_cast<const u32x4*>(DB > 8 && d >= kEight ? y + v_up + 4 * (d - kEight) : y + 4 * d);
          to[d] = z[0]; to[d + 1] = z[1]; to[d + 2] = z[2]; to[d + 3] = z[3];
        }
      }
    }
    if constexpr (E4M3) v_sc = c.v_scale[(int64_t)(lane < 32 ? p.p[0] : p.p[1]) * c.Hkv + t.hk];
  };
  auto scale_of = [&](int bytes, int m) { return E4M3 ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane(bytes, 32 * m) << 23) : 1.f; };

  Acc acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int v = 0; v < NA; ++v) acc[d][v] = 0.f;
  float m_run = kUnset, l_run = 0.f;
  bool bad = false;

  Pages now{{0, 0}, {false, false}};
  if (some) {
    now = pages_of(entry0);
    load_k(now, n);
    if (!LATE) load_v(now, n);
  }
  for (; n >= w.n0; n -= 4) {
    const int key0 = n * kKeys;
    float sc[NS];
#pragma unroll
    for (int y = 0; y < TILES; ++y) {
      Acc z;
#pragma unroll
      for (int v = 0; v < NA; ++v) z[v] = 0.f;
      const float ks = ROWS == 32 ? (r < 16 ? scale_of(k_sc, 0) : scale_of(k_sc, 1)) : scale_of(k_sc, y);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const u32x4 k = kr[y][j];
        if constexpr (BF && E4M3) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const u32x4 f = {bf16_of_e4m3<false>(k[2 * x], ks), bf16_of_e4m3<true>(k[2 * x], ks), bf16_of_e4m3<false>(k[2 * x + 1], ks), bf16_of_e4m3<true>(k[2 * x + 1], ks)};
            z = M::mul(__builtin_bit_cast(bf16x8, f), qf[2 * j + x], z);
          }
        } else if constexpr (BF) {
          z = M::mul(__builtin_bit_cast(bf16x8, k), qf[j], z);
        } else if (GROUPS * EPC * j < D) {
          const float* q = qs + r * QS + (GROUPS * j + g) * EPC;
#pragma unroll
          for (int x = 0; x < EPC; x += 4) {
            const f32x4 qv = *reinterpret_cast<const f32x4*>(q + x);
            float f[4];
            if constexpr (E4M3) {
              const float2 lo = e4m3_pair<false>(k[x / 4]), hi = e4m3_pair<true>(k[x / 4]);
              f[0] = lo.x * ks; f[1] = lo.y * ks; f[2] = hi.x * ks; f[3] = hi.y * ks;
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(k[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) z = M::mul(f[e], qv[e], z);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < NA; ++v) sc[NA * y + v] = z[v];
    }
    // the keys' registers are free for the next block's
    const Pages next = pages_of(entry);
    const bool more = n - 4 >= w.n0;
    const bool whole = key0 >= w.all_lo && key0 + kKeys <= w.all_hi && now.ok[0] && now.ok[1];
    if (LATE) load_v(now, n);
    if (more) {
      if (!LATE) load_k(next, n - 4);
      entry = table_at(max(n - 8, w.n0));
    }

    if constexpr (MOD) {
      const float x0 = (float)(near - key0 - M::row(0, g));
#pragma unroll
      for (int v = 0; v < NS; ++v) {
        if (cap) sc[v] = BF ? fmaf(-2.f * k1, cap_r(sc[v], c2), k1) : k1 * tanhf(sc[v] * (a.scale / a.cap));
        else sc[v] *= c2;
        sc[v] = fmaf(-slope2, fabsf(x0 - (float)M::row(v, 0)), sc[v]);
      }
    }
    if (!whole) {
      const int l0 = see.lo - key0 - M::row(0, g), h0 = see.hi - key0 - M::row(0, g);
#pragma unroll
      for (int v = 0; v < NS; ++v) {
        const int key = M::row(v, 0);
        sc[v] = key >= l0 && key < h0 && now.ok[key / 16] ? sc[v] : -INFINITY;
      }
    }
    // The reference of the exponents is lazy: it moves where a block's sum says that some exponent was large
    float p[NS], sum;
    auto exponentials = [&]() {
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < NS; ++v) {
        p[v] = __builtin_amdgcn_exp2f(MOD ? sc[v] - m_run : fmaf(sc[v], c2, -m_run));
        sum += p[v];
      }
    };
    exponentials();
    if (__builtin_expect(__any(sum > kSumMost), 0)) {
      float top = -INFINITY;
#pragma unroll
      for (int v = 0; v < NS; ++v) top = fmaxf(top, sc[v]);
      const float m_new = fmaxf(m_run, M::max(MOD ? top : top * c2));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < NA; ++v) acc[d][v] *= alpha;
      exponentials();
    }
    l_run += sum;

    if (!whole) {                                      // nothing of what no row sees; of the rest, what is not finite is added at the end
      uint32_t found = 0, beyond[2] = {0, 0};
      if constexpr (E4M3) {                            // the scale of a half without a token that is seen may be anything: what is zero times it is to stay so
        const bool low = now.ok[0] && key0 < w.hi && key0 + 16 > w.lo, high = now.ok[1] && key0 + 16 < w.hi && key0 + 32 > w.lo;
        v_sc = (lane < 32 ? low : high) ? v_sc : 127;
        beyond[0] = e4m3_beyond(__builtin_amdgcn_readlane(v_sc, 0));
        beyond[1] = e4m3_beyond(__builtin_amdgcn_readlane(v_sc, 32));
      }
#pragma unroll
      for (int v = 0; v < NS; ++v) {
        const int key = key0 + M::row(v, g);
        const bool in = key >= w.lo && key < w.hi && now.ok[M::row(v, 0) / 16];
#pragma unroll
        for (int d = 0; d < VW; ++d) {
          vr[v][d] = in ? vr[v][d] : 0;
          found |= drop_not_finite<S>(vr[v][d], beyond[M::row(v, 0) / 16]);
        }
      }
      bad = bad || __any(found != 0);
    }
    if constexpr (BF) {
#pragma unroll
      for (int m = 0; m < NS / 8; ++m) {               // eight keys a lane: the contraction of one matrix instruction
        u32x4 hi, lo;                                  // probabilities as the sum of two bf16: 2^-16 of them is left out
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = p[8 * m + 2 * e], y = p[8 * m + 2 * e + 1];
          hi[e] = pack_bf16(x, y);
          lo[e] = pack_bf16(x - __uint_as_float(hi[e] << 16), y - __uint_as_float(hi[e] & 0xffff0000u));
        }
#pragma unroll
        for (int d = 0; d < DB; d += 2) {
          u32x4 f[2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {                // values of one column by pairs of keys
            const int v = 8 * m + 2 * e;
            const float vs = scale_of(v_sc, M::row(v, 0) / 16);
            if constexpr (E4M3) {
              const uint32_t z = __builtin_amdgcn_perm(vr[v + 1][d / 4], vr[v][d / 4], d % 4 ? 0x07030602 : 0x05010400);
              f[0][e] = bf16_of_e4m3<false>(z, vs);
              f[1][e] = bf16_of_e4m3<true>(z, vs);
            } else {
              f[0][e] = __builtin_amdgcn_perm(vr[v + 1][d / 2], vr[v][d / 2], 0x05040100);
              f[1][e] = __builtin_amdgcn_perm(vr[v + 1][d / 2], vr[v][d / 2], 0x07060302);
            }
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            acc[d + x] = M::mul(__builtin_bit_cast(bf16x8, f[x]), __builtin_bit_cast(bf16x8, hi), acc[d + x]);
            acc[d + x] = M::mul(__builtin_bit_cast(bf16x8, f[x]), __builtin_bit_cast(bf16x8, lo), acc[d + x]);
          }
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < NS; ++v) {
        const float vs = scale_of(v_sc, M::row(v, 0) / 16);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          float f;
          if constexpr (E4M3) {
            const float2 z = (d & 2) ? e4m3_pair<true>(vr[v][d / 4]) : e4m3_pair<false>(vr[v][d / 4]);
            f = ((d & 1) ? z.y : z.x) * vs;
          } else {
            f = __uint_as_float(vr[v][d]);
          }
          acc[d] = M::mul(f, p[v], acc[d]);
        }
      }
    }
    if (more) {
      if (LATE) load_k(next, n - 4);
      else load_v(next, n - 4);
    }
    now = next;
  }

  // ---- the four wavefronts' sums, against the highest of their references
  const float l = M::sum(l_run);
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
      for (int v = 0; v < NA; ++v) {
        float* to = fold + (wave * ROWS + r) * FS + PW * M::row(v, g);
#pragma unroll
        for (int d = 0; d < PW; ++d) to[d] = acc[PW * pass + d][v] * weight;
      }
    __syncthreads();
    for (int x = tid; x < live * ROWS; x += 256) {
      const int y = x / ROWS, rho = x % ROWS, d0 = DB * rho + PW * pass;
      const int R = t.tile * ROWS + y, yi = R / G, yh = t.hk * G + R - yi * G;
      if (!BF && d0 >= D) continue;
      const float top = fmaxf(fmaxf(stat_m[0][y], stat_m[1][y]), fmaxf(stat_m[2][y], stat_m[3][y]));
      float sum = 0.f, o[PW];
#pragma unroll
      for (int d = 0; d < PW; ++d) o[d] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sum += stat_l[k][y] * __builtin_amdgcn_exp2f(stat_m[k][y] - top);
#pragma unroll
        for (int d = 0; d < PW; ++d) o[d] += fold[(k * ROWS + y) * FS + PW * rho + d];
      }
      // Values that are not finite: the blocks at the masks' edges left them out, and in whole ones an infinity times both parts of a probability,
      // or times one that fp32 does not hold, is NaN.  Where this row sees any, they are what its columns have.
      bool odd = any_bad;
#pragma unroll
      for (int d = 0; d < PW; ++d) odd = odd || !is_finite(o[d]);
      if (__builtin_expect(odd, 0)) {
        const RowSpan ys = row_span(a, s, yi);
        const int k0 = max(ys.lo, w.n0 * kKeys), k1 = min(ys.hi, w.n1 * kKeys);
        float found[PW];
#pragma unroll
        for (int d = 0; d < PW; ++d) found[d] = 0.f;
        for (int key = k0 & ~(kScan - 1); key < k1; key += kScan) {
          const int page = page_of(c, t.b, key >> c.shift);
          if (page < 0) continue;
          const S* from = (const S*)(vbase + ((int64_t)page * c.v.sb + (int64_t)(key & ((1 << c.shift) - 1)) * c.v.ss) * (int)sizeof(S)) + d0;
          const uint8_t scale = E4M3 ? c.v_scale[(int64_t)page * c.Hkv + t.hk] : (uint8_t)127;
#pragma unroll
          for (int u = 0; u < kScan; ++u)
#pragma unroll
            for (int d = 0; d < PW; ++d) {
              const float z = stored(from + u * c.v.ss + d, scale);
              found[d] += key + u >= k0 && key + u < k1 && !is_finite(z) ? z : 0.f;
            }
        }
        if (sum == sum) {                              // (a score that is NaN makes all columns so)
#pragma unroll
          for (int d = 0; d < PW; ++d) o[d] = found[d] == 0.f ? o[d] : found[d];
        }
      }
      if (part) {
        float* to = a.part_o + (a.plan.base + (int64_t)t.state * ROWS + y) * D + d0;
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
    if (part) a.part_row[a.plan.base + (int64_t)t.state * ROWS + r] = make_float4(m_all, sum, besides, 0.f);
    else a.lse[(int64_t)h * a.T + s.r.first + i] = sum != 0.f ? m_all * kScoreLn2 + logf(sum) + besides : -INFINITY;
  }
}

// ---- joining the states of rows whose walk was split

// Where the states of a row are: n of them (1: the row is whole), step rows apart
struct RowStates {
  int n;
  int64_t first, step;
};
__device__ __forceinline__ RowStates states_of(const CacheAttnArgs& a, int64_t row, int first, int end) {
  const int t = (int)(row / a.Hq), h = (int)(row - (int64_t)t * a.Hq), G = a.Hq / a.c.Hkv;
  RowStates y{1, 0, 0};
  if (t < first || t >= end) return y;
  const int4 at = a.info[t];
  const int shares = at.y & 0xffff, tile_rows = at.y >> 16;
  // (where starts are no starts, a token may not have been told of: nothing is read outside the states, and no number leaves its type)
  if (shares <= 1 || tile_rows <= 0 || tile_rows > kPromptRows || at.x < 0 || at.z <= 0 || at.z > a.state_rows || at.w < 0 || at.w >= a.T) return y;
  const int hk = h / G, R = at.w * G + h - hk * G, tile = R / tile_rows;
  y.first = at.x + ((int64_t)(at.z - 1 - tile) * a.c.Hkv + hk) * tile_rows + (R - tile * tile_rows);
  y.step = (int64_t)at.z * a.c.Hkv * tile_rows;
  if (tile < at.z && y.first + (shares - 1) * y.step < a.state_rows) y.n = shares;
  return y;
}
__device__ __forceinline__ void store_joined(const CacheAttnArgs& a, const RowStates& s, int64_t row, int x, f32x4 o, float m, float sum, float besides, int bf16) {
  o *= sum != 0.f ? 1.f / sum : 0.f;
  if (__builtin_expect(!(is_finite(o[0]) && is_finite(o[1]) && is_finite(o[2]) && is_finite(o[3])) && sum == sum, 0)) {
    // an infinity times the weight of a state that counts for nothing is NaN: what is not finite in any state is what the row has
    f32x4 found = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < s.n; ++k) {
      const f32x4 z = *reinterpret_cast<const f32x4*>(a.part_o + (s.first + k * s.step) * a.c.D + 4 * x);
#pragma unroll
      for (int e = 0; e < 4; ++e) found[e] += is_finite(z[e]) ? 0.f : z[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = found[e] == 0.f ? o[e] : found[e];
  }
  const int64_t to = row * a.c.D + 4 * x, t = row / a.Hq;
  if (a.o) *reinterpret_cast<f32x4*>(a.o + to) = o;
  if (a.o_lowp && bf16) *reinterpret_cast<u32x2*>((uint16_t*)a.o_lowp + to) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
  else if (a.o_lowp) *reinterpret_cast<f32x4*>((float*)a.o_lowp + to) = o;
  if (x == 0) a.lse[(row - t * a.Hq) * a.T + t] = sum != 0.f ? m * kScoreLn2 + logf(sum) + besides : -INFINITY;
}

// O, not divided by its row sum yet, against the reference m
struct Joined {
  float m, sum, besides;
  f32x4 o;
};
__device__ __forceinline__ Joined join(const Joined& a, const Joined& b) {
  const float m = fmaxf(a.m, b.m), p = __builtin_amdgcn_exp2f(a.m - m), q = __builtin_amdgcn_exp2f(b.m - m);
  return Joined{m, a.sum * p + b.sum * q, a.besides, a.o * p + b.o * q};
}
// states k0, k0 + all, ... of a row, N of them under way
template <int N>
__device__ __forceinline__ Joined join_states(const CacheAttnArgs& a, const RowStates& s, int k0, int all, int x) {
  Joined y{kUnset, 0.f, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int k = k0; k < s.n; k += N * all) {
    f32x4 z[N];
    float4 st[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t from = s.first + (k + u * all) * s.step;
      z[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      st[u] = make_float4(kUnset, 0.f, 0.f, 0.f);
      if (k + u * all < s.n) {
        z[u] = *reinterpret_cast<const f32x4*>(a.part_o + from * a.c.D + 4 * x);
        st[u] = a.part_row[from];
      }
    }
    float top = y.m;
#pragma unroll
    for (int u = 0; u < N; ++u) top = fmaxf(top, st[u].x);
    const float old = __builtin_amdgcn_exp2f(y.m - top);
    y.m = top;
    y.sum *= old;
    y.o *= old;
    y.besides = st[0].z;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float w = __builtin_amdgcn_exp2f(st[u].x - top);
      y.sum += st[u].y * w;
      y.o += z[u] * w;
    }
  }
  return y;
}

// Many states of few rows: a workgroup a row, 64 D / 4 lanes' worth of its states side by side in each wavefront
__global__ __launch_bounds__(64 * kManyWaves) void cache_combine_many_kernel(const CacheAttnArgs a, int bf16) {
  __shared__ Joined fold[kManyWaves * 64];
  const int lane = threadIdx.x & 63, vecs = a.c.D / 4, side = 64 / vecs, x = lane % vecs, y = lane / vecs, all = kManyWaves * side;
  const int first = max(min(a.starts[0], a.T), 0), end = max(min(a.starts[a.c.B], a.T), 0);
  const RowStates s = states_of(a, blockIdx.x, first, end);
  if (s.n <= 1) return;
  const int k0 = uniform(threadIdx.x >> 6) * side + y;
  if (y < side) fold[k0 * vecs + x] = join_states<8>(a, s, k0, all, x);
  __syncthreads();
  if (threadIdx.x >= vecs) return;
  Joined z = fold[x];
  for (int k = 1; k < min(all, s.n); ++k) z = join(z, fold[k * vecs + x]);
  store_joined(a, s, blockIdx.x, x, z.o, z.m, z.sum, z.besides, bf16);
}
// Few states of many rows: 64 D / 4 lanes' worth of rows side by side, each lane through its row's states, four under way; `rounds` times a
// wavefront.  With alone = 1, for more states, a row at a time and its states side by side.  Rows that are whole cost a look.
__global__ __launch_bounds__(256) void cache_combine_kernel(const CacheAttnArgs a, int rounds, int alone, int bf16) {
  const int lane = threadIdx.x & 63, vecs = a.c.D / 4, side = 64 / vecs, per = alone ? 1 : side, x = lane % vecs, y = lane / vecs;
  const int first = max(min(a.starts[0], a.T), 0), end = max(min(a.starts[a.c.B], a.T), 0);
  const int64_t rows = (int64_t)a.T * a.Hq, base = ((int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6)) * rounds * per, stop = min(base + rounds * per, rows);
  for (int64_t row0 = base; row0 < stop; row0 += per) {
    const int64_t row = row0 + (alone ? 0 : y);
    RowStates s{1, 0, 0};
    if (y < side && row < stop) s = states_of(a, row, first, end);
    if (!__any(s.n > 1)) {                             // nor are the other heads of the last token split
      row0 = (min(row0 + per, stop) - 1) / a.Hq * a.Hq + a.Hq - per;
      continue;
    }
    Joined z = join_states<4>(a, s.n > 1 ? s : RowStates{0, 0, 0}, alone ? y : 0, alone ? side : 1, x);
    if (alone) {
      for (int u = 1; u < side; ++u) {
        const int from = lane + u * vecs;
        const Joined other{__shfl(z.m, from), __shfl(z.sum, from), 0.f, f32x4{__shfl(z.o[0], from), __shfl(z.o[1], from), __shfl(z.o[2], from), __shfl(z.o[3], from)}};
        if (y == 0) z = join(z, other);
      }
      if (y != 0) continue;
    }
    if (s.n > 1) store_joined(a, s, row, x, z.o, z.m, z.sum, z.besides, bf16);
  }
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnArgs& a, bool bf16, hipStream_t stream) {
  if (a.plan.grid <= 0 || a.plan.grid > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("cache_attn", stream);
  const dim3 grid((unsigned)a.plan.grid), block(256);
  const bool mod = a.cap > 0.f || a.slopes, few = a.plan.rows == 16;
  auto go = [&](auto plain, auto modified) { hipLaunchKernelGGL(mod ? modified : plain, grid, block, 0, stream, a); };
#define ST_STREAM_FEW(T, S, DP) go(cache_stream_kernel<T, S, 16, DP, false>, cache_stream_kernel<T, S, 16, DP, true>)
#define ST_STREAM(T, S, DP) (few ? ST_STREAM_FEW(T, S, DP) : go(cache_stream_kernel<T, S, 32, DP, false>, cache_stream_kernel<T, S, 32, DP, true>))
  const int D = a.c.D;
  if (!few && D > kTallCacheHead) return hipErrorInvalidValue;
  if (bf16 && a.c.dtype == ST_E4M3) D == 128 ? ST_STREAM(uint16_t, uint8_t, 128) : ST_STREAM(uint16_t, uint8_t, 64);
  else if (bf16) D == 128 ? ST_STREAM(uint16_t, uint16_t, 128) : ST_STREAM(uint16_t, uint16_t, 64);
  else if (a.c.dtype == ST_E4M3) D > kTallCacheHead ? ST_STREAM_FEW(float, uint8_t, 256) : D > 64 ? ST_STREAM(float, uint8_t, 128) : ST_STREAM(float, uint8_t, 64);
  else D > kTallCacheHead ? ST_STREAM_FEW(float, float, 256) : D > 64 ? ST_STREAM(float, float, 128) : ST_STREAM(float, float, 64);
#undef ST_STREAM
#undef ST_STREAM_FEW
  return hipGetLastError();
}

hipError_t launch_cache_combine(const CacheAttnArgs& a, bool bf16, int states, hipStream_t stream) {
  const int64_t rows = (int64_t)a.T * a.Hq;
  if (rows <= 0) return hipSuccess;
  ProfScope prof("cache_combine", stream);
  if (states >= 16 && rows <= kManyRows) {
    hipLaunchKernelGGL(cache_combine_many_kernel, dim3((unsigned)rows), dim3(64 * kManyWaves), 0, stream, a, bf16 ? 1 : 0);
    return hipGetLastError();
  }
  const int alone = states >= 4;
  const int64_t per = alone ? 1 : 64 / (a.c.D / 4), groups = (rows + per - 1) / per, rounds = (groups + 8191) / 8192, blocks = (groups + 4 * rounds - 1) / (4 * rounds);
  if (rounds > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(cache_combine_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a, (int)rounds, alone, bf16 ? 1 : 0);
  return hipGetLastError();
}

}  // namespace st
