// New keys and values into a cache of pages, and chunks of it out again.
//
//   n = x rsqrt(mean(x^2) + eps) w,  (a, b) -> (a cos t - b sin t, a sin t + b cos t)      queries and keys, as st_rope.hip
//   e = max(e of the rows that are there, least e with max |x| <= 448 2^e)                 of a page and head, pages in e4m3
//   stored = e4m3(x 2^-e);  rows that are there: e4m3(stored 2^(e - e'))                   (exact but below the least value)
//
// Appending: a workgroup has the new rows of a page and head, keys or values, whose scale it needs before it stores any; up to four rows a lane
// stay in registers meanwhile, so that everything is read once.  Queries are a workgroup's of eight tokens, whose angles all heads share.
// Prompts of 11000 tokens (32/8 heads of 128 in 8 bits) take 61 us for 248 MB, 4.0 TB/s: memory, and the vector unit over half of the time (22 of
// 40 million cycles), for keys in fp64 above all.  One token each of 16 sequences: 7.5 us, a launch and its chain of latencies.
#include <algorithm>

#include "st_cache.h"
#include "st_rope_rows.h"

namespace st {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kTokensMost = 8;                       // tokens whose angles a workgroup holds for the queries

// ---- arithmetic of the keys: fp32 as the queries' for pages in fp32, otherwise fp64, so that a value is rounded as one of the 64-bit
// definition is (in fp32 one of 30000 bf16 keys fell to the other side; the prompts above to bf16 pages: 70 us for 270 MB)

// sine and cosine of x turns, |x| <= 1/2: x is taken to the nearest quarter, |r| <= pi / 4 from there, and both series of r are cut where the
// next term is below 1e-16
__device__ __forceinline__ void sincos_turns(double x, double& s, double& c) {
  const double n = rint(4.0 * x), r = (x - 0.25 * n) * 6.283185307179586477, z = r * r;
  const double ps = r * (1.0 + z * (-1.0 / 6 + z * (1.0 / 120 + z * (-1.0 / 5040 + z * (1.0 / 362880 + z * (-1.0 / 39916800 + z * (1.0 / 6227020800.0 - z / 1307674368000.0)))))));
  const double pc = 1.0 + z * (-0.5 + z * (1.0 / 24 + z * (-1.0 / 720 + z * (1.0 / 40320 + z * (-1.0 / 3628800 + z * (1.0 / 479001600.0 + z * (-1.0 / 87178291200.0 + z / 20922789888000.0)))))));
  const int k = (int)n & 3;
  const double u = k & 1 ? pc : ps, v = k & 1 ? ps : pc;
  s = k & 2 ? -u : u;
  c = (k + 1) & 2 ? -v : v;
}
// Sine and cosine of p f, f in 64ths of a turn: those of the nearest 64th from a table, and of the rest, at most pi / 64, from series whose next
// terms are below 1e-15.  The angle itself is off by 2^-52 of p f at most: f and its unit are rounded.  The product is rounded to a whole number by an addition to 1.5 2^52, whose last bits are that number's.
constexpr int kParts = 64;
__device__ __forceinline__ void sincos_part(double p, double f, const double2* table, double& s, double& c) {
  constexpr double kWhole = 6755399441055744.0, t = 6.283185307179586477 / kParts;
  const double w = fma(p, f, kWhole), r = fma(p, f, kWhole - w), z = r * r;
  const double2 at = table[(uint32_t)__double_as_longlong(w) % kParts];
  const double ps = r * (t + z * (-t * t * t / 6 + z * (t * t * t * t * t / 120 - z * (t * t * t * t * t * t * t / 5040))));
  const double pc = 1.0 + z * (-t * t / 2 + z * (t * t * t * t / 24 - z * (t * t * t * t * t * t / 720)));
  s = at.x * pc + at.y * ps;
  c = at.y * pc - at.x * ps;
}

// To fp32 so that a second rounding, to fewer bits, gives what one rounding of x would: cut off behind 23 bits, with a one in the last of them
// where anything was cut off.
__device__ __forceinline__ float sticky(double x) {
  const uint64_t u = __double_as_longlong(x);
  const uint32_t low = (uint32_t)u;
  return (float)__longlong_as_double((u & 0xffffffff00000000ull) | (low & 0xe0000000u) | min(low & 0x1fffffffu, 1u) << 29);
}

template <typename A>
__device__ __forceinline__ A lanes_sum(A x, int lanes) {
  for (int d = 1; d < lanes; d *= 2) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float inv_root(float x) { return rsqrtf(x); }
// (the instruction's 2^-26 by two steps of Newton's; zero of an infinity, as of fp32)
__device__ __forceinline__ double inv_root(double x) {
  double y = __builtin_amdgcn_rsq(x);
#pragma unroll
  for (int k = 0; k < 2; ++k) y = fma(0.5 * y, fma(-x * y, y, 1.0), y);
  return x == INFINITY ? 0.0 : y;
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= 3.402823466e38f; }
// The least e, -126 at the least, with top <= 448 2^e = 1.75 2^(e + 8)
__device__ __forceinline__ int exponent_for(float top) {
  const uint32_t u = __float_as_uint(top);
  return max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0), -126);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 0x00400000u); }   // -127 .. 127

// Position of packed row t for a pair: that of its token, `place`, or from a table
__device__ __forceinline__ double position_of(const RopeArgs& g, double place, int t, int pair) {
  if (!g.positions) return place;
  int axis = 0, end = 0;                             // (no index that is known at run time only: the list would be copied to memory)
#pragma unroll
  for (int y = 0; y + 1 < ST_ROPE_MAX_AXES; ++y) {
    end += g.axis_pairs[y];
    axis += y + 1 < g.n_axes && pair >= end;
  }
  return (double)g.positions[(int64_t)axis * g.S + t];
}
__device__ __forceinline__ double fraction(double turns) { return turns - rint(turns); }
constexpr double kPerTurn = 0.15915494309189533577;

// What a workgroup has of the new rows: those of sequence b whose tokens lie in one page
struct Piece {
  int b, j, slot0;           // sequence, page of its pages, token of its first row
  int lo, hi;                // tokens
  int row0;                  // packed row of token lo
};
// Sequence b has at most n_b / page + 2 such pieces, so the workgroups from starts[b] / page + 2 b on are enough for it (the number before the
// next one's is at least that), and a workgroup finds its sequence by a look at all of them, a thread each.
__device__ __forceinline__ bool find_piece(const AppendArgs& a, Piece& p, int* found) {
  const int u = blockIdx.x, tid = threadIdx.x, shift = a.c.shift, T = a.g.S;
  if (tid == 0) *found = -1;
  __syncthreads();
  for (int b = tid; b < a.c.B; b += kThreads) {
    const SeqRows r = seq_rows(a.starts, b, T);
    if (u >= (r.first >> shift) + 2 * b && u < ((r.first + r.n) >> shift) + 2 * b + 2) *found = b;
  }
  __syncthreads();
  p.b = __builtin_amdgcn_readfirstlane(*found);
  if (p.b < 0) return false;
  const SeqRows r = seq_rows(a.starts, p.b, T);
  const int len = a.c.lens[p.b];
  p.slot0 = len - r.n;
  p.j = (max(p.slot0, 0) >> shift) + u - (r.first >> shift) - 2 * p.b;
  p.lo = (int)min(max((int64_t)max(p.slot0, 0), (int64_t)p.j << shift), (int64_t)max(len, 0));
  p.hi = (int)min((int64_t)len, ((int64_t)p.j + 1) << shift);
  p.row0 = r.first + p.lo - p.slot0;
  return p.lo < p.hi;
}

// T: of the rows; A: of the arithmetic of keys; S: what the pages hold
template <typename T, typename A, typename S, int V, int U, bool NEXT>
__device__ __forceinline__ void append_rows(const AppendArgs& a, const Piece& p, int h, bool key, int lanes, int* shared, double2* parts) {
  constexpr bool E4M3 = std::is_same<S, uint8_t>::value, F64 = std::is_same<A, double>::value;
  const RopeArgs& g = a.g;
  const int tid = threadIdx.x, chunk = tid & (lanes - 1), group = tid / lanes, groups = kThreads / lanes, half = g.rot / 2;
  if (p.j >= a.c.width) return;
  const int page = __builtin_amdgcn_readfirstlane(page_of(a.c, p.b, p.j));
  if (page < 0) return;
  const View& in = key ? g.k : a.v_in;
  const View& to = key ? a.c.k : a.c.v;
  const T* src = (const T*)in.ptr + (int64_t)p.row0 * in.ss + (int64_t)h * in.sh;
  S* dst = (S*)const_cast<void*>(to.ptr) + (int64_t)page * to.sb + (int64_t)h * to.sh;
  const int begun = p.lo & ((1 << a.c.shift) - 1), n = p.hi - p.lo;
  Place<V, NEXT> at[U];
  double f[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = place_of<V, NEXT>(g, chunk + u * lanes);
#pragma unroll
    for (int e = 0; e < V; ++e) f[u][e] = key && at[u].pair + e < half ? g.freq[at[u].pair + e] * (kPerTurn * (F64 ? kParts : 1)) : 0.0;
  }
  if (F64 && key) {
    if (tid < kParts) {
      double sn, cs;
      sincos_turns(tid < kParts / 2 ? tid / (double)kParts : tid / (double)kParts - 1.0, sn, cs);
      parts[tid] = make_double2(sn, cs);
    }
    __syncthreads();
  }
  const double place0 = (double)(g.offset + p.lo);
  auto load_row = [&](int row, Vec<V> (&x)[U], Vec<V> (&z)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) load_pairs<V, NEXT>(src + row * in.ss, at[u], x[u], z[u]);
  };
  auto finish = [&](int row, Vec<V> (&x)[U], Vec<V> (&z)[U]) {   // of rows as they are stored, before they are rounded
    if (!key) return;
    A r = 1;
    if (g.norm) {
      A sum = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += at[u].live ? (A)x[u].x[e] * (A)x[u].x[e] + (A)z[u].x[e] * (A)z[u].x[e] : (A)0;
      r = inv_root(lanes_sum(sum, lanes) / (A)g.D + (A)g.eps);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      A y[V], w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = (A)x[u].x[e], w[e] = (A)z[u].x[e];
      if (g.norm) {
        Vec<V> wa, wb;
        if (g.k_weight) load_pairs<V, NEXT>(g.k_weight, at[u], wa, wb);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          y[e] *= g.k_weight ? r * (A)wa.x[e] : r;
          w[e] *= g.k_weight ? r * (A)wb.x[e] : r;
        }
      }
      if (at[u].pair < half) {                         // (a lane's pairs turn all or none; those as they are: zero times infinity is NaN)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const double place = position_of(g, place0 + (double)row, p.row0 + row, at[u].pair + e);
          A c, s;
          if constexpr (F64) sincos_part(place, f[u][e], parts, s, c);
          else sincospif((float)(2.0 * fraction(place * f[u][e])), &s, &c);
          const A m = y[e] * c - w[e] * s;
          w[e] = y[e] * s + w[e] * c;
          y[e] = m;
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if constexpr (E4M3) x[u].x[e] = sticky(y[e]), z[u].x[e] = sticky(w[e]);
        else x[u].x[e] = (float)y[e], z[u].x[e] = (float)w[e];
      }
    }
  };
  auto make = [&](int row, Vec<V> (&x)[U], Vec<V> (&z)[U]) {
    load_row(row, x, z);
    finish(row, x, z);
  };
  bool all_finite = true;
  auto store_row = [&](int row, Vec<V> (&x)[U], Vec<V> (&z)[U], float unit) {
    S* to_row = dst + (int64_t)(begun + row) * to.ss;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (E4M3) {
        if (__builtin_expect(!all_finite, 0))
#pragma unroll
          for (int e = 0; e < V; ++e) {
            x[u].x[e] = is_finite(x[u].x[e]) ? x[u].x[e] : NAN;
            z[u].x[e] = is_finite(z[u].x[e]) ? z[u].x[e] : NAN;
          }
#pragma unroll
        for (int e = 0; e < V; ++e) x[u].x[e] *= unit, z[u].x[e] *= unit;
      }
      if (at[u].live) store_pairs<V, NEXT>(to_row, at[u], x[u], z[u]);
    }
  };
  if constexpr (!E4M3) {
    for (int row = group; row < n; row += groups) {
      Vec<V> x[U], z[U];
      make(row, x, z);
      store_row(row, x, z, 1.f);
    }
  } else {
    uint8_t* scale = (key ? a.c.k_scale : a.c.v_scale) + (int64_t)page * g.Hkv + h;
    const int had = begun > 0 ? min(max((int)*scale - 127, -126), 127) : -126;
    // the highest magnitude, as the bits of one, which are in order: an infinity or NaN is above all finite ones
    uint32_t top = 0;
    auto highest = [&](const Vec<V> (&x)[U], const Vec<V> (&z)[U], uint32_t below) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at[u].live)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const uint32_t y = __float_as_uint(x[u].x[e]) & 0x7fffffff, w = __float_as_uint(z[u].x[e]) & 0x7fffffff;
            top = max(top, max(y < below ? y : 0, w < below ? w : 0));
          }
    };
    auto of_all = [&]() {
      for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      if ((tid & 63) == 0) shared[tid >> 6] = (int)top;
      __syncthreads();
      top = max(max((uint32_t)shared[0], (uint32_t)shared[1]), max((uint32_t)shared[2], (uint32_t)shared[3]));
    };
    constexpr uint32_t kInfinity = 0x7f800000u;
    // The first rows of a lane stay in registers until the scale is known, the others are made again (pages of up to 64 tokens of 128: none)
    constexpr int kHeld = 4;
    Vec<V> x[kHeld][U], z[kHeld][U];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) load_row(min(group + k * groups, n - 1), x[k], z[k]);
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (group + k * groups < n) {
        finish(group + k * groups, x[k], z[k]);
        highest(x[k], z[k], 0xffffffffu);
      }
    for (int row = group + kHeld * groups; row < n; row += groups) {
      Vec<V> y[U], w[U];
      make(row, y, w);
      highest(y, w, 0xffffffffu);
    }
    of_all();
    if (__builtin_expect(top >= kInfinity, 0)) {       // the highest of the finite ones
      all_finite = false;
      top = 0;
      for (int row = group; row < n; row += groups) {
        Vec<V> y[U], w[U];
        make(row, y, w);
        highest(y, w, kInfinity);
      }
      __syncthreads();
      of_all();
    }
    const int e = max(had, exponent_for(__uint_as_float(top)));
    const float unit = power_of_two(-e);
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (group + k * groups < n) store_row(group + k * groups, x[k], z[k], unit);
    for (int row = group + kHeld * groups; row < n; row += groups) {
      Vec<V> y[U], w[U];
      make(row, y, w);
      store_row(row, y, w, unit);
    }
    if (e > had && begun > 0) {
      const int less = e - had;
      const float by = less < 32 ? power_of_two(-less) : 0.f;
      for (int row = group; row < begun; row += groups)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          S* to_row = dst + (int64_t)row * to.ss;
          Vec<V> y, w;
          load_pairs<V, NEXT>(to_row, at[u], y, w);
#pragma unroll
          for (int v = 0; v < V; ++v) y.x[v] *= by, w.x[v] *= by;
          if (at[u].live) store_pairs<V, NEXT>(to_row, at[u], y, w);
        }
    }
    if (tid == 0) *scale = (uint8_t)(e + 127);
  }
}

// grid (pieces, 2 Hkv + eights of a page's tokens): keys and values of a head, or all query heads of eight tokens
template <typename T, typename S, int V, int U, bool NEXT>
__global__ __launch_bounds__(kThreads, (std::is_same<S, uint8_t>::value ? 4 : 1)) void cache_append_kernel(const AppendArgs a, int lanes) {
  constexpr bool F64 = sizeof(S) < 4;
  __shared__ __attribute__((aligned(16))) float2 angles[kTokensMost * kMaxPairs];
  __shared__ int shared[4];
  const RopeArgs& g = a.g;
  Piece p;
  if (!find_piece(a, p, shared)) return;
  __syncthreads();
  const int y = blockIdx.y;
  if (y < 2 * g.Hkv) {
    // (four pairs a lane in fp64: with eight the registers leave two wavefronts a SIMD)
    constexpr int VK = F64 && V == 8 ? 4 : V;
    append_rows<T, typename std::conditional<F64, double, float>::type, S, VK, U, NEXT>(a, p, y >> 1, (y & 1) == 0, lanes * (V / VK), shared, (double2*)angles);
    return;
  }
  const int t0 = (y - 2 * g.Hkv) * kTokensMost, n = min(kTokensMost, p.hi - p.lo - t0), half = g.rot / 2;
  if (n <= 0) return;
  const int tid = threadIdx.x, chunk = tid & (lanes - 1), group = tid / lanes, groups = kThreads / lanes;
  // row / heads = row inv_heads / 2^32 while rows x heads stay below 2^32: at most 16384 heads of eight tokens
  const uint32_t heads = (uint32_t)g.Hq, rows = heads * (uint32_t)n, inv_heads = 0xffffffffu / heads + 1;
  Place<V, NEXT> at[U];
#pragma unroll
  for (int u = 0; u < U; ++u) at[u] = place_of<V, NEXT>(g, chunk + u * lanes);
  Vec<V> x[U], z[U], wa[U], wb[U];
  auto fetch = [&](uint32_t row) {
    row = min(row, rows - 1);
    const uint32_t t = heads > 1 ? __umulhi(row, inv_heads) : row;
    const T* src = (const T*)g.q.ptr + (int64_t)(p.row0 + t0 + (int)t) * g.q.ss + (int64_t)(row - t * heads) * g.q.sh;
#pragma unroll
    for (int u = 0; u < U; ++u) load_pairs<V, NEXT>(src, at[u], x[u], z[u]);
  };
  fetch(group);
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < V; ++e) wa[u].x[e] = wb[u].x[e] = 1.f;
    if (g.q_weight) load_pairs<V, NEXT>(g.q_weight, at[u], wa[u], wb[u]);
  }
  const double place0 = (double)(g.offset + p.lo + t0);
  for (int e = tid; e < n * half; e += kThreads) {
    const int t = e / half, j = e - t * half;
    float2 w;
    sincospif((float)(2.0 * fraction(position_of(g, place0 + (double)t, p.row0 + t0 + t, j) * (g.freq[j] * kPerTurn))), &w.y, &w.x);
    angles[e] = w;
  }
  __syncthreads();
  for (uint32_t row = group; row < rows; row += groups) {
    const uint32_t t = heads > 1 ? __umulhi(row, inv_heads) : row;
    T* dst = (T*)const_cast<void*>(g.q_out.ptr) + (int64_t)(p.row0 + t0 + (int)t) * g.q_out.ss + (int64_t)(row - t * heads) * g.q_out.sh;
    Vec<V> ya[U], yb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) ya[u] = x[u], yb[u] = z[u];
    if (row + groups < rows) fetch(row + groups);
    float r = 1.f;
    if (g.norm) {
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += at[u].live ? ya[u].x[e] * ya[u].x[e] + yb[u].x[e] * yb[u].x[e] : 0.f;
      r = rsqrtf(row_sum(sum, lanes) / (float)g.D + g.eps);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (g.norm) {
#pragma unroll
        for (int e = 0; e < V; ++e) ya[u].x[e] *= r * wa[u].x[e], yb[u].x[e] *= r * wb[u].x[e];
      }
      if (at[u].pair < half) {                         // (a lane's pairs turn all or none; those as they are: zero times infinity is NaN)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 w = angles[t * half + at[u].pair + e];
          const float m = ya[u].x[e], o = yb[u].x[e];
          ya[u].x[e] = m * w.x - o * w.y;
          yb[u].x[e] = m * w.y + o * w.x;
        }
      }
      if (at[u].live) store_pairs<V, NEXT>(dst, at[u], ya[u], yb[u]);
    }
  }
}

// ---- chunks

// Bound by memory: 32768 tokens of 8 heads of 128 in 8 bits to bf16 (201 MB, in part from the last cache) take 32 us.  A workgroup takes
// `tokens` neighbouring tokens of a sequence, whose pages it looks up first, and a thread 16 bytes of the chunk at a time, four of them under
// way; grid (., B, 2: keys and values).  vecs: such pieces of a row, inv: 2^32 / pieces of a token and of a row.
constexpr int kReadTokens = 64, kReadAtOnce = 4;

template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const ReadArgs a, int tokens, uint32_t vecs, uint32_t inv_token, uint32_t inv_row) {
  constexpr int V = 16 / (int)sizeof(T);
  __shared__ int pages[kReadTokens];
  const CacheArgs& c = a.c;
  const View& out = blockIdx.z ? a.v_out : a.k_out;
  if (!out.ptr) return;
  const View& in = blockIdx.z ? c.v : c.k;
  const uint8_t* scales = blockIdx.z ? c.v_scale : c.k_scale;
  const int b = blockIdx.y, tid = threadIdx.x, i0 = blockIdx.x * tokens, n = min(tokens, a.count - i0), mask = (1 << c.shift) - 1;
  const int64_t first = (a.first ? a.first[b] : 0) + (int64_t)i0;
  if (tid < n) {
    const int64_t token = first + tid;
    pages[tid] = token >= 0 && token < seq_len(c, b) ? page_of(c, b, (int)(token >> c.shift)) : -1;
  }
  __syncthreads();
  const uint32_t token_vecs = vecs * (uint32_t)c.Hkv, all = token_vecs * (uint32_t)n;
  T* dst = (T*)const_cast<void*>(out.ptr) + b * out.sb;
  for (uint32_t x0 = tid; x0 < all; x0 += kThreads * kReadAtOnce) {
    Vec<V> y[kReadAtOnce];
    float unit[kReadAtOnce];
    int page[kReadAtOnce], i[kReadAtOnce], h[kReadAtOnce], d[kReadAtOnce];
#pragma unroll
    for (int u = 0; u < kReadAtOnce; ++u) {
      const uint32_t x = min(x0 + u * kThreads, all - 1), t = tokens == 1 ? 0 : token_vecs > 1 ? __umulhi(x, inv_token) : x, w = x - t * token_vecs;
      const uint32_t z = vecs > 1 ? __umulhi(w, inv_row) : w;
      i[u] = (int)t;
      h[u] = (int)z;
      d[u] = (int)(w - z * vecs) * V;
      page[u] = pages[t];
      unit[u] = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) y[u].x[e] = 0.f;
      if (page[u] >= 0) {
        y[u] = load<V>((const S*)in.ptr + (int64_t)page[u] * in.sb + (int64_t)((int)(first + i[u]) & mask) * in.ss + (int64_t)h[u] * in.sh + d[u]);
        if constexpr (std::is_same<S, uint8_t>::value) unit[u] = scale_value(scales[(int64_t)page[u] * c.Hkv + h[u]]);
      }
    }
#pragma unroll
    for (int u = 0; u < kReadAtOnce; ++u) {
      if (x0 + u * kThreads >= all) break;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if constexpr (std::is_same<S, uint8_t>::value) y[u].x[e] *= unit[u];
      }
      store<V>(dst + (int64_t)(i0 + i[u]) * out.ss + (int64_t)h[u] * out.sh + d[u], y[u]);
    }
  }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, bool bf16, hipStream_t stream) {
  const RopeArgs& g = a.g;
  if (g.S <= 0 || a.c.B <= 0) return hipSuccess;
  const int64_t pieces = ((int64_t)g.S >> a.c.shift) + 2 * (int64_t)a.c.B;
  const int y = 2 * g.Hkv + (g.Hq > 0 ? (1 << a.c.shift) / kTokensMost : 0);
  if (pieces > (1 << 23) || y > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)pieces, (unsigned)y), block(kThreads);
  ProfScope prof("cache_append", stream);
  with_pairs(g, [&](auto v, auto u, auto next) {
    constexpr int V = decltype(v)::value, U = decltype(u)::value;
    constexpr bool NEXT = decltype(next)::value;
    const int lanes = lanes_of(g.D, V);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, lanes); };
    if (a.c.dtype == ST_E4M3) bf16 ? go(cache_append_kernel<uint16_t, uint8_t, V, U, NEXT>) : go(cache_append_kernel<float, uint8_t, V, U, NEXT>);
    else bf16 ? go(cache_append_kernel<uint16_t, uint16_t, V, U, NEXT>) : go(cache_append_kernel<float, float, V, U, NEXT>);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const ReadArgs& a, int out_dtype, hipStream_t stream) {
  if (a.count <= 0 || a.c.B <= 0) return hipSuccess;
  const uint32_t vecs = (uint32_t)(a.c.D / (out_dtype == ST_BF16 ? 8 : 4)), token_vecs = vecs * (uint32_t)a.c.Hkv;
  // eight rounds of a workgroup; fewer where that leaves the chip less than four workgroups a compute unit
  const int64_t full = std::max<int64_t>(2 * (int64_t)a.count * a.c.B / 1024, 1);
  const int tokens = (int)std::min<int64_t>(std::min<int64_t>(std::max<int64_t>(2048 / token_vecs, 1), kReadTokens), full);
  const int64_t blocks = ((int64_t)a.count + tokens - 1) / tokens;
  if (blocks > (1 << 23)) return hipErrorInvalidValue;
  // x / y = x inv / 2^32 while x y stays below 2^32: the 2048 pieces of several tokens, or those of one token of 16384 heads by those of a row
  const uint32_t inv_token = 0xffffffffu / token_vecs + 1, inv_row = 0xffffffffu / vecs + 1;
  const dim3 grid((unsigned)blocks, (unsigned)a.c.B, 2), block(kThreads);
  ProfScope prof("cache_read", stream);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, tokens, vecs, inv_token, inv_row); };
  if (a.c.dtype == ST_E4M3) out_dtype == ST_BF16 ? go(cache_read_kernel<uint8_t, uint16_t>) : go(cache_read_kernel<uint8_t, float>);
  else out_dtype == ST_BF16 ? go(cache_read_kernel<uint16_t, uint16_t>) : go(cache_read_kernel<float, float>);
  return hipGetLastError();
}

}  // namespace st
