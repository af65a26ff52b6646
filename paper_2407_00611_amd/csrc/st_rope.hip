// RMS norm of every query and key head and the rotation by the token's position, in one pass over both, and its gradients.
//
//   n = x rsqrt(mean(x^2) + eps) w              over the D values of a head (left out where no norm is asked for)
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = p f    for each rotated pair, p its axis' position, f its frequency
//   backward  dn = R^T dy,  g = dn w,  dx = r (g - xh mean(g xh)),  dw = sum dn xh,  xh = x r,  r = rsqrt(mean(x^2) + eps)
//
// Bounded by HBM: x is read and y written once (24 heads of 64 x 16384 tokens, three axes: 201 MB in 40.5 us, 5.0 TB/s; the gradients of
// 32/8 heads x 4096 tokens behind their forward: 252 MB in 55 us).  A token's angles serve all of its heads: a workgroup takes some tokens, makes their
// sines and cosines once (LDS), and its lanes then take the heads' rows.  Angles of far positions need more than fp32: p f / 2 pi is
// taken in fp64 and only its fraction rounded (positions below 2^31: 1e-7 of a turn at most, from the fp64 frequency itself).
//
// A row is held by D / 2V neighbouring lanes, V pairs a lane, both values of a pair in the same lane: two vectors half the rotated
// values apart, or, for neighbouring pairs, two in a row.  Values behind the rotated ones are pairs with the angle zero.
#include <algorithm>

#include "st_rope_rows.h"

namespace st {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kTokensMost = 8;                       // tokens whose angles a workgroup holds at a time

// sines and cosines of tokens [t0, t0 + n) into LDS
__device__ __forceinline__ void make_angles(const RopeArgs& g, int64_t t0, int n, float2* angles, int tid) {
  const int half = g.rot / 2;
  for (int x = tid; x < n * half; x += kThreads) {
    const int t = x / half, j = x - t * half;
    const int64_t token = t0 + t, b = token / g.S;
    const int i = (int)(token - b * g.S);
    double p;
    if (g.positions) {
      int axis = 0, end = 0;                         // (no index that is known at run time only: the list would be copied to memory)
#pragma unroll
      for (int y = 0; y + 1 < ST_ROPE_MAX_AXES; ++y) {
        end += g.axis_pairs[y];
        axis += y + 1 < g.n_axes && j >= end;
      }
      p = (double)g.positions[((int64_t)axis * g.B + b) * g.S + i];
    } else {
      p = (double)(g.seg > 0 && i >= g.seg ? g.offset2 + (i - g.seg) : g.offset + i);
    }
    const double turns = p * (g.freq[j] * 0.15915494309189533577);
    float2 y;
    sincospif((float)(2.0 * (turns - rint(turns))), &y.y, &y.x);
    angles[x] = y;
  }
}

template <typename T>
struct Rows {                // of one token and head
  const T* in;
  T* out;
  int t, h;                  // token of the workgroup's, head (keys behind the queries)
};
template <typename T>
__device__ __forceinline__ Rows<T> row_of(const RopeArgs& g, int64_t t0, uint32_t row, uint32_t inv_heads) {
  Rows<T> y;
  const uint32_t heads = (uint32_t)(g.Hq + g.Hkv), t = heads > 1 ? __umulhi(row, inv_heads) : row;
  y.t = (int)t;
  y.h = (int)(row - t * heads);
  const int64_t token = t0 + y.t, b = token / g.S, i = token - b * g.S;
  const bool key = y.h >= g.Hq;
  const View &in = key ? g.k : g.q, &out = key ? g.k_out : g.q_out;
  const int64_t h = key ? y.h - g.Hq : y.h;
  y.in = (const T*)in.ptr + b * in.sb + i * in.ss + h * in.sh;
  y.out = (T*)const_cast<void*>(out.ptr) + b * out.sb + i * out.ss + h * out.sh;
  return y;
}

template <int V>
__device__ __forceinline__ void angle_pairs(const float2* angles, const RopeArgs& g, int t, int pair, Vec<V>& c, Vec<V>& s) {
  const int half = g.rot / 2;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const bool turned = pair + e < half;
    const float2 y = turned ? angles[t * half + pair + e] : make_float2(1.f, 0.f);
    c.x[e] = y.x;
    s.x[e] = y.y;
  }
}

// U: chunks of V pairs a lane holds (head sizes beyond 128 whose halves have an odd number of pairs need two)
template <typename T, int V, int U, bool NEXT>
__global__ __launch_bounds__(kThreads) void rope_fwd_kernel(const RopeArgs g, int lanes, int tokens) {
  __shared__ float2 angles[kTokensMost * kMaxPairs];
  const int tid = threadIdx.x, chunk = tid & (lanes - 1), group = tid / lanes, groups = kThreads / lanes;
  const int64_t all = (int64_t)g.B * g.S, t0 = (int64_t)blockIdx.x * tokens;
  const int n = (int)min((int64_t)tokens, all - t0);
  // row / heads = row inv_heads / 2^32 while rows x heads stay below 2^32: at most 16384 heads of eight tokens
  const uint32_t heads = (uint32_t)(g.Hq + g.Hkv), rows = heads * (uint32_t)n, inv_heads = 0xffffffffu / heads + 1;
  Place<V, NEXT> p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) p[u] = place_of<V, NEXT>(g, chunk + u * lanes);
  Vec<V> a[U], b[U];
  auto fetch = [&](uint32_t row) {
    const Rows<T> y = row_of<T>(g, t0, min(row, rows - 1), inv_heads);
#pragma unroll
    for (int u = 0; u < U; ++u) load_pairs<V, NEXT>(y.in, p[u], a[u], b[u]);
    return y;
  };
  Rows<T> at = fetch(group);
  make_angles(g, t0, n, angles, tid);
  __syncthreads();
  for (uint32_t row = group; row < rows; row += groups) {
    const Rows<T> y = at;
    Vec<V> x[U], z[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = a[u], z[u] = b[u];
    if (row + groups < rows) at = fetch(row + groups);
    if (g.norm) {
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) sum += p[u].live ? x[u].x[e] * x[u].x[e] + z[u].x[e] * z[u].x[e] : 0.f;
      const float r = rsqrtf(row_sum(sum, lanes) / (float)g.D + g.eps);
      const float* w = y.h >= g.Hq ? g.k_weight : g.q_weight;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Vec<V> wa, wb;
        if (w) load_pairs<V, NEXT>(w, p[u], wa, wb);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          x[u].x[e] *= w ? r * wa.x[e] : r;
          z[u].x[e] *= w ? r * wb.x[e] : r;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Vec<V> c, s, ya, yb;
      angle_pairs<V>(angles, g, y.t, p[u].pair, c, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        ya.x[e] = x[u].x[e] * c.x[e] - z[u].x[e] * s.x[e];
        yb.x[e] = x[u].x[e] * s.x[e] + z[u].x[e] * c.x[e];
      }
      if (p[u].live) store_pairs<V, NEXT>(y.out, p[u], ya, yb);
    }
  }
}

// The same rows with the gradient dy (TD) beside them; sums of dw stay in registers until the workgroup has done all its tokens.
// Held to 128 registers, four wavefronts on a SIMD: the 1024 workgroups are on the chip at once (32/8 heads x 4096 tokens, forward and
// backward: 59 us, 68 with 160 registers and a quarter of the workgroups left over).
template <typename T, typename TD, int V, int U, bool NEXT>
__global__ __launch_bounds__(kThreads, 4) void rope_bwd_kernel(const RopeArgs g, int lanes, int tokens, int64_t blocks) {
  __shared__ float2 angles[kTokensMost * kMaxPairs];
  __shared__ float sums[kThreads * V * U * 2];
  const int tid = threadIdx.x, chunk = tid & (lanes - 1), group = tid / lanes, groups = kThreads / lanes;
  const int64_t all = (int64_t)g.B * g.S;
  const uint32_t heads = (uint32_t)(g.Hq + g.Hkv), inv_heads = 0xffffffffu / heads + 1;
  Place<V, NEXT> p[U];
  Vec<V> dwa[2][U], dwb[2][U];                       // of the query weights and the key weights
#pragma unroll
  for (int u = 0; u < U; ++u) {
    p[u] = place_of<V, NEXT>(g, chunk + u * lanes);
#pragma unroll
    for (int e = 0; e < V; ++e) dwa[0][u].x[e] = dwa[1][u].x[e] = dwb[0][u].x[e] = dwb[1][u].x[e] = 0.f;
  }
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int64_t t0 = blk * tokens;
    const int n = (int)min((int64_t)tokens, all - t0);
    const uint32_t rows = heads * (uint32_t)n;
    __syncthreads();
    make_angles(g, t0, n, angles, tid);
    __syncthreads();
    for (uint32_t row = group; row < rows; row += groups) {
      const Rows<T> y = row_of<T>(g, t0, row, inv_heads);
      const bool key = y.h >= g.Hq;
      const View& dv = key ? g.dk : g.dq;
      const int64_t token = t0 + y.t, bb = token / g.S, i = token - bb * g.S;
      const TD* drow = (const TD*)dv.ptr + bb * dv.sb + i * dv.ss + (key ? y.h - g.Hq : y.h) * dv.sh;
      Vec<V> x[U], z[U], ga[U], gb[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (g.norm) load_pairs<V, NEXT>(y.in, p[u], x[u], z[u]);
        load_pairs<V, NEXT>(drow, p[u], ga[u], gb[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {                  // dn = R^T dy
        Vec<V> c, s;
        angle_pairs<V>(angles, g, y.t, p[u].pair, c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float a = ga[u].x[e], b = gb[u].x[e];
          ga[u].x[e] = a * c.x[e] + b * s.x[e];
          gb[u].x[e] = b * c.x[e] - a * s.x[e];
        }
      }
      if (g.norm) {
        const float* w = key ? g.k_weight : g.q_weight;
        float xx = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) xx += p[u].live ? x[u].x[e] * x[u].x[e] + z[u].x[e] * z[u].x[e] : 0.f;
        const float r = rsqrtf(row_sum(xx, lanes) / (float)g.D + g.eps);
        float gx = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          Vec<V> wa, wb;
          if (w) load_pairs<V, NEXT>(w, p[u], wa, wb);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            x[u].x[e] *= r;
            z[u].x[e] *= r;
            const float da = ga[u].x[e] * x[u].x[e], db = gb[u].x[e] * z[u].x[e];
            dwa[0][u].x[e] += key ? 0.f : da;
            dwb[0][u].x[e] += key ? 0.f : db;
            dwa[1][u].x[e] += key ? da : 0.f;
            dwb[1][u].x[e] += key ? db : 0.f;
            if (w) ga[u].x[e] *= wa.x[e], gb[u].x[e] *= wb.x[e];
            gx += p[u].live ? ga[u].x[e] * x[u].x[e] + gb[u].x[e] * z[u].x[e] : 0.f;
          }
        }
        const float mean = row_sum(gx, lanes) / (float)g.D;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            ga[u].x[e] = r * (ga[u].x[e] - x[u].x[e] * mean);
            gb[u].x[e] = r * (gb[u].x[e] - z[u].x[e] * mean);
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p[u].live) store_pairs<V, NEXT>(y.out, p[u], ga[u], gb[u]);
    }
  }
  if (!g.dw_parts) return;
  // over the groups of lanes, in their order; parts [workgroup][queries, keys][D]
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sums[((u * 2) * V + e) * kThreads + tid] = dwa[k][u].x[e];
        sums[((u * 2 + 1) * V + e) * kThreads + tid] = dwb[k][u].x[e];
      }
    __syncthreads();
    for (int x = tid; x < U * 2 * V * lanes; x += kThreads) {
      const int l = x & (lanes - 1), what = x / lanes, e = what % V, second = what / V % 2, u = what / (2 * V);
      const Place<V, NEXT> q = place_of<V, NEXT>(g, l + u * lanes);
      if (!q.live) continue;
      float sum = 0.f;
      for (int y = 0; y < groups; ++y) sum += sums[what * kThreads + y * lanes + l];
      // element of the row that value e of the first or second of the pairs is
      const int d = NEXT ? 2 * (q.pair + e) + second : (second ? q.b : q.a) + e;
      g.dw_parts[((int64_t)blockIdx.x * 2 + k) * g.D + d] = sum;
    }
  }
}

// dw += (or =) the workgroups' sums in their order: 16 columns a workgroup, sixty-four runs of the sums side by side, four loads
// of each in flight
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* __restrict__ parts, int32_t n, int32_t D, float* dwq, float* dwk, int32_t assign) {
  __shared__ float fold[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), y = threadIdx.x >> 4;
  float sum = 0.f;
  if (c < 2 * D)
    for (int k = y; k < n; k += 256) {
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = k + 64 * u < n ? parts[(int64_t)(k + 64 * u) * 2 * D + c] : 0.f;
      sum += (x[0] + x[1]) + (x[2] + x[3]);
    }
  fold[y][threadIdx.x & 15] = sum;
  __syncthreads();
  if (y != 0 || c >= 2 * D) return;
  float* out = c < D ? dwq : dwk;
  if (!out) return;
  out += c < D ? c : c - D;
  float all = assign ? 0.f : *out;
  for (int k = 0; k < 64; ++k) all += fold[k][threadIdx.x & 15];
  *out = all;
}

// tokens of a workgroup: one while that does not fill the chip, then as many as keep four workgroups for every compute unit; where
// there are more of them than compute units, as many as give every lane a row
int tokens_each(const RopeArgs& g) {
  const int64_t tokens = (int64_t)g.B * g.S, groups = kThreads / lanes_of(g.D, pairs_per_lane(g.D, g.rot));
  const int64_t full = std::min<int64_t>((groups + g.Hq + g.Hkv - 1) / (g.Hq + g.Hkv), std::max<int64_t>(tokens / 256, 1));
  return (int)std::min<int64_t>(std::max<int64_t>(tokens / 1024, full), kTokensMost);
}

int bwd_blocks(const RopeArgs& g) {
  const int64_t tokens = (int64_t)g.B * g.S;
  const int each = tokens_each(g);
  return (int)std::min<int64_t>((tokens + each - 1) / each, kRopeBlocksMost);
}

}  // namespace

hipError_t launch_rope_fwd(const RopeArgs& g, bool bf16, hipStream_t stream) {
  const int64_t tokens = (int64_t)g.B * g.S;
  if (tokens <= 0) return hipSuccess;
  const int each = tokens_each(g);
  const int64_t blocks = (tokens + each - 1) / each;
  if (blocks > (1 << 23)) return hipErrorInvalidValue;
  ProfScope prof("qk_rope_fwd", stream);
  with_pairs(g, [&](auto v, auto u, auto next) {
    constexpr int V = decltype(v)::value, U = decltype(u)::value;
    constexpr bool NEXT = decltype(next)::value;
    const dim3 grid((unsigned)blocks), block(kThreads);
    if (bf16) hipLaunchKernelGGL((rope_fwd_kernel<uint16_t, V, U, NEXT>), grid, block, 0, stream, g, lanes_of(g.D, V), each);
    else hipLaunchKernelGGL((rope_fwd_kernel<float, V, U, NEXT>), grid, block, 0, stream, g, lanes_of(g.D, V), each);
  });
  return hipGetLastError();
}

hipError_t launch_rope_bwd(const RopeArgs& g, bool bf16, bool d_bf16, float* dwq, float* dwk, bool assign, hipStream_t stream) {
  const int64_t tokens = (int64_t)g.B * g.S;
  const int each = tokens_each(g);
  const int64_t blocks = (tokens + each - 1) / each;
  if (tokens > 0) {
    ProfScope prof("qk_rope_bwd", stream);
    const dim3 grid((unsigned)bwd_blocks(g)), block(kThreads);
    with_pairs(g, [&](auto v, auto u, auto next) {
      constexpr int V = decltype(v)::value, U = decltype(u)::value;
      constexpr bool NEXT = decltype(next)::value;
      const int lanes = lanes_of(g.D, V);
      if (bf16 && d_bf16) hipLaunchKernelGGL((rope_bwd_kernel<uint16_t, uint16_t, V, U, NEXT>), grid, block, 0, stream, g, lanes, each, blocks);
      else if (bf16) hipLaunchKernelGGL((rope_bwd_kernel<uint16_t, float, V, U, NEXT>), grid, block, 0, stream, g, lanes, each, blocks);
      else hipLaunchKernelGGL((rope_bwd_kernel<float, float, V, U, NEXT>), grid, block, 0, stream, g, lanes, each, blocks);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!dwq && !dwk) return hipSuccess;
  ProfScope prof("qk_rope_dw", stream);
  hipLaunchKernelGGL(rope_dw_kernel, dim3((unsigned)((2 * g.D + 15) / 16)), dim3(1024), 0, stream, g.dw_parts, tokens > 0 ? bwd_blocks(g) : 0, g.D, dwq, dwk, assign ? 1 : 0);
  return hipGetLastError();
}

}  // namespace st
