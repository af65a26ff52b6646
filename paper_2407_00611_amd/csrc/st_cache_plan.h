// How the attention of a batch of sequences is cut into the workgroups of a launch.  Lengths and rows are in device memory, and differ from
// sequence to sequence by orders of magnitude; a workgroup finds its piece of the work from them by itself.
//
// Sequence b has S_b row tiles, each of which walks about L_b key blocks.  With c key blocks a share, c = sum S_b L_b Hkv / target or the
// least, sequence b is cut into ceil(L_b / c) shares: at most target + sum S_b Hkv workgroups, and of sequences with several shares
// at most 2 target, each of which leaves a partial state.
#pragma once

#include "st_cache.h"

namespace st {

struct CacheItem {
  int b, hk, tile, share;    // b < 0: none
  int shares, tiles;         // of the sequence
  int first_state, state;    // of the sequence and of this item; only with several shares
};

struct SeqSpan {
  SeqRows r;                 // n: at most max_rows
  int len;
  int64_t pos;               // of the first row
};
__device__ __forceinline__ SeqSpan seq_span(const CacheAttnArgs& a, int b) {
  SeqSpan y;
  y.r = seq_rows(a.starts, b, a.T);
  y.len = seq_len(a.c, b);
  y.pos = a.q_first ? a.q_first[b] : (int64_t)a.c.lens[b] - y.r.n;
  y.r.n = min(y.r.n, a.max_rows);
  return y;
}
// The tokens [lo, hi) that row i of a sequence sees (empty: lo >= hi)
struct RowSpan {
  int lo, hi;
};
__device__ __forceinline__ int to_token(int64_t p, int len) { return (int)min(max(p, (int64_t)0), (int64_t)len); }
__device__ __forceinline__ RowSpan row_span(const CacheAttnArgs& a, const SeqSpan& s, int i) {
  const int64_t p = s.pos + i;
  RowSpan y;
  y.lo = a.window > 0 ? to_token(p - a.window + 1, s.len) : 0;
  y.hi = a.causal ? to_token(p + 1, s.len) : s.len;
  return y;
}

template <typename T>
__device__ __forceinline__ T wave_scan(T x) {        // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

struct PlanRoom {
  int64_t sums[8];
  CacheItem item;
};
// 256 threads; room: LDS
template <int ROWS, int KEYS>
__device__ __forceinline__ CacheItem find_item(const CacheAttnArgs& a, PlanRoom* room) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = a.Hq / a.c.Hkv;
  auto work = [&](int b, int& S, int& L) {
    S = L = 0;
    if (b >= a.c.B) return;
    const SeqSpan s = seq_span(a, b);
    const int M = s.r.n * G;
    if (M <= a.plan.rows_from || M > a.plan.rows_to) return;
    S = (M + ROWS - 1) / ROWS;
    const RowSpan first = row_span(a, s, 0), last = row_span(a, s, s.r.n - 1);
    L = max((last.hi + KEYS - 1) / KEYS - first.lo / KEYS, 0);
  };
  int S0, L0;
  work(tid, S0, L0);
  int64_t sum = (int64_t)S0 * L0;
  for (int b = tid + 256; b < a.c.B; b += 256) {
    int S, L;
    work(b, S, L);
    sum += (int64_t)S * L;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) room->sums[wave] = sum;
  if (tid == 0) room->item.b = -1;
  __syncthreads();
  const int64_t all = (room->sums[0] + room->sums[1] + room->sums[2] + room->sums[3]) * a.c.Hkv;
  const int c = (int)min(max((all + a.plan.target - 1) / a.plan.target, (int64_t)a.plan.least), (int64_t)1 << 30);
  const int64_t me = blockIdx.x;
  int64_t items_before = 0, states_before = 0;
  for (int b0 = 0; b0 < a.c.B; b0 += 256) {
    if (b0 > 0) work(b0 + tid, S0, L0);
    const int shares = max((L0 + c - 1) / c, 1);
    const int64_t n = (int64_t)S0 * shares * a.c.Hkv, m = shares > 1 ? n : 0;
    int64_t x = wave_scan(n), y = wave_scan(m);
    __syncthreads();
    if (lane == 63) room->sums[wave] = x, room->sums[4 + wave] = y;
    __syncthreads();
    int64_t nx = 0, ny = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) x += room->sums[w], y += room->sums[4 + w];
      nx += room->sums[w];
      ny += room->sums[4 + w];
    }
    x += items_before - n;
    y += states_before - m;
    if (me >= x && me < x + n) {
      const int at = (int)(me - x), rest = at / a.c.Hkv;
      CacheItem& t = room->item;
      t.b = b0 + tid;
      t.hk = at - rest * a.c.Hkv;
      t.share = rest / S0;
      t.tile = S0 - 1 - (rest - t.share * S0);       // later rows see more: first
      t.shares = shares;
      t.tiles = S0;
      // (starts that are no starts may name more rows than there are: what there is no room for is left out)
      t.first_state = (int)min(y, (int64_t)1 << 30);
      t.state = (int)min(y + at, (int64_t)1 << 30);
      if (shares > 1 && t.state >= a.plan.states) t.b = -1;
    }
    __syncthreads();
    items_before += nx;
    states_before += ny;
    if (items_before > me) break;
  }
  CacheItem t = room->item;
  t.b = __builtin_amdgcn_readfirstlane(t.b);
  t.hk = __builtin_amdgcn_readfirstlane(t.hk);
  t.tile = __builtin_amdgcn_readfirstlane(t.tile);
  t.share = __builtin_amdgcn_readfirstlane(t.share);
  t.shares = __builtin_amdgcn_readfirstlane(t.shares);
  t.tiles = __builtin_amdgcn_readfirstlane(t.tiles);
  t.first_state = __builtin_amdgcn_readfirstlane(t.first_state);
  t.state = __builtin_amdgcn_readfirstlane(t.state);
  return t;
}

// The key blocks [n0, n1) of a tile's walk, and what its rows see; of a share of it
struct CacheWalk {
  int lo, hi;                // tokens that some row sees
  int all_lo, all_hi;        // tokens that all of them see
  int n0, n1;
};
template <int ROWS, int KEYS>
__device__ __forceinline__ CacheWalk cache_walk(const CacheAttnArgs& a, const SeqSpan& s, const CacheItem& t, int G) {
  const int first = t.tile * ROWS / G, last = min(t.tile * ROWS + ROWS, s.r.n * G) - 1;
  const RowSpan x = row_span(a, s, first), y = row_span(a, s, last / G);
  CacheWalk w;
  w.lo = x.lo;
  w.hi = y.hi;
  w.all_lo = y.lo;
  w.all_hi = x.hi;
  const int b0 = w.lo / KEYS, n = max((w.hi + KEYS - 1) / KEYS - b0, 0);
  w.n0 = b0 + (int)((int64_t)n * t.share / t.shares);
  w.n1 = b0 + (int)((int64_t)n * (t.share + 1) / t.shares);
  return w;
}
// Says where the states of the tile's tokens are
template <int ROWS>
__device__ __forceinline__ void tell_rows(const CacheAttnArgs& a, const SeqSpan& s, const CacheItem& t, int G) {
  if (t.share != 0 || t.hk != 0 || !a.info) return;
  const int i0 = (t.tile * ROWS + G - 1) / G, i1 = min((t.tile * ROWS + ROWS + G - 1) / G, s.r.n);   // their first head is in this tile
  for (int i = i0 + threadIdx.x; i < i1; i += 256) a.info[s.r.first + i] = make_int4(t.first_state, t.shares, t.tiles, i);
}

}  // namespace st
