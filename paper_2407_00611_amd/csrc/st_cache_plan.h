// How the attention of a batch of sequences is cut into the workgroups of a launch.  Lengths and rows are in device memory, and differ from
// sequence to sequence by orders of magnitude; a workgroup finds its piece of the work from them by itself.
//
// Sequence b has S_b row tiles, each of which walks about L_b key blocks.  With c key blocks a share, c = sum S_b L_b Hkv / target or the
// least, sequence b is cut into L_b / c shares, rounded: at most target + sum S_b Hkv workgroups, and of sequences with several shares
// at most 4/3 target (x rounded is at most 4/3 x where it is 2 or more), each of which leaves a partial state.
#pragma once

#include "st_cache.h"
#include "st_mfma.h"

namespace st {

// Reference of the exponents of a row that has met no key: the lowest number, so that whatever fp32 holds of a score counts
constexpr float kUnset = -3.402823466e38f;

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
  y.pos = a.q_first ? min(max(a.q_first[b], -((int64_t)1 << 62)), (int64_t)1 << 62) : (int64_t)a.c.lens[b] - y.r.n;
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

// Sums over the wavefront's lanes, by data parallel primitives: inclusive, in a fixed order
template <typename T>
__device__ __forceinline__ T from_lanes_before(T x, T none, int how) {
  const int i = __builtin_bit_cast(int, x), z = __builtin_bit_cast(int, none);
  int y;
  switch (how) {
    case 0: y = __builtin_amdgcn_update_dpp(z, i, 0x111, 0xf, 0xf, false); break;   // row_shr 1, 2, 4, 8
    case 1: y = __builtin_amdgcn_update_dpp(z, i, 0x112, 0xf, 0xf, false); break;
    case 2: y = __builtin_amdgcn_update_dpp(z, i, 0x114, 0xf, 0xf, false); break;
    case 3: y = __builtin_amdgcn_update_dpp(z, i, 0x118, 0xf, 0xf, false); break;
    case 4: y = __builtin_amdgcn_update_dpp(z, i, 0x142, 0xa, 0xf, false); break;   // lane 15 of a row to the next row: rows 1 and 3
    default: y = __builtin_amdgcn_update_dpp(z, i, 0x143, 0xc, 0xf, false);         // lane 31 to the upper half
  }
  return __builtin_bit_cast(T, y);
}
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
#pragma unroll
  for (int d = 0; d < 6; ++d) x += from_lanes_before(x, T(0), d);
  return x;
}
__device__ __forceinline__ float wave_last(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ int wave_last(int x) { return __builtin_amdgcn_readlane(x, 63); }

// Every wavefront for itself, a sequence a lane: no barrier, and one look at the lengths is all the memory that a batch of 64 waits for.  Larger
// batches cost every workgroup two rounds for each 64 sequences (the same 560 MB in 64 sequences 123.5 us, 256 144, 512 171, 4096 2.1 ms).
// The span of the sequence found comes with it.
template <int ROWS, int KEYS>
__device__ __forceinline__ CacheItem find_item(const CacheAttnArgs& a, SeqSpan& span) {
  const int lane = threadIdx.x & 63, G = a.Hq / a.c.Hkv;
  auto work = [&](int b, SeqSpan& s, int& S, int& L) {
    S = L = 0;
    s = SeqSpan{SeqRows{0, 0}, 0, 0};
    if (b >= a.c.B) return;
    s = seq_span(a, b);
    const int M = s.r.n * G;
    if (M <= a.plan.rows_from || M > a.plan.rows_to) return;
    S = (M + ROWS - 1) / ROWS;
    const RowSpan first = row_span(a, s, 0), last = row_span(a, s, s.r.n - 1);
    L = max((last.hi + KEYS - 1) / KEYS - first.lo / KEYS, 0);
  };
  SeqSpan s0;
  int S0, L0;
  work(lane, s0, S0, L0);
  // (fp32 with some room above: the same sum in every wavefront, and shares that are never too many)
  float all = wave_last(wave_scan((float)S0 * (float)L0));
  for (int b = lane + 64; b - lane < a.c.B; b += 64) {
    SeqSpan s;
    int S, L;
    work(b, s, S, L);
    all += wave_last(wave_scan((float)S * (float)L));
  }
  const int c = max((int)fminf(all * (float)a.c.Hkv / (float)a.plan.target * 1.0001f + 1.f, 1e9f), a.plan.least);
  // Sequences of few rows read every key once: the heads of one run of tokens, whose rows lie side by side, go to the workgroups of one XCD at
  // about the same time (64 ragged sequences 127 us, 139 in the order of the numbers).
  int me = blockIdx.x;
  if (ROWS == 16) {
    const int x = me % kDispatchXcds, y = me / kDispatchXcds, z = y / a.c.Hkv;
    me = (z * kDispatchXcds + x) * a.c.Hkv + y - z * a.c.Hkv;
  }
  CacheItem t;
  t.b = -1;
  int items_before = 0, states_before = 0;
  for (int b0 = 0; b0 < a.c.B; b0 += 64) {
    if (b0 > 0) work(b0 + lane, s0, S0, L0);
    const int shares = max((int)(((int64_t)L0 + c / 2) / c), 1);
    // (a launch has at most 2^22 workgroups: what starts that are no starts name beyond that is left out)
    const int n = (int)min((int64_t)S0 * shares * a.c.Hkv, (int64_t)1 << 24), m = shares > 1 ? n : 0;
    const int x = wave_scan(n), y = wave_scan(m);
    const uint64_t mine = __ballot(me - items_before >= x - n && me - items_before < x);
    if (mine) {
      const int l = __ffsll((unsigned long long)mine) - 1;
      auto of = [&](int z) { return __builtin_amdgcn_readlane(z, l); };
      t.b = b0 + l;
      const int at = me - items_before - of(x - n), rest = at / a.c.Hkv;
      t.tiles = of(S0);
      t.shares = of(shares);
      t.hk = at - rest * a.c.Hkv;
      t.share = rest / t.tiles;
      t.tile = t.tiles - 1 - (rest - t.share * t.tiles);   // later rows see more: first
      t.first_state = states_before + of(y - m);
      t.state = t.first_state + at;
      if (t.shares > 1 && (t.state < 0 || t.state >= a.plan.states)) t.b = -1;
      span.r.first = of(s0.r.first);
      span.r.n = of(s0.r.n);
      span.len = of(s0.len);
      span.pos = (int64_t)((uint64_t)(uint32_t)of((int)s0.pos) | (uint64_t)(uint32_t)of((int)(s0.pos >> 32)) << 32);
      return t;
    }
    items_before = (int)min((int64_t)items_before + wave_last(x), (int64_t)1 << 30);
    states_before = (int)min((int64_t)states_before + wave_last(y), (int64_t)1 << 30);
  }
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
  for (int i = i0 + threadIdx.x; i < i1; i += 256) a.info[s.r.first + i] = make_int4((int)(a.plan.base + (int64_t)t.first_state * ROWS), t.shares | ROWS << 16, t.tiles, i);
  if (t.tile != t.tiles - 1) return;                   // rows that are not computed have no states
  for (int i = s.r.n + threadIdx.x, n = seq_rows(a.starts, t.b, a.T).n; i < n; i += 256) a.info[s.r.first + i] = make_int4(0, 0, 0, 0);
}

}  // namespace st
