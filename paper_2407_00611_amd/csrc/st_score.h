// Attention with modified scores, what its kernels share: arguments, the keys a row sees, the score arithmetic.
//
//   u = scale <q, k>                    y = cap tanh(u / cap), or u without a cap
//   s = y - slope |p_q - p_k|           over the keys p_k of the row's interval
//   P = softmax(s), O = P V;  backward  dU = P (dP - Delta) (1 - (y / cap)^2)
//
// The keys that a row sees are one interval [lo, hi) of the chunk, whatever made it: the causal order, a document, a prefix, the
// padding of a batch.  A tile is skipped, taken whole or masked by four numbers of its rows.
//
// Distances are taken from the nearest key that the row sees: |p_q - t| = |x - t| + rest with x = p_q clamped to [lo, hi - 1],
// for every key t of the interval.  x and t are small integers, so the bias inside a chunk far from the row is exact in fp32, and
// slope * rest is a constant of the row, which leaves the softmax alone and is taken off lse at the end.
#pragma once

#include "st_internal.h"
#include "st_mfma.h"

namespace st {

struct ScoreArgs {
  Shape s;
  View q, k, v;
  int64_t k_offset;
  float cap;                 // 0: none
  const float* slopes;       // fp32 [Hq], nullable
  const int64_t* spans;      // [B, Sq, 2], nullable
  // forward; a split launch (n_split > 1) writes state y at part_o + y B Sq Hq D, part_lse + y B Hq Sq instead
  float* o;                  // nullable, fp32 [B,Sq,Hq,D]
  float* lse;                // fp32 [B,Hq,Sq]
  void* o_lowp;              // nullable, [B,Sq,Hq,D] in the storage type
  int32_t n_split;
  float *part_o, *part_lse;
  // backward
  View d_o;
  const float* lse_in;       // final
  const float* delta;
  float *dq, *dk, *dv;       // nullable fp32, added to or (assign) overwritten
  void *dq_lowp, *dk_lowp, *dv_lowp;   // nullable, storage type
  int32_t assign;
  // shares of a query tile's keys and of a key tile's rows; with more than one, share y writes part_dq + y B Sq Hq D
  // (part_dk, part_dv + y B Sk Hkv D), and a last launch adds them up in order
  int32_t q_split, kv_split;
  float *part_dq, *part_dk, *part_dv;
  // bf16, made by launch_score_rows, [B, Hkv, ceil(Sq G / 32)]: what every run of 32 rows sees (BlockSpan), and the statistics of its
  // rows, kRowStats floats
  int4* blocks;
  float* rows;
};
// of 32 rows: lse less the cap (log2 units, as if the nearest key had no bias; inf: a row without gradients), minus Delta, the keys it sees and
// the nearest of them, slope (log2 units)
constexpr int kRowStats = 8 * 32;
enum { kRowLse = 0, kRowDelta = 1, kRowLo = 2, kRowHi = 3, kRowX = 4, kRowSlope = 5 };

constexpr float kScoreLog2e = 1.4426950408889634f;
constexpr float kScoreLn2 = 0.6931471805599453f;

hipError_t launch_mask_spans(const Shape& s, const int64_t* bounds, int32_t n_docs, const int64_t* prefix, int64_t* spans, hipStream_t stream);
hipError_t launch_score_fwd_bf16(const ScoreArgs& a, hipStream_t stream);
hipError_t launch_score_fwd_f32(const ScoreArgs& a, hipStream_t stream);
hipError_t launch_score_combine(const ScoreArgs& a, int bf16, hipStream_t stream);
hipError_t launch_score_rows(const ScoreArgs& a, hipStream_t stream);
hipError_t launch_score_bwd_bf16(const ScoreArgs& a, hipStream_t stream);
hipError_t launch_score_bwd_f32(const ScoreArgs& a, hipStream_t stream);
hipError_t launch_score_add_parts(const ScoreArgs& a, int bf16, hipStream_t stream);

// rows of the kernels' tiles: 32 in a wavefront, packed over the query heads of a KV head (row R is token R / G, head R % G of the
// group), so that a tile of keys is read once for all of them and a single token fills the tile with its heads
constexpr int kScoreRows = 128;      // bf16: rows of a query tile's workgroup
constexpr int kScoreKeys = 128;      // bf16: keys of a key tile's workgroup

constexpr int score_f32_halves(int D) { return D > 128 ? 2 : 1; }   // fp32: workgroups that share a key tile, by columns

constexpr int64_t kScoreGridMost = 1 << 22;   // workgroups of a launch: a dimension of a grid holds fewer than 2^32 threads

// shares of each of `jobs` workgroups that fill `slots` places, where a workgroup walks `steps` tiles
int score_split(int64_t jobs, int64_t slots, int64_t steps, int64_t least_steps, int most);

// ---- device side

// The keys [lo, hi) of the chunk that token i sees (empty: lo = hi = 0), and the nearest of them to the token
struct RowView {
  int lo, hi, x;
  float rest;                // distance from the token to x
};
__device__ __forceinline__ int key_clamp(int64_t p, int64_t k0, int Sk) {
  if (p <= k0) return 0;
  const uint64_t d = (uint64_t)p - (uint64_t)k0;
  return d < (uint64_t)Sk ? (int)d : Sk;
}
__device__ __forceinline__ RowView row_view(const ScoreArgs& a, int b, int i) {
  const Shape& s = a.s;
  const int64_t pos = q_pos(s, i);
  RowView v;
  v.lo = 0;
  v.hi = s.Sk;
  if (a.spans) {
    const longlong2 w = *reinterpret_cast<const longlong2*>(a.spans + 2 * ((int64_t)b * s.Sq + i));
    v.lo = key_clamp(w.x, a.k_offset, s.Sk);
    v.hi = key_clamp(w.y, a.k_offset, s.Sk);
  }
  if (s.causal) v.hi = pos < a.k_offset ? 0 : min(v.hi, key_clamp(pos + 1, a.k_offset, s.Sk));
  if (v.lo >= v.hi) v.lo = v.hi = 0;
  const int64_t last = a.k_offset + v.hi - 1, first = a.k_offset + v.lo;
  const int64_t near = pos < first ? first : pos > last ? last : pos;
  v.x = (int)(near - a.k_offset);
  v.rest = (float)(pos > near ? pos - near : near - pos);
  return v;
}

template <typename F>
__device__ __forceinline__ int wave_fold(int x, F f) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = f(x, __shfl_xor(x, d));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_min(int x) { return wave_fold(x, [](int p, int q) { return min(p, q); }); }
__device__ __forceinline__ int wave_max(int x) { return wave_fold(x, [](int p, int q) { return max(p, q); }); }

// What a set of rows sees: some row the keys in [lo, hi) at most (empty: lo >= hi), all rows those in [all_lo, all_hi)
struct BlockSpan {
  int lo, hi, all_lo, all_hi;
};
__device__ __forceinline__ BlockSpan span_of(const RowView& v) {
  const bool none = v.lo >= v.hi;
  return BlockSpan{none ? 0x7fffffff : v.lo, none ? 0 : v.hi, v.lo, v.hi};
}
__device__ __forceinline__ BlockSpan span_join(const BlockSpan& p, const BlockSpan& q) {
  return BlockSpan{min(p.lo, q.lo), max(p.hi, q.hi), max(p.all_lo, q.all_lo), min(p.all_hi, q.all_hi)};
}

// scores, from the products <q, k>: in log2 units without the row's constants
struct ScoreConst {
  float c;                   // scale log2 e; with a cap 2 scale log2 e / cap, the exponent of tanh
  float k1;                  // cap log2 e
};
__device__ __forceinline__ ScoreConst score_const(const ScoreArgs& a) {
  ScoreConst k;
  k.c = a.cap > 0.f ? 2.f * kScoreLog2e * (a.s.scale / a.cap) : a.s.scale * kScoreLog2e;
  k.k1 = a.cap * kScoreLog2e;
  return k;
}
// r = 1 / (1 + e^(2 u / cap)): tanh(u / cap) = 1 - 2 r and 1 - tanh^2 = 4 r (1 - r), for any u.  Both functions are the hardware's, r some
// 2^-24 off, and the score 2 cap times that: caps are at most kCapMost.
constexpr float kCapMost = 1024.f;
__device__ __forceinline__ float cap_r(float u, float c) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * c));
}

// A lane's operand reads from a swizzled LDS tile (swz of st_mfma.h): three addresses in registers, the rest of a fragment's place
// is an exclusive or with a constant and the instruction's own offset.  (Left to the compiler, every fragment's address of a loop
// has a register of its own, some sixty that the accumulators need.)
template <int D>
struct LaneReads {
  uint32_t nat, lo, hi;
  __device__ __forceinline__ explicit LaneReads(int lane) {
    const int g = lane >> 5, r = lane & 31, s16 = lane & 15, half = (lane >> 4) & 1;
    nat = (uint32_t)swz<D>(r, g);
    const int row = 4 * g + (s16 >> 2);
    lo = (uint32_t)(swz<D>(row, 2 * half + ((s16 & 3) >> 1)) + (s16 & 1) * 8);
    hi = (lo + 8 * D * 2) ^ 32;                        // eight rows on: the swizzle flips the second chunk bit
  }
  // as lds_frag: row row0 + r, elements 16 ks + 8 g .. + 7
  __device__ __forceinline__ bf16x8 frag(uint32_t tile, int row0, int ks) const {
    return lds_read_b128((const ST_LDS char*)(uintptr_t)((tile + nat) ^ (uint32_t)(32 * ks)) + row0 * D * 2);
  }
  // as lds_frag_tr: column 32 db + r at rows row0 + 4 g .. + 3 and row0 + 8 + 4 g .. + 3
  __device__ __forceinline__ bf16x8 frag_tr(uint32_t tile, int row0, int db) const {
    const u32x2 x = lds_read_tr16((const ST_LDS char*)(uintptr_t)((tile + lo) ^ (uint32_t)(64 * db)) + row0 * D * 2);
    const u32x2 y = lds_read_tr16((const ST_LDS char*)(uintptr_t)((tile + hi) ^ (uint32_t)(64 * db)) + row0 * D * 2);
    return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
  }
};

// What a lane holds of a row's scores against a block of keys until their exponentials are taken, so that each costs as few
// instructions as can be: with a cap r of cap_r, which falls as the score rises; otherwise the score over c, the bias included.
template <bool CAP, bool BIAS>
struct ScoreTile {
  float c, k1, slope, x;     // x: the row's nearest key, from the lane's first key of the block on
  __device__ __forceinline__ ScoreTile(const ScoreConst& k, float slope2, int x0) : c(k.c), k1(k.k1), slope(CAP ? slope2 : slope2 / k.c), x((float)x0) {}
  // with both, the exponent itself.  raw: any tile; raw_side: all its keys on one side of the row, and the bias but for that of the
  // lane's first key
  __device__ __forceinline__ float raw(float u, int key) const {
    if (CAP && !BIAS) return cap_r(u, c);
    const float y = CAP ? fmaf(-2.f * k1, cap_r(u, c), k1) : u;
    return BIAS ? fmaf(-slope, fabsf(x - (float)key), y) : y;
  }
  __device__ __forceinline__ float raw_side(float u, int key, float side) const {
    if (CAP && !BIAS) return cap_r(u, c);
    const float y = CAP ? fmaf(-2.f * k1, cap_r(u, c), k1) : u;
    return BIAS ? fmaf(side, (float)key, y) : y;
  }
  __device__ __forceinline__ float lowest() const { return CAP && !BIAS ? INFINITY : -INFINITY; }
  __device__ __forceinline__ float higher(float a, float b) const { return CAP && !BIAS ? fminf(a, b) : fmaxf(a, b); }
  // log2 units, less m
  __device__ __forceinline__ float exponent(float y, float m) const {
    if (CAP) return BIAS ? y - m : fmaf(-2.f * k1, y, k1 - m);
    return fmaf(y, c, -m);
  }
};

// bf16 values with the infinities and NaN among them made the largest finite value of their sign.  As signed integers those with a
// plus are the highest, as unsigned ones those with a minus: two packed instructions for a pair.
__device__ __forceinline__ bf16x8 finite_bf16(bf16x8 x) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  const s16x8 y = __builtin_elementwise_min(__builtin_bit_cast(s16x8, x), (s16x8)(short)0x7f7f);
  return __builtin_bit_cast(bf16x8, __builtin_elementwise_min(__builtin_bit_cast(u16x8, y), (u16x8)(unsigned short)0xff7f));
}

}  // namespace st
