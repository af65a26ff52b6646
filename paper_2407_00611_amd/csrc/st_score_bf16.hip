// bf16 attention with modified scores (st_score.h), head size 128 or 64: forward, dQ and dK/dV on v_mfma_f32_32x32x16_bf16.
//
// Products <q, k> of the stored values are exact in the matrix unit's fp32 sums; scale, cap, bias and softmax are fp32, Q itself is
// not rounded again.  P and dU are rounded to bf16 for the second contractions, relative 2^-9 at most each, as those of the other
// bf16 kernels here; sums and statistics stay fp32.
//
// Rows whose tile a mask edge crosses: the matrix unit multiplies what a row does not see by zero, and 0 * inf is NaN.  In such a
// tile the operand's infinities and NaN are set to zero.  The forward adds them to the rows that do see them once O is stored; in
// the backward, a row that sees a key with such values has NaN in P or dU already, and so has its contribution.
#include <algorithm>

#include "st_score.h"

namespace st {
namespace {

constexpr int kBN = 64;              // keys of a streamed tile
constexpr float kGap = 8.f;          // log2 units a tile's maximum may exceed the row's exponent reference by

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Tiles of 64 keys that a query tile's workgroup walks: those its rows' hull touches, its share of them
struct Walk {
  int t0, t1;
};
__device__ __forceinline__ Walk walk_of(int lo, int hi, int n_split, int share) {
  if (lo >= hi) return Walk{0, 0};
  const int first = lo / kBN, n = (hi + kBN - 1) / kBN - first;
  const int64_t y = share;
  return Walk{first + (int)(n * y / n_split), first + (int)(n * (y + 1) / n_split)};
}

// Block id -> (row tile, KV head, batch entry).  Every XCD has a contiguous range of the (KV head, batch entry) pairs, whose keys and
// values stay in its L2; under a causal mask the later tiles, which see more, come first.
__device__ __forceinline__ void tile_block(const ScoreArgs& a, int n_qt, int& qt, int& hk, int& b) {
  int hb;
  qtile_block(blockIdx.x, gridDim.x, n_qt, a.s.causal, qt, hb);
  hk = uniform(hb % a.s.Hkv);
  b = uniform(hb / a.s.Hkv);
  qt = uniform(qt);
}

// =============================================================================================
// forward: 128 rows per workgroup, 32 per wavefront; lane = row (C layout column)
// =============================================================================================
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void score_fwd_kernel(const ScoreArgs a) {
  constexpr int KB = kBN / 32, KS = D / 16, DB = D / 32;
  constexpr int kTile = kBN * D * 2;
  __shared__ __attribute__((aligned(1024))) char smem_raw[4 * kTile];   // 2 stages x (K, V)
  __shared__ int hull[8];
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G;
  const int n_qt = (M + kScoreRows - 1) / kScoreRows;
  int qt, hk, b;
  tile_block(a, n_qt, qt, hk, b);

  const int R = qt * kScoreRows + wave * 32 + r, row = min(R, M - 1);
  const int i = row / G, h = hk * G + row % G;
  const RowView see = row_view(a, b, i);
  const BlockSpan own = span_of(see);
  BlockSpan w;                                         // of the wavefront's rows
  w.lo = wave_min(own.lo); w.hi = wave_max(own.hi); w.all_lo = wave_max(own.all_lo); w.all_hi = wave_min(own.all_hi);
  if (lane == 0) {
    hull[wave] = w.lo;
    hull[4 + wave] = w.hi;
  }
  // Q fragments (B operand): row r, elements 16 ks + 8 g .. + 7
  bf16x8 qf[KS];
  const char* qrow = (const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)i * a.q.ss + (int64_t)h * a.q.sh) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + (16 * ks + 8 * g) * 2);
  const ScoreConst k = score_const(a);
  const float slope2 = BIAS ? a.slopes[h] * kScoreLog2e : 0.f;
  __syncthreads();
  const int lo = uniform(min(min(hull[0], hull[1]), min(hull[2], hull[3]))), hi = uniform(max(max(hull[4], hull[5]), max(hull[6], hull[7])));
  const Walk walk = walk_of(lo, hi, a.n_split, blockIdx.y);

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  uint32_t bad = 0;

  const char* kb_ = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh) * 2;
  const char* vb_ = (const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh) * 2;
  auto issue_load = [&](int t, int stage) {
    stage_dma<D, kBN>(kb_, a.k.ss, t * kBN, s.Sk, smem + stage * 2 * kTile, tid);
    stage_dma<D, kBN>(vb_, a.v.ss, t * kBN, s.Sk, smem + stage * 2 * kTile + kTile, tid);
  };
  int buf = 0;
  if (walk.t0 < walk.t1) issue_load(walk.t0, 0);
  __syncthreads();
  for (int t = walk.t0; t < walk.t1; ++t) {
    if (t + 1 < walk.t1) issue_load(t + 1, buf ^ 1);
    const int key0 = t * kBN;
    if (w.lo < key0 + kBN && w.hi > key0) {            // some row of this wavefront sees some key of the tile
      const bool masked = w.all_lo > key0 || w.all_hi < key0 + kBN;
      const ST_LDS char* ktile = smem + buf * 2 * kTile;
      const ST_LDS char* vtile = ktile + kTile;
      f32x16 sc[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[kb][v] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) sc[kb] = mfma32(lds_frag<D>(ktile, 32 * kb, ks, lane), qf[ks], sc[kb]);
      const float x = (float)(see.x - key0 - 4 * g);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float e = CAP ? fmaf(-2.f * k.k1, cap_r(sc[kb][v], k.c), k.k1) : BIAS ? sc[kb][v] * k.c : sc[kb][v];
          if (BIAS) e = fmaf(-slope2, fabsf(x - (float)(32 * kb + 8 * (v / 4) + v % 4)), e);
          sc[kb][v] = e;
        }
      constexpr bool kRaw = !CAP && !BIAS;             // the exponents are c times what sc holds
      if (masked) {
        const int l0 = see.lo - key0 - 4 * g, h0 = see.hi - key0 - 4 * g;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = 32 * kb + 8 * (v / 4) + v % 4;
            if (key < l0 || key >= h0) sc[kb][v] = -INFINITY;
          }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sc[kb][v]);
      mx = xhalf_max(mx);
      if (kRaw) mx *= k.c;
      // The reference of the exponents moves only when a tile exceeds it by more than kGap, which is rare after the first tiles
      const bool jump = mx - m_run > kGap || (m_run == -INFINITY && mx != -INFINITY);
      if (__builtin_expect(__any(jump), 0)) {
        const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= alpha;
        m_run = m_new;
#pragma unroll
        for (int db = 0; db < DB; ++db) scale_in_place(acc[db], alpha);
      }
      const float mc = m_run == -INFINITY ? 0.f : m_run;
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float p = __builtin_amdgcn_exp2f(kRaw ? fmaf(sc[kb][v], k.c, -mc) : sc[kb][v] - mc);
          sc[kb][v] = p;
          sum += p;
        }
      l_run += sum;
      auto contract = [&](auto scrub) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf16x8 pf = pack_c_as_b(sc[kb], m);
#pragma unroll
            for (int db = 0; db < DB; ++db)
              acc[db] = mfma32(scrub(lds_frag_tr<D>(vtile, 32 * kb + 16 * m, 32 * db, lane)), pf, acc[db]);
          }
      };
      if (masked) contract([&](bf16x8 f) { return scrub_bf16(f, bad); });
      else contract([](bf16x8 f) { return f; });
    }
    __syncthreads();
    buf ^= 1;
  }

  // ---- O = acc / l, lse = m ln 2 + ln l, less the bias of the nearest key
  const float l = xhalf_sum(l_run);
  const float inv = l != 0.f ? 1.f / l : 0.f;
  const int64_t n_o = (int64_t)s.B * s.Sq * s.Hq;
  const bool part = a.n_split > 1;
  float* o = part ? a.part_o + blockIdx.y * n_o * D : a.o;
  uint16_t* olow = part ? nullptr : (uint16_t*)a.o_lowp;
  const int64_t orow = (((int64_t)b * s.Sq + i) * s.Hq + h) * D;
  const bool any_bad = __any(bad != 0);
  if (R < M) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int d = 32 * db + 8 * q4 + 4 * g;
        const float4 y = make_float4(acc[db][4 * q4] * inv, acc[db][4 * q4 + 1] * inv, acc[db][4 * q4 + 2] * inv, acc[db][4 * q4 + 3] * inv);
        if (o) *reinterpret_cast<float4*>(o + orow + d) = y;
        if (olow) *reinterpret_cast<uint2*>(olow + orow + d) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
      }
    if (g == 0) {
      float x = l != 0.f ? m_run * kScoreLn2 + logf(l) : -INFINITY;
      if (BIAS) x = fmaf(-a.slopes[h], see.rest, x);
      (part ? a.part_lse + blockIdx.y * n_o : a.lse)[((int64_t)b * s.Hq + h) * s.Sq + i] = x;
    }
    if (any_bad)
      // what the masked tiles of this wavefront left out: V[t][d] of the keys that this row sees
      for (int t = walk.t0; t < walk.t1; ++t) {
        if (!(w.all_lo > t * kBN || w.all_hi < (t + 1) * kBN)) continue;
        for (int key = max(see.lo, t * kBN); key < min(see.hi, (t + 1) * kBN); ++key)
          for (int d = 4 * g; d < D; d += 8)
            for (int e = 0; e < 4; ++e) {
              const float y = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(vb_ + ((int64_t)key * a.v.ss + d + e) * 2) << 16);
              if (fabsf(y) <= 3.402823466e38f) continue;
              if (o) o[orow + d + e] += y;
              if (olow) {
                const float z = __uint_as_float((uint32_t)olow[orow + d + e] << 16) + y;
                olow[orow + d + e] = (uint16_t)pack_bf16(z, z);
              }
            }
      }
  }
}

// =============================================================================================
// dQ: as the forward, with dP beside S
// =============================================================================================
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void score_dq_kernel(const ScoreArgs a) {
  constexpr int KB = kBN / 32, KS = D / 16, DB = D / 32;
  constexpr int kTile = kBN * D * 2;
  __shared__ __attribute__((aligned(1024))) char smem_raw[4 * kTile];
  __shared__ int hull[8];
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G;
  const int n_qt = (M + kScoreRows - 1) / kScoreRows;
  int qt, hk, b;
  tile_block(a, n_qt, qt, hk, b);

  const int R = qt * kScoreRows + wave * 32 + r, row = min(R, M - 1);
  const int i = row / G, h = hk * G + row % G;
  RowView see = row_view(a, b, i);
  const int64_t stat = ((int64_t)b * s.Hq + h) * s.Sq + i;
  const float slope = BIAS ? a.slopes[h] : 0.f, slope2 = slope * kScoreLog2e;
  const float lse = a.lse_in[stat], dlt = a.delta[stat];
  if (lse == -INFINITY) see.lo = see.hi = 0;           // an empty row
  // the row's constant: s log2 e = e + const with e from the nearest key on
  const float lse2 = (BIAS ? fmaf(slope, see.rest, lse) : lse) * kScoreLog2e;
  const BlockSpan own = span_of(see);
  BlockSpan w;
  w.lo = wave_min(own.lo); w.hi = wave_max(own.hi); w.all_lo = wave_max(own.all_lo); w.all_hi = wave_min(own.all_hi);
  if (lane == 0) {
    hull[wave] = w.lo;
    hull[4 + wave] = w.hi;
  }
  bf16x8 qf[KS], dof[KS];
  const char* qrow = (const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)i * a.q.ss + (int64_t)h * a.q.sh) * 2;
  const char* drow = (const char*)a.d_o.ptr + ((int64_t)b * a.d_o.sb + (int64_t)i * a.d_o.ss + (int64_t)h * a.d_o.sh) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + (16 * ks + 8 * g) * 2);
    dof[ks] = *reinterpret_cast<const bf16x8*>(drow + (16 * ks + 8 * g) * 2);
  }
  const ScoreConst k = score_const(a);
  __syncthreads();
  const int lo = uniform(min(min(hull[0], hull[1]), min(hull[2], hull[3]))), hi = uniform(max(max(hull[4], hull[5]), max(hull[6], hull[7])));
  const Walk walk = walk_of(lo, hi, a.q_split, blockIdx.y);

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  uint32_t bad = 0;
  const char* kb_ = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh) * 2;
  const char* vb_ = (const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh) * 2;
  auto issue_load = [&](int t, int stage) {
    stage_dma<D, kBN>(kb_, a.k.ss, t * kBN, s.Sk, smem + stage * 2 * kTile, tid);
    stage_dma<D, kBN>(vb_, a.v.ss, t * kBN, s.Sk, smem + stage * 2 * kTile + kTile, tid);
  };
  int buf = 0;
  if (walk.t0 < walk.t1) issue_load(walk.t0, 0);
  __syncthreads();
  for (int t = walk.t0; t < walk.t1; ++t) {
    if (t + 1 < walk.t1) issue_load(t + 1, buf ^ 1);
    const int key0 = t * kBN;
    if (w.lo < key0 + kBN && w.hi > key0) {
      const bool masked = w.all_lo > key0 || w.all_hi < key0 + kBN;
      const ST_LDS char* ktile = smem + buf * 2 * kTile;
      const ST_LDS char* vtile = ktile + kTile;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        f32x16 sc, dp;
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[v] = dp[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          sc = mfma32(lds_frag<D>(ktile, 32 * kb, ks, lane), qf[ks], sc);
          dp = mfma32(lds_frag<D>(vtile, 32 * kb, ks, lane), dof[ks], dp);
        }
        const float x = (float)(see.x - key0 - 32 * kb - 4 * g);
        const int l0 = see.lo - key0 - 32 * kb - 4 * g, h0 = see.hi - key0 - 32 * kb - 4 * g;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = 8 * (v / 4) + v % 4;
          float e, f = 1.f;
          if (CAP) {
            const float rr = cap_r(sc[v], k.c);
            e = fmaf(-2.f * k.k1, rr, k.k1 - lse2);
            f = 4.f * rr * (1.f - rr);
          } else {
            e = fmaf(sc[v], k.c, -lse2);
          }
          if (BIAS) e = fmaf(-slope2, fabsf(x - (float)key), e);
          float ds = __builtin_amdgcn_exp2f(e) * (dp[v] - dlt);
          if (CAP) ds *= f;
          if (masked) ds = key >= l0 && key < h0 ? ds : 0.f;
          sc[v] = ds;
        }
        auto contract = [&](auto scrub) {
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf16x8 dsf = pack_c_as_b(sc, m);
#pragma unroll
            for (int db = 0; db < DB; ++db)
              acc[db] = mfma32(scrub(lds_frag_tr<D>(ktile, 32 * kb + 16 * m, 32 * db, lane)), dsf, acc[db]);
          }
        };
        if (masked) contract([&](bf16x8 f) { return scrub_bf16(f, bad); });
        else contract([](bf16x8 f) { return f; });
      }
    }
    __syncthreads();
    buf ^= 1;
  }
  if (R >= M) return;
  const int64_t orow = (((int64_t)b * s.Sq + i) * s.Hq + h) * D;
  const bool part = a.q_split > 1;
  float* out = part ? a.part_dq + blockIdx.y * ((int64_t)s.B * s.Sq * s.Hq * D) : a.dq;
  uint16_t* low = part ? nullptr : (uint16_t*)a.dq_lowp;
  const bool add = !part && !a.assign;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int d = 32 * db + 8 * q4 + 4 * g;
      float4 y = make_float4(acc[db][4 * q4] * s.scale, acc[db][4 * q4 + 1] * s.scale, acc[db][4 * q4 + 2] * s.scale, acc[db][4 * q4 + 3] * s.scale);
      if (add) {
        const float4 z = *reinterpret_cast<const float4*>(out + orow + d);
        y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
      }
      if (out) *reinterpret_cast<float4*>(out + orow + d) = y;
      if (low) *reinterpret_cast<uint2*>(low + orow + d) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    }
}

// =============================================================================================
// dK, dV: 128 keys of one KV head per workgroup, 32 per wavefront, K and V fragments resident; the group's rows stream by in blocks
// of 32.  lane = key (C layout column), registers = 16 rows
// =============================================================================================
constexpr int kBlockList = 1024;     // row blocks that a workgroup looks through at a time

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void score_dkv_kernel(const ScoreArgs a) {
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int kTile = 32 * D * 2, kStats = 6 * 32 * 4;
  constexpr int kStage = 2 * kTile + kStats;           // Q, dO, and of each row lse, Delta, lo, hi, x, slope
  __shared__ __attribute__((aligned(16))) char smem_raw[2 * kStage];
  __shared__ int4 list[kBlockList];                    // block, hull of its rows, 1: every row sees every key of the workgroup
  __shared__ int count[5];
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G, n_blk = (M + 31) / 32;
  const int n_kt = (s.Sk + kScoreKeys - 1) / kScoreKeys;
  const int logical = xcd_logical_block(blockIdx.x, gridDim.x);
  const int kt = uniform(logical % n_kt), bh = logical / n_kt;
  const int b = uniform(bh % s.B), hk = uniform(bh / s.B);
  const int key0 = kt * kScoreKeys, key_end = min(key0 + kScoreKeys, s.Sk);
  const int wkey0 = key0 + wave * 32, wkey_end = min(wkey0 + 32, s.Sk);
  const int key = wkey0 + r, key_row = min(key, s.Sk - 1);
  const uint32_t inv_g = G > 1 ? 0xffffffffu / (uint32_t)G + 1 : 0;      // x / G = x inv_g / 2^32 for the small x below

  const char* kp = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh + (int64_t)key_row * a.k.ss) * 2;
  const char* vp = (const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh + (int64_t)key_row * a.v.ss) * 2;
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = *reinterpret_cast<const bf16x8*>(kp + (16 * ks + 8 * g) * 2);
    vf[ks] = *reinterpret_cast<const bf16x8*>(vp + (16 * ks + 8 * g) * 2);
  }
  const ScoreConst k = score_const(a);
  f32x16 acc_k[DB], acc_v[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc_k[db][v] = acc_v[db][v] = 0.f;
  uint32_t bad = 0;

  // what the rows of block j see; without spans a row sees a run from the chunk's first key on, longer from row to row
  auto block_span = [&](int j) {
    if (a.blocks) {
      const int4 x = a.blocks[(int64_t)b * n_blk + j];
      return BlockSpan{x.x, x.y, x.z, x.w};
    }
    if (!s.causal) return BlockSpan{0, s.Sk, 0, s.Sk};
    auto seen = [&](int i) {
      const int64_t pos = q_pos(s, i);
      return pos < a.k_offset ? 0 : key_clamp(pos + 1, a.k_offset, s.Sk);
    };
    const int first = seen(32 * j / G), last = seen(min(32 * j + 31, M - 1) / G);
    return BlockSpan{last > 0 ? 0 : 0x7fffffff, last, 0, first};
  };

  u32x4 rq[D / 64], rd[D / 64];                        // a block on its way: 32 rows x D / 8 pieces over 256 threads
  float st_lse = 0.f, st_dlt = 0.f, st_x = 0.f, st_slope = 0.f;
  int st_lo = 0, st_hi = 0;
  auto row_at = [&](int j, int x, int& i, int& h) {    // row x of block j
    const int base = 32 * j / G;                       // uniform
    const uint32_t n = (uint32_t)(32 * j - base * G + x), q = G > 1 ? __umulhi(n, inv_g) : n;
    i = base + (int)q;
    h = hk * G + (int)(n - q * (uint32_t)G);
  };
  auto load_block = [&](int j) {
    j = uniform(j);
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      const int p = tid + 256 * u;
      int i, h;
      row_at(j, min(p / (D / 8), M - 1 - 32 * j), i, h);
      rq[u] = *reinterpret_cast<const u32x4*>((const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)i * a.q.ss + (int64_t)h * a.q.sh + p % (D / 8) * 8) * 2);
      rd[u] = *reinterpret_cast<const u32x4*>((const char*)a.d_o.ptr + ((int64_t)b * a.d_o.sb + (int64_t)i * a.d_o.ss + (int64_t)h * a.d_o.sh + p % (D / 8) * 8) * 2);
    }
    if (tid < 32) {
      int i, h;
      const int x = min(tid, M - 1 - 32 * j);
      row_at(j, x, i, h);
      const RowView see = row_view(a, b, i);
      const int64_t stat = ((int64_t)b * s.Hq + h) * s.Sq + i;
      const float lse = a.lse_in[stat];
      st_slope = BIAS ? a.slopes[h] : 0.f;
      const bool none = x < tid || lse == -INFINITY;   // a row that does not exist, or an empty one: P = 0
      st_lse = none ? INFINITY : (BIAS ? fmaf(st_slope, see.rest, lse) : lse) * kScoreLog2e;
      st_slope *= kScoreLog2e;
      st_dlt = a.delta[stat];
      st_lo = none ? 0 : see.lo;
      st_hi = none ? 0 : see.hi;
      st_x = (float)see.x;
    }
  };
  auto store_block = [&](int stage) {
    ST_LDS char* p0 = smem + stage * kStage;
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      const int p = tid + 256 * u;
      *reinterpret_cast<ST_LDS u32x4*>(p0 + swz<D>(p / (D / 8), p % (D / 8))) = rq[u];
      *reinterpret_cast<ST_LDS u32x4*>(p0 + kTile + swz<D>(p / (D / 8), p % (D / 8))) = rd[u];
    }
    if (tid < 32) {
      ST_LDS float* f = reinterpret_cast<ST_LDS float*>(p0 + 2 * kTile) + tid;
      f[0] = st_lse;
      f[32] = st_dlt;
      f[64] = __int_as_float(st_lo);
      f[96] = __int_as_float(st_hi);
      f[128] = st_x;
      f[160] = st_slope;
    }
  };

  // the blocks of this share: every kv_split-th, so that shares of a mask's edge and of its inside are alike
  const int n_share = a.kv_split, share = blockIdx.y, mine = (n_blk - share + n_share - 1) / n_share;
  for (int at = 0; at < mine; at += kBlockList) {
    // ---- the visible ones among the next blocks, in order
    int total = 0;
    for (int c0 = 0; c0 < kBlockList; c0 += 256) {
      const int x = at + c0 + tid, j = share + x * n_share;
      BlockSpan y{0x7fffffff, 0, 0, 0};
      if (x < mine) y = block_span(j);
      const bool seen = y.lo < key_end && y.hi > key0;
      const uint64_t votes = __ballot(seen);
      if (lane == 0) count[wave] = __popcll(votes);
      __syncthreads();
      int before = total;
      for (int x2 = 0; x2 < wave; ++x2) before += count[x2];
      if (seen) list[before + __popcll(votes & (((uint64_t)1 << lane) - 1))] =
          make_int4(j, y.lo, y.hi, y.all_lo <= key0 && y.all_hi >= key_end && 32 * j + 32 <= M ? 1 : 0);
      total += count[0] + count[1] + count[2] + count[3];
      __syncthreads();
    }
    total = uniform(total);
    if (total == 0) continue;
    load_block(list[0].x);
    store_block(0);
    __syncthreads();
    int buf = 0;
    for (int n = 0; n < total; ++n) {
      const int4 blk = list[n];
      const bool more = n + 1 < total;
      if (more) load_block(list[n + 1].x);
      const int blk_lo = uniform(blk.y), blk_hi = uniform(blk.z);
      const bool masked = !uniform(blk.w);
      if (blk_lo < wkey_end && blk_hi > wkey0) {
        const ST_LDS char* qtile = smem + buf * kStage;
        const ST_LDS char* dotile = qtile + kTile;
        const ST_LDS float* stats = reinterpret_cast<const ST_LDS float*>(qtile + 2 * kTile);
        f32x16 sc, dp;
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[v] = dp[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          sc = mfma32(lds_frag<D>(qtile, 0, ks, lane), kf[ks], sc);
          dp = mfma32(lds_frag<D>(dotile, 0, ks, lane), vf[ks], dp);
        }
        const float kx = (float)key;
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const int at4 = 8 * j4 + 4 * g;
          const f32x4 lse2 = *reinterpret_cast<const ST_LDS f32x4*>(stats + at4);
          const f32x4 dlt = *reinterpret_cast<const ST_LDS f32x4*>(stats + 32 + at4);
          f32x4 x = {}, slope2 = {};
          if (BIAS) {
            x = *reinterpret_cast<const ST_LDS f32x4*>(stats + 128 + at4);
            slope2 = *reinterpret_cast<const ST_LDS f32x4*>(stats + 160 + at4);
          }
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            const int v = 4 * j4 + e4;
            float e, f = 1.f;
            if (CAP) {
              const float rr = cap_r(sc[v], k.c);
              e = fmaf(-2.f * k.k1, rr, k.k1) - lse2[e4];
              f = 4.f * rr * (1.f - rr);
            } else {
              e = fmaf(sc[v], k.c, -lse2[e4]);
            }
            if (BIAS) e = fmaf(-slope2[e4], fabsf(x[e4] - kx), e);
            const float p = __builtin_amdgcn_exp2f(e);
            float ds = p * (dp[v] - dlt[e4]);
            if (CAP) ds *= f;
            sc[v] = p;
            dp[v] = ds;
          }
        }
        auto contract = [&](auto scrub) {
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf16x8 pf = pack_c_as_b(sc, m), dsf = pack_c_as_b(dp, m);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              acc_v[db] = mfma32(scrub(lds_frag_tr<D>(dotile, 16 * m, 32 * db, lane)), pf, acc_v[db]);
              acc_k[db] = mfma32(scrub(lds_frag_tr<D>(qtile, 16 * m, 32 * db, lane)), dsf, acc_k[db]);
            }
          }
        };
        if (masked) {
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int row = 8 * (v / 4) + 4 * g + v % 4;
            const int lo = __float_as_int(stats[64 + row]), hi = __float_as_int(stats[96 + row]);
            const bool see = key >= lo && key < hi;
            sc[v] = see ? fmaf(0.f, dp[v], sc[v]) : 0.f;   // (a row whose dO is not finite: NaN, as the scrubbed dO no longer says it)
            dp[v] = see ? dp[v] : 0.f;
          }
          contract([&](bf16x8 f) { return scrub_bf16(f, bad); });
        } else {
          contract([](bf16x8 f) { return f; });
        }
      }
      if (more) store_block(buf ^ 1);
      __syncthreads();
      buf ^= 1;
    }
  }

  if (key >= s.Sk) return;
  const int64_t n_kv = (int64_t)s.B * s.Sk * s.Hkv * D, orow = (((int64_t)b * s.Sk + key) * s.Hkv + hk) * D;
  const bool part = n_share > 1, add = !part && !a.assign;
  auto store = [&](const f32x16 (&acc)[DB], float c, float* out, uint16_t* low) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int d = 32 * db + 8 * q4 + 4 * g;
        float4 y = make_float4(acc[db][4 * q4] * c, acc[db][4 * q4 + 1] * c, acc[db][4 * q4 + 2] * c, acc[db][4 * q4 + 3] * c);
        if (add) {
          const float4 z = *reinterpret_cast<const float4*>(out + orow + d);
          y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
        }
        if (out) *reinterpret_cast<float4*>(out + orow + d) = y;
        if (low) *reinterpret_cast<uint2*>(low + orow + d) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
      }
  };
  store(acc_k, s.scale, part ? a.part_dk + share * n_kv : a.dk, part ? nullptr : (uint16_t*)a.dk_lowp);
  store(acc_v, 1.f, part ? a.part_dv + share * n_kv : a.dv, part ? nullptr : (uint16_t*)a.dv_lowp);
}

// f(integral D, cap, bias)
template <typename F>
hipError_t with_score(const ScoreArgs& a, F f) {
  using std::integral_constant;
  auto mods = [&](auto d) {
    constexpr integral_constant<bool, true> yes;
    constexpr integral_constant<bool, false> no;
    if (a.cap > 0.f) return a.slopes ? f(d, yes, yes) : f(d, yes, no);
    return a.slopes ? f(d, no, yes) : f(d, no, no);
  };
  if (a.s.D == 128) return mods(integral_constant<int, 128>());
  if (a.s.D == 64) return mods(integral_constant<int, 64>());
  return hipErrorInvalidValue;
}

int64_t row_tiles(const Shape& s) {
  const int64_t rows = (int64_t)s.Sq * (s.Hq / s.Hkv);
  return (rows + kScoreRows - 1) / kScoreRows * s.Hkv * s.B;
}

}  // namespace

hipError_t launch_score_fwd_bf16(const ScoreArgs& a, hipStream_t stream) {
  const int64_t total = row_tiles(a.s);
  if (total <= 0) return hipSuccess;
  if (total > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("score_fwd_bf16", stream);
  return with_score(a, [&](auto d, auto cap, auto bias) {
    hipLaunchKernelGGL((score_fwd_kernel<decltype(d)::value, decltype(cap)::value, decltype(bias)::value>), dim3((unsigned)total, (unsigned)a.n_split), dim3(256), 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_score_bwd_bf16(const ScoreArgs& a, hipStream_t stream) {
  const int64_t total = row_tiles(a.s), keys = (int64_t)((a.s.Sk + kScoreKeys - 1) / kScoreKeys) * a.s.Hkv * a.s.B;
  if (total > kScoreGridMost || keys > kScoreGridMost) return hipErrorInvalidValue;
  if (keys > 0) {
    ProfScope prof("score_dkv_bf16", stream);
    const hipError_t e = with_score(a, [&](auto d, auto cap, auto bias) {
      hipLaunchKernelGGL((score_dkv_kernel<decltype(d)::value, decltype(cap)::value, decltype(bias)::value>), dim3((unsigned)keys, (unsigned)a.kv_split), dim3(256), 0, stream, a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (total <= 0) return hipSuccess;
  ProfScope prof("score_dq_bf16", stream);
  return with_score(a, [&](auto d, auto cap, auto bias) {
    hipLaunchKernelGGL((score_dq_kernel<decltype(d)::value, decltype(cap)::value, decltype(bias)::value>), dim3((unsigned)total, (unsigned)a.q_split), dim3(256), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace st
