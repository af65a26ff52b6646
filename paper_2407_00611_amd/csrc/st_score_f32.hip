// fp32 attention with modified scores (st_score.h), any D <= 256 that is a multiple of 8, on v_mfma_f32_32x32x2_f32: the tiles and
// the layout of work of the other fp32 kernels (st_f32_tiles.h).  A query tile is 32 rows of one head, whose keys the wavefronts
// share; a key tile is 32 keys, whose (query head, row tile) pairs they share; every sum has one owner and a fixed order.
//
// Bound by the fp32 matrix instruction where there is work for all SIMDs (16 heads x 2000 rows of 128, causal, forward and backward:
// 1.06 ms), by the chain of one tile where there is not: 8/2 heads x 500 rows of 80 take 88 us, of which a wavefront's one block of
// dK/dV is 18: 13 of products, four of exponentials and tanh.
#include "st_f32_tiles.h"
#include "st_score.h"

namespace st {
namespace {

// score of a product <q, k> without the bias, and the factor of its gradient
template <bool CAP>
__device__ __forceinline__ float score_of(float u, const ScoreArgs& a, float& f) {
  u *= a.s.scale;
  f = 1.f;
  if (!CAP) return u;
  const float t = tanhf(u / a.cap);
  f = 1.f - t * t;
  return a.cap * t;
}

// A piece of a tile that a mask edge crosses, with its infinities and NaN taken as zero; true if it had some.  (Looking at the tile
// once more beforehand was a chain of loads: 8/2 heads x 500 rows of 80, forward and backward, 95 us, 89 so.)
template <int DP, int N>
__device__ __forceinline__ bool make_finite(Piece<N>& f) {
  bool bad = false;
#pragma unroll
  for (int k = 0; k < piece_rows<DP, N>() * (DP / 32); ++k) {
    const bool fine = finite(f.x[k]);
    bad = bad || !fine;
    f.x[k] = fine ? f.x[k] : 0.f;
  }
  return bad;
}

template <int DP, bool FULL, bool CAP>
__global__ __launch_bounds__(waves<DP>() * 64) void score_fwd_f32_kernel(const ScoreArgs a) {
  constexpr int NW = waves<DP>(), DB = DP / 32, N = DP == 128 ? 16 : 32, R = DP < 128 ? 3 : DP == 128 ? 4 : 2;
  constexpr int NR = row_pieces<DP, N>(), NC = col_pieces<DP, N>(), kPieces = NR + NC;
  __shared__ __attribute__((aligned(16))) float qs[kT * lds_stride<DP>()];
  __shared__ float fold[NW / 2 * DB * 16 * 64];
  __shared__ float fold_m[NW / 2 * 64], fold_l[NW / 2 * 64];
  __shared__ int any_dirty;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int n_qt = (s.Sq + kT - 1) / kT;
  int qt, hb;
  qtile_block(blockIdx.x, gridDim.x, n_qt, s.causal, qt, hb);
  const int h = (int)sgpr(hb % s.Hq), b = (int)sgpr(hb / s.Hq), hk = (int)sgpr(h / (s.Hq / s.Hkv));
  const int row0 = (int)sgpr(qt * kT);
  stage_tile<DP>(qs, (const float*)a.q.ptr + b * a.q.sb + h * a.q.sh, a.q.ss, row0, s.Sq, s.D, tid);
  if (tid == 0) any_dirty = 0;
  const int i = min(row0 + r, s.Sq - 1);
  const RowView see = row_view(a, b, i);
  BlockSpan w = span_of(see);
  w.lo = wave_min(w.lo); w.hi = wave_max(w.hi); w.all_lo = wave_max(w.all_lo); w.all_hi = wave_min(w.all_hi);
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  const float *k0 = (const float*)a.k.ptr + b * a.k.sb + hk * a.k.sh, *v0 = (const float*)a.v.ptr + b * a.v.sb + hk * a.v.sh;
  __syncthreads();

  float m = -INFINITY, l = 0.f;
  f32x16 acc[DB];
  zero_acc(acc);
  const int first = w.lo < w.hi ? w.lo / kT : 0, n = w.lo < w.hi ? (w.hi + kT - 1) / kT - first : 0;
  const int t0 = first + (int)((int64_t)n * blockIdx.y / a.n_split), t1 = first + (int)((int64_t)n * (blockIdx.y + 1) / a.n_split);
  for (int t = t0 + wave; t < t1; t += NW) {
    const int key0 = t * kT, limit = min(kT, s.Sk - key0);
    const float *kb = k0 + (int64_t)key0 * a.k.ss, *vb = v0 + (int64_t)key0 * a.v.ss;
    const bool masked = w.all_lo > key0 || w.all_hi < key0 + kT;
    const float* krow = kb + (int64_t)min(r, limit - 1) * a.k.ss;
    Piece<N> f[R];
    auto load = [&](int x) {
      if (x >= kPieces) return;
      if (x < NR) load_rows<DP, FULL>(f[x % R], krow, x, s.D, g);
      else load_cols<DP, FULL>(f[x % R], vb, a.v.ss, limit, x - NR, s.D, r, g);
      __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 p;
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] = 0.f;
#pragma unroll
    for (int x = 0; x < R - 1; ++x) load(x);
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      load(x + R - 1);
      contract_d<DP>(p, f[x % R], qs, x, r, g);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = key0 + c_row(v, g);
      float unused;
      const float e = fmaf(-slope, fabsf((float)(see.x - key)), score_of<CAP>(p[v], a, unused));
      p[v] = key >= see.lo && key < see.hi ? e : -INFINITY;
      mx = fmaxf(mx, p[v]);
    }
    const float m_new = fmaxf(m, xhalf_max(mx));
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = expf(p[v] - m_use);
      sum += p[v];
    }
    const float alpha = expf(m - m_use);
    l = l * alpha + sum;
    m = m_new;
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
    }
    bool bad = false;
#pragma unroll
    for (int x = NR; x < kPieces; ++x) {
      load(x + R - 1);
      if (masked) bad = make_finite<DP>(f[x % R]) || bad;
      contract_rows<DP>(acc, f[x % R], p, x - NR);
    }
    if (bad) any_dirty = 1;
  }
  for (int y = NW / 2; y > 0; y /= 2) {
    if (wave >= y && wave < 2 * y) {
      put_acc(fold + (wave - y) * DB * 16 * 64, acc, lane);
      fold_m[(wave - y) * 64 + lane] = m;
      fold_l[(wave - y) * 64 + lane] = l;
    }
    __syncthreads();
    if (wave < y) {
      const float mo = fold_m[wave * 64 + lane], lo = fold_l[wave * 64 + lane];
      const float mn = fmaxf(m, mo), mu = mn == -INFINITY ? 0.f : mn;
      const float own = expf(m - mu), other = expf(mo - mu);
      add_acc(fold + wave * DB * 16 * 64, acc, own, other, lane);
      l = own * l + other * lo;
      m = mn;
    }
    __syncthreads();
  }
  if (wave != 0 || row0 + r >= s.Sq) return;
  l = xhalf_sum(l);
  const float inv = l != 0.f ? 1.f / l : 0.f;
  const bool part = a.n_split > 1;
  const int64_t n_rows = (int64_t)s.B * s.Sq * s.Hq, at = (((int64_t)b * s.Sq + i) * s.Hq + h) * s.D;
  float* o = part ? a.part_o + blockIdx.y * n_rows * s.D + at : a.o ? a.o + at : nullptr;
  float* ol = !part && a.o_lowp ? (float*)a.o_lowp + at : nullptr;
  if (o == nullptr) {                                        // the storage type is fp32: one output serves as both
    o = ol;
    ol = nullptr;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < DB; ++q) {
      const int d = block_column<DB>(j, q, g);
      if (d >= s.D) continue;
      const float4 x = acc_block(acc, j, q, inv);
      *reinterpret_cast<float4*>(o + d) = x;
      if (ol) *reinterpret_cast<float4*>(ol + d) = x;
    }
  if (g == 0)
    (part ? a.part_lse + blockIdx.y * n_rows : a.lse)[((int64_t)b * s.Hq + h) * s.Sq + i] = l != 0.f ? fmaf(-slope, see.rest, m + logf(l)) : -INFINITY;
  if (any_dirty)
    for (int t = t0; t < t1; ++t)
      if (w.all_lo > t * kT || w.all_hi < (t + 1) * kT)
        add_nonfinite<DB>(o, ol, v0, a.v.ss, max(see.lo, t * kT), min(see.hi, (t + 1) * kT), s.D, g, false);
}

// ---------------------------------------------------------------- dQ
template <int DP, bool FULL, bool CAP>
__global__ __launch_bounds__(waves<DP>() * 64) void score_dq_f32_kernel(const ScoreArgs a) {
  constexpr int NW = waves<DP>(), DB = DP / 32, N = DP == 128 ? 16 : 32, R = DP < 128 ? 3 : DP == 128 ? 4 : 2;
  constexpr int NR = row_pieces<DP, N>(), NC = col_pieces<DP, N>(), kPieces = 2 * NR + NC;
  __shared__ __attribute__((aligned(16))) float qs[kT * lds_stride<DP>()];
  __shared__ __attribute__((aligned(16))) float dos[kT * lds_stride<DP>()];
  __shared__ float fold[NW / 2 * DB * 16 * 64];
  __shared__ int any_dirty;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int n_qt = (s.Sq + kT - 1) / kT;
  int qt, hb;
  qtile_block(blockIdx.x, gridDim.x, n_qt, s.causal, qt, hb);
  const int h = (int)sgpr(hb % s.Hq), b = (int)sgpr(hb / s.Hq), hk = (int)sgpr(h / (s.Hq / s.Hkv));
  const int row0 = (int)sgpr(qt * kT);
  stage_tile<DP>(qs, (const float*)a.q.ptr + b * a.q.sb + h * a.q.sh, a.q.ss, row0, s.Sq, s.D, tid);
  stage_tile<DP>(dos, (const float*)a.d_o.ptr + b * a.d_o.sb + h * a.d_o.sh, a.d_o.ss, row0, s.Sq, s.D, tid);
  if (tid == 0) any_dirty = 0;
  const int i = min(row0 + r, s.Sq - 1);
  RowView see = row_view(a, b, i);
  const int64_t stat = ((int64_t)b * s.Hq + h) * s.Sq + i;
  const float slope = a.slopes ? a.slopes[h] : 0.f, lse_row = a.lse_in[stat], dl = a.delta[stat];
  if (lse_row == -INFINITY) see.lo = see.hi = 0;             // an empty row
  const float lse = fmaf(slope, see.rest, lse_row);
  BlockSpan w = span_of(see);
  w.lo = wave_min(w.lo); w.hi = wave_max(w.hi); w.all_lo = wave_max(w.all_lo); w.all_hi = wave_min(w.all_hi);
  const float *k0 = (const float*)a.k.ptr + b * a.k.sb + hk * a.k.sh, *v0 = (const float*)a.v.ptr + b * a.v.sb + hk * a.v.sh;
  __syncthreads();

  f32x16 acc[DB];
  zero_acc(acc);
  const int first = w.lo < w.hi ? w.lo / kT : 0, n = w.lo < w.hi ? (w.hi + kT - 1) / kT - first : 0;
  const int t0 = first + (int)((int64_t)n * blockIdx.y / a.q_split), t1 = first + (int)((int64_t)n * (blockIdx.y + 1) / a.q_split);
  for (int t = t0 + wave; t < t1; t += NW) {
    const int key0 = t * kT, limit = min(kT, s.Sk - key0);
    const float *kb = k0 + (int64_t)key0 * a.k.ss, *vb = v0 + (int64_t)key0 * a.v.ss;
    const bool masked = w.all_lo > key0 || w.all_hi < key0 + kT;
    const float* krow = kb + (int64_t)min(r, limit - 1) * a.k.ss;
    const float* vrow = vb + (int64_t)min(r, limit - 1) * a.v.ss;
    Piece<N> f[R];
    auto load = [&](int x) {
      if (x >= kPieces) return;
      if (x < 2 * NR) load_rows<DP, FULL>(f[x % R], x < NR ? krow : vrow, x < NR ? x : x - NR, s.D, g);
      else load_cols<DP, FULL>(f[x % R], kb, a.k.ss, limit, x - 2 * NR, s.D, r, g);
      __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 p, ds;
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] = ds[v] = 0.f;
#pragma unroll
    for (int x = 0; x < R - 1; ++x) load(x);
#pragma unroll
    for (int x = 0; x < 2 * NR; ++x) {
      load(x + R - 1);
      if (x < NR) contract_d<DP>(p, f[x % R], qs, x, r, g);
      else contract_d<DP>(ds, f[x % R], dos, x - NR, r, g);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = key0 + c_row(v, g);
      float f2;
      const float e = fmaf(-slope, fabsf((float)(see.x - key)), score_of<CAP>(p[v], a, f2));
      ds[v] = key >= see.lo && key < see.hi ? expf(e - lse) * (ds[v] - dl) * f2 : 0.f;
    }
    bool bad = false;
#pragma unroll
    for (int x = 2 * NR; x < kPieces; ++x) {
      load(x + R - 1);
      if (masked) bad = make_finite<DP>(f[x % R]) || bad;
      contract_rows<DP>(acc, f[x % R], ds, x - 2 * NR);
    }
    if (bad) any_dirty = 1;
  }
  for (int y = NW / 2; y > 0; y /= 2) {
    if (wave >= y && wave < 2 * y) put_acc(fold + (wave - y) * DB * 16 * 64, acc, lane);
    __syncthreads();
    if (wave < y) add_acc(fold + wave * DB * 16 * 64, acc, 1.f, 1.f, lane);
    __syncthreads();
  }
  if (wave != 0 || row0 + r >= s.Sq) return;
  const bool part = a.q_split > 1;
  const int64_t n_q = (int64_t)s.B * s.Sq * s.Hq * s.D, at = (((int64_t)b * s.Sq + i) * s.Hq + h) * s.D;
  float* out = part ? a.part_dq + blockIdx.y * n_q + at : a.dq ? a.dq + at : nullptr;
  float* low = !part && a.dq_lowp ? (float*)a.dq_lowp + at : nullptr;
  if (out == nullptr) {
    out = low;
    low = nullptr;
  }
  const bool add_old = !part && !a.assign;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < DB; ++q) {
      const int d = block_column<DB>(j, q, g);
      if (d >= s.D) continue;
      float4 x = acc_block(acc, j, q, s.scale);
      if (add_old) x = add(x, *reinterpret_cast<const float4*>(out + d));
      *reinterpret_cast<float4*>(out + d) = x;
      if (low) *reinterpret_cast<float4*>(low + d) = x;
    }
  if (any_dirty)
    for (int t = t0; t < t1; ++t)
      if (w.all_lo > t * kT || w.all_hi < (t + 1) * kT)
        add_nonfinite<DB>(out, low, k0, a.k.ss, max(see.lo, t * kT), min(see.hi, (t + 1) * kT), s.D, g, true);
}

// ---------------------------------------------------------------- dK, dV
// block = key tile + ceil(Sk / 32) (KV head + Hkv batch entry); share y takes every kv_split-th group of a wavefront each's pairs
// Head sizes beyond 128: the accumulators of 32 keys are more than the registers, so a workgroup has half of the gradients' columns and
// makes S and dP for itself (8/2 heads x 400 rows of 256, forward and backward: 163 us; 229 with all columns, 640 values of them in
// scratch memory).
template <int DP, bool FULL, bool CAP>
__global__ __launch_bounds__(512) void score_dkv_f32_kernel(const ScoreArgs a) {
  constexpr int NW = 8, H = score_f32_halves(DP), DH = DP / H, DB = DH / 32, N = 16, R = DP < 128 ? 4 : 2;   // DH: columns of this workgroup
  constexpr int NR = row_pieces<DP, N>(), NC = col_pieces<DH, N>(), kPieces = 2 * NR + 2 * NC;
  constexpr int kStat = 5 * kT;                              // of every row lse, Delta, lo, hi, x
  __shared__ __attribute__((aligned(16))) float ks[kT * lds_stride<DP>()];
  __shared__ __attribute__((aligned(16))) float vs[kT * lds_stride<DP>()];
  __shared__ __attribute__((aligned(16))) float stats[NW * kStat];
  __shared__ float fold[NW / 2 * DB * 16 * 64];
  __shared__ int any_dirty;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int tile = (int)(blockIdx.x / H), first = (int)sgpr((int)(blockIdx.x % H) * DH), columns = min(DH, s.D - first);
  const int n_kt = (s.Sk + kT - 1) / kT, outer = tile / n_kt;
  const int key0 = (int)sgpr((tile - outer * n_kt) * kT), hk = (int)sgpr(outer % s.Hkv), b = (int)sgpr(outer / s.Hkv);
  const int keys = min(kT, s.Sk - key0), key = key0 + r;
  const int G = s.Hq / s.Hkv;
  if (tid < waves<DP>() * 64) {
    stage_tile<DP>(ks, (const float*)a.k.ptr + b * a.k.sb + hk * a.k.sh, a.k.ss, key0, s.Sk, s.D, tid);
    stage_tile<DP>(vs, (const float*)a.v.ptr + b * a.v.sb + hk * a.v.sh, a.v.ss, key0, s.Sk, s.D, tid);
  }
  if (tid == 0) any_dirty = 0;
  __syncthreads();
  f32x16 acc_k[DB], acc_v[DB];
  zero_acc(acc_k);
  zero_acc(acc_v);
  const int per_head = (s.Sq + kT - 1) / kT;
  const int64_t pairs = (int64_t)G * per_head;
  float* st = stats + wave * kStat;
  for (int64_t x = (int64_t)blockIdx.y * NW + wave; x < pairs; x += (int64_t)NW * a.kv_split) {
    const int hg = (int)sgpr((int)(x / per_head)), h = hk * G + hg, i0 = (int)sgpr((int)(x - (int64_t)hg * per_head)) * kT;
    const int limit = min(kT, s.Sq - i0), i = i0 + min(r, limit - 1);
    const int64_t stat = ((int64_t)b * s.Hq + h) * s.Sq + i;
    const float slope = a.slopes ? a.slopes[h] : 0.f, lse_row = a.lse_in[stat];
    RowView see = row_view(a, b, i);
    if (r >= limit || lse_row == -INFINITY) see.lo = see.hi = 0;        // a row that does not exist, or an empty one
    BlockSpan w = span_of(see);
    w.lo = wave_min(w.lo); w.hi = wave_max(w.hi); w.all_lo = wave_max(w.all_lo); w.all_hi = wave_min(w.all_hi);
    if (w.lo >= key0 + keys || w.hi <= key0) continue;
    const bool masked = w.all_lo > key0 || w.all_hi < key0 + keys;
    const float* qb = (const float*)a.q.ptr + b * a.q.sb + h * a.q.sh + (int64_t)i0 * a.q.ss;
    const float* db_ = (const float*)a.d_o.ptr + b * a.d_o.sb + h * a.d_o.sh + (int64_t)i0 * a.d_o.ss;
    const float* qrow = qb + (int64_t)min(r, limit - 1) * a.q.ss;
    const float* drow = db_ + (int64_t)min(r, limit - 1) * a.d_o.ss;
    Piece<N> f[R];
    auto load = [&](int x) {
      if (x >= kPieces) return;
      if (x < 2 * NR) load_rows<DP, FULL>(f[x % R], x < NR ? qrow : drow, x < NR ? x : x - NR, s.D, g);
      else if (x < 2 * NR + NC) load_cols<DH, FULL>(f[x % R], db_ + first, a.d_o.ss, limit, x - 2 * NR, columns, r, g);
      else load_cols<DH, FULL>(f[x % R], qb + first, a.q.ss, limit, x - 2 * NR - NC, columns, r, g);
      __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 p, ds;
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] = ds[v] = 0.f;
#pragma unroll
    for (int x = 0; x < R - 1; ++x) load(x);
#pragma unroll
    for (int x = 0; x < 2 * NR; ++x) {
      load(x + R - 1);
      if (x < NR) contract_d<DP>(p, f[x % R], ks, x, r, g);
      else contract_d<DP>(ds, f[x % R], vs, x - NR, r, g);
    }
    if (g == 0) {
      st[r] = fmaf(slope, see.rest, lse_row);
      st[2 * kT + r] = __int_as_float(see.lo);
      st[3 * kT + r] = __int_as_float(see.hi);
    } else {
      st[kT + r] = a.delta[stat];
      st[4 * kT + r] = __int_as_float(see.x);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int row = c_row(v, g);
      const bool live = key >= __float_as_int(st[2 * kT + row]) && key < __float_as_int(st[3 * kT + row]);
      float f2;
      const float e = fmaf(-slope, fabsf((float)(__float_as_int(st[4 * kT + row]) - key)), score_of<CAP>(p[v], a, f2));
      p[v] = live ? expf(e - st[row]) : 0.f;
      ds[v] = live ? p[v] * (ds[v] - st[kT + row]) * f2 : 0.f;
    }
    __builtin_amdgcn_wave_barrier();
    bool bad = false;
#pragma unroll
    for (int x = 2 * NR; x < kPieces; ++x) {
      load(x + R - 1);
      if (masked) bad = make_finite<DH>(f[x % R]) || bad;
      if (x < 2 * NR + NC) contract_rows<DH>(acc_v, f[x % R], p, x - 2 * NR);
      else contract_rows<DH>(acc_k, f[x % R], ds, x - 2 * NR - NC);
    }
    if (bad) any_dirty = 1;
  }
  for (int n = NW / 2; n > 0; n /= 2) {
    float* slot = fold + (wave - (wave >= n ? n : 0)) * DB * 16 * 64;
    if (wave >= n && wave < 2 * n) put_acc(slot, acc_k, lane);
    __syncthreads();
    if (wave < n) add_acc(slot, acc_k, 1.f, 1.f, lane);
    __syncthreads();
    if (wave >= n && wave < 2 * n) put_acc(slot, acc_v, lane);
    __syncthreads();
    if (wave < n) add_acc(slot, acc_v, 1.f, 1.f, lane);
    __syncthreads();
  }
  if (wave != 0 || key >= s.Sk) return;
  const bool part = a.kv_split > 1, add_old = !part && !a.assign;
  const int64_t n_kv = (int64_t)s.B * s.Sk * s.Hkv * s.D, at = (((int64_t)b * s.Sk + key) * s.Hkv + hk) * s.D + first;
  auto place = [&](float* parts, float* out, void* low, float*& o, float*& o2) {
    o = part ? parts + blockIdx.y * n_kv + at : out ? out + at : nullptr;
    o2 = !part && low ? (float*)low + at : nullptr;
    if (o == nullptr) {
      o = o2;
      o2 = nullptr;
    }
  };
  float *ok, *ok2, *ov, *ov2;
  place(a.part_dk, a.dk, a.dk_lowp, ok, ok2);
  place(a.part_dv, a.dv, a.dv_lowp, ov, ov2);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < DB; ++q) {
      const int d = block_column<DB>(j, q, g);
      if (d >= columns) continue;
      float4 x = acc_block(acc_k, j, q, s.scale), y = acc_block(acc_v, j, q, 1.f);
      if (add_old) {
        x = add(x, *reinterpret_cast<const float4*>(ok + d));
        y = add(y, *reinterpret_cast<const float4*>(ov + d));
      }
      *reinterpret_cast<float4*>(ok + d) = x;
      *reinterpret_cast<float4*>(ov + d) = y;
      if (ok2) *reinterpret_cast<float4*>(ok2 + d) = x;
      if (ov2) *reinterpret_cast<float4*>(ov2 + d) = y;
    }
  if (any_dirty)
    // what this share's masked tiles left out, row by row
    for (int64_t x = 0; x < pairs; ++x) {
      if (x / NW % a.kv_split != blockIdx.y) continue;
      const int hg = (int)(x / per_head), h = hk * G + hg, i0 = (int)(x - (int64_t)hg * per_head) * kT;
      const float* qb = (const float*)a.q.ptr + b * a.q.sb + h * a.q.sh;
      const float* db_ = (const float*)a.d_o.ptr + b * a.d_o.sb + h * a.d_o.sh;
      for (int i = i0; i < min(i0 + kT, s.Sq); ++i) {
        const RowView see = row_view(a, b, i);
        if (key < see.lo || key >= see.hi || a.lse_in[((int64_t)b * s.Hq + h) * s.Sq + i] == -INFINITY) continue;
        add_nonfinite<DB>(ok, ok2, qb + first, a.q.ss, i, i + 1, columns, g, true);
        add_nonfinite<DB>(ov, ov2, db_ + first, a.d_o.ss, i, i + 1, columns, g, false);
      }
    }
}

}  // namespace

hipError_t launch_score_fwd_f32(const ScoreArgs& a, hipStream_t stream) {
  const int64_t total = (int64_t)((a.s.Sq + kT - 1) / kT) * a.s.Hq * a.s.B;
  if (total <= 0) return hipSuccess;
  if (total > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("score_fwd_f32", stream);
  return with_padded_d(a.s.D, [&](auto dp, auto full) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool FULL = decltype(full)::value;
    const dim3 grid((unsigned)total, (unsigned)a.n_split), block(waves<DP>() * 64);
    if (a.cap > 0.f) hipLaunchKernelGGL((score_fwd_f32_kernel<DP, FULL, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((score_fwd_f32_kernel<DP, FULL, false>), grid, block, 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_score_bwd_f32(const ScoreArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)((a.s.Sq + kT - 1) / kT) * a.s.Hq * a.s.B, keys = (int64_t)((a.s.Sk + kT - 1) / kT) * a.s.Hkv * a.s.B;
  if (rows > kScoreGridMost || keys * score_f32_halves(a.s.D) > kScoreGridMost) return hipErrorInvalidValue;
  return with_padded_d(a.s.D, [&](auto dp, auto full) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool FULL = decltype(full)::value;
    const dim3 block(waves<DP>() * 64);
    if (keys > 0) {
      ProfScope prof("score_dkv_f32", stream);
      const dim3 grid((unsigned)(keys * score_f32_halves(DP)), (unsigned)a.kv_split);
      if (a.cap > 0.f) hipLaunchKernelGGL((score_dkv_f32_kernel<DP, FULL, true>), grid, dim3(512), 0, stream, a);
      else hipLaunchKernelGGL((score_dkv_f32_kernel<DP, FULL, false>), grid, dim3(512), 0, stream, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (rows > 0) {
      ProfScope prof("score_dq_f32", stream);
      const dim3 grid((unsigned)rows, (unsigned)a.q_split);
      if (a.cap > 0.f) hipLaunchKernelGGL((score_dq_f32_kernel<DP, FULL, true>), grid, block, 0, stream, a);
      else hipLaunchKernelGGL((score_dq_f32_kernel<DP, FULL, false>), grid, block, 0, stream, a);
      return hipGetLastError();
    }
    return hipSuccess;
  });
}

}  // namespace st
