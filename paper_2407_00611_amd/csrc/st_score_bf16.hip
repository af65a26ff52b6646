// bf16 attention with modified scores (st_score.h), head size 128 or 64: forward, dQ and dK/dV on v_mfma_f32_32x32x16_bf16.
//
// Products <q, k> of the stored values are exact in the matrix unit's fp32 sums; scale, cap, bias and softmax are fp32, Q itself is
// not rounded again.  P and dU are rounded to bf16 for the second contractions, relative 2^-8 at most each, as those of the other
// bf16 kernels here; sums and statistics stay fp32.
//
// Rows whose tile a mask edge crosses: the matrix unit multiplies what a row does not see by zero, and 0 * inf is NaN.  In such a
// tile the operand's infinities and NaN are made finite.  The forward adds them to the rows that do see them once O is stored; in
// the backward, P or dU of a row that sees a key with such values is NaN, and so is its contribution.
#include <algorithm>
#include <type_traits>

#include "st_score.h"

namespace st {
namespace {

constexpr int kBN = 64;              // keys of a streamed tile
// A lane's sum over sixteen keys beyond which a row's exponent reference moves up: one of its exponents exceeds the reference by 8
// log2 units then; while all are below that, none does.
constexpr float kSumMost = 4096.f;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Whether 32 rows of an LDS tile hold an infinity or NaN: their products with zeros are NaN then, whatever place a matrix instruction
// takes an operand's values for.  Eight short ones, where a look at every operand's bits is some 96 others; operands are made finite
// only where it is true.
template <int D>
__device__ __forceinline__ bool not_finite(const LaneReads<D>& reads, uint32_t tile) {
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
  const bf16x8 zero = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(reads.frag_tr(tile, 16 * m, db), zero, z, 0, 0, 0);
  return __any((z[0] + z[1]) + (z[2] + z[3]) != 0.f);
}

// Tiles of 64 keys that a query tile's workgroup walks: those that the hull of its rows touches.  The general ones come first (a
// mask edge crosses them, or a biased row lies in them), then the rest, the whole ones, in two ranges of the chunk: nearest first,
// so that a bias that falls with the distance finds the largest exponents early.  The two kinds have loops of their own: as two
// ways through one loop's body they cost copies of all accumulators and the masks' compares in every tile (32/8 heads x 8192 rows,
// capped: 358 us).  A share of a split walk is a run of this order.
struct Walk {
  int t0, a0, a1, a2;        // general [t0, a0), [a1, a2) and from a3 on; whole [a0, a1) from its end, [a2, a3) from its start
  int n_gen, n0, n1;         // general tiles; this share
  __device__ __forceinline__ int tile(int n) const {
    if (n < n_gen) {
      const int g1 = a0 - t0, g2 = g1 + a2 - a1;
      return n < g1 ? t0 + n : n < g2 ? a1 + n - g1 : a3 + n - g2;
    }
    n -= n_gen;
    return n < a1 - a0 ? a1 - 1 - n : a2 + n - (a1 - a0);
  }
  int a3;
};
// x_lo, x_hi: where the rows' nearest keys lie (bias only)
__device__ __forceinline__ Walk walk_of(const BlockSpan& w, bool bias, int x_lo, int x_hi, int n_split, int share) {
  Walk y;
  const bool any = w.lo < w.hi;
  y.t0 = any ? w.lo / kBN : 0;
  const int t1 = any ? (w.hi + kBN - 1) / kBN : 0;
  const int f0 = min(max((w.all_lo + kBN - 1) / kBN, y.t0), t1), f1 = max(min(w.all_hi / kBN, t1), f0);   // whole tiles
  y.a0 = f0;
  y.a1 = f1;
  y.a2 = y.a3 = f1;
  if (bias) {                                          // only those with all rows on one side
    y.a1 = max(min(f1, (x_lo + 1) / kBN), f0);
    y.a2 = min(max(y.a1, (x_hi + kBN - 1) / kBN), f1);
    y.a3 = f1;
    if (y.a2 < y.a1) y.a2 = y.a1;
  }
  const int whole = y.a1 - y.a0 + y.a3 - y.a2, n = t1 - y.t0;
  y.n_gen = n - whole;
  const int64_t s = share;
  y.n0 = (int)(n * s / n_split);
  y.n1 = (int)(n * (s + 1) / n_split);
  return y;
}

// The nth of a batch entry's row tiles, of 256 at a time those with the most keys first: what spans leave to a tile differs, and one
// that holds the end of a document and the start of the next walks both, behind the mask of each.  Launched last such a tile runs on
// while the chip is empty.  The order is by half octaves of the keys that the first and the last row see, and the tile's number.
constexpr int kTileLevels = 16;
__device__ __forceinline__ int ordered_tile(const ScoreArgs& a, int b, int n_qt, int nth, int* lds) {   // lds: 4 kTileLevels + 1 ints
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), G = s.Hq / s.Hkv;
  const int c0 = nth & ~255, t = n_qt - 1 - (c0 + tid);
  int level = -1;
  if (t >= 0) {
    const BlockSpan w = span_join(span_of(row_view(a, b, t * kScoreRows / G)), span_of(row_view(a, b, min((t * kScoreRows + kScoreRows - 1) / G, s.Sq - 1))));
    const float hull = (float)max(w.hi - w.lo, 0), cost = fmaxf(2.f * hull - (float)max(w.all_hi - w.all_lo, 0), 0.f);
    const int below = (__float_as_int(2.f * (float)s.Sk) >> 22) - (__float_as_int(cost) >> 22);
    level = max(kTileLevels - 1 - below, 0);
  }
  uint64_t mine = 0;
#pragma unroll
  for (int x = 0; x < kTileLevels; ++x) {
    const uint64_t m = __ballot(level == x);
    if (level == x) mine = m;
    if (lane == 0) lds[4 * x + wave] = __popcll(m);
  }
  __syncthreads();
  int rank = __popcll(mine & (((uint64_t)1 << lane) - 1));
#pragma unroll
  for (int x = 0; x < kTileLevels; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      if (x > level || (x == level && y < wave)) rank += lds[4 * x + y];
  if (level >= 0 && rank == nth - c0) lds[4 * kTileLevels] = t;
  __syncthreads();
  return uniform(lds[4 * kTileLevels]);
}

// Block id -> (row tile, KV head, batch entry).  Every XCD has a contiguous range of the (KV head, batch entry) pairs, whose keys and
// values stay in its L2; under a causal mask the later tiles, which see more, come first.
// Workgroups whose order is worth its making, 2 us of each.  The spans are on the device, so a rule on the host goes by the number of
// workgroups: more than the chip holds at once, and so few turns of them that a long last one shows.  Forward without and with an
// order, in us:
//   long documents   24 heads of 64 x 8192 rows, six of them (1536 workgroups) 135, 114; 32/8 heads of 128, eight x 4096 (1024) 56, 53,
//                    three x 8192 (2048) 258, 243
//   what has the same work in every tile loses: 32/8 heads x 8192 rows, 31 documents 72, 79, a window of 64 keys 60, 69
//   beyond 2048      32/8 heads, three documents x 16384 (4096) 896, 890, x 32768 (8192) 3370, 3430; window of 64 keys x 16384 121, 138;
//                    but six documents, 24 heads of 64 x 16384 (3072), 448, 407
constexpr int kOrderFrom = 512, kOrderUpTo = 2048;
__device__ __forceinline__ void tile_block(const ScoreArgs& a, int block, int blocks, int n_qt, int* lds, int& qt, int& hk, int& b) {
  int hb;
  qtile_block(block, blocks, n_qt, a.s.causal || a.spans, qt, hb);
  hk = uniform(hb % a.s.Hkv);
  b = uniform(hb / a.s.Hkv);
  qt = uniform(qt);
  if (a.spans && blocks > kOrderFrom && blocks <= kOrderUpTo) qt = ordered_tile(a, b, n_qt, n_qt - 1 - qt, lds);
}

// what the rows of the workgroup see together, from what those of each wavefront do; hull: 6 x 4 ints of LDS
__device__ __forceinline__ BlockSpan workgroup_span(int* hull, const BlockSpan& w, int x_lo, int x_hi, int wave, int lane, int& wg_x_lo, int& wg_x_hi) {
  if (lane == 0) {
    hull[wave] = w.lo; hull[4 + wave] = w.hi; hull[8 + wave] = w.all_lo; hull[12 + wave] = w.all_hi; hull[16 + wave] = x_lo; hull[20 + wave] = x_hi;
  }
  __syncthreads();
  auto lowest = [&](int o) { return uniform(min(min(hull[o], hull[o + 1]), min(hull[o + 2], hull[o + 3]))); };
  auto highest = [&](int o) { return uniform(max(max(hull[o], hull[o + 1]), max(hull[o + 2], hull[o + 3]))); };
  wg_x_lo = lowest(16);
  wg_x_hi = highest(20);
  return BlockSpan{lowest(0), highest(4), highest(8), lowest(12)};
}

// Direct loads of a whole 64-key tile (in assembly: the compiler would wait for builtin ones ahead of every LDS read, those of the
// tile in hand too; landed() is the wait): the lane's place in the tile's first rows, the rest of the address is uniform
__device__ __forceinline__ void landed() {
  wait_vmcnt<0>();
  __syncthreads();
}
template <int D>
struct TileLoads {
  const char* at;
  int64_t row;               // bytes
  __device__ __forceinline__ TileLoads(const char* base, int64_t stride, int lane, int wave) : row(stride * 2) {
    constexpr int PPR = D / 8, RPI = 64 / PPR;
    const int r = wave * RPI + lane / PPR, f = swz<D>(r, 0) - r * D * 2;
    at = base + r * row + (((lane % PPR) << 4) ^ f);
  }
  __device__ __forceinline__ void issue(int key0, uint32_t tile, int wave) const {
    constexpr int N = kBN * D * 2 / 4096, STEP = 4 * 64 / (D / 8);
#pragma unroll
    for (int j = 0; j < N; ++j) dma16_asm(at + (key0 + STEP * j) * row, tile + (4 * j + wave) * 1024);
  }
};

// =============================================================================================
// Forward: S^T = K Q^T and O^T += V^T P^T, so that a lane has one row (C layout column) of a wavefront's 32: its reference, sum and
// span are registers, and the exponentials of S^T are the second product's operand as they stand.  128 rows a workgroup, packed over
// the heads of a KV head, two workgroups a compute unit at head size 128, three at 64.  One pass over the keys: O and the row sum
// against a reference m, O = acc / l, lse = m ln 2 + ln l.
//
// Bound by the matrix units and the vector unit together, whose work hardly overlaps with two wavefronts on a SIMD (two runs of rows,
// 32/8 heads x 4096 x 2048 keys: busy 42 % and 61 % of the time), and by power: 32/8 heads x 8192 x 4096 keys of 128 take 590 us,
// 930 TFLOP/s at 1.8 GHz (capped 650 us; 24 or 32 heads of 64, vector unit busy 82 %: 900 TFLOP/s).  Wavefronts of 64 rows, half the
// operand reads a product, leave one on a SIMD and took 951 us; products and softmax interleaved by hand gained 3 % there and
// nothing where masks are.  Packed images (24 heads of 64 x 8192 rows) take 110 us, prompts with prefixes (32/8
// x 4096) 53 to 56 us, spans included.
// =============================================================================================
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void score_fwd_kernel(const ScoreArgs a) {
  constexpr int KB = kBN / 32, KS = D / 16, DB = D / 32;
  constexpr int kTile = kBN * D * 2;
  constexpr float kUnset = -1e30f;                     // reference of a row that has met no key: whatever comes exceeds it
  __shared__ __attribute__((aligned(1024))) char smem_raw[4 * kTile];   // 2 stages x (K, V)
  __shared__ int hull[24], order[4 * kTileLevels + 1];
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G;
  const int n_qt = (M + kScoreRows - 1) / kScoreRows;
  int qt, hk, b;
  tile_block(a, blockIdx.x, gridDim.x, n_qt, order, qt, hk, b);

  const int R = qt * kScoreRows + wave * 32 + r, row = min(R, M - 1);
  const int i = row / G, h = hk * G + row % G;
  const RowView see = row_view(a, b, i);
  BlockSpan w = span_of(see);                          // of the wavefront's rows
  w.lo = wave_min(w.lo); w.hi = wave_max(w.hi); w.all_lo = wave_max(w.all_lo); w.all_hi = wave_min(w.all_hi);
  // Q fragments (B operand): row r, elements 16 ks + 8 g .. + 7
  bf16x8 qf[KS];
  const char* qrow = (const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)i * a.q.ss + (int64_t)h * a.q.sh) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + (16 * ks + 8 * g) * 2);
  const ScoreConst k = score_const(a);
  const float slope2 = BIAS ? a.slopes[h] * kScoreLog2e : 0.f;
  int x_lo = 0, x_hi = 0;
  if (BIAS) x_lo = wave_min(see.x), x_hi = wave_max(see.x);
  const BlockSpan wg = workgroup_span(hull, w, x_lo, x_hi, wave, lane, x_lo, x_hi);
  const Walk walk = walk_of(wg, BIAS, x_lo, x_hi, a.n_split, blockIdx.y);

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  float m_run = kUnset, l_run = 0.f;
  bool bad = false;

  const char* kb_ = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh) * 2;
  const char* vb_ = (const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh) * 2;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)smem;
  const TileLoads<D> k_loads(kb_, a.k.ss, lane, wave), v_loads(vb_, a.v.ss, lane, wave);
  auto issue_load = [&](int n, int stage) {
    const int t = walk.tile(n);
    const uint32_t at = smem_addr + stage * 2 * kTile;
    if (n < walk.n_gen) {                              // it may be the ragged end of the chunk
      stage_dma_asm<D, kBN>(kb_, a.k.ss, t * kBN, s.Sk, at, tid);
      stage_dma_asm<D, kBN>(vb_, a.v.ss, t * kBN, s.Sk, at + kTile, tid);
    } else {
      k_loads.issue(t * kBN, at, wave);
      v_loads.issue(t * kBN, at + kTile, wave);
    }
  };
  const LaneReads<D> reads(lane);

  // 32 keys against the wavefront's rows, in three steps
  struct Block {
    f32x16 sc;
    u32x4 pf[2];
  };
  auto products = [&](Block& y, uint32_t ktile) {
#pragma unroll
    for (int v = 0; v < 16; ++v) y.sc[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) y.sc = mfma32(reads.frag(ktile, 0, ks), qf[ks], y.sc);
  };
  // In a whole tile the bias is slope (key - x) or slope (x - key) for all keys: the part of it that no key changes goes into the reference.
  auto softmax = [&](auto general, Block& y, int key0) {
    constexpr bool GEN = decltype(general)::value;
    const int x0 = see.x - key0 - 4 * g;
    const ScoreTile<CAP, BIAS> f(k, slope2, x0);
    const float side = x0 > 0 ? f.slope : -f.slope;    // (left of the row the bias rises with the key)
    const float off = BIAS && !GEN ? slope2 * fabsf((float)x0) : 0.f;
    const int l0 = see.lo - key0 - 4 * g, h0 = see.hi - key0 - 4 * g;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = 8 * (v / 4) + v % 4;
      y.sc[v] = GEN ? f.raw(y.sc[v], key) : f.raw_side(y.sc[v], key, side);
      if (GEN) y.sc[v] = key >= l0 && key < h0 ? y.sc[v] : f.lowest();
    }
    // The reference m_run of the exponents is lazy.  It moves where the block's sum says that some exponent was large (or too large
    // for its exponential): nothing of the block has been used by then.
    float p[16], sum;
    auto exponentials = [&]() {
      const float m = m_run + off;
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        p[v] = __builtin_amdgcn_exp2f(f.exponent(y.sc[v], m));
        sum += p[v];
      }
    };
    exponentials();
    if (__builtin_expect(__any(sum > kSumMost), 0)) {
      float top = f.lowest();
#pragma unroll
      for (int v = 0; v < 16; ++v) top = f.higher(top, y.sc[v]);
      const float m_new = fmaxf(m_run, xhalf_max(f.exponent(top, off)));
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
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) y.pf[m][e] = pack_bf16(p[8 * m + 2 * e], p[8 * m + 2 * e + 1]);
  };
  auto contract = [&](auto scrub, const Block& y, uint32_t vtile) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 vf = reads.frag_tr(vtile, 16 * m, db);
        acc[db] = mfma32(decltype(scrub)::value ? finite_bf16(vf) : vf, __builtin_bit_cast(bf16x8, y.pf[m]), acc[db]);
      }
  };

  int buf = 0, n = walk.n0;
  if (n < walk.n1) issue_load(n, 0);
  landed();
  for (; n < min(walk.n1, walk.n_gen); ++n) {
    if (n + 1 < walk.n1) issue_load(n + 1, buf ^ 1);
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
    if (w.lo < key0 + kBN && w.hi > key0) {            // some row of this wavefront sees some key of the tile
      Block y[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) products(y[kb], ktile + 32 * kb * D * 2);
      const bool dirty = (w.all_lo > key0 || w.all_hi < key0 + kBN) &&
                         (not_finite<D>(reads, ktile + kTile) || not_finite<D>(reads, ktile + kTile + 32 * D * 2));
      bad = bad || dirty;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t vblock = ktile + kTile + 32 * kb * D * 2;
        softmax(std::true_type(), y[kb], key0 + 32 * kb);
        if (__builtin_expect(dirty, 0)) contract(std::true_type(), y[kb], vblock);
        else contract(std::false_type(), y[kb], vblock);
      }
    }
    landed();
    buf ^= 1;
  }
  for (; n < walk.n1; ++n) {
    if (n + 1 < walk.n1) issue_load(n + 1, buf ^ 1);
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
    // both blocks' products first: the second's run over the softmax of the first
    Block y[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) products(y[kb], ktile + 32 * kb * D * 2);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      softmax(std::false_type(), y[kb], key0 + 32 * kb);
      contract(std::false_type(), y[kb], ktile + kTile + 32 * kb * D * 2);
    }
    landed();
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
  if (R >= M) return;
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
  if (bad)
    // what the general tiles of this wavefront left out: V[t][d] of the keys that this row sees
    for (int y = walk.n0; y < min(walk.n1, walk.n_gen); ++y) {
      const int key0 = walk.tile(y) * kBN;
      for (int key = max(see.lo, key0); key < min(see.hi, key0 + kBN); ++key)
        for (int d = 4 * g; d < D; d += 8)
          for (int e = 0; e < 4; ++e) {
            const float x = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(vb_ + ((int64_t)key * a.v.ss + d + e) * 2) << 16);
            if (fabsf(x) <= 3.402823466e38f) continue;
            if (o) o[orow + d + e] += x;
            if (olow) {
              const float z = __uint_as_float((uint32_t)olow[orow + d + e] << 16) + x;
              olow[orow + d + e] = (uint16_t)pack_bf16(z, z);
            }
          }
    }
}

// =============================================================================================
// dQ: as the forward, with dP^T = V dO^T beside S^T and P from the final lse: dQ^T += K^T dU^T.  Seven contractions for both passes of
// the backward, where five would do in one: dQ of one pass would be added up by atomics, in no order.
// =============================================================================================
template <int D, bool CAP, bool BIAS>
__device__ __forceinline__ void score_dq(const ScoreArgs& a, int block_x, int blocks, int share, char* smem_raw) {
  constexpr int KB = kBN / 32, KS = D / 16, DB = D / 32;
  constexpr int kTile = kBN * D * 2;
  int* hull = (int*)(smem_raw + 4 * kTile);
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G;
  const int n_qt = (M + kScoreRows - 1) / kScoreRows;
  int qt, hk, b;
  tile_block(a, block_x, blocks, n_qt, hull + 24, qt, hk, b);

  const int R = qt * kScoreRows + wave * 32 + r, row = min(R, M - 1);
  const int i = row / G, h = hk * G + row % G;
  RowView see = row_view(a, b, i);
  const int64_t stat = ((int64_t)b * s.Hq + h) * s.Sq + i;
  const float slope = BIAS ? a.slopes[h] : 0.f, slope2 = slope * kScoreLog2e;
  const float lse = a.lse_in[stat], dlt = a.delta[stat];
  if (lse == -INFINITY) see.lo = see.hi = 0;           // an empty row
  // the row's constant: s log2 e = e + const with e from the nearest key on
  const float lse2 = (BIAS ? fmaf(slope, see.rest, lse) : lse) * kScoreLog2e;
  BlockSpan w = span_of(see);
  w.lo = wave_min(w.lo); w.hi = wave_max(w.hi); w.all_lo = wave_max(w.all_lo); w.all_hi = wave_min(w.all_hi);
  bf16x8 qf[KS], dof[KS];
  const char* qrow = (const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)i * a.q.ss + (int64_t)h * a.q.sh) * 2;
  const char* drow = (const char*)a.d_o.ptr + ((int64_t)b * a.d_o.sb + (int64_t)i * a.d_o.ss + (int64_t)h * a.d_o.sh) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + (16 * ks + 8 * g) * 2);
    dof[ks] = *reinterpret_cast<const bf16x8*>(drow + (16 * ks + 8 * g) * 2);
  }
  const ScoreConst k = score_const(a);
  int unused;
  const BlockSpan wg = workgroup_span(hull, w, 0, 0, wave, lane, unused, unused);
  const Walk walk = walk_of(wg, false, 0, 0, a.q_split, share);

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  const char* kb_ = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh) * 2;
  const char* vb_ = (const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh) * 2;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)smem;
  const TileLoads<D> k_loads(kb_, a.k.ss, lane, wave), v_loads(vb_, a.v.ss, lane, wave);
  auto issue_load = [&](int n, int stage) {
    const int t = walk.tile(n);
    const uint32_t at = smem_addr + stage * 2 * kTile;
    if (n < walk.n_gen) {
      stage_dma_asm<D, kBN>(kb_, a.k.ss, t * kBN, s.Sk, at, tid);
      stage_dma_asm<D, kBN>(vb_, a.v.ss, t * kBN, s.Sk, at + kTile, tid);
    } else {
      k_loads.issue(t * kBN, at, wave);
      v_loads.issue(t * kBN, at + kTile, wave);
    }
  };
  const LaneReads<D> reads(lane);
  auto block = [&](auto general, uint32_t ktile, uint32_t vtile, int key0) {
    constexpr bool GEN = decltype(general)::value;
    f32x16 sc, dp;
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = dp[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sc = mfma32(reads.frag(ktile, 0, ks), qf[ks], sc);
      dp = mfma32(reads.frag(vtile, 0, ks), dof[ks], dp);
    }
    const float x = (float)(see.x - key0 - 4 * g);
    const int l0 = see.lo - key0 - 4 * g, h0 = see.hi - key0 - 4 * g;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = 8 * (v / 4) + v % 4;
      float e, f = 1.f;
      if (CAP) {
        const float rr = cap_r(sc[v], k.c);
        e = fmaf(-2.f * k.k1, rr, k.k1 - lse2);
        f = fmaf(-rr, rr, rr);                         // a quarter of 1 - tanh^2
      } else {
        e = fmaf(sc[v], k.c, -lse2);
      }
      if (BIAS) e = fmaf(-slope2, fabsf(x - (float)key), e);
      float ds = __builtin_amdgcn_exp2f(e) * (dp[v] - dlt);
      if (CAP) ds *= f;
      if (GEN) ds = key >= l0 && key < h0 ? fmaf(0.f, sc[v], ds) : 0.f;
      sc[v] = ds;
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const bf16x8 dsf = pack_c_as_b(sc, m);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 ktf = reads.frag_tr(ktile, 16 * m, db);
        acc[db] = mfma32(GEN ? finite_bf16(ktf) : ktf, dsf, acc[db]);
      }
    }
  };
  int buf = 0, n = walk.n0;
  if (n < walk.n1) issue_load(n, 0);
  landed();
  for (; n < min(walk.n1, walk.n_gen); ++n) {
    if (n + 1 < walk.n1) issue_load(n + 1, buf ^ 1);
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
    if (w.lo < key0 + kBN && w.hi > key0)
#pragma unroll 1
      for (int kb = 0; kb < KB; ++kb)
        block(std::true_type(), ktile + 32 * kb * D * 2, ktile + kTile + 32 * kb * D * 2, key0 + 32 * kb);
    landed();
    buf ^= 1;
  }
  for (; n < walk.n1; ++n) {
    if (n + 1 < walk.n1) issue_load(n + 1, buf ^ 1);
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      block(std::false_type(), ktile + 32 * kb * D * 2, ktile + kTile + 32 * kb * D * 2, key0 + 32 * kb);
    landed();
    buf ^= 1;
  }
  if (R >= M) return;
  const int64_t orow = (((int64_t)b * s.Sq + i) * s.Hq + h) * D;
  const bool part = a.q_split > 1;
  float* out = part ? a.part_dq + share * ((int64_t)s.B * s.Sq * s.Hq * D) : a.dq;
  uint16_t* low = part ? nullptr : (uint16_t*)a.dq_lowp;
  const bool add = !part && !a.assign;
  const float c = CAP ? 4.f * s.scale : s.scale;
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
}

// =============================================================================================
// dK, dV: 128 keys of one KV head per workgroup, 32 per wavefront; the group's rows stream by in blocks of 32, so that the gradients
// of shared heads are sums in registers.  lane = key (C layout column), registers = 16 rows.  K fragments stay in registers, V in LDS,
// so that two workgroups fit a compute unit: one's softmax runs under the other's products (with V in registers too and one workgroup:
// 516 us for 32/8 heads x 4096 x 2048 keys, biased; 301 so, with rows and statistics straight to LDS).  Both gradients and dQ of 32/8 heads x 8192 x 4096 keys of 128: 1.9 ms, 1010
// TFLOP/s of the seven contractions (capped 2.05 ms; 32 heads of 64: 1.0 ms, 960).
// =============================================================================================
constexpr int kBlockList = 512;      // row blocks that a workgroup looks through at a time

template <int D>
constexpr int dkv_lds() { return kScoreKeys * D * 2 + 2 * (2 * 32 * D * 2 + kRowStats * 4) + kBlockList * 16 + 8 * 4; }

template <int D, bool CAP, bool BIAS>
__device__ __forceinline__ void score_dkv(const ScoreArgs& a, int block_x, int blocks, int share, char* smem_raw) {
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int kTile = 32 * D * 2, kStage = 2 * kTile + kRowStats * 4;   // Q, dO and the statistics of 32 rows
  constexpr int kKeyTile = kScoreKeys * D * 2;
  int4* list = (int4*)(smem_raw + kKeyTile + 2 * kStage);                 // block and hull of its rows: whole ones from the front, the others from the back
  int* count = (int*)(list + kBlockList);
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  ST_LDS char* stages = smem + kKeyTile;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 5, r = lane & 31;
  const int G = s.Hq / s.Hkv, M = s.Sq * G, n_blk = (M + 31) / 32;
  const int n_kt = (s.Sk + kScoreKeys - 1) / kScoreKeys;
  const int logical = xcd_logical_block(block_x, blocks);
  const int kt = uniform(logical % n_kt), bh = logical / n_kt;
  const int b = uniform(bh % s.B), hk = uniform(bh / s.B);
  const int key0 = kt * kScoreKeys, key_end = min(key0 + kScoreKeys, s.Sk);
  const int wkey0 = key0 + wave * 32, wkey_end = min(wkey0 + 32, s.Sk);
  const int key = wkey0 + r, key_row = min(key, s.Sk - 1);
  const uint32_t inv_g = G > 1 ? 0xffffffffu / (uint32_t)G + 1 : 0;      // x / G = x inv_g / 2^32 for the small x below

  stage_dma_asm<D, kScoreKeys>((const char*)a.v.ptr + ((int64_t)b * a.v.sb + (int64_t)hk * a.v.sh) * 2, a.v.ss, key0, s.Sk, (uint32_t)(uintptr_t)smem, tid);
  const char* kp = (const char*)a.k.ptr + ((int64_t)b * a.k.sb + (int64_t)hk * a.k.sh + (int64_t)key_row * a.k.ss) * 2;
  bf16x8 kf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const bf16x8*>(kp + (16 * ks + 8 * g) * 2);
  const ScoreConst k = score_const(a);
  f32x16 acc_k[DB], acc_v[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc_k[db][v] = acc_v[db][v] = 0.f;

  // a block's rows and statistics, straight to LDS: two of the 16-byte pieces of each tile a lane (one at head size 64)
  constexpr int PPR = D / 8, RPI = 64 / PPR;
  const int piece_row = wave * RPI + lane / PPR, piece = ((lane % PPR) << 4) ^ (swz<D>(piece_row, 0) - piece_row * D * 2);
  const char* q_base = (const char*)a.q.ptr + ((int64_t)b * a.q.sb + (int64_t)hk * G * a.q.sh) * 2 + piece;
  const char* d_base = (const char*)a.d_o.ptr + ((int64_t)b * a.d_o.sb + (int64_t)hk * G * a.d_o.sh) * 2 + piece;
  const char* stat_base = (const char*)(a.rows + ((int64_t)b * s.Hkv + hk) * n_blk * kRowStats) + lane * 16;
  auto load_block = [&](int j, int stage) {
    j = uniform(j);
    const uint32_t at = (uint32_t)(uintptr_t)stages + stage * kStage;
    const int base = 32 * j / G, rem = 32 * j - base * G;                // uniform
#pragma unroll
    for (int u = 0; u < 32 / (4 * RPI); ++u) {
      const uint32_t x = (uint32_t)(rem + min(piece_row + 4 * RPI * u, M - 1 - 32 * j)), q = G > 1 ? __umulhi(x, inv_g) : x;
      const int64_t i = base + (int)q, h = (int)(x - q * (uint32_t)G);
      dma16_asm(q_base + (i * a.q.ss + h * a.q.sh) * 2, at + (4 * u + wave) * 1024);
      dma16_asm(d_base + (i * a.d_o.ss + h * a.d_o.sh) * 2, at + kTile + (4 * u + wave) * 1024);
    }
    if (wave == 0) dma16_asm(stat_base + (int64_t)j * kRowStats * 4, at + 2 * kTile);
  };

  const LaneReads<D> reads(lane);
  const uint32_t v_rows = (uint32_t)(uintptr_t)smem + wave * 32 * D * 2, stage_addr = (uint32_t)(uintptr_t)stages;
  const float kx = (float)key;
  auto block = [&](auto general, int stage) {
    constexpr bool GEN = decltype(general)::value;
    const uint32_t qtile = stage_addr + stage * kStage, dotile = qtile + kTile;
    const ST_LDS float* stats = reinterpret_cast<const ST_LDS float*>(stages + stage * kStage + 2 * kTile);
    auto rows4 = [&](int what, int j4) { return *reinterpret_cast<const ST_LDS f32x4*>(stats + 32 * what + 8 * j4 + 4 * g); };
    f32x16 sc, dp;
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4) {
      const f32x4 dlt = rows4(kRowDelta, j4);          // minus Delta: what the products of dP are added to
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[4 * j4 + e] = 0.f, dp[4 * j4 + e] = dlt[e];
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sc = mfma32(reads.frag(qtile, 0, ks), kf[ks], sc);
      dp = mfma32(reads.frag(dotile, 0, ks), reads.frag(v_rows, 0, ks), dp);
    }
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4) {
      const f32x4 lse2 = rows4(kRowLse, j4);
      f32x4 x = {}, slope2 = {}, lo = {}, hi = {};
      if (BIAS) x = rows4(kRowX, j4), slope2 = rows4(kRowSlope, j4);
      if (GEN) lo = rows4(kRowLo, j4), hi = rows4(kRowHi, j4);
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const int v = 4 * j4 + e4;
        float e, f = 1.f;
        if (CAP) {
          const float rr = cap_r(sc[v], k.c);
          e = fmaf(-2.f * k.k1, rr, -lse2[e4]);        // (k1 is in the row's statistics)
          f = fmaf(-rr, rr, rr);                       // a quarter of 1 - tanh^2
        } else {
          e = fmaf(sc[v], k.c, -lse2[e4]);
        }
        if (BIAS) e = fmaf(-slope2[e4], fabsf(x[e4] - kx), e);
        float p = __builtin_amdgcn_exp2f(e), ds = p * dp[v];
        if (CAP) ds *= f;
        if (GEN) {
          const bool see = key >= __float_as_int(lo[e4]) && key < __float_as_int(hi[e4]);
          p = see ? fmaf(0.f, ds, p) : 0.f;            // (NaN for a row whose dO, or below Q, is not finite: the operand no longer says it)
          ds = see ? fmaf(0.f, sc[v], ds) : 0.f;
        }
        sc[v] = p;
        dp[v] = ds;
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const bf16x8 pf = pack_c_as_b(sc, m), dsf = pack_c_as_b(dp, m);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 x = reads.frag_tr(dotile, 16 * m, db), y = reads.frag_tr(qtile, 16 * m, db);
        acc_v[db] = mfma32(GEN ? finite_bf16(x) : x, pf, acc_v[db]);
        acc_k[db] = mfma32(GEN ? finite_bf16(y) : y, dsf, acc_k[db]);
      }
    }
  };

  // the blocks of this share: every kv_split-th, so that shares of a mask's edge and of its inside are alike
  const int n_share = a.kv_split, mine = (n_blk - share + n_share - 1) / n_share;
  for (int at = 0; at < mine; at += kBlockList) {
    // ---- the visible ones among the next blocks, in order
    int whole = 0, edge = 0;
    for (int c0 = 0; c0 < kBlockList && at + c0 < mine; c0 += 256) {
      const int x = at + c0 + tid, j = share + x * n_share;
      int4 y = make_int4(0x7fffffff, 0, 0, 0);
      if (x < mine) y = a.blocks[((int64_t)b * s.Hkv + hk) * n_blk + j];
      const bool seen = y.x < key_end && y.y > key0, all = seen && y.z <= key0 && y.w >= key_end;
      const uint64_t v_all = __ballot(all), v_edge = __ballot(seen && !all), before = ((uint64_t)1 << lane) - 1;
      if (lane == 0) {
        count[wave] = __popcll(v_all);
        count[4 + wave] = __popcll(v_edge);
      }
      __syncthreads();
      int p = whole, q = edge;
      for (int x2 = 0; x2 < wave; ++x2) p += count[x2], q += count[4 + x2];
      if (seen) list[all ? p + __popcll(v_all & before) : kBlockList - 1 - q - __popcll(v_edge & before)] = make_int4(j, y.x, y.y, 0);
      whole += count[0] + count[1] + count[2] + count[3];
      edge += count[4] + count[5] + count[6] + count[7];
      __syncthreads();
    }
    whole = uniform(whole);
    edge = uniform(edge);
    const int total = whole + edge;
    if (total == 0) continue;
    auto entry = [&](int n) { return n < edge ? kBlockList - 1 - n : n - edge; };
    load_block(list[entry(0)].x, 0);
    landed();
    int buf = 0, n = 0;
    for (; n < edge; ++n) {
      if (n + 1 < total) load_block(list[entry(n + 1)].x, buf ^ 1);
      const int4 y = list[entry(n)];
      if (uniform(y.y) < wkey_end && uniform(y.z) > wkey0) block(std::true_type(), buf);
      landed();
      buf ^= 1;
    }
    for (; n < total; ++n) {
      if (n + 1 < total) load_block(list[n + 1 - edge].x, buf ^ 1);
      block(std::false_type(), buf);
      landed();
      buf ^= 1;
    }
  }

  landed();                                            // (V, also where no block was visible)
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
  store(acc_k, CAP ? 4.f * s.scale : s.scale, part ? a.part_dk + share * n_kv : a.dk, part ? nullptr : (uint16_t*)a.dk_lowp);
  store(acc_v, 1.f, part ? a.part_dv + share * n_kv : a.dv, part ? nullptr : (uint16_t*)a.dv_lowp);
}

// Both in one launch, the key tiles first: those of a causal or packed batch do unlike amounts of work, and the query tiles fill
// the places that the short ones leave (32/8 heads x 8192 packed rows: 1111 and 419 us in launches of their own).
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void score_bwd_kernel(const ScoreArgs a, int key_tiles, int query_tiles) {
  constexpr int kQueryLds = 4 * kBN * D * 2 + (24 + 4 * kTileLevels + 1) * 4;
  __shared__ __attribute__((aligned(1024))) char smem[dkv_lds<D>() > kQueryLds ? dkv_lds<D>() : kQueryLds];
  const int n_kv = key_tiles * a.kv_split, block = blockIdx.x;      // (either number of tiles may be zero)
  if (block < n_kv) score_dkv<D, CAP, BIAS>(a, block % key_tiles, key_tiles, block / key_tiles, smem);
  else score_dq<D, CAP, BIAS>(a, (block - n_kv) % query_tiles, query_tiles, (block - n_kv) / query_tiles, smem);
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
  const int64_t rows = row_tiles(a.s), keys = (int64_t)((a.s.Sk + kScoreKeys - 1) / kScoreKeys) * a.s.Hkv * a.s.B;
  const int64_t total = keys * a.kv_split + rows * a.q_split;
  if (total <= 0) return hipSuccess;
  if (total > 4 * kScoreGridMost - 1) return hipErrorInvalidValue;
  ProfScope prof("score_bwd_bf16", stream);
  return with_score(a, [&](auto d, auto cap, auto bias) {
    hipLaunchKernelGGL((score_bwd_kernel<decltype(d)::value, decltype(cap)::value, decltype(bias)::value>), dim3((unsigned)total), dim3(256), 0, stream, a,
                       (int)keys, (int)rows);
    return hipGetLastError();
  });
}

}  // namespace st
