// Attention of prompts against a cache of pages, bf16: 128 packed rows a workgroup, keys and values of 64 tokens at a time through LDS.
//
//   S^T = K Q^T and O^T += V^T P^T, as st_score_bf16.hip: a lane has one row of its wavefront's 32.
// Pages in bf16 come to LDS by direct loads; those in 8 bits through registers, where they become bf16 by a power of two, exactly, once for
// the workgroup's 128 rows.  Probabilities are rounded to bf16 for the second product, 2^-8 relative at most (as in st_score_bf16.hip: a second
// part is half of all matrix instructions more); those of sequences whose rows fit one tile meet it in two parts, 2^-16, as everywhere else.
//
// Bound by the matrix and the vector unit in turn: 2048 rows against 18432 tokens in 8 bits (32/8 heads of 128, 584 GFLOP) take 620 to 685 us
// as cards differ, 850 to 940 TFLOP/s; of all cycles the matrix units are busy 41 %, exponentials, sums and conversions take about as many, and
// two wavefronts on a SIMD, which is what 128 accumulators and operands leave room for, overlap little of both.  Raised priority around the
// products won 1 % here and lost 2 % of mixed batches; conversions spread over the products' loop lost more than they hid.
#include <type_traits>

#include "st_cache_plan.h"
#include "st_score.h"

namespace st {
namespace {

constexpr int kRows = kPromptRows, kBN = kPromptKeys;
constexpr float kSumMost = 4096.f;                   // a lane's sum over sixteen keys beyond which a row's reference moves

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= 3.402823466e38f; }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Whether 32 rows of an LDS tile hold an infinity or NaN: their products with zeros are NaN then
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

__device__ __forceinline__ void landed() {
  wait_vmcnt<0>();
  __syncthreads();
}

// The tiles of a workgroup's walk in the order it takes them: first the general ones, which a mask edge crosses (all of them where a page is
// missing) or in which a biased row lies, then the whole ones, those before the rows from the nearest one down, those behind them from the
// nearest one up.  General are [t0, a0), [a1, a2) and [a3, t1), whole [a0, a1) and [a2, a3).
struct TileWalk {
  int t0, a0, a1, a2, a3, t1, n_gen;
  __device__ __forceinline__ int tile(int n) const {
    if (n < n_gen) {
      if (n < t1 - a3) return t1 - 1 - n;
      n -= t1 - a3;
      return n < a2 - a1 ? a2 - 1 - n : a0 - 1 - (n - (a2 - a1));
    }
    n -= n_gen;
    return n < a1 - a0 ? a1 - 1 - n : a2 + n - (a1 - a0);
  }
};

template <typename S, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void cache_prompt_kernel(const CacheAttnArgs a) {
  constexpr bool E4M3 = std::is_same<S, uint8_t>::value;
  constexpr int KB = kBN / 32, KS = D / 16, DB = D / 32;
  constexpr int kTile = kBN * D * 2;
  constexpr int PASSES = kBN * D / 16 / 256;           // 16-byte pieces of a tile in 8 bits a thread: 2 or 1
  __shared__ __attribute__((aligned(1024))) char smem_raw[4 * kTile];   // 2 stages x (K, V)
  __shared__ int missing;
  ST_LDS char* smem = (ST_LDS char*)smem_raw;
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 5, r = lane & 31, G = a.Hq / c.Hkv;
  SeqSpan s;
  const CacheItem t = find_item<kRows, kBN>(a, s);
  if (t.b < 0) return;
  const int all_rows = s.r.n * G;
  tell_rows<kRows>(a, s, t, G);
  if (tid == 0) missing = 0;

  const int R = t.tile * kRows + wave * 32 + r, row = min(R, all_rows - 1), i = row / G, h = t.hk * G + row - i * G;
  const RowSpan see = row_span(a, s, i);
  bf16x8 qf[KS];
  const char* qrow = (const char*)a.q.ptr + ((int64_t)(s.r.first + i) * a.q.ss + (int64_t)h * a.q.sh) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qrow + (16 * ks + 8 * g) * 2);

  // what the workgroup's rows see, and those of the wavefront
  const int first = t.tile * kRows, last = min(first + kRows, all_rows) - 1;
  const RowSpan x0 = row_span(a, s, first / G), x1 = row_span(a, s, last / G);
  const int w_first = min(first + wave * 32, last), w_last = min(first + wave * 32 + 31, last);
  const RowSpan y0 = row_span(a, s, w_first / G), y1 = row_span(a, s, w_last / G);
  const int32_t* table = c.table + (int64_t)t.b * c.width;
  TileWalk walk;
  walk.t0 = x0.lo / kBN;
  walk.t1 = max((x1.hi + kBN - 1) / kBN, walk.t0);
  __syncthreads();
  bool hole = false;                                   // a page that is not there makes every tile a general one
  for (int p = (walk.t0 * kBN >> c.shift) + tid; p < c.width && ((int64_t)p << c.shift) < (int64_t)x1.hi; p += 256) {
    const int page = table[p];
    hole = hole || page < 0 || page >= c.n_pages;
  }
  if (__any(hole) && lane == 0) missing = 1;
  __syncthreads();
  walk.a0 = min(max((x1.lo + kBN - 1) / kBN, walk.t0), walk.t1);
  walk.a3 = max(min(x0.hi / kBN, walk.t1), walk.a0);
  // Rows that fit one tile have probabilities in two parts, as those of other kernels, whatever batch their sequence is in, and general tiles
  const bool fine = all_rows <= kRows;
  if (missing || fine) walk.a0 = walk.a3 = walk.t1;
  walk.a1 = walk.a2 = walk.a3;
  if (BIAS) {                                          // whole: with all rows on one side
    const int64_t p0 = s.pos + first / G, p1 = s.pos + last / G;
    walk.a1 = max(min((int)(min(max(p0 + 1, (int64_t)0), (int64_t)s.len) / kBN), walk.a3), walk.a0);
    walk.a2 = max(min((int)((min(max(p1, (int64_t)0), (int64_t)s.len) + kBN - 1) / kBN), walk.a3), walk.a1);
  }
  walk.n_gen = walk.a0 - walk.t0 + walk.a2 - walk.a1 + walk.t1 - walk.a3;
  const int n_all = walk.t1 - walk.t0;
  const int n0 = (int)((int64_t)n_all * t.share / t.shares), n1 = (int)((int64_t)n_all * (t.share + 1) / t.shares);

  ScoreConst k;
  k.c = CAP ? 2.f * kScoreLog2e * (a.scale / a.cap) : a.scale * kScoreLog2e;
  k.k1 = a.cap * kScoreLog2e;
  const float slope = BIAS ? a.slopes[h] : 0.f, slope2 = slope * kScoreLog2e;
  int near = 0;                                        // the nearest token that the row sees
  float besides = 0.f;                                 // what the bias of that one adds to lse
  if (BIAS && see.lo < see.hi) {
    const int64_t p = s.pos + i;
    near = (int)min(max(p, (int64_t)see.lo), (int64_t)see.hi - 1);
    besides = -slope * (float)(p > near ? p - near : near - p);
  }

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  float m_run = kUnset, l_run = 0.f;
  bool bad = false;

  const char* kb_ = (const char*)c.k.ptr + (int64_t)t.hk * c.k.sh * (int)sizeof(S);
  const char* vb_ = (const char*)c.v.ptr + (int64_t)t.hk * c.v.sh * (int)sizeof(S);
  const uint32_t smem_addr = (uint32_t)(uintptr_t)smem;

  // Pages of a tile's four runs of 16 keys, run x in lanes x, x + 4, ...; in 8 bits their scales beside them, of keys in lanes 0 .. 3, of values in 4 .. 7
  auto pages_at = [&](int tile) {
    const int p = table[min((tile * kBN + 16 * (lane & 3)) >> c.shift, c.width - 1)];
    return p >= 0 && p < c.n_pages ? p : -1;
  };
  auto scales_at = [&](int pages) -> int {
    if constexpr (!E4M3) return 0;
    else return (lane & 4 ? c.v_scale : c.k_scale)[(int64_t)max(pages, 0) * c.Hkv + t.hk];
  };
  auto run_base = [&](const char* base, const View& v, int pages, int tile, int run) {
    const int p = max(__builtin_amdgcn_readlane(pages, run), 0);
    return base + ((int64_t)p * v.sb + (int64_t)((tile * kBN + 16 * run) & ((1 << c.shift) - 1)) * v.ss) * (int)sizeof(S);
  };
  u32x4 raw[E4M3 ? 2 * PASSES : 1];
  constexpr int kPieces = D / 16;                      // of a row in 8 bits; a wavefront takes 64 / kPieces rows, all of one run
  // in an order in which sixteen lanes' stores to LDS meet no bank twice: four (two) rows apart where the swizzle differs in its last bit
  const int at_row = lane / kPieces, my_row = wave * (64 / kPieces) + (D == 128 ? (at_row & 1) * 4 + (at_row >> 1) : (at_row & 1) | (at_row >> 1 & 1) << 2 | (at_row >> 2 & 1) << 1 | (at_row >> 3) << 3);
  auto load_raw = [&](int tile, int pages) {
    if constexpr (E4M3) {
#pragma unroll
      for (int x = 0; x < PASSES; ++x) {
        const int row = x * (256 / kPieces) + my_row, run = x * (256 / kPieces / 16) + wave * (64 / kPieces) / 16;
        raw[x] = *reinterpret_cast<const u32x4*>(run_base(kb_, c.k, pages, tile, run) + (row & 15) * c.k.ss + (tid % kPieces) * 16);
        raw[PASSES + x] = *reinterpret_cast<const u32x4*>(run_base(vb_, c.v, pages, tile, run) + (row & 15) * c.v.ss + (tid % kPieces) * 16);
      }
    }
  };
  auto store_raw = [&](int scales, int stage) {
    if constexpr (E4M3) {
#pragma unroll
      for (int x = 0; x < 2 * PASSES; ++x) {
        const int y = x % PASSES, row = y * (256 / kPieces) + my_row, run = y * (256 / kPieces / 16) + wave * (64 / kPieces) / 16, chunk = 2 * (tid % kPieces);
        const float sc = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(scales, run + (x < PASSES ? 0 : 4)) << 23);
        ST_LDS char* to = smem + (2 * stage + (x < PASSES ? 0 : 1)) * kTile;
        auto pair = [&](uint32_t w, bool high) {
          return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, true))
                      : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, false));
        };
#pragma unroll
        for (int z = 0; z < 2; ++z)
          *reinterpret_cast<ST_LDS u32x4*>(to + swz<D>(row, chunk + z)) =
              u32x4{pair(raw[x][2 * z], false), pair(raw[x][2 * z], true), pair(raw[x][2 * z + 1], false), pair(raw[x][2 * z + 1], true)};
      }
    }
  };
  // direct loads of a tile in bf16: a wavefront's instruction covers 64 / (D / 8) rows, all of one run
  auto load_direct = [&](int tile, int pages, int stage) {
    if constexpr (!E4M3) {
      constexpr int PPR = D / 8, RPI = 64 / PPR, N = kBN / RPI / 4;
      const int rl = lane / PPR;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int row = (j * 4 + wave) * RPI, run = row / 16, at = row + rl;
        const uint32_t off = (uint32_t)(swz<D>(at, lane % PPR) - at * D * 2);      // the piece that belongs at this place
        dma16_asm(run_base(kb_, c.k, pages, tile, run) + (int64_t)(at & 15) * c.k.ss * 2 + off, smem_addr + 2 * stage * kTile + row * D * 2);
        dma16_asm(run_base(vb_, c.v, pages, tile, run) + (int64_t)(at & 15) * c.v.ss * 2 + off, smem_addr + (2 * stage + 1) * kTile + row * D * 2);
      }
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
  // seen: the keys' runs of 16 that have a page (general tiles)
  auto softmax = [&](auto general, Block& y, int key0, int seen, u32x4* rest = nullptr) {
    constexpr bool GEN = decltype(general)::value;
    const int d0 = near - key0 - 4 * g;
    const ScoreTile<CAP, BIAS> f(k, slope2, d0);
    const float side = d0 > 0 ? f.slope : -f.slope;    // (before the row the bias rises with the key)
    const float off = BIAS && !GEN ? slope2 * fabsf((float)d0) : 0.f;
    const int l0 = see.lo - key0 - 4 * g, h0 = see.hi - key0 - 4 * g;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = 8 * (v / 4) + v % 4;
      y.sc[v] = GEN ? f.raw(y.sc[v], key) : f.raw_side(y.sc[v], key, side);
      if (GEN) y.sc[v] = key >= l0 && key < h0 && (seen >> (v / 8) & 1) ? y.sc[v] : f.lowest();
    }
    // The reference of the exponents is lazy: it moves where the block's sum says that some exponent was large
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
      for (int e = 0; e < 4; ++e) {
        const float a0 = p[8 * m + 2 * e], a1 = p[8 * m + 2 * e + 1];
        y.pf[m][e] = pack_bf16(a0, a1);
        if (rest) rest[m][e] = pack_bf16(a0 - __uint_as_float(y.pf[m][e] << 16), a1 - __uint_as_float(y.pf[m][e] & 0xffff0000u));
      }
  };
  auto contract = [&](auto scrub, const u32x4* pf, uint32_t vtile, const u32x4* rest = nullptr) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        bf16x8 vf = reads.frag_tr(vtile, 16 * m, db);
        if (decltype(scrub)::value) vf = finite_bf16(vf);
        acc[db] = mfma32(vf, __builtin_bit_cast(bf16x8, pf[m]), acc[db]);
        if (rest) acc[db] = mfma32(vf, __builtin_bit_cast(bf16x8, rest[m]), acc[db]);
      }
  };

  // A tile's values are under way while the one before is worked on, its pages one tile longer.
  int n = n0, buf = 0, pages = 0, pages_next = 0, scales_next = 0;
  auto tile_of = [&](int n) { return walk.tile(min(n, n1 - 1)); };
  if (n < n1) {
    pages = pages_at(tile_of(n));
    pages_next = pages_at(tile_of(n + 1));
    const int scales = scales_at(pages);
    load_raw(tile_of(n), pages);
    load_direct(tile_of(n), pages, 0);
    store_raw(scales, 0);
  }
  landed();
  int pages_then = 0;
  auto fetch = [&]() {                                 // of the next tile; all of its addresses are there, past the end the last one's again
    if (n + 1 < n1) {
      scales_next = scales_at(pages_next);
      load_raw(tile_of(n + 1), pages_next);
      load_direct(tile_of(n + 1), pages_next, buf ^ 1);
      pages_then = pages_at(tile_of(n + 2));
    }
  };
  auto arrived = [&]() {
    if (n + 1 < n1) store_raw(scales_next, buf ^ 1);
    landed();
    pages = pages_next;
    pages_next = pages_then;
    buf ^= 1;
  };
  for (; fine && n < n1; ++n) {                        // a block at a time: registers for the second parts
    fetch();
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
#pragma unroll 1
    for (int kb = 0; kb < KB; ++kb) {
      const int at = key0 + 32 * kb;
      if (first + wave * 32 > last || y0.lo >= at + 32 || y1.hi <= at) continue;      // no rows, or none that sees any of the block
      const uint32_t vblock = ktile + kTile + 32 * kb * D * 2;
      const int seen = (__builtin_amdgcn_readlane(pages, 2 * kb) >= 0 ? 1 : 0) | (__builtin_amdgcn_readlane(pages, 2 * kb + 1) >= 0 ? 2 : 0);
      const bool dirty = (seen != 3 || y1.lo > at || y0.hi < at + 32) && not_finite<D>(reads, vblock);
      bad = bad || dirty;
      Block y;
      u32x4 rest[2];
      products(y, ktile + 32 * kb * D * 2);
      softmax(std::true_type(), y, at, seen, rest);
      if (__builtin_expect(dirty, 0)) contract(std::true_type(), y.pf, vblock, rest);
      else contract(std::false_type(), y.pf, vblock, rest);
    }
    arrived();
  }
  for (; n < min(n1, walk.n_gen); ++n) {
    fetch();
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
    if (y0.lo < key0 + kBN && y1.hi > key0) {          // some row of this wavefront may see some key of the tile
      Block y[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) products(y[kb], ktile + 32 * kb * D * 2);
      const bool cut = missing || y1.lo > key0 || y0.hi < key0 + kBN;
      const bool dirty = cut && (not_finite<D>(reads, ktile + kTile) || not_finite<D>(reads, ktile + kTile + 32 * D * 2));
      bad = bad || dirty;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t vblock = ktile + kTile + 32 * kb * D * 2;
        const int seen = (__builtin_amdgcn_readlane(pages, 2 * kb) >= 0 ? 1 : 0) | (__builtin_amdgcn_readlane(pages, 2 * kb + 1) >= 0 ? 2 : 0);
        softmax(std::true_type(), y[kb], key0 + 32 * kb, seen);
        if (__builtin_expect(dirty, 0)) contract(std::true_type(), y[kb].pf, vblock);
        else contract(std::false_type(), y[kb].pf, vblock);
      }
    }
    arrived();
  }
  for (; n < n1; ++n) {
    fetch();
    const int key0 = walk.tile(n) * kBN;
    const uint32_t ktile = smem_addr + buf * 2 * kTile;
    // both blocks' products first: the second's run over the softmax of the first
    Block y[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) products(y[kb], ktile + 32 * kb * D * 2);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      softmax(std::false_type(), y[kb], key0 + 32 * kb, 3);
      contract(std::false_type(), y[kb].pf, ktile + kTile + 32 * kb * D * 2);
    }
    arrived();
  }

  // ---- O = acc / l, lse = m ln 2 + ln l; or the state of a share
  const float l = xhalf_sum(l_run);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) bad = bad || !is_finite(acc[db][v]);
  if (__builtin_expect(__any(bad), 0)) {
    // Values that are not finite: general tiles left them out, and in whole ones an infinity times a probability that bf16 does not hold is
    // NaN.  What of them a row sees is what its columns have.  A lane looks at a key of the tile, then all at the columns of those that have any.
    uint32_t had[DB];                                  // columns that met one, a bit each
#pragma unroll
    for (int db = 0; db < DB; ++db) had[db] = 0;
    for (int y = n0; y < n1; ++y) {
      const int key0 = walk.tile(y) * kBN, mine = key0 + lane;
      auto row_of = [&](int key, int page) {
        return (const S*)(vb_ + ((int64_t)page * c.v.sb + (int64_t)(key & ((1 << c.shift) - 1)) * c.v.ss) * (int)sizeof(S));
      };
      auto value = [&](S x, float scale) {
        if constexpr (E4M3) return e4m3_pair<false>(x).x * scale;
        else return __uint_as_float((uint32_t)x << 16);
      };
      const int page = mine < y1.hi ? page_of(c, t.b, mine >> c.shift) : -1;
      float scale = 1.f;
      uint32_t some = 0;
      if (page >= 0) {
        const uint32_t byte = E4M3 ? c.v_scale[(int64_t)page * c.Hkv + t.hk] : 127, more = E4M3 ? e4m3_beyond(byte) : 0x00800080u;
        const uint32_t bits = E4M3 ? 0x7f7f7f7fu : 0x7fff7fffu;
        scale = scale_value((uint8_t)byte);
        const S* from = row_of(mine, page);
        for (int d = 0; d < D; d += 16 / (int)sizeof(S)) {
          const u32x4 z = *reinterpret_cast<const u32x4*>(from + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) some |= ((z[e] & bits) + more) & ~bits;
        }
      }
      for (uint64_t left = __ballot(some != 0); left; left &= left - 1) {
        const int at = __ffsll((unsigned long long)left) - 1, key = key0 + at;
        const S* from = row_of(key, __builtin_amdgcn_readlane(page, at));
        const float sc = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(scale), at));
        if (key < see.lo || key >= see.hi || l != l) continue;      // (a score that is NaN makes all columns so)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float z = value(from[32 * db + 8 * (v / 4) + 4 * g + v % 4], sc);
            const uint32_t lost = is_finite(z) ? 0 : 1u << v;
            acc[db][v] = lost ? (had[db] & lost ? acc[db][v] : 0.f) + z : acc[db][v];
            had[db] |= lost;
            if (v % 4 == 3) asm volatile("" ::: "memory");         // (four at a time: masks of more have no registers)
          }
      }
    }
  }
  if (R >= all_rows) return;
  const bool part = t.shares > 1;
  const float inv = part ? 1.f : l != 0.f ? 1.f / l : 0.f;
  const int64_t state = a.plan.base + (int64_t)t.state * kRows + wave * 32 + r;
  const int64_t orow = part ? state * D : ((int64_t)(s.r.first + i) * a.Hq + h) * D;
  float* o = part ? a.part_o : a.o;
  uint16_t* olow = part ? nullptr : (uint16_t*)a.o_lowp;
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
    if (part) a.part_row[state] = make_float4(m_run, l, besides, 0.f);
    else a.lse[(int64_t)h * a.T + s.r.first + i] = l != 0.f ? m_run * kScoreLn2 + logf(l) + besides : -INFINITY;
  }
}

}  // namespace

hipError_t launch_cache_prompt(const CacheAttnArgs& a, hipStream_t stream) {
  if (a.plan.grid <= 0 || a.plan.grid > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("cache_prompt", stream);
  const dim3 grid((unsigned)a.plan.grid), block(256);
  auto go = [&](auto plain, auto cap, auto bias, auto both) {
    hipLaunchKernelGGL(a.cap > 0.f ? (a.slopes ? both : cap) : a.slopes ? bias : plain, grid, block, 0, stream, a);
  };
#define ST_PROMPT(S, D) go(cache_prompt_kernel<S, D, false, false>, cache_prompt_kernel<S, D, true, false>, cache_prompt_kernel<S, D, false, true>, cache_prompt_kernel<S, D, true, true>)
  if (a.c.dtype == ST_E4M3) a.c.D == 128 ? ST_PROMPT(uint8_t, 128) : ST_PROMPT(uint8_t, 64);
  else a.c.D == 128 ? ST_PROMPT(uint16_t, 128) : ST_PROMPT(uint16_t, 64);
#undef ST_PROMPT
  return hipGetLastError();
}

}  // namespace st
