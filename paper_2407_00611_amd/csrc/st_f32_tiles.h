// Tiles of the fp32 kernels (st_f32.hip, st_score_f32.hip): operand loads, contractions on v_mfma_f32_32x32x2_f32, the fold of a
// workgroup's wavefronts, and the table of key tiles.
#pragma once

#include <type_traits>

#include "st_internal.h"
#include "st_mfma.h"
#include "st_walk.h"

namespace st {
namespace {

constexpr int kT = 32;             // rows of every tile

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// wavefronts per workgroup: eight (two per SIMD, which hide each other's loads) as long as a wavefront's accumulators
// and operands fit 256 registers
template <int DP>
constexpr int waves() { return DP <= 128 ? 8 : 4; }

// number of leading keys of a chunk that query position qpos may see
__device__ __forceinline__ int visible_keys(const Shape& s, int64_t qpos, int64_t k0) {
  if (!s.causal) return s.Sk;
  int64_t n = qpos - k0 + 1;
  return n < 0 ? 0 : (n > s.Sk ? s.Sk : (int)n);
}

// row of a tile that register v of a C tile holds in half g
__device__ __forceinline__ int c_row(int v, int g) { return 8 * (v / 4) + 4 * g + v % 4; }

// ---- streamed operands, in pieces of N (32 or 16) registers.  While one piece is contracted (N instructions of 64
// cycles) the next one is on its way; two pieces and the accumulators are what fits beside a second wavefront.
// FULL: D == DP.  Otherwise the columns at or beyond D read as zero.
template <int N>
struct Piece {
  float x[N];
};
template <int DP, int N>
constexpr int row_pieces() { return (DP + 2 * N - 1) / (2 * N); }           // 2 N columns each
template <int DP, int N>
constexpr int piece_rows() {                                                // registers v of a C tile per column piece
  int n = 16;
  while (n * (DP / 32) > N) n /= 2;
  return n;
}
template <int DP, int N>
constexpr int col_pieces() { return 16 / piece_rows<DP, N>(); }

// Row r of a tile as the k-along-D operand: columns 2 N n + 8 j + 4 g .. + 3
template <int DP, bool FULL, int N>
__device__ __forceinline__ void load_rows(Piece<N>& f, const float* row, int n, int D, int g) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    const int d = 2 * N * n + 8 * j;
    if (d >= DP) continue;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (FULL || d < D) x = *reinterpret_cast<const float4*>(row + d + 4 * g);
    f.x[4 * j] = x.x; f.x[4 * j + 1] = x.y; f.x[4 * j + 2] = x.z; f.x[4 * j + 3] = x.w;
  }
}

// a pointer said to be global, where the compiler does not see it (it would load with flat loads, which wait for LDS too)
typedef const __attribute__((address_space(1))) float* GlobalFloats;
__device__ const __attribute__((aligned(16))) float zero_row[256] = {};
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
// The column that row m of accumulator db stands for, which is free as long as the results are stored so (acc_block).  A lane's
// columns are neighbours, one load of up to four floats a row, where their number is even.  Three would be three loads again, at
// strides of three floats: head size 96 has them 32 apart, a row's loads of a wavefront in one piece.
template <int DB>
__device__ __forceinline__ constexpr int column(int m, int db) { return DB % 2 == 0 ? DB * m + db : 32 * db + m; }
// The transposed operand of a tile X: lane r = columns column(r, 0 .. DB - 1), register v = row c_row(v, g).
// Rows at or beyond `limit` (tile-relative, >= 1) are zero: their weight is, but a row that exists, read in their place, may
// hold an infinity, and 0 * inf is NaN.
template <int DP, bool FULL, int N>
__device__ __forceinline__ void load_cols(Piece<N>& f, const float* tile, int64_t stride, int limit, int n, int D, int r, int g) {
  constexpr int DB = DP / 32;
  int mine = limit - 4 * g;
  asm volatile("" : "+v"(mine));                     // compared anew for every piece: kept, the masks of all rows spill
#pragma unroll
  for (int u = 0; u < piece_rows<DP, N>(); ++u) {
    const int v = n * piece_rows<DP, N>() + u, row = 8 * (v / 4) + v % 4;
    GlobalFloats p = (GlobalFloats)tile + (int64_t)(4 * g) * stride + (int64_t)row * stride;
    if (limit < kT) p = row < mine ? p : (GlobalFloats)zero_row;
    p += column<DB>(r, 0);
    float* x = f.x + DB * u;
    if constexpr (DB % 2 == 0) {
      constexpr int W = DB % 4 == 0 ? 4 : 2;
      typedef typename std::conditional<W == 4, f32x4v, f32x2v>::type Vec;
#pragma unroll
      for (int q = 0; q < DB; q += W) {
        Vec y = {};
        if (FULL || DB * r + q < D) y = *reinterpret_cast<const __attribute__((address_space(1))) Vec*>(p + q);   // D is a multiple of 8
#pragma unroll
        for (int e = 0; e < W; ++e) x[q + e] = y[e];
      }
    } else {
#pragma unroll
      for (int db = 0; db < DB; ++db) x[db] = FULL || column<DB>(r, db) < D ? p[32 * db] : 0.f;
    }
  }
}

// ---- resident tile in LDS: kT rows of D floats, rows padded by 4 floats so that 16-byte reads of one column by
// consecutive rows spread over the banks; rows at or beyond `limit` and columns at or beyond D are zero
template <int DP>
constexpr int lds_stride() { return DP + 4; }
template <int DP>
__device__ __forceinline__ void stage_tile(float* lds, const float* base, int64_t stride, int row0, int limit, int D, int tid) {
  for (int p = tid; p < kT * (DP / 4); p += waves<DP>() * 64) {
    const int row = p / (DP / 4), d = p % (DP / 4) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row0 + row < limit && d < D) x = *reinterpret_cast<const float4*>(base + (int64_t)(row0 + row) * stride + d);
    *reinterpret_cast<float4*>(lds + row * lds_stride<DP>() + d) = x;
  }
}

// C tile (rows: the streamed tile's, columns: the LDS tile's rows) += contraction along its row piece n
template <int DP, int N>
__device__ __forceinline__ void contract_d(f32x16& c, const Piece<N>& f, const float* lds, int n, int r, int g) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    const int d = 2 * N * n + 8 * j;
    if (d >= DP) continue;
    const float4 y = *reinterpret_cast<const float4*>(lds + r * lds_stride<DP>() + d + 4 * g);
    c = mfma_f32(f.x[4 * j], y.x, c);
    c = mfma_f32(f.x[4 * j + 1], y.y, c);
    c = mfma_f32(f.x[4 * j + 2], y.z, c);
    c = mfma_f32(f.x[4 * j + 3], y.w, c);
  }
}

// acc^T[d][column] += sum over the rows of column piece n of X[row][d] w[row][column]
template <int DP, int N>
__device__ __forceinline__ void contract_rows(f32x16 (&acc)[DP / 32], const Piece<N>& f, const f32x16& w, int n) {
  constexpr int DB = DP / 32;
#pragma unroll
  for (int u = 0; u < piece_rows<DP, N>(); ++u)
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = mfma_f32(f.x[DB * u + db], w[n * piece_rows<DP, N>() + u], acc[db]);
}

// ---- infinities and NaN in a tile that a mask edge crosses.  The matrix instruction multiplies a row that a column
// does not see by a weight of zero, and 0 * inf is NaN; a row must not reach a column that it is masked from.  Such a
// tile ("dirty", found by reading it once more: only tiles on the edge are looked at) is contracted with those values
// taken as zero, and the workgroup adds them to the stored result of the columns that do see them.
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

__device__ __forceinline__ bool tile_dirty(const float* tile, int64_t stride, int limit, int D, int lane) {
  bool bad = false;
  for (int p = lane; p < limit * (D / 4); p += 64) {
    const float4 x = *reinterpret_cast<const float4*>(tile + (int64_t)(p / (D / 4)) * stride + p % (D / 4) * 4);
    bad = bad || !(finite(x.x) && finite(x.y) && finite(x.z) && finite(x.w));
  }
  return __any(bad);
}

template <int N>
__device__ __forceinline__ void scrub(Piece<N>& f) {
#pragma unroll
  for (int k = 0; k < N; ++k) f.x[k] = finite(f.x[k]) ? f.x[k] : 0.f;
}

// out[d] += X[t][d] wherever that is no finite number, for the rows t in [lo, hi); as_nan: their weight may have either sign
template <int DB>
__device__ __forceinline__ void add_nonfinite(float* out, float* out2, const float* x0, int64_t stride, int lo, int hi, int D, int g, bool as_nan) {
#pragma unroll 1
  for (int t = lo; t < hi; ++t)
#pragma unroll 1
    for (int d = 0; d < D; ++d) {
      const float x = x0[(int64_t)t * stride + d];
      if (((DB % 2 == 0 ? d / DB / 4 : d / 4) & 1) != g || finite(x)) continue;       // acc_block's half
      out[d] += as_nan ? __builtin_nanf("") : x;
      if (out2) out2[d] = out[d];
    }
}

template <int N>
__device__ __forceinline__ void zero_acc(f32x16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
}

// Four neighbouring results of a lane, the columns from block_column on: number q of the DB that block j of its accumulators holds
template <int DB>
__device__ __forceinline__ int block_column(int j, int q, int g) { return DB % 2 == 0 ? 4 * (DB * (2 * j + g) + q) : 32 * q + 8 * j + 4 * g; }
template <int DB>
__device__ __forceinline__ float4 acc_block(const f32x16 (&acc)[DB], int j, int q, float c) {
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = c * (DB % 2 == 0 ? acc[(4 * q + e) % DB][4 * j + (4 * q + e) / DB] : acc[q][4 * j + e]);
  return make_float4(x[0], x[1], x[2], x[3]);
}

__device__ __forceinline__ float4 add(float4 x, float4 y) { return make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); }

// One tree step of the fold of the wavefronts' accumulators: the upper half of `n` wavefronts puts its values down.
template <int N>
__device__ __forceinline__ void put_acc(float* slot, const f32x16 (&acc)[N], int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) slot[(16 * i + v) * 64 + lane] = acc[i][v];
}
template <int N>
__device__ __forceinline__ void add_acc(const float* slot, f32x16 (&acc)[N], float own, float other, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[i][v] = own * acc[i][v] + other * slot[(16 * i + v) * 64 + lane];
}

// The 32-key tiles a query tile's workgroups walk, numbered through the chunks.  A share is a run of them, and the workgroup's
// wavefronts take the tiles of the run in turn: shares differ by one tile at most, whatever the mask and the chunks (dealt out
// in turns of eight, 104 tiles make four shares of 32 and 24: 4 heads x 400 rows x 8 chunks of 400 keys at head size 128 59 us,
// 51 so).  The table is in LDS because arguments come from host memory: a read of them is 0.7 us, and every chunk that the
// walk comes to would need some.
struct KeyTable {
  int32_t end[kMaxTable];                            // tiles up to and with this chunk that the workgroup's last row sees
  int64_t k_offset[kMaxTable];
  const float* k[kMaxTable];                         // of this head and batch entry
  const float* v[kMaxTable];
};
// by one wavefront, a lane per chunk; a barrier has to follow
__device__ __forceinline__ void build_key_table(KeyTable& tab, const Shape& s, const ChunkTable& t, int64_t last_pos, int b, int hk, int lane) {
  static_assert(kMaxTable == 64, "a lane per chunk");
  const int64_t k0 = t.k_offset[lane];               // the whole table is read: the loads need not wait for its length
  const float* k = (const float*)t.k[lane] + (int64_t)b * t.ksb + (int64_t)hk * t.ksh;
  const float* v = (const float*)t.v[lane] + (int64_t)b * t.vsb + (int64_t)hk * t.vsh;
  const int n = lane < t.n ? (visible_keys(s, last_pos, k0) + kT - 1) / kT : 0;
  int total;
  tab.end[lane] = lane_scan(n, total) + n;
  tab.k_offset[lane] = k0;
  tab.k[lane] = k;
  tab.v[lane] = v;
}
// tiles [lo, hi) of share y
__device__ __forceinline__ void key_share(int end, int n_split, int y, int& lo, int& hi) {
  const uint32_t total = (uint32_t)__builtin_amdgcn_readlane(end, 63), n = (uint32_t)max(n_split, 1), each = total / n, rest = total % n;
  lo = (int)(each * y + rest * y / n);
  hi = (int)(each * (y + 1) + rest * (y + 1) / n);
}
// Tile x of the walk, x below the last `end`; end = this lane's entry of the table
struct KeyTile {
  int key0;                                          // first key in its chunk
  int64_t k_offset;
  const float *k, *v;                                // at that key
};
__device__ __forceinline__ uint64_t uniform64(uint64_t x) { return (uint64_t)sgpr((uint32_t)x) | (uint64_t)sgpr((uint32_t)(x >> 32)) << 32; }
__device__ __forceinline__ const float* uniform_ptr(const float* p) { return (const float*)(GlobalFloats)uniform64((uint64_t)p); }
__device__ __forceinline__ KeyTile key_tile(const KeyTable& tab, const ChunkTable& t, int end, int x) {
  const int c = __popcll(__ballot(end <= x));
  const int first = c > 0 ? __builtin_amdgcn_readlane(end, c - 1) : 0;
  KeyTile y;
  y.key0 = (x - first) * kT;
  y.k_offset = (int64_t)uniform64((uint64_t)tab.k_offset[c]);
  y.k = uniform_ptr(tab.k[c]) + (int64_t)y.key0 * t.kss;
  y.v = uniform_ptr(tab.v[c]) + (int64_t)y.key0 * t.vss;
  return y;
}

// f(integral constant, full): the kernels are built for these D, and for smaller ones with zero-filled columns
template <typename F>
hipError_t with_padded_d(int D, F f) {
  using std::integral_constant;
  constexpr integral_constant<bool, true> full;
  constexpr integral_constant<bool, false> padded;
  if (D == 64) return f(integral_constant<int, 64>(), full);
  if (D == 128) return f(integral_constant<int, 128>(), full);
  if (D == 256) return f(integral_constant<int, 256>(), full);
  if (D <= 32) return f(integral_constant<int, 32>(), padded);
  if (D <= 64) return f(integral_constant<int, 64>(), padded);
  if (D <= 96) return f(integral_constant<int, 96>(), padded);
  if (D <= 128) return f(integral_constant<int, 128>(), padded);
  if (D <= 192) return f(integral_constant<int, 192>(), padded);
  if (D <= 256) return f(integral_constant<int, 256>(), padded);
  return hipErrorInvalidValue;
}

}  // namespace
}  // namespace st
