// Small passes beside the kernels of attention with modified scores: the row spans of documents and prefixes, what runs of 32 rows
// see, and the sum of the shares of split gradients.
#include "st_score.h"

namespace st {
namespace {

// Row at position p of a packed batch entry: its document is the last one that starts at or before p (empty documents start where
// the next one does, and are passed over).  bounds [B, n_docs + 1] rise; a row before the first or behind the last sees nothing.
// A launch's time (2.5 us for 8192 rows of 8 documents); counting the bounds, loads side by side, instead of searching is no faster.
__global__ __launch_bounds__(256) void mask_spans_kernel(const Shape s, const int64_t* __restrict__ bounds, int32_t n_docs, const int64_t* __restrict__ prefix, int64_t* __restrict__ spans) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= (int64_t)s.B * s.Sq) return;
  const int64_t b = x / s.Sq, p = q_pos(s, (int)(x - b * s.Sq));
  const int64_t* e = bounds + b * (n_docs + 1);
  int lo = 0, hi = n_docs + 1;                         // entries before lo are <= p, those from hi on are not
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (e[mid] <= p) lo = mid + 1;
    else hi = mid;
  }
  longlong2 w = make_longlong2(0, 0);
  if (lo >= 1 && lo <= n_docs) {
    w.x = e[lo - 1];
    w.y = e[lo];
    if (s.causal) {
      const int64_t len = w.y - w.x, pre = prefix ? min(max(prefix[b * n_docs + lo - 1], (int64_t)0), len) : 0;
      w.y = min(w.y, max(p + 1, w.x + pre));
    }
  }
  *reinterpret_cast<longlong2*>(spans + 2 * x) = w;
}

// Half a wavefront per run of 32 packed rows of a KV head: what every key tile needs to know of them, made once (2 us of kernel for
// 32/8 heads x 8192 rows; every key tile reads 128 bytes a row otherwise strewn over lse, Delta and spans).
__global__ __launch_bounds__(256) void score_rows_kernel(const ScoreArgs a, int32_t n_blk) {
  const int64_t x = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, n = (int64_t)a.s.B * a.s.Hkv * n_blk;
  const int r = threadIdx.x & 31, G = a.s.Hq / a.s.Hkv, M = a.s.Sq * G;
  const int64_t at = min(x, n - 1), bh = at / n_blk;
  const int j = (int)(at - bh * n_blk), b = (int)(bh / a.s.Hkv), hk = (int)(bh - (int64_t)b * a.s.Hkv);
  const int R = 32 * j + r, row = min(R, M - 1), i = row / G, h = hk * G + row - i * G;
  const int64_t stat = ((int64_t)b * a.s.Hq + h) * a.s.Sq + i;
  const float lse = a.lse_in[stat], slope = a.slopes ? a.slopes[h] : 0.f;
  RowView see = row_view(a, b, i);
  const bool none = R >= M || lse == -INFINITY;        // a row that does not exist, or an empty one: P = 0
  if (none) see.lo = see.hi = 0;
  BlockSpan w = span_of(see);
#pragma unroll
  for (int d = 1; d < 32; d *= 2)
    w = span_join(w, BlockSpan{__shfl_xor(w.lo, d), __shfl_xor(w.hi, d), __shfl_xor(w.all_lo, d), __shfl_xor(w.all_hi, d)});
  if (x >= n) return;
  if (r == 0) a.blocks[x] = make_int4(w.lo, w.hi, w.all_lo, w.all_hi);
  float* f = a.rows + x * kRowStats + r;
  f[32 * kRowLse] = none ? INFINITY : (fmaf(slope, see.rest, lse) - a.cap) * kScoreLog2e;
  f[32 * kRowDelta] = -a.delta[stat];
  f[32 * kRowLo] = __int_as_float(see.lo);
  f[32 * kRowHi] = __int_as_float(see.hi);
  f[32 * kRowX] = (float)see.x;
  f[32 * kRowSlope] = slope * kScoreLog2e;
}

// Many partial states of few rows (a split walk of a token or a few): a workgroup per row, eight states side by side, where the
// general combine has a thread go through all of them (64 states of 32 rows of 128: 55 us).  Weights as there: an empty state is 0
// whatever its O holds, a row that is empty in all of them stays empty, one that is NaN in any of them becomes NaN.
__global__ __launch_bounds__(256) void score_combine_kernel(const float* __restrict__ o, const float* __restrict__ lse, int32_t n, int32_t Sq, int32_t Hq, int32_t D,
                                                            int64_t n_rows, float* o_out, float* __restrict__ lse_out, void* low, int32_t bf16) {
  __shared__ float w[kMaxTable];
  __shared__ float4 fold[256];
  const int64_t row = blockIdx.x;                      // (b Sq + i) Hq + h
  const int64_t bi = row / Hq, h = row - bi * Hq, b = bi / Sq, i = bi - b * Sq, stat = (b * Hq + h) * Sq + i;
  const int tid = threadIdx.x, vecs = D / 4, lanes = 256 / vecs;
  if (tid < 64) {
    const float l = tid < n ? lse[tid * n_rows + stat] : -INFINITY;
    float m = l;
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    // (fmaxf passes over NaN: with none but such states beside empty ones the sum of all lse is NaN, with empty ones alone -inf)
    const bool none = m == -INFINITY;
    const float e = none ? l : expf(l - m);
    float sum = e;
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    w[tid] = !none ? e / sum : sum == -INFINITY ? 0.f : sum;
    if (tid == 0) lse_out[stat] = none ? sum : m + logf(sum);
  }
  __syncthreads();
  const int x = tid % vecs, y = tid / vecs;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  if (y < lanes)
    for (int k0 = y; k0 < n; k0 += 4 * lanes) {        // four loads in flight
      float4 p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) p[u] = *reinterpret_cast<const float4*>(o + (min(k0 + u * lanes, n - 1) * n_rows + row) * D + 4 * x);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float c = k0 + u * lanes < n ? w[k0 + u * lanes] : 0.f;
        if (c != 0.f) r = make_float4(fmaf(c, p[u].x, r.x), fmaf(c, p[u].y, r.y), fmaf(c, p[u].z, r.z), fmaf(c, p[u].w, r.w));
      }
    }
  fold[tid] = r;
  __syncthreads();
  if (y != 0) return;
  for (int k = 1; k < lanes; ++k) {
    const float4 p = fold[k * vecs + x];
    r.x += p.x; r.y += p.y; r.z += p.z; r.w += p.w;
  }
  if (o_out) *reinterpret_cast<float4*>(o_out + row * D + 4 * x) = r;
  if (low && bf16) *reinterpret_cast<uint2*>((uint16_t*)low + row * D + 4 * x) = make_uint2(pack_bf16(r.x, r.y), pack_bf16(r.z, r.w));
  else if (low) *reinterpret_cast<float4*>((float*)low + row * D + 4 * x) = r;
}

struct PartSum {
  const float* part;         // n sums of `floats` floats, one behind the other; null: nothing to add up
  float* out;                // nullable; added to unless assign
  void* low;                 // nullable
  int32_t n;
  int64_t floats;
};
struct PartSums {
  PartSum x[3];
  int32_t assign, bf16;
};
// Four neighbouring floats a thread, in the order of the shares: memory-bound (two shares of dK and dV of 8 KV heads x 8192 keys of 128,
// to bf16: 33 us, 5 TB/s).
__global__ __launch_bounds__(256) void score_add_parts_kernel(const PartSums a) {
  const PartSum& p = a.x[blockIdx.y];
  for (int64_t e = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); e < p.floats && p.part; e += (int64_t)gridDim.x * 1024) {
    float4 y = *reinterpret_cast<const float4*>(p.part + e);
    for (int k = 1; k < p.n; ++k) {
      const float4 z = *reinterpret_cast<const float4*>(p.part + k * p.floats + e);
      y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
    }
    if (!a.assign) {
      const float4 z = *reinterpret_cast<const float4*>(p.out + e);
      y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
    }
    if (p.out) *reinterpret_cast<float4*>(p.out + e) = y;
    if (p.low && a.bf16) *reinterpret_cast<uint2*>((uint16_t*)p.low + e) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    else if (p.low) *reinterpret_cast<float4*>((float*)p.low + e) = y;
  }
}

}  // namespace

int score_split(int64_t jobs, int64_t slots, int64_t steps, int64_t least_steps, int most) {
  if (jobs <= 0) return 1;
  int64_t n = slots / jobs;
  n = n > most ? most : n;
  n = n > steps / least_steps ? steps / least_steps : n;
  return n < 1 ? 1 : (int)n;
}

hipError_t launch_mask_spans(const Shape& s, const int64_t* bounds, int32_t n_docs, const int64_t* prefix, int64_t* spans, hipStream_t stream) {
  const int64_t n = (int64_t)s.B * s.Sq;
  if (n <= 0) return hipSuccess;
  if ((n + 255) / 256 > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("mask_spans", stream);
  hipLaunchKernelGGL(mask_spans_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, s, bounds, n_docs, prefix, spans);
  return hipGetLastError();
}

hipError_t launch_score_combine(const ScoreArgs& a, int bf16, hipStream_t stream) {
  const int64_t rows = (int64_t)a.s.B * a.s.Sq * a.s.Hq;
  if (rows > kScoreGridMost || a.n_split > kMaxTable) return hipErrorInvalidValue;
  ProfScope prof("score_combine", stream);
  hipLaunchKernelGGL(score_combine_kernel, dim3((unsigned)rows), dim3(256), 0, stream, a.part_o, a.part_lse, a.n_split, a.s.Sq, a.s.Hq, a.s.D, rows, a.o, a.lse, a.o_lowp, bf16);
  return hipGetLastError();
}

hipError_t launch_score_rows(const ScoreArgs& a, hipStream_t stream) {
  const int64_t n_blk = ((int64_t)a.s.Sq * (a.s.Hq / a.s.Hkv) + 31) / 32, n = n_blk * a.s.B * a.s.Hkv;
  if (n <= 0) return hipSuccess;
  if ((n + 7) / 8 > kScoreGridMost) return hipErrorInvalidValue;
  ProfScope prof("score_rows", stream);
  hipLaunchKernelGGL(score_rows_kernel, dim3((unsigned)((n + 7) / 8)), dim3(256), 0, stream, a, (int32_t)n_blk);
  return hipGetLastError();
}

hipError_t launch_score_add_parts(const ScoreArgs& a, int bf16, hipStream_t stream) {
  PartSums p{};
  const int64_t n_q = (int64_t)a.s.B * a.s.Sq * a.s.Hq * a.s.D, n_kv = (int64_t)a.s.B * a.s.Sk * a.s.Hkv * a.s.D;
  int64_t most = 0;
  if (a.q_split > 1) p.x[0] = PartSum{a.part_dq, a.dq, a.dq_lowp, a.q_split, n_q}, most = n_q;
  if (a.kv_split > 1) {
    p.x[1] = PartSum{a.part_dk, a.dk, a.dk_lowp, a.kv_split, n_kv};
    p.x[2] = PartSum{a.part_dv, a.dv, a.dv_lowp, a.kv_split, n_kv};
    most = most > n_kv ? most : n_kv;
  }
  if (most == 0) return hipSuccess;
  p.assign = a.assign;
  p.bf16 = bf16;
  const int64_t blocks = (most / 4 + 255) / 256;
  ProfScope prof("score_add_parts", stream);
  hipLaunchKernelGGL(score_add_parts_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096), 3), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace st
