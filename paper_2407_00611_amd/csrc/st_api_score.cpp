// C ABI of the attention with modified scores, of the row spans it takes, and of the norms and rotations of queries and keys:
// argument checks, workspace layout, launches.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "st_checks.h"
#include "st_rope.h"
#include "st_score.h"

using namespace st::checks;
using st::fail;
using st::hip_fail;

namespace {

st_status check_score(const st_block_desc* d, const st_score* m) {
  if (d == nullptr) return fail(ST_ERR_INVALID_ARG, "null descriptor");
  ST_TRY(check_shape(d->dtype, d->B, d->Hq, d->Hkv, d->D, d->Sq, d->Sk));
  ST_TRY(check_scale(d->scale));
  ST_TRY(check_segments(d->Sq, d->q_offset, d->q_seg, d->q_offset2));
  if ((int64_t)d->Sq * (d->Hq / d->Hkv) > 0x7fffff00) return fail(ST_ERR_UNSUPPORTED, "more than 2^31 rows of a KV head's group");
  const int64_t rows = d->dtype == ST_BF16 ? ((int64_t)d->Sq * (d->Hq / d->Hkv) + st::kScoreRows - 1) / st::kScoreRows * d->Hkv : ((int64_t)d->Sq + 31) / 32 * d->Hq;
  const int64_t keys = ((int64_t)d->Sk + 31) / 32 * d->Hkv * (d->dtype == ST_F32 ? st::score_f32_halves(d->D) : 1);
  if (std::max(rows, keys) * d->B > st::kScoreGridMost) return fail(ST_ERR_UNSUPPORTED, "more than %lld tiles", (long long)st::kScoreGridMost);
  if (m == nullptr) return ST_OK;
  if (!(m->softcap >= 0.f) || m->softcap > 3.0e38f) return fail(ST_ERR_INVALID_ARG, "softcap must be 0 or finite and positive");
  if (m->softcap > 0.f && !std::isfinite(2.f * st::kScoreLog2e * (d->scale / m->softcap))) return fail(ST_ERR_INVALID_ARG, "scale / softcap is too large");
  if (m->softcap > 0.f && !std::isfinite(m->softcap * st::kScoreLog2e)) return fail(ST_ERR_INVALID_ARG, "softcap is too large");
  if (d->dtype == ST_BF16 && m->softcap > st::kCapMost) return fail(ST_ERR_UNSUPPORTED, "bf16 path needs softcap <= %g (0: no cap)", (double)st::kCapMost);
  if (m->slopes && d->Sk > 1 << 24) return fail(ST_ERR_UNSUPPORTED, "slopes need chunks of at most 2^24 keys, whose numbers fp32 holds");
  if (reinterpret_cast<uintptr_t>(m->slopes) % 4) return fail(ST_ERR_ALIGNMENT, "slopes: not 4-byte aligned");
  if (reinterpret_cast<uintptr_t>(m->spans) % 16) return fail(ST_ERR_ALIGNMENT, "spans: not 16-byte aligned");
  return ST_OK;
}

st::ScoreArgs score_args(const st_block_desc* d, const st_score* m) {
  st::ScoreArgs a;
  memset(&a, 0, sizeof(a));
  a.s = shape_of(d);
  a.k_offset = d->k_offset;
  if (m) {
    a.cap = m->softcap;
    a.slopes = m->slopes;
    a.spans = m->spans;
  }
  a.n_split = a.q_split = a.kv_split = 1;
  return a;
}

// How the launches are split and where in the workspace their sums lie (byte offsets).
constexpr int64_t kSplitBytesMost = (int64_t)256 << 20;
// A share is at least so many products of a tile; fewer where that leaves compute units without a workgroup.  Forward and backward of
// 12/4 heads x 2 x 1000 packed rows take 78 us with 96, 83 with 64 and 80 with 128; of 16/4 x 200, too few for the chip, 41 us with
// 32, 50 with 64.
constexpr int64_t kLeastShare = 96, kLeastShareOfFew = 32;
// More partial states than this are joined by a workgroup a row, fewer by a thread for each value: one token of four sequences, 16
// states, 33.2 us in all against 35.1; 4 heads x 1000 rows, two states, 21.9 against 19.9.
constexpr int kJoinedSideBySide = 4;
struct ScorePlan {
  int n_split, q_split, kv_split;
  size_t lse, dk, dv, blocks, rows, bytes;
};
ScorePlan fwd_plan(const st::Shape& s, int dtype) {
  const int G = s.Hq / s.Hkv;
  const bool bf16 = dtype == ST_BF16;
  const int64_t tiles = bf16 ? ((int64_t)s.Sq * G + st::kScoreRows - 1) / st::kScoreRows : ((int64_t)s.Sq + 31) / 32;
  const int64_t n_o = (int64_t)s.B * s.Sq * s.Hq * s.D * 4, n_l = (int64_t)s.B * s.Sq * s.Hq * 4;
  ScorePlan p{};
  // One row tile of a token or a few is a stream of keys from memory, which two workgroups on each of 256 compute units keep
  // busy; more rows are work enough for one.
  p.n_split = st::score_split(tiles * (bf16 ? s.Hkv : s.Hq) * s.B, tiles == 1 ? 512 : 256, bf16 ? ((int64_t)s.Sk + 63) / 64 : ((int64_t)s.Sk + 255) / 256, bf16 ? 4 : 1,
                              st::kMaxTable);
  while (p.n_split > 1 && p.n_split * n_o > kSplitBytesMost) --p.n_split;
  if (p.n_split > 1) {
    p.lse = align_up((size_t)(p.n_split * n_o), 256);
    p.bytes = p.lse + align_up((size_t)(p.n_split * n_l), 256);
  }
  return p;
}
// Key tiles and query tiles share a launch.  A share of one is about what a place of the chip has to do on the average, where a tile
// is longer; the work is counted in products of 32 x 32 x D, four of a key tile's 32 rows for each 32 keys and three of a query
// tile's.  A mask leaves the longest key tiles, which come first, and takes from the average: half of it, or, where one of two runs
// of rows is past most keys, a quarter.  (The size of the workspace must not depend on the offsets.)  32/8 heads x 8192 packed
// rows, capped: 857 + 33 us in two shares, 947 in one; x 4096 rows in two runs and 2048 keys: 403 + 12 in three, 470 + 10 in two.
ScorePlan bwd_plan(const st::Shape& s, int dtype, bool spans) {
  const int G = s.Hq / s.Hkv;
  const bool bf16 = dtype == ST_BF16;
  const int64_t row_blocks = bf16 ? ((int64_t)s.Sq * G + 31) / 32 : ((int64_t)s.Sq + 31) / 32 * G, key_blocks = ((int64_t)s.Sk + 31) / 32;
  const int halves = bf16 ? 1 : st::score_f32_halves(s.D);
  const int64_t rows = bf16 ? ((int64_t)s.Sq * G + st::kScoreRows - 1) / st::kScoreRows * s.Hkv * s.B : ((int64_t)s.Sq + 31) / 32 * s.Hq * s.B;
  const int64_t keys = bf16 ? ((int64_t)s.Sk + st::kScoreKeys - 1) / st::kScoreKeys * s.Hkv * s.B : key_blocks * s.Hkv * s.B * halves;
  const int64_t n_q = (int64_t)s.B * s.Sq * s.Hq * s.D * 4, n_kv = (int64_t)s.B * s.Sk * s.Hkv * s.D * 4;
  const int64_t kv_len = (halves > 1 ? 3 : 4) * row_blocks, q_len = 3 * key_blocks;
  const int64_t each = (keys * kv_len + rows * q_len) / 512;
  const int quarters = !bf16 ? 4 : spans || (s.causal && s.q_seg <= 0) ? 2 : s.causal ? 3 : 4;
  ScorePlan p{};
  auto shares = [](int64_t len, int64_t most, int64_t eighths) { return (int)std::min<int64_t>(std::max<int64_t>((8 * len + eighths * most) / (8 * most), 1), 16); };
  auto split = [&](int64_t least) {
    p.q_split = shares(q_len, std::max(each, least), 4);
    p.kv_split = shares(kv_len, std::max(each * quarters / 4, least), quarters < 4 ? 7 : 4);
  };
  split(bf16 ? kLeastShare : 8);
  if (bf16 && keys * p.kv_split + rows * p.q_split < 256) split(kLeastShareOfFew);
  while (p.q_split > 1 && p.q_split * n_q > kSplitBytesMost) --p.q_split;
  while (p.kv_split > 1 && p.kv_split * n_kv * 2 > kSplitBytesMost) --p.kv_split;
  p.dk = p.q_split > 1 ? align_up((size_t)(p.q_split * n_q), 256) : 0;
  const size_t kv = p.kv_split > 1 ? align_up((size_t)(p.kv_split * n_kv), 256) : 0;
  p.dv = p.dk + kv;
  p.blocks = p.dv + kv;
  const int64_t blocks = ((int64_t)s.Sq * G + 31) / 32 * s.Hkv * s.B;
  p.rows = p.blocks + (bf16 ? align_up((size_t)blocks * sizeof(int4), 256) : 0);
  p.bytes = p.rows + (bf16 ? (size_t)blocks * st::kRowStats * 4 : 0);
  return p;
}

st_status check_workspace(const void* ws, size_t bytes, size_t need, const char* what) {
  if (need == 0) return ST_OK;
  if (ws == nullptr || bytes < need) return fail(ST_ERR_WORKSPACE, "%s workspace needs %zu bytes", what, need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(ST_ERR_ALIGNMENT, "workspace: not 256-byte aligned");
  return ST_OK;
}

st_status check_low(const char* name, const void* p) {
  if (reinterpret_cast<uintptr_t>(p) % 16) return fail(ST_ERR_ALIGNMENT, "%s: not 16-byte aligned", name);
  return ST_OK;
}

st_status check_rope(const st_rope_desc* d, const int32_t* positions, const double* freq) {
  if (d == nullptr) return fail(ST_ERR_INVALID_ARG, "null descriptor");
  if (d->dtype != ST_F32 && d->dtype != ST_BF16) return fail(ST_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->B < 0 || d->S < 0 || d->Hkv < 0) return fail(ST_ERR_INVALID_ARG, "negative size");
  if (d->Hq <= 0 || d->D <= 0) return fail(ST_ERR_INVALID_ARG, "Hq and D must be positive");
  if (d->D > 256 || d->D % 8 != 0) return fail(ST_ERR_UNSUPPORTED, "D <= 256 and D %% 8 == 0 are needed (D=%d)", d->D);
  if ((int64_t)d->Hq + d->Hkv > 16384) return fail(ST_ERR_UNSUPPORTED, "more than 16384 heads");
  if ((int64_t)d->B * d->S > (int64_t)1 << 25) return fail(ST_ERR_UNSUPPORTED, "more than 2^25 tokens");
  if (d->rot < 0 || d->rot > d->D || d->rot % 2) return fail(ST_ERR_INVALID_ARG, "rot = %d must be even, 0 .. D", d->rot);
  if (d->pairing != ST_ROPE_HALVES && d->pairing != ST_ROPE_NEIGHBOURS) return fail(ST_ERR_INVALID_ARG, "unknown pairing %d", d->pairing);
  if (d->norm != 0 && d->norm != 1) return fail(ST_ERR_INVALID_ARG, "unknown norm %d", d->norm);
  if (d->norm && !(d->eps >= 0.f && d->eps <= 3.0e38f)) return fail(ST_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (d->n_axes < 1 || d->n_axes > ST_ROPE_MAX_AXES) return fail(ST_ERR_INVALID_ARG, "n_axes must be in 1..%d", ST_ROPE_MAX_AXES);
  int64_t pairs = 0;
  for (int x = 0; x < d->n_axes; ++x) {
    if (d->axis_pairs[x] < 0) return fail(ST_ERR_INVALID_ARG, "axis_pairs[%d] is negative", x);
    pairs += d->axis_pairs[x];
  }
  if (pairs != d->rot / 2) return fail(ST_ERR_INVALID_ARG, "axis_pairs add up to %lld, rot has %d pairs", (long long)pairs, d->rot / 2);
  ST_TRY(check_segments(d->S, d->offset, d->seg, d->offset2));
  if (positions == nullptr && d->n_axes != 1) return fail(ST_ERR_INVALID_ARG, "more than one axis needs positions");
  if (positions != nullptr && d->seg != 0) return fail(ST_ERR_INVALID_ARG, "positions and a second run of rows exclude each other");
  if (d->rot > 0 && (int64_t)d->B * d->S > 0 && freq == nullptr) return fail(ST_ERR_INVALID_ARG, "freq: null pointer");
  if (reinterpret_cast<uintptr_t>(freq) % 8 || reinterpret_cast<uintptr_t>(positions) % 4) return fail(ST_ERR_ALIGNMENT, "freq needs 8-byte, positions 4-byte alignment");
  return ST_OK;
}

st_status check_weight(const char* name, const void* p) {
  if (reinterpret_cast<uintptr_t>(p) % 16) return fail(ST_ERR_ALIGNMENT, "%s: not 16-byte aligned", name);
  return ST_OK;
}

st::RopeArgs rope_args(const st_rope_desc* d) {
  st::RopeArgs g;
  memset(&g, 0, sizeof(g));
  g.B = d->B; g.S = d->S; g.Hq = d->Hq; g.Hkv = d->Hkv; g.D = d->D; g.rot = d->rot;
  g.next = d->pairing == ST_ROPE_NEIGHBOURS;
  g.norm = d->norm;
  g.eps = d->eps;
  g.n_axes = d->n_axes;
  for (int x = 0; x < ST_ROPE_MAX_AXES; ++x) g.axis_pairs[x] = d->axis_pairs[x];
  g.offset = d->offset; g.seg = d->seg; g.offset2 = d->offset2;
  return g;
}

}  // namespace

extern "C" {

st_status st_mask_spans(int32_t B, int32_t Sq, int64_t q_offset, int32_t q_seg, int64_t q_offset2, int32_t causal, const int64_t* bounds,
                        int32_t n_docs, const int64_t* prefix, int64_t* spans, void* hip_stream) {
  if (B < 0 || Sq < 0 || n_docs < 0) return fail(ST_ERR_INVALID_ARG, "negative size");
  ST_TRY(check_segments(Sq, q_offset, q_seg, q_offset2));
  if ((int64_t)B * Sq == 0) return ST_OK;
  if (bounds == nullptr || spans == nullptr) return fail(ST_ERR_INVALID_ARG, "bounds / spans: null pointer");
  if (reinterpret_cast<uintptr_t>(bounds) % 8 || reinterpret_cast<uintptr_t>(prefix) % 8 || reinterpret_cast<uintptr_t>(spans) % 16)
    return fail(ST_ERR_ALIGNMENT, "bounds and prefix need 8-byte, spans 16-byte alignment");
  if (((int64_t)B * Sq + 255) / 256 > st::kScoreGridMost) return fail(ST_ERR_UNSUPPORTED, "more than 2^30 rows");
  if (n_docs >= 1 << 30) return fail(ST_ERR_UNSUPPORTED, "2^30 documents or more");   // (the search adds two of their numbers)
  st::Shape s;
  memset(&s, 0, sizeof(s));
  s.B = B; s.Sq = Sq; s.q_offset = q_offset; s.q_seg = q_seg; s.q_offset2 = q_offset2; s.causal = causal ? 1 : 0;
  ST_HIP(st::launch_mask_spans(s, bounds, n_docs, prefix, spans, (hipStream_t)hip_stream), "st_mask_spans launch");
  return ST_OK;
}

size_t st_attn_score_workspace_bytes(const st_block_desc* d, const st_score* m, int32_t backward) {
  if (check_score(d, m) != ST_OK || (int64_t)d->B * d->Sq == 0) return 0;
  const st::Shape s = shape_of(d);
  return backward ? std::max(bwd_plan(s, d->dtype, true).bytes, bwd_plan(s, d->dtype, false).bytes) : fwd_plan(s, d->dtype).bytes;
}

st_status st_attn_score_fwd(const st_block_desc* d, const st_score* m, const st_tensor* q, const st_tensor* k, const st_tensor* v,
                            float* o_part, float* lse_part, void* o_lowp, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ST_TRY(check_score(d, m));
  const int64_t n_q = (int64_t)d->B * d->Sq * d->Hq * d->D, n_kv = (int64_t)d->B * d->Sk * d->Hkv * d->D;
  ST_TRY(check_tensor("q", q, d->dtype, n_q));
  ST_TRY(check_tensor("k", k, d->dtype, n_kv));
  ST_TRY(check_tensor("v", v, d->dtype, n_kv));
  if (n_q == 0) return ST_OK;
  if (o_part == nullptr && o_lowp == nullptr) return fail(ST_ERR_INVALID_ARG, "o_part and o_lowp: one of them is needed");
  if ((void*)o_part == o_lowp) return fail(ST_ERR_INVALID_ARG, "o_lowp aliases o_part");
  if (o_part) ST_TRY(check_f32("o_part", o_part, n_q));
  ST_TRY(check_low("o_lowp", o_lowp));
  ST_TRY(check_f32("lse_part", lse_part, n_q));
  st::ScoreArgs a = score_args(d, m);
  a.q = view_of(q);
  a.k = view_of(k);
  a.v = view_of(v);
  a.o = o_part;
  a.lse = lse_part;
  a.o_lowp = o_lowp;
  const ScorePlan p = fwd_plan(a.s, d->dtype);
  ST_TRY(check_workspace(workspace, workspace_bytes, p.bytes, "score forward"));
  a.n_split = p.n_split;
  a.part_o = (float*)workspace;
  a.part_lse = (float*)((char*)workspace + p.lse);
  ST_HIP(d->dtype == ST_BF16 ? st::launch_score_fwd_bf16(a, (hipStream_t)hip_stream) : st::launch_score_fwd_f32(a, (hipStream_t)hip_stream), "st_attn_score_fwd launch");
  if (a.n_split <= 1) return ST_OK;
  if (a.n_split > kJoinedSideBySide) {
    ST_HIP(st::launch_score_combine(a, d->dtype == ST_BF16, (hipStream_t)hip_stream), "st_attn_score_fwd combine");
    return ST_OK;
  }
  st::CombineArgs c;
  memset(&c, 0, sizeof(c));
  c.n = a.n_split;
  const int64_t n_l = (int64_t)d->B * d->Sq * d->Hq;
  for (int x = 0; x < c.n; ++x) {
    c.o[x] = a.part_o + x * n_q;
    c.lse[x] = a.part_lse + x * n_l;
  }
  c.B = d->B; c.Sq_in = c.Sq_out = d->Sq; c.Hq = d->Hq; c.D = d->D;
  c.o_out = o_part ? o_part : d->dtype == ST_F32 ? (float*)o_lowp : a.part_o;   // (a thread reads all states of what it writes)
  c.lse_out = lse_part;
  c.o_lowp = c.o_out == (float*)o_lowp ? nullptr : o_lowp;
  ST_HIP(st::launch_combine(c, d->dtype, (hipStream_t)hip_stream), "st_attn_score_fwd combine");
  return ST_OK;
}

st_status st_attn_score_bwd(const st_block_desc* d, const st_score* m, const st_tensor* q, const st_tensor* k, const st_tensor* v,
                            const st_tensor* d_o, const float* lse_final, const float* delta, int32_t flags, float* dq_acc, float* dk_acc,
                            float* dv_acc, void* dq_lowp, void* dk_lowp, void* dv_lowp, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ST_TRY(check_score(d, m));
  const int64_t n_q = (int64_t)d->B * d->Sq * d->Hq * d->D, n_kv = (int64_t)d->B * d->Sk * d->Hkv * d->D;
  if (flags & ~ST_GRAD_ASSIGN) return fail(ST_ERR_INVALID_ARG, "unknown flags %d", flags);
  const bool assign = (flags & ST_GRAD_ASSIGN) != 0;
  ST_TRY(check_tensor("q", q, d->dtype, n_q));
  ST_TRY(check_tensor("d_o", d_o, d->dtype, n_q));
  ST_TRY(check_tensor("k", k, d->dtype, n_kv));
  ST_TRY(check_tensor("v", v, d->dtype, n_kv));
  ST_TRY(check_f32("lse_final", lse_final, n_q));
  ST_TRY(check_f32("delta", delta, n_q));
  struct { const char* name; float* acc; void* low; int64_t n; } out[3] = {{"dq", dq_acc, dq_lowp, n_q}, {"dk", dk_acc, dk_lowp, n_kv}, {"dv", dv_acc, dv_lowp, n_kv}};
  for (const auto& o : out) {
    if (o.n == 0) continue;
    if (!assign && o.acc == nullptr) return fail(ST_ERR_INVALID_ARG, "%s_acc: null pointer (nothing to add to)", o.name);
    if (o.acc == nullptr && o.low == nullptr) return fail(ST_ERR_INVALID_ARG, "%s_acc and %s_lowp: one of them is needed", o.name, o.name);
    if ((void*)o.acc == o.low) return fail(ST_ERR_INVALID_ARG, "%s_lowp aliases %s_acc", o.name, o.name);
    if (o.acc) ST_TRY(check_f32(o.name, o.acc, o.n));
    ST_TRY(check_low(o.name, o.low));
  }
  const void* written[] = {dq_acc, dk_acc, dv_acc, dq_lowp, dk_lowp, dv_lowp};
  for (int x = 0; x < 6; ++x)
    for (int y = 0; y < x; ++y)
      if (written[x] && written[x] == written[y]) return fail(ST_ERR_INVALID_ARG, "two gradients share their memory");
  if (n_q == 0 && n_kv == 0) return ST_OK;
  st::ScoreArgs a = score_args(d, m);
  a.q = view_of(q);
  a.k = view_of(k);
  a.v = view_of(v);
  a.d_o = view_of(d_o);
  a.lse_in = lse_final;
  a.delta = delta;
  a.assign = assign ? 1 : 0;
  a.dq = dq_acc; a.dk = dk_acc; a.dv = dv_acc;
  a.dq_lowp = dq_lowp; a.dk_lowp = dk_lowp; a.dv_lowp = dv_lowp;
  if (n_q > 0) {
    const ScorePlan p = bwd_plan(a.s, d->dtype, a.spans != nullptr);
    ST_TRY(check_workspace(workspace, workspace_bytes, p.bytes, "score backward"));
    a.q_split = p.q_split;
    a.kv_split = p.kv_split;
    a.part_dq = (float*)workspace;
    a.part_dk = (float*)((char*)workspace + p.dk);
    a.part_dv = (float*)((char*)workspace + p.dv);
    if (d->dtype == ST_BF16) {
      a.blocks = (int4*)((char*)workspace + p.blocks);
      a.rows = (float*)((char*)workspace + p.rows);
      ST_HIP(st::launch_score_rows(a, (hipStream_t)hip_stream), "row statistics launch");
    }
  }
  ST_HIP(d->dtype == ST_BF16 ? st::launch_score_bwd_bf16(a, (hipStream_t)hip_stream) : st::launch_score_bwd_f32(a, (hipStream_t)hip_stream), "st_attn_score_bwd launch");
  ST_HIP(st::launch_score_add_parts(a, d->dtype == ST_BF16, (hipStream_t)hip_stream), "st_attn_score_bwd sums");
  return ST_OK;
}

st_status st_qk_rope_fwd(const st_rope_desc* d, const st_tensor* q, const st_tensor* k, const float* q_weight, const float* k_weight,
                         const double* freq, const int32_t* positions, const st_tensor* q_out, const st_tensor* k_out, void* hip_stream) {
  ST_TRY(check_rope(d, positions, freq));
  const int64_t n_q = (int64_t)d->B * d->S * d->Hq * d->D, n_k = (int64_t)d->B * d->S * d->Hkv * d->D;
  ST_TRY(check_tensor("q", q, d->dtype, n_q));
  ST_TRY(check_tensor("q_out", q_out, d->dtype, n_q));
  if (n_k > 0) {
    ST_TRY(check_tensor("k", k, d->dtype, n_k));
    ST_TRY(check_tensor("k_out", k_out, d->dtype, n_k));
  }
  ST_TRY(check_weight("q_weight", q_weight));
  ST_TRY(check_weight("k_weight", k_weight));
  if (!d->norm && (q_weight || k_weight)) return fail(ST_ERR_INVALID_ARG, "weights need norm = 1");
  if (n_q == 0) return ST_OK;
  st::RopeArgs g = rope_args(d);
  g.q = view_of(q);
  g.q_out = view_of(q_out);
  if (n_k > 0) {
    g.k = view_of(k);
    g.k_out = view_of(k_out);
  }
  g.q_weight = q_weight;
  g.k_weight = k_weight;
  g.freq = freq;
  g.positions = positions;
  ST_HIP(st::launch_rope_fwd(g, d->dtype == ST_BF16, (hipStream_t)hip_stream), "st_qk_rope_fwd launch");
  return ST_OK;
}

size_t st_qk_rope_bwd_workspace_bytes(const st_rope_desc* d) {
  if (d == nullptr || d->B <= 0 || d->S <= 0 || d->D <= 0 || !d->norm) return 0;
  return align_up((size_t)std::min<int64_t>((int64_t)d->B * d->S, st::kRopeBlocksMost) * 2 * d->D * 4, 256);
}

st_status st_qk_rope_bwd(const st_rope_desc* d, const st_tensor* q, const st_tensor* k, const st_tensor* d_q, const st_tensor* d_k,
                         int32_t d_dtype, const float* q_weight, const float* k_weight, const double* freq, const int32_t* positions,
                         int32_t flags, const st_tensor* dx_q, const st_tensor* dx_k, float* dw_q, float* dw_k, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
  ST_TRY(check_rope(d, positions, freq));
  if (d_dtype != ST_F32 && d_dtype != d->dtype) return fail(ST_ERR_INVALID_ARG, "d_dtype must be ST_F32 or the storage dtype");
  if (flags & ~ST_GRAD_ASSIGN) return fail(ST_ERR_INVALID_ARG, "unknown flags %d", flags);
  const int64_t n_q = (int64_t)d->B * d->S * d->Hq * d->D, n_k = (int64_t)d->B * d->S * d->Hkv * d->D;
  if (d->norm) ST_TRY(check_tensor("q", q, d->dtype, n_q));
  ST_TRY(check_tensor("d_q", d_q, d_dtype, n_q));
  ST_TRY(check_tensor("dx_q", dx_q, d->dtype, n_q));
  if (n_k > 0) {
    if (d->norm) ST_TRY(check_tensor("k", k, d->dtype, n_k));
    ST_TRY(check_tensor("d_k", d_k, d_dtype, n_k));
    ST_TRY(check_tensor("dx_k", dx_k, d->dtype, n_k));
  }
  ST_TRY(check_weight("q_weight", q_weight));
  ST_TRY(check_weight("k_weight", k_weight));
  ST_TRY(check_weight("dw_q", dw_q));
  ST_TRY(check_weight("dw_k", dw_k));
  if (!d->norm && (q_weight || k_weight || dw_q || dw_k)) return fail(ST_ERR_INVALID_ARG, "weights and their gradients need norm = 1");
  if ((dw_q && dw_q == dw_k)) return fail(ST_ERR_INVALID_ARG, "dw_q aliases dw_k");
  st::RopeArgs g = rope_args(d);
  if (n_q > 0) {
    if (d->norm) g.q = view_of(q);
    g.dq = view_of(d_q);
    g.q_out = view_of(dx_q);
    if (n_k > 0) {
      if (d->norm) g.k = view_of(k);
      g.dk = view_of(d_k);
      g.k_out = view_of(dx_k);
    }
    if (dw_q || dw_k) {
      const size_t need = st_qk_rope_bwd_workspace_bytes(d);
      ST_TRY(check_workspace(workspace, workspace_bytes, need, "rope backward"));
      g.dw_parts = (float*)workspace;
    }
  }
  g.q_weight = q_weight;
  g.k_weight = k_weight;
  g.freq = freq;
  g.positions = positions;
  ST_HIP(st::launch_rope_bwd(g, d->dtype == ST_BF16, d_dtype == ST_BF16, dw_q, dw_k, (flags & ST_GRAD_ASSIGN) != 0, (hipStream_t)hip_stream), "st_qk_rope_bwd launch");
  return ST_OK;
}

}  // extern "C"
