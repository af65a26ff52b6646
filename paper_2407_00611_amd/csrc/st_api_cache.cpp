// C ABI of the cache of keys and values in pages: argument checks, workspace layout, launches.
#include <algorithm>
#include <cmath>

#include "st_cache.h"
#include "st_checks.h"
#include "st_score.h"

using namespace st::checks;
using st::fail;
using st::hip_fail;

namespace {

// A share of a walk is at least so many blocks of keys: two of 32 for each wavefront of a tile of 16 or 32 rows (one in fp32, where a block is
// four times the work: 3 rows of four sequences 20 us, 23 with two), four of 64 of a prompt's tile (102 rows of 18 sequences 34 us, 46 with
// eight).
constexpr int kLeastBlocks = 8, kLeastOfPrompts = 4;
// bf16 walks of so many blocks and more, of so many tiles and heads, have workgroups enough with shares of twice that (4000 tokens of 16
// sequences, 8 heads 40 us, 44 with eight blocks; 1500 tokens of 8 ragged ones 15.6, 13.7).
constexpr int kLongBlocks = 96, kLongJobs = 64;
// Workgroups that shares are made for: sequences of up to 16 rows wait for memory, and more workgroups than the chip holds at once even out
// what the lengths leave (64 ragged sequences 124 us, 140 with 1024); those of more rows are work, and each share has so many rows of O to
// join (fp32, D = 256, 256 rows of two sequences 96 us, 120 with 1024, 168 with 2048).
constexpr int kPlacesOfFew = 2048, kPlaces = 512;
// Sequences of up to so many rows are read again for every 32 of them (16 heads x 24 rows x 2048 tokens as fast either way, 64 rows 30 us and
// 40); of up to kFewOfShort where there are few tiles, and a step's latency is what counts (246 rows of six sequences 27 us, 31).
constexpr int kFewRows = 128, kFewOfShort = 256, kShortTiles = 64;
// Beside sequences of more, those of up to so many rows are taken in tiles of 16, and only those behind in a prompt's tiles, with probabilities
// in two parts up to 128 rows (six of 20 rows beside two prompts 101 us, 136 in a prompt's tile; fifteen of 32 beside one 135, 195; of 64 200, 170).
constexpr int kFewBesides = 32;

// Where no walk of bf16 rows has more blocks than this, none is split and no join launched: a step of a workgroup's four wavefronts is 1.1 us,
// a launch that joins 3 and more.  kWhole blocks for one sequence (400 tokens 9.5 us, 11.1 split; 700 tokens 12.2, 11.3), three times as many where
// there are a workgroup or two for each compute unit (1200 tokens of 32 sequences, 8 heads 19 us, 26; of 64 ragged ones 26, 28; 2000 tokens of
// those 46, 44), kWholeOfMany where the last of many have the chip for themselves (32 sequences of 24 heads of 64, 700 tokens 23 us, 25; 980 tokens
// 32, 30).
constexpr int kWhole = 16, kWholeOfMany = 24;

st_status check_cache(const st_cache* c) {
  if (c == nullptr) return fail(ST_ERR_INVALID_ARG, "null cache");
  if (c->dtype != ST_F32 && c->dtype != ST_BF16 && c->dtype != ST_E4M3) return fail(ST_ERR_INVALID_ARG, "cache: unknown dtype %d", c->dtype);
  if (c->n_pages < 0 || c->B < 0 || c->width < 0) return fail(ST_ERR_INVALID_ARG, "cache: negative size");
  if (c->Hkv <= 0 || c->D <= 0) return fail(ST_ERR_INVALID_ARG, "cache: Hkv and D must be positive");
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1))) return fail(ST_ERR_UNSUPPORTED, "cache: pages of 16, 32, 64, 128 or 256 tokens (page=%d)", c->page);
  if (c->D > 256 || c->D % 8 != 0) return fail(ST_ERR_UNSUPPORTED, "cache: D <= 256 and D %% 8 == 0 are needed (D=%d)", c->D);
  if (c->dtype == ST_E4M3 && c->D % 16 != 0) return fail(ST_ERR_UNSUPPORTED, "cache: D %% 16 == 0 is needed in 8 bits (D=%d)", c->D);
  if (c->Hkv > 16384) return fail(ST_ERR_UNSUPPORTED, "cache: more than 16384 heads");
  if (c->B > 65535) return fail(ST_ERR_UNSUPPORTED, "cache: B must not exceed 65535");
  if ((int64_t)c->width * c->page > (int64_t)1 << 30) return fail(ST_ERR_UNSUPPORTED, "cache: more than 2^30 tokens a sequence");
  const int64_t n = (int64_t)c->n_pages * c->page * c->Hkv * c->D;
  ST_TRY(check_tensor("cache k", &c->k, c->dtype, n));
  ST_TRY(check_tensor("cache v", &c->v, c->dtype, n));
  // (kernels add places inside a page in 32 bits)
  if (std::max(c->k.stride_s, c->v.stride_s) >= (int64_t)1 << 20) return fail(ST_ERR_UNSUPPORTED, "cache: tokens of a page are 2^20 values or more apart");
  if (c->dtype == ST_E4M3 && n > 0 && (c->k_scale == nullptr || c->v_scale == nullptr)) return fail(ST_ERR_INVALID_ARG, "cache: pages in 8 bits need k_scale and v_scale");
  if (c->dtype != ST_E4M3 && (c->k_scale || c->v_scale)) return fail(ST_ERR_INVALID_ARG, "cache: scales belong to pages in 8 bits");
  if (c->B > 0 && (c->lens == nullptr || (c->table == nullptr && c->width > 0))) return fail(ST_ERR_INVALID_ARG, "cache: table / lens: null pointer");
  if (reinterpret_cast<uintptr_t>(c->table) % 4 || reinterpret_cast<uintptr_t>(c->lens) % 4) return fail(ST_ERR_ALIGNMENT, "cache: table and lens need 4-byte alignment");
  return ST_OK;
}

st_status check_starts(const st_cache* c, const int32_t* starts, int64_t T) {
  if (c->B == 0 || T == 0) return ST_OK;
  if (starts == nullptr) return fail(ST_ERR_INVALID_ARG, "starts: null pointer");
  if (reinterpret_cast<uintptr_t>(starts) % 4) return fail(ST_ERR_ALIGNMENT, "starts: not 4-byte aligned");
  return ST_OK;
}

st::CacheArgs cache_args(const st_cache* c) {
  st::CacheArgs a;
  memset(&a, 0, sizeof(a));
  // (without a page no sequence has a token)
  a.dtype = c->dtype; a.n_pages = c->n_pages; a.shift = __builtin_ctz((unsigned)c->page); a.Hkv = c->Hkv; a.D = c->D; a.B = c->B; a.width = c->n_pages > 0 ? c->width : 0;
  a.k = view_of(&c->k);
  a.v = view_of(&c->v);
  a.k_scale = c->k_scale; a.v_scale = c->v_scale; a.table = c->table; a.lens = c->lens;
  return a;
}

st_status check_rows(const st_cache_rows* r, const st_cache* c) {
  if (r == nullptr) return fail(ST_ERR_INVALID_ARG, "null descriptor");
  ST_TRY(check_cache(c));
  if (r->dtype != ST_F32 && r->dtype != ST_BF16) return fail(ST_ERR_INVALID_ARG, "unknown dtype %d", r->dtype);
  if (c->dtype != ST_E4M3 && c->dtype != r->dtype) return fail(ST_ERR_UNSUPPORTED, "rows and pages of different dtypes");
  if (r->T < 0 || r->max_rows < 0 || r->window < 0) return fail(ST_ERR_INVALID_ARG, "negative size");
  if (r->Hq <= 0 || r->Hq % c->Hkv != 0) return fail(ST_ERR_INVALID_ARG, "need Hq %% Hkv == 0 (Hq=%d Hkv=%d)", r->Hq, c->Hkv);
  if (r->dtype == ST_BF16 && c->D != 128 && c->D != 64) return fail(ST_ERR_UNSUPPORTED, "bf16 path is built for D = 64 or 128 (D=%d)", c->D);
  if (r->Hq > 65535) return fail(ST_ERR_UNSUPPORTED, "Hq must not exceed 65535");
  if (r->T > 1 << 25) return fail(ST_ERR_UNSUPPORTED, "more than 2^25 rows");
  if ((int64_t)r->T * (r->Hq / c->Hkv) > 0x7fffff00) return fail(ST_ERR_UNSUPPORTED, "more than 2^31 rows of a KV head's group");
  ST_TRY(check_scale(r->scale));
  if (!(r->softcap >= 0.f) || r->softcap > 3.0e38f) return fail(ST_ERR_INVALID_ARG, "softcap must be 0 or finite and positive");
  if (r->softcap > 0.f && !std::isfinite(2.f * st::kScoreLog2e * (r->scale / r->softcap))) return fail(ST_ERR_INVALID_ARG, "scale / softcap is too large");
  if (r->softcap > 0.f && !std::isfinite(r->softcap * st::kScoreLog2e)) return fail(ST_ERR_INVALID_ARG, "softcap is too large");
  if (r->dtype == ST_BF16 && r->softcap > st::kCapMost) return fail(ST_ERR_UNSUPPORTED, "bf16 path needs softcap <= %g (0: no cap)", (double)st::kCapMost);
  if (r->slopes && (int64_t)c->width * c->page > 1 << 24) return fail(ST_ERR_UNSUPPORTED, "slopes need sequences of at most 2^24 tokens, whose numbers fp32 holds");
  if (reinterpret_cast<uintptr_t>(r->slopes) % 4) return fail(ST_ERR_ALIGNMENT, "slopes: not 4-byte aligned");
  if (((int64_t)r->T * (r->Hq / c->Hkv) / 16 + c->B) * c->Hkv > st::kScoreGridMost / 2) return fail(ST_ERR_UNSUPPORTED, "more than %lld tiles", (long long)st::kScoreGridMost / 2);
  return ST_OK;
}

// Row tiles of all sequences together there can be, and how their walks are split: a launch for tiles of `rows` rows
st::CachePlan launch_plan(const st_cache_rows* r, const st_cache* c, int rows, int from, int to, int64_t base) {
  const int64_t G = r->Hq / c->Hkv, some = std::min(c->B, r->T), most_rows = std::min<int64_t>((int64_t)std::min(r->max_rows, r->T) * G, to);
  const int64_t tiles = std::min(r->T * G / rows + some, some * ((most_rows + rows - 1) / rows));
  const int keys = rows == st::kPromptRows ? st::kPromptKeys : st::kCacheKeys;
  int64_t blocks = ((int64_t)c->width * c->page + keys - 1) / keys;
  if (r->causal && r->window > 0) blocks = std::min(blocks, ((int64_t)r->window + std::min(r->max_rows, r->T) - 1 + keys - 1) / keys + 1);
  st::CachePlan p{};
  p.rows = rows;
  p.rows_from = from;
  p.rows_to = to;
  p.least = rows == st::kPromptRows ? kLeastOfPrompts : r->dtype == ST_F32 ? kLeastBlocks / 2 : kLeastBlocks;
  p.target = most_rows <= 16 || (r->dtype == ST_BF16 && rows == 16) ? kPlacesOfFew : kPlaces;
  const int64_t jobs = tiles * c->Hkv;
  if (r->dtype == ST_BF16 && rows != st::kPromptRows && blocks <= (jobs <= kPlaces ? std::min(kWhole + jobs / 8, 3 * (int64_t)kWhole) : kWholeOfMany)) p.least = 4 * kWhole;
  else if (r->dtype == ST_BF16 && rows != st::kPromptRows && blocks >= kLongBlocks && jobs >= kLongJobs) p.least = 2 * kLeastBlocks;
  const int64_t most = std::max<int64_t>((blocks + p.least / 2) / p.least, 1);
  p.most = (int32_t)most;
  p.grid = std::min(p.target + jobs, jobs * most);
  if (rows == 16) p.grid = (p.grid + 8 * c->Hkv - 1) / (8 * c->Hkv) * (8 * c->Hkv);   // (whole rounds of the order in which they take their pieces)
  // (as many as with the shortest shares: a window, which shortens walks, never needs more room than none)
  p.states = most > 1 ? (int32_t)std::min<int64_t>(p.target * 4 / 3 + 1, jobs * std::max(most, (blocks + kLeastBlocks / 2) / kLeastBlocks)) : 0;
  p.base = base;
  p.jobs = jobs;
  return p;
}
// The launches of a call: sequences of few rows and those of more have kernels of their own where there may be both
struct Plans {
  int n;
  st::CachePlan p[2];
  int64_t rows;              // of all states
  int states;                // of a row, on the average
};
Plans plans_of(const st_cache_rows* r, const st_cache* c) {
  constexpr int kAll = 0x7fffffff;
  const int64_t most = (int64_t)std::min(r->max_rows, r->T) * (r->Hq / c->Hkv);
  const bool tall = r->dtype == ST_BF16 && most > kFewRows && (most > kFewOfShort || launch_plan(r, c, st::kPromptRows, 0, kAll, 0).jobs > kShortTiles);
  const int large = tall ? st::kPromptRows : 32, few = tall ? kFewBesides : 16;
  Plans y{};
  y.n = 1;
  if (most <= 16 || (r->dtype == ST_F32 && c->D > st::kTallCacheHead)) {
    y.p[0] = launch_plan(r, c, 16, 0, kAll, 0);
  } else if (most <= kFewRows || c->B == 1 || (most <= kFewOfShort && !tall)) {
    y.p[0] = launch_plan(r, c, large, 0, kAll, 0);
  } else {
    y.n = 2;
    y.p[0] = launch_plan(r, c, large, few, kAll, 0);
    y.p[1] = launch_plan(r, c, 16, 0, few, (int64_t)y.p[0].states * large);
  }
  for (int x = 0; x < y.n; ++x) y.rows += (int64_t)y.p[x].states * y.p[x].rows;
  y.states = y.n == 1 ? (int)std::min<int64_t>(y.p[0].states / y.p[0].jobs, y.p[0].most) : 1;
  return y;
}
struct Room {
  size_t rows, info, bytes;
};
Room room_of(const Plans& p, const st_cache_rows* r, const st_cache* c) {
  Room y{};
  if (p.rows == 0) return y;
  y.rows = align_up((size_t)p.rows * c->D * 4, 256);
  y.info = y.rows + align_up((size_t)p.rows * 16, 256);
  y.bytes = y.info + align_up((size_t)r->T * 16, 256);
  return y;
}

}  // namespace

extern "C" {

st_status st_cache_append(const st_rope_desc* d, const st_cache* c, const int32_t* starts, const st_tensor* q, const st_tensor* k, const st_tensor* v,
                          const float* q_weight, const float* k_weight, const double* freq, const int32_t* positions, const st_tensor* q_out,
                          void* hip_stream) {
  ST_TRY(check_cache(c));
  ST_TRY(check_rope(d, positions, freq, 0));
  if (d->B != 1 || d->seg != 0) return fail(ST_ERR_INVALID_ARG, "packed rows: B = 1 and seg = 0");
  if (d->Hkv != c->Hkv || d->D != c->D) return fail(ST_ERR_INVALID_ARG, "the rows have %d heads of %d, the cache %d of %d", d->Hkv, d->D, c->Hkv, c->D);
  if (c->dtype != ST_E4M3 && c->dtype != d->dtype) return fail(ST_ERR_UNSUPPORTED, "rows and pages of different dtypes");
  ST_TRY(check_starts(c, starts, d->S));
  const int64_t n_q = (int64_t)d->S * d->Hq * d->D, n_k = (int64_t)d->S * d->Hkv * d->D;
  ST_TRY(check_tensor("k", k, d->dtype, n_k));
  ST_TRY(check_tensor("v", v, d->dtype, n_k));
  if (n_q > 0) {
    ST_TRY(check_tensor("q", q, d->dtype, n_q));
    ST_TRY(check_tensor("q_out", q_out, d->dtype, n_q));
  }
  ST_TRY(check_weight("q_weight", q_weight));
  ST_TRY(check_weight("k_weight", k_weight));
  if (!d->norm && (q_weight || k_weight)) return fail(ST_ERR_INVALID_ARG, "weights need norm = 1");
  if (n_k == 0 || c->B == 0) return ST_OK;
  st::AppendArgs a;
  memset(&a, 0, sizeof(a));
  a.g = rope_args(d);
  a.c = cache_args(c);
  a.g.k = view_of(k);
  a.v_in = view_of(v);
  if (n_q > 0) {
    a.g.q = view_of(q);
    a.g.q_out = view_of(q_out);
  }
  a.g.q_weight = q_weight;
  a.g.k_weight = k_weight;
  a.g.freq = freq;
  a.g.positions = positions;
  a.starts = starts;
  ST_HIP(st::launch_cache_append(a, d->dtype == ST_BF16, (hipStream_t)hip_stream), "st_cache_append launch");
  return ST_OK;
}

st_status st_cache_read(const st_cache* c, const int32_t* first, int32_t count, int32_t dtype, const st_tensor* k_out, const st_tensor* v_out,
                        void* hip_stream) {
  ST_TRY(check_cache(c));
  if (dtype != ST_F32 && dtype != ST_BF16) return fail(ST_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (c->dtype != ST_E4M3 && c->dtype != dtype) return fail(ST_ERR_UNSUPPORTED, "chunks and pages of different dtypes");
  if (count < 0) return fail(ST_ERR_INVALID_ARG, "negative size");
  if (reinterpret_cast<uintptr_t>(first) % 4) return fail(ST_ERR_ALIGNMENT, "first: not 4-byte aligned");
  const int64_t n = (int64_t)count * c->Hkv * c->D;
  if (count > 1 << 28 || n >= (int64_t)1 << 34) return fail(ST_ERR_UNSUPPORTED, "more than 2^28 tokens or 2^34 values of a sequence");
  if (n == 0 || c->B == 0) return ST_OK;
  if (k_out == nullptr && v_out == nullptr) return fail(ST_ERR_INVALID_ARG, "k_out and v_out: one of them is needed");
  st::ReadArgs a;
  memset(&a, 0, sizeof(a));
  a.c = cache_args(c);
  a.first = first;
  a.count = count;
  if (k_out) {
    ST_TRY(check_tensor("k_out", k_out, dtype, n));
    a.k_out = view_of(k_out);
  }
  if (v_out) {
    ST_TRY(check_tensor("v_out", v_out, dtype, n));
    a.v_out = view_of(v_out);
  }
  if (a.k_out.ptr == a.v_out.ptr) return fail(ST_ERR_INVALID_ARG, "v_out aliases k_out");
  ST_HIP(st::launch_cache_read(a, dtype, (hipStream_t)hip_stream), "st_cache_read launch");
  return ST_OK;
}

size_t st_attn_cache_workspace_bytes(const st_cache_rows* r, const st_cache* c) {
  if (check_rows(r, c) != ST_OK || c->B == 0 || r->T == 0 || r->max_rows == 0) return 0;
  return room_of(plans_of(r, c), r, c).bytes;
}

st_status st_attn_cache(const st_cache_rows* r, const st_cache* c, const int32_t* starts, const int64_t* q_first, const st_tensor* q, float* o_part,
                        float* lse_part, void* o_lowp, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ST_TRY(check_rows(r, c));
  ST_TRY(check_starts(c, starts, r->T));
  if (reinterpret_cast<uintptr_t>(q_first) % 8) return fail(ST_ERR_ALIGNMENT, "q_first: not 8-byte aligned");
  const int64_t n_q = (int64_t)r->T * r->Hq * c->D;
  ST_TRY(check_tensor("q", q, r->dtype, n_q));
  if (n_q == 0 || c->B == 0 || r->max_rows == 0) return ST_OK;
  if (o_part == nullptr && o_lowp == nullptr) return fail(ST_ERR_INVALID_ARG, "o_part and o_lowp: one of them is needed");
  if ((void*)o_part == o_lowp) return fail(ST_ERR_INVALID_ARG, "o_lowp aliases o_part");
  if (o_part) ST_TRY(check_f32("o_part", o_part, n_q));
  ST_TRY(check_low("o_lowp", o_lowp));
  ST_TRY(check_f32("lse_part", lse_part, n_q));
  st::CacheAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.c = cache_args(c);
  a.q = view_of(q);
  a.starts = starts;
  a.q_first = q_first;
  a.T = r->T; a.Hq = r->Hq; a.max_rows = r->max_rows; a.causal = r->causal ? 1 : 0; a.window = r->window;
  a.scale = r->scale; a.cap = r->softcap; a.slopes = r->slopes;
  a.o = o_part;
  a.lse = lse_part;
  a.o_lowp = o_lowp;
  const Plans plans = plans_of(r, c);
  const Room room = room_of(plans, r, c);
  ST_TRY(check_workspace(workspace, workspace_bytes, room.bytes, "cache attention"));
  if (room.bytes > 0) {
    a.part_o = (float*)workspace;
    a.part_row = (float4*)((char*)workspace + room.rows);
    a.info = (int4*)((char*)workspace + room.info);
  }
  a.state_rows = plans.rows;
  for (int x = 0; x < plans.n; ++x) {
    a.plan = plans.p[x];
    ST_HIP(a.plan.rows == st::kPromptRows ? st::launch_cache_prompt(a, (hipStream_t)hip_stream) : st::launch_cache_attn(a, r->dtype == ST_BF16, (hipStream_t)hip_stream),
           "st_attn_cache launch");
  }
  if (plans.rows > 0) ST_HIP(st::launch_cache_combine(a, r->dtype == ST_BF16, plans.states, (hipStream_t)hip_stream), "st_attn_cache combine");
  return ST_OK;
}

}  // extern "C"
