// A cache of keys and values in pages: what its kernels share.  Token x of sequence b is row x % page of page table[b][x / page].
//
// Everything that changes from step to step is in device memory, and a wrong number there must not become an address: rows are held
// to [0, T), tokens to the table's width, and an entry of the table that is no page holds nothing.
#pragma once

#include "st_e4m3.h"
#include "st_internal.h"
#include "st_rope.h"

namespace st {

struct CacheArgs {
  int32_t dtype, n_pages, shift, Hkv, D, B, width;   // page = 1 << shift
  View k, v;                                         // [page, token, head]
  uint8_t *k_scale, *v_scale;                        // [n_pages, Hkv], e4m3 only
  const int32_t *table, *lens;
};

struct AppendArgs {
  RopeArgs g;                                        // B = 1, S = T; k: the new keys
  CacheArgs c;
  View v_in;
  const int32_t* starts;
};

struct ReadArgs {
  CacheArgs c;
  const int32_t* first;                              // nullable
  int32_t count;
  View k_out, v_out;                                 // ptr null: not asked for
};

// Which sequences a launch takes and how it is split (st_cache_plan.h)
struct CachePlan {
  int32_t rows;                                      // of a tile: 16, 32, or 128 (prompts)
  int32_t rows_from, rows_to;                        // packed rows (token, head of a group) of a sequence: rows_from < rows <= rows_to
  int32_t least;                                     // key blocks of a share, at least
  int32_t target;                                    // workgroups that the shares are made for
  int32_t states;                                    // partial states there is room for
  int32_t most;                                      // shares of a walk, at most
  int64_t base;                                      // rows of the states of launches before
  int64_t jobs, grid;                                // tiles times KV heads, at most; workgroups
};

struct CacheAttnArgs {
  CacheArgs c;
  View q;                                            // sb unused
  const int32_t* starts;
  const int64_t* q_first;                            // nullable
  int32_t T, Hq, max_rows, causal, window;
  float scale, cap;
  const float* slopes;                               // nullable
  float* o;                                          // nullable, fp32 [T,Hq,D]
  float* lse;                                        // [Hq,T]
  void* o_lowp;                                      // nullable
  CachePlan plan;
  // of a split walk: a state has the rows of its tile, O not divided by its row sum yet, and for each row the reference of its exponents,
  // the sum, and what its lse has besides
  float* part_o;                                     // [state rows, D]
  float4* part_row;                                  // [state rows]
  int64_t state_rows;
  int4* info;                                        // [T]: row of the sequence's first state, shares | rows of a tile << 16, row tiles, row of the sequence
};

constexpr int kCacheKeys = 32;                       // keys of a block
constexpr int kTallCacheHead = 128;                  // the largest head with tiles of 32 rows: of larger ones a lane has no room for its part of O,
                                                     // keys and values (D = 256, fp32: 4 x 20 rows of a group against 2000 tokens 46 us so, 31 in tiles of 16)
constexpr int kPromptRows = 128, kPromptKeys = 64;   // of the kernel for prompts

hipError_t launch_cache_append(const AppendArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_cache_read(const ReadArgs& a, int out_dtype, hipStream_t stream);
hipError_t launch_cache_attn(const CacheAttnArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_cache_prompt(const CacheAttnArgs& a, hipStream_t stream);
// states: so many a row, on the average of what there is room for
hipError_t launch_cache_combine(const CacheAttnArgs& a, bool bf16, int states, hipStream_t stream);

// ---- device side

// rows of sequence b among the T packed ones
struct SeqRows {
  int first, n;
};
__device__ __forceinline__ SeqRows seq_rows(const int32_t* starts, int b, int T) {
  const int s0 = min(max(starts[b], 0), T), s1 = min(max(starts[b + 1], 0), T);
  return SeqRows{s0, max(s1 - s0, 0)};
}
// tokens of sequence b that the table has room for
__device__ __forceinline__ int seq_len(const CacheArgs& c, int b) { return (int)min((int64_t)max(c.lens[b], 0), (int64_t)c.width << c.shift); }
// the page of a sequence's pages j (0 <= j < width), or -1
__device__ __forceinline__ int page_of(const CacheArgs& c, int b, int j) {
  const int p = c.table[(int64_t)b * c.width + j];
  return p >= 0 && p < c.n_pages ? p : -1;
}
// 2^(scale - 127)
__device__ __forceinline__ float scale_value(uint8_t s) { return __uint_as_float((uint32_t)s << 23); }

}  // namespace st
