// Argument checks of the C ABI's entry points, and how a failure is reported.
#pragma once

#include <cstddef>
#include <cstdint>

#include "st_internal.h"

namespace st {

// st_last_error() of the calling thread becomes this text; returns s
st_status fail(st_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
st_status hip_fail(hipError_t e, const char* what);

namespace checks {

inline size_t elem_size(int dtype) { return dtype == ST_BF16 ? 2 : 4; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline st_status check_scale(float scale) {
  if (!(scale > 0.f) || scale > 3.0e38f) return fail(ST_ERR_INVALID_ARG, "scale must be finite and positive");
  return ST_OK;
}

inline st_status check_shape(int dtype, int B, int Hq, int Hkv, int D, int Sq, int Sk) {
  if (dtype != ST_F32 && dtype != ST_BF16) return fail(ST_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (B < 0 || Sq < 0 || Sk < 0) return fail(ST_ERR_INVALID_ARG, "negative size");
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return fail(ST_ERR_INVALID_ARG, "need Hq %% Hkv == 0 (Hq=%d Hkv=%d)", Hq, Hkv);
  if (D <= 0) return fail(ST_ERR_INVALID_ARG, "D must be positive");
  if (dtype == ST_F32 && (D > 256 || D % 8 != 0)) return fail(ST_ERR_UNSUPPORTED, "fp32 path needs D <= 256 and D %% 8 == 0 (D=%d)", D);
  if (dtype == ST_BF16 && D != 128 && D != 64) return fail(ST_ERR_UNSUPPORTED, "bf16 path is built for D = 64 or 128 (D=%d)", D);
  if (B > 65535 || Hq > 65535) return fail(ST_ERR_UNSUPPORTED, "B and Hq must not exceed 65535");
  return ST_OK;
}

// a [B,S,heads,D] view whose rows must be 16-byte aligned
inline st_status check_view(const char* name, const void* ptr, int64_t sb, int64_t ss, int64_t sh, int dtype,
                     int64_t n_elems) {
  if (n_elems == 0) return ST_OK;
  if (ptr == nullptr) return fail(ST_ERR_INVALID_ARG, "%s: null pointer", name);
  const int64_t per16 = 16 / (int64_t)elem_size(dtype);
  if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return fail(ST_ERR_ALIGNMENT, "%s: base pointer is not 16-byte aligned", name);
  if (sb % per16 || ss % per16 || sh % per16) return fail(ST_ERR_ALIGNMENT, "%s: strides must be multiples of %lld elements", name, (long long)per16);
  if (sb < 0 || ss < 0 || sh < 0) return fail(ST_ERR_INVALID_ARG, "%s: negative stride", name);
  return ST_OK;
}

inline st_status check_tensor(const char* name, const st_tensor* t, int dtype, int64_t n_elems) {
  if (t == nullptr) return fail(ST_ERR_INVALID_ARG, "%s: null st_tensor", name);
  return check_view(name, t->ptr, t->stride_b, t->stride_s, t->stride_h, dtype, n_elems);
}

inline st_status check_f32(const char* name, const void* p, int64_t n_elems) {
  if (n_elems == 0) return ST_OK;
  if (p == nullptr) return fail(ST_ERR_INVALID_ARG, "%s: null pointer", name);
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(ST_ERR_ALIGNMENT, "%s: not 16-byte aligned", name);
  return ST_OK;
}

inline st::View view_of(const st_tensor* t) { return st::View{t->ptr, t->stride_b, t->stride_s, t->stride_h}; }

inline st::Shape shape_of(const st_block_desc* d) {
  return st::Shape{d->B, d->Hq, d->Hkv, d->D, d->Sq, d->Sk, d->q_offset, d->causal ? 1 : 0, d->scale, d->q_seg, d->q_offset2};
}
inline st::Shape shape_of(const st_ring_desc* d) {
  return st::Shape{d->B, d->Hq, d->Hkv, d->D, d->Sq, d->Sk, d->q_offset, d->causal ? 1 : 0, d->scale, d->q_seg, d->q_offset2};
}

// two runs of query rows: the second must not start before the first ends (positions rise with the row index)
inline st_status check_segments(int32_t Sq, int64_t q_offset, int32_t q_seg, int64_t q_offset2) {
  if (q_seg == 0) return ST_OK;
  if (q_seg < 0 || q_seg >= Sq) return fail(ST_ERR_INVALID_ARG, "q_seg = %d must be 0 or inside the %d query rows", q_seg, Sq);
  if (q_offset2 < q_offset + q_seg) return fail(ST_ERR_INVALID_ARG, "second run of query rows starts before the first ends");
  return ST_OK;
}

#define ST_TRY(expr)                  \
  do {                                \
    st_status _s = (expr);            \
    if (_s != ST_OK) return _s;       \
  } while (0)
#define ST_HIP(expr, what)                        \
  do {                                            \
    hipError_t _e = (expr);                       \
    if (_e != hipSuccess) return hip_fail(_e, what); \
  } while (0)

}  // namespace checks
}  // namespace st
