// Native argument marshalling of the calls a training step makes many times: torch tensors, lists and numbers straight into
// the structs of the C ABI (include/startrail.h).  Bounded by nothing but instructions; through ctypes a ring call with 8
// chunks took 15 us (forward) and 30 us (backward) of Python beside the 4 to 13 us its launches take, more with more chunks,
// and small shares were that much host time: 128 rows of one fp32 head 68 us a pass for 43 us of kernels.
//
// Every function returns the status of the call, or None without having called anything when an argument is not what the
// short way takes (another sequence type, a tensor subclass, a shape or dtype that does not fit ...): the Python wrapper
// then goes the general way, which accepts what is acceptable and raises the error that belongs to the rest.
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/startrail.h"

namespace {

// ---- arguments; false: not for the short way
using Tensor = const at::Tensor*;

bool tensor(PyObject* o, Tensor* t) {
  if (!THPVariable_CheckExact(o)) return false;
  *t = &THPVariable_Unpack(o);
  const at::Tensor& x = **t;
  if (!x.defined() || x.layout() != at::kStrided || !x.is_cuda() || !x.has_storage()) return false;
  // wrappers of transforms, fake and lazy tensors and views with a pending operation have other keys
  const auto plain = c10::DispatchKeySet({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView,
                                          c10::DispatchKey::AutocastCUDA});
  return ((x.key_set() - plain).raw_repr() & ~c10::full_backend_mask) == 0;
}
void* address(Tensor t) { return t->numel() ? t->data_ptr() : nullptr; }
bool pointer(PyObject* o, void** p) {          // None: null
  *p = nullptr;
  Tensor t;
  if (o == Py_None) return true;
  if (!tensor(o, &t)) return false;
  *p = address(t);
  return true;
}
bool dtype_code(Tensor t, int32_t* code) {
  *code = t->scalar_type() == at::kFloat ? ST_F32 : ST_BF16;
  return t->scalar_type() == at::kFloat || t->scalar_type() == at::kBFloat16;
}
bool dense_f32(PyObject* o, at::IntArrayRef shape, float** p) {
  Tensor t;
  if (!tensor(o, &t) || t->scalar_type() != at::kFloat || t->sizes() != shape || !t->is_contiguous()) return false;
  *p = (float*)address(t);
  return true;
}
bool strides_fit(Tensor t) { return t->dim() == 4 && (t->stride(3) == 1 || t->size(3) <= 1); }
bool view(PyObject* o, Tensor* t, st_tensor* v) {
  if (!tensor(o, t) || !strides_fit(*t)) return false;
  *v = st_tensor{address(*t), (*t)->stride(0), (*t)->stride(1), (*t)->stride(2)};
  return true;
}
bool integer(PyObject* o, int64_t* x) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  *x = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0;
}
bool integer(PyObject* o, int32_t* x) {
  int64_t y;
  if (!integer(o, &y) || y < INT32_MIN || y > INT32_MAX) return false;
  *x = (int32_t)y;
  return true;
}
bool real(PyObject* o, float* x) {
  if (!PyFloat_CheckExact(o)) return false;
  *x = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
bool truth(PyObject* o, int32_t* x) {
  *x = o == Py_True;
  return o == Py_True || o == Py_False;
}
bool handle(PyObject* o, void** p) {
  int64_t x;
  if (!integer(o, &x)) return false;
  *p = (void*)x;
  return true;
}
struct Items {
  Py_ssize_t n = 0;
  PyObject** at = nullptr;
};
bool items(PyObject* o, Items* s) {
  if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
  s->n = PySequence_Fast_GET_SIZE(o);
  s->at = PySequence_Fast_ITEMS(o);
  return true;
}
bool integers(PyObject* o, int32_t* to, Py_ssize_t most, Py_ssize_t* n) {
  Items s;
  if (!items(o, &s) || s.n > most) return false;
  for (Py_ssize_t i = 0; i < s.n; ++i)
    if (!integer(s.at[i], to + i)) return false;
  *n = s.n;
  return true;
}
template <typename Desc>
bool where(PyObject* o, Desc* d) {             // position of row 0, or (position, rows of the first run, position of the second)
  d->q_seg = 0;
  d->q_offset2 = 0;
  if (!PyTuple_CheckExact(o)) return integer(o, &d->q_offset);
  return PyTuple_GET_SIZE(o) == 3 && integer(PyTuple_GET_ITEM(o, 0), &d->q_offset) && integer(PyTuple_GET_ITEM(o, 1), &d->q_seg) &&
         integer(PyTuple_GET_ITEM(o, 2), &d->q_offset2);
}
template <typename Desc>
bool shape(Tensor q, Desc* d) {
  if (q->dim() != 4 || !dtype_code(q, &d->dtype)) return false;
  for (int i = 0; i < 4; ++i)
    if (q->size(i) > INT32_MAX) return false;
  d->B = (int32_t)q->size(0);
  d->Sq = (int32_t)q->size(1);
  d->Hq = (int32_t)q->size(2);
  d->D = (int32_t)q->size(3);
  return true;
}
bool bytes_of(PyObject* o, void** p, size_t* n) {   // first 256-byte boundary of a buffer and what is left from there
  Tensor t;
  if (!tensor(o, &t)) return false;
  const uintptr_t at = (uintptr_t)t->data_ptr(), up = (at + 255) / 256 * 256;
  const size_t have = (size_t)t->numel() * t->element_size();
  if (have < up - at) return false;
  *p = (void*)up;
  *n = have - (up - at);
  return true;
}

// the tables of a ring call
struct Ring {
  st_ring_desc d;
  Tensor q, k0;
  st_tensor tq;
  const void *k[ST_MAX_CHUNKS], *v[ST_MAX_CHUNKS];
  int64_t k_offset[ST_MAX_CHUNKS];
  int32_t order[ST_MAX_CHUNKS];
  Py_ssize_t n_visit;
  int32_t mode;

  bool chunks(PyObject* o, const void** to, Tensor first, int64_t* strides) {
    Items s;
    if (!items(o, &s) || s.n != d.n_chunks) return false;
    Tensor t0 = nullptr;
    for (Py_ssize_t i = 0; i < s.n; ++i) {
      Tensor t;
      if (!tensor(s.at[i], &t)) return false;
      if (i == 0) {
        t0 = t;
        if (!strides_fit(t)) return false;
        if (first == nullptr) first = k0 = t;
      }
      if (t->sizes() != first->sizes() || t->strides() != t0->strides() || t->scalar_type() != q->scalar_type()) return false;
      to[i] = t->data_ptr();
    }
    for (int i = 0; i < 3; ++i) strides[i] = t0->stride(i);
    return true;
  }
  bool read(PyObject* oq, PyObject* ks, PyObject* vs, PyObject* q_where, PyObject* k_offsets, PyObject* causal, PyObject* scale,
            PyObject* visit, PyObject* mode_) {
    Items off;
    if (!items(k_offsets, &off) || off.n < 1 || off.n > ST_MAX_CHUNKS) return false;
    d.n_chunks = (int32_t)off.n;
    for (Py_ssize_t i = 0; i < off.n; ++i)
      if (!integer(off.at[i], k_offset + i)) return false;
    if (!view(oq, &q, &tq) || !shape(q, &d) || !where(q_where, &d) || !truth(causal, &d.causal) || !real(scale, &d.scale)) return false;
    if (!chunks(ks, k, nullptr, &d.k_stride_b) || !chunks(vs, v, k0, &d.v_stride_b)) return false;
    if (k0->size(1) > INT32_MAX || k0->size(2) > INT32_MAX) return false;
    d.Sk = (int32_t)k0->size(1);
    d.Hkv = (int32_t)k0->size(2);
    d.k_ptr = k;
    d.v_ptr = v;
    d.k_offset = k_offset;
    return integers(visit, order, ST_MAX_CHUNKS, &n_visit) && integer(mode_, &mode);
  }
  at::IntArrayRef q_shape() const { return q->sizes(); }
  std::array<int64_t, 3> stat_shape() const { return {d.B, d.Hq, d.Sq}; }
};
static_assert(offsetof(st_ring_desc, k_stride_h) == offsetof(st_ring_desc, k_stride_b) + 16 &&
              offsetof(st_ring_desc, v_stride_h) == offsetof(st_ring_desc, v_stride_b) + 16, "strides lie side by side");

// gradient accumulators (fp32) or their copies (low: the dtype of q) per chunk, None where there is none
bool tables(PyObject* o, const Ring& r, bool low, void** to) {
  Items s;
  if (!items(o, &s) || s.n != r.d.n_chunks) return false;
  for (Py_ssize_t i = 0; i < s.n; ++i) {
    to[i] = nullptr;
    if (s.at[i] == Py_None) continue;
    Tensor t;
    if (!tensor(s.at[i], &t) || t->scalar_type() != (low ? r.q->scalar_type() : at::kFloat) || t->sizes() != r.k0->sizes() || !t->is_contiguous()) return false;
    to[i] = t->data_ptr();
  }
  return true;
}

struct Unlocked {                              // other Python threads run meanwhile
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
PyObject* call(F f) {
  st_status s;
  {
    Unlocked u;
    s = f();
  }
  return PyLong_FromLong(s);
}
// Python calls in through C: an exception of a tensor's accessors (memory that may not be touched, a copy on write that does not
// fit) must not leave here.  Nothing has been called yet then; the general way meets the same exception and raises it.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (...) {
    Py_RETURN_NONE;
  }
}
#define ST_SHORT(cond) \
  if (!(cond)) Py_RETURN_NONE

// ring_fwd(q, ks, vs, where, k_offsets, causal, scale, order, members, mode, o, lse, o_low, workspace, stream)
PyObject* ring_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 15);
  Ring r;
  int32_t members[ST_MAX_CHUNKS];
  Py_ssize_t n_members = 0;
  float *o, *lse;
  void *low, *ws, *stream;
  size_t ws_bytes;
  ST_SHORT(r.read(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[9]));
  const bool has_members = a[8] != Py_None;
  ST_SHORT(!has_members || (integers(a[8], members, ST_MAX_CHUNKS, &n_members) && n_members == r.n_visit));
  ST_SHORT(dense_f32(a[10], r.q_shape(), &o) && dense_f32(a[11], r.stat_shape(), &lse) && pointer(a[12], &low) &&
           bytes_of(a[13], &ws, &ws_bytes) && handle(a[14], &stream));
  return call([&] {
    return st_ring_fwd(&r.d, &r.tq, r.order, has_members ? members : nullptr, (int32_t)r.n_visit, r.mode, o, lse, low, ws, ws_bytes, stream);
  });
}

// ring_bwd(q, ks, vs, d_o, o, lse, where, k_offsets, causal, scale, order, dq, dk, dv, assign, dk_low, dv_low, mode, workspace,
// stream): st_ring_bwd_last, or st_ring_bwd_noalloc where the workspace is None (then without assign and copies)
PyObject* ring_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 20);
  Ring r;
  Tensor t_do, t_o;
  st_tensor tdo, to;
  int32_t o_dtype, assign;
  float *lse, *dq;
  void *dk[ST_MAX_CHUNKS], *dv[ST_MAX_CHUNKS], *lk[ST_MAX_CHUNKS], *lv[ST_MAX_CHUNKS], *ws = nullptr, *stream;
  size_t ws_bytes = 0;
  ST_SHORT(r.read(a[0], a[1], a[2], a[6], a[7], a[8], a[9], a[10], a[17]));
  ST_SHORT(view(a[3], &t_do, &tdo) && view(a[4], &t_o, &to) && dtype_code(t_o, &o_dtype) && dense_f32(a[5], r.stat_shape(), &lse) &&
           dense_f32(a[11], r.q_shape(), &dq) && tables(a[12], r, false, dk) && tables(a[13], r, false, dv) && truth(a[14], &assign));
  const bool low_k = a[15] != Py_None, low_v = a[16] != Py_None, own = a[18] == Py_None;
  ST_SHORT((!low_k || tables(a[15], r, true, lk)) && (!low_v || tables(a[16], r, true, lv)) && handle(a[19], &stream));
  ST_SHORT(own ? !assign && !low_k && !low_v : bytes_of(a[18], &ws, &ws_bytes));
  return call([&] {
    if (own)
      return st_ring_bwd_noalloc(&r.d, &r.tq, &tdo, &to, o_dtype, lse, r.order, (int32_t)r.n_visit, r.mode, dq, (float* const*)dk, (float* const*)dv, stream);
    return st_ring_bwd_last(&r.d, &r.tq, &tdo, &to, o_dtype, lse, r.order, (int32_t)r.n_visit, r.mode, dq, (float* const*)dk, (float* const*)dv,
                            assign ? ST_KV_ASSIGN : 0, low_k ? lk : nullptr, low_v ? lv : nullptr, ws, ws_bytes, stream);
  });
}

bool block(PyObject* oq, PyObject* ok, PyObject* ov, PyObject* q_where, PyObject* k_offset, PyObject* causal, PyObject* scale, st_block_desc* d,
           Tensor* q, Tensor* k, st_tensor* tq, st_tensor* tk, st_tensor* tv) {
  Tensor v;
  if (!view(oq, q, tq) || !view(ok, k, tk) || !view(ov, &v, tv) || !shape(*q, d) || !where(q_where, d) || !integer(k_offset, &d->k_offset) ||
      !truth(causal, &d->causal) || !real(scale, &d->scale))
    return false;
  if ((*k)->size(1) > INT32_MAX || (*k)->size(2) > INT32_MAX) return false;
  d->Sk = (int32_t)(*k)->size(1);
  d->Hkv = (int32_t)(*k)->size(2);
  return true;
}

// block_fwd(q, k, v, where, k_offset, causal, scale, o, lse, stream)
PyObject* block_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 10);
  st_block_desc d;
  Tensor q, k;
  st_tensor tq, tk, tv;
  float *o, *lse;
  void* stream;
  ST_SHORT(block(a[0], a[1], a[2], a[3], a[4], a[5], a[6], &d, &q, &k, &tq, &tk, &tv));
  ST_SHORT(dense_f32(a[7], q->sizes(), &o) && dense_f32(a[8], {d.B, d.Hq, d.Sq}, &lse) && handle(a[9], &stream));
  return call([&] { return st_attn_block_fwd(&d, &tq, &tk, &tv, o, lse, stream); });
}

// block_bwd(q, k, v, d_o, lse, delta, where, k_offset, causal, scale, dq, dk, dv, workspace, stream)
PyObject* block_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 15);
  st_block_desc d;
  Tensor q, k, t_do;
  st_tensor tq, tk, tv, tdo;
  float *lse, *delta, *dq, *dk, *dv;
  void *ws, *stream;
  size_t ws_bytes;
  ST_SHORT(block(a[0], a[1], a[2], a[6], a[7], a[8], a[9], &d, &q, &k, &tq, &tk, &tv));
  ST_SHORT(view(a[3], &t_do, &tdo) && dense_f32(a[4], {d.B, d.Hq, d.Sq}, &lse) && dense_f32(a[5], {d.B, d.Hq, d.Sq}, &delta) &&
           dense_f32(a[10], q->sizes(), &dq) && dense_f32(a[11], {d.B, d.Sk, d.Hkv, d.D}, &dk) && dense_f32(a[12], {d.B, d.Sk, d.Hkv, d.D}, &dv) &&
           bytes_of(a[13], &ws, &ws_bytes) && handle(a[14], &stream));
  return call([&] { return st_attn_block_bwd(&d, &tq, &tk, &tv, &tdo, lse, delta, dq, dk, dv, ws, ws_bytes, stream); });
}

// a dense copy of shape `s` in out_dtype, or None
bool low_copy(PyObject* o, at::IntArrayRef s, int32_t out_dtype, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  Tensor t;
  int32_t code;
  if (!tensor(o, &t) || t->sizes() != s || !t->is_contiguous() || !dtype_code(t, &code) || code != out_dtype) return false;
  *p = address(t);
  return true;
}

// merge(o, lse, o_part, lse_part, out_dtype, o_low, stream)
PyObject* merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 7);
  Tensor t;
  float *o, *lse, *op, *lp;
  void *low, *stream;
  int32_t out;
  ST_SHORT(tensor(a[0], &t) && t->dim() == 4 && dense_f32(a[0], t->sizes(), &o) && dense_f32(a[2], t->sizes(), &op));
  const int64_t B = t->size(0), S = t->size(1), H = t->size(2), D = t->size(3);
  ST_SHORT(B <= INT32_MAX && S <= INT32_MAX && H <= INT32_MAX && D <= INT32_MAX);
  ST_SHORT(dense_f32(a[1], {B, H, S}, &lse) && dense_f32(a[3], {B, H, S}, &lp) && integer(a[4], &out) && low_copy(a[5], t->sizes(), out, &low) &&
           handle(a[6], &stream));
  return call([&] { return st_attn_merge(o, lse, op, lp, (int32_t)B, (int32_t)S, (int32_t)H, (int32_t)D, out, low, stream); });
}

// combine(o_parts, lse_parts, row0, rows, out_dtype, o, lse, o_low, stream)
PyObject* combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 9);
  Items so, sl;
  const float *op[ST_MAX_CHUNKS], *lp[ST_MAX_CHUNKS];
  int32_t row0, rows, out;
  ST_SHORT(items(a[0], &so) && items(a[1], &sl) && so.n == sl.n && so.n > 0 && so.n <= ST_MAX_CHUNKS && integer(a[2], &row0) && integer(a[3], &rows) &&
           integer(a[4], &out));
  Tensor t;
  ST_SHORT(tensor(so.at[0], &t) && t->dim() == 4);
  const int64_t B = t->size(0), S = t->size(1), H = t->size(2), D = t->size(3);
  ST_SHORT(B <= INT32_MAX && S <= INT32_MAX && H <= INT32_MAX && D <= INT32_MAX && rows >= 0);
  for (Py_ssize_t i = 0; i < so.n; ++i)
    ST_SHORT(dense_f32(so.at[i], t->sizes(), (float**)&op[i]) && dense_f32(sl.at[i], {B, H, S}, (float**)&lp[i]));
  float *o, *lse;
  void *low, *stream;
  ST_SHORT(dense_f32(a[5], {B, rows, H, D}, &o) && dense_f32(a[6], {B, H, rows}, &lse) && low_copy(a[7], {B, rows, H, D}, out, &low) &&
           handle(a[8], &stream));
  return call([&] {
    return st_attn_combine(op, lp, (int32_t)so.n, (int32_t)B, (int32_t)S, (int32_t)H, (int32_t)D, row0, rows, o, lse, out, low, stream);
  });
}

// delta(d_o, o, delta, stream)
PyObject* delta(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 4);
  st_block_desc d;
  memset(&d, 0, sizeof(d));
  Tensor t_do, t_o;
  st_tensor tdo, to;
  int32_t o_dtype;
  float* out;
  void* stream;
  ST_SHORT(view(a[0], &t_do, &tdo) && view(a[1], &t_o, &to) && shape(t_do, &d) && dtype_code(t_o, &o_dtype) &&
           dense_f32(a[2], {d.B, d.Hq, d.Sq}, &out) && handle(a[3], &stream));
  d.Hkv = d.Hq;
  d.scale = 1.f;
  return call([&] { return st_attn_delta(&d, &tdo, &to, o_dtype, out, stream); });
}

// cast(src, dst, dst_dtype, stream)
PyObject* cast(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 4);
  Tensor src, dst;
  int32_t out, code;
  void* stream;
  ST_SHORT(tensor(a[0], &src) && tensor(a[1], &dst) && integer(a[2], &out) && handle(a[3], &stream));
  ST_SHORT(src->scalar_type() == at::kFloat && src->is_contiguous() && dst->is_contiguous() && dst->numel() == src->numel() &&
           dtype_code(dst, &code) && code == out);
  float* from = (float*)address(src);
  void* to = address(dst);
  const int64_t count = src->numel();
  return call([&] { return st_cast_from_f32(from, to, count, out, stream); });
}

// ---- the calls that make their own outputs: (status, outputs...) or None.  Tensors have to be on the current device, which the
// caller says, as the outputs and the workspace are made on it.
struct Made {
  at::Tensor t[4];
  at::TensorOptions on;
  float* f32(int i, at::IntArrayRef s) { return (float*)made(i, s, at::kFloat); }
  void* made(int i, at::IntArrayRef s, at::ScalarType type) {
    t[i] = at::empty(s, on.dtype(type));
    return address(&t[i]);
  }
};
bool here(Tensor t, int64_t device) { return t->get_device() == device; }
bool dense_of(PyObject* o, at::IntArrayRef shape, at::ScalarType type, int64_t device, void** p) {
  Tensor t;
  if (!tensor(o, &t) || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous() || !here(t, device)) return false;
  *p = address(t);
  return true;
}
bool dense_or_none(PyObject* o, at::IntArrayRef shape, at::ScalarType type, int64_t device, void** p) {
  *p = nullptr;
  return o == Py_None || dense_of(o, shape, type, device, p);
}
// a workspace that the caller gives, or one of `need` bytes
bool workspace_of(PyObject* o, size_t need, int64_t device, Made* m, int slot, void** p, size_t* n) {
  *p = nullptr;
  *n = 0;
  if (o != Py_None) {
    Tensor t;
    return tensor(o, &t) && here(t, device) && bytes_of(o, p, n);
  }
  if (need == 0) return true;
  *p = m->made(slot, {(int64_t)need}, at::kByte);    // (the allocator's blocks lie on 512-byte boundaries)
  *n = need;
  return (uintptr_t)*p % 256 == 0;
}
PyObject* answer(PyObject* status, std::initializer_list<PyObject*> out) {
  if (status == nullptr) return nullptr;
  PyObject* all = PyTuple_New(1 + (Py_ssize_t)out.size());
  if (all == nullptr) return nullptr;
  PyTuple_SET_ITEM(all, 0, status);
  Py_ssize_t i = 1;
  for (PyObject* x : out) PyTuple_SET_ITEM(all, i++, x);
  return all;
}
PyObject* given_or(PyObject* o, const at::Tensor& t) {
  if (!t.defined()) {
    Py_INCREF(o);
    return o;
  }
  return THPVariable_Wrap(t);
}

// mask_spans(bounds, rows, where, causal, prefix, spans, device, stream)
PyObject* mask_spans(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 8);
  Tensor b;
  st_block_desc d;
  int64_t device;
  int32_t causal;
  void *prefix, *spans, *stream;
  ST_SHORT(tensor(a[0], &b) && b->dim() == 2 && b->size(1) >= 1 && b->scalar_type() == at::kLong && b->is_contiguous() && integer(a[6], &device) && here(b, device));
  ST_SHORT(b->size(0) <= INT32_MAX && b->size(1) <= INT32_MAX && integer(a[1], &d.Sq) && d.Sq >= 0 && where(a[2], &d) && truth(a[3], &causal));
  const int64_t B = b->size(0), docs = b->size(1) - 1;
  ST_SHORT(dense_or_none(a[4], {B, docs}, at::kLong, device, &prefix) && dense_or_none(a[5], {B, d.Sq, 2}, at::kLong, device, &spans) && handle(a[7], &stream));
  Made m;
  m.on = b->options();
  if (a[5] == Py_None) spans = m.made(0, {B, d.Sq, 2}, at::kLong);
  const int64_t* bounds = (const int64_t*)address(b);
  PyObject* s = call([&] {
    return st_mask_spans((int32_t)B, d.Sq, d.q_offset, d.q_seg, d.q_offset2, causal, bounds, (int32_t)docs, (const int64_t*)prefix, (int64_t*)spans, stream);
  });
  return answer(s, {given_or(a[5], m.t[0])});
}

// q, k, v, where, k_offset, causal, scale at a[0 .. 6]; softcap, slopes, spans at a[at]
bool scored(PyObject* const* a, PyObject* const* mods, int64_t device, st_block_desc* d, st_score* m, Tensor* q, Tensor* k, st_tensor* tq, st_tensor* tk, st_tensor* tv) {
  Tensor v;
  if (!block(a[0], a[1], a[2], a[3], a[4], a[5], a[6], d, q, k, tq, tk, tv) || !tensor(a[2], &v)) return false;
  if (v->sizes() != (*k)->sizes() || (*k)->size(0) != d->B || (*k)->size(3) != d->D || (*k)->scalar_type() != (*q)->scalar_type() || v->scalar_type() != (*q)->scalar_type()) return false;
  if (!here(*q, device) || !here(*k, device) || !here(v, device) || !real(mods[0], &m->softcap)) return false;
  return dense_or_none(mods[1], {d->Hq}, at::kFloat, device, (void**)&m->slopes) && dense_or_none(mods[2], {d->B, d->Sq, 2}, at::kLong, device, (void**)&m->spans);
}

// score_fwd(q, k, v, where, k_offset, causal, scale, softcap, slopes, spans, o, lse, o_low, lowp, workspace, device, stream): O (the
// fp32 one where it is written) and lse
PyObject* score_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 17);
  st_block_desc d;
  st_score m;
  Tensor q, k;
  st_tensor tq, tk, tv;
  int64_t device;
  int32_t lowp;
  void *o, *lse, *low, *ws, *stream;
  size_t ws_bytes;
  ST_SHORT(integer(a[15], &device) && scored(a, a + 7, device, &d, &m, &q, &k, &tq, &tk, &tv) && truth(a[13], &lowp) && handle(a[16], &stream));
  ST_SHORT(dense_or_none(a[10], q->sizes(), at::kFloat, device, &o) && dense_or_none(a[11], {d.B, d.Hq, d.Sq}, at::kFloat, device, &lse) &&
           dense_or_none(a[12], q->sizes(), q->scalar_type(), device, &low));
  Made x;
  x.on = q->options();
  const bool want_low = a[12] == Py_None && lowp, want_o = a[10] == Py_None && a[12] == Py_None && !lowp;
  ST_SHORT(workspace_of(a[14], st_attn_score_workspace_bytes(&d, &m, 0), device, &x, 2, &ws, &ws_bytes));
  if (want_low) low = x.made(0, q->sizes(), q->scalar_type());
  if (want_o) o = x.f32(0, q->sizes());
  if (a[11] == Py_None) lse = x.f32(1, {d.B, d.Hq, d.Sq});
  PyObject* s = call([&] { return st_attn_score_fwd(&d, &m, &tq, &tk, &tv, (float*)o, (float*)lse, low, ws, ws_bytes, stream); });
  PyObject* first = a[10] != Py_None ? given_or(a[10], at::Tensor()) : given_or(a[12], x.t[0]);
  return answer(s, {first, given_or(a[11], x.t[1])});
}

// score_bwd(q, k, v, where, k_offset, causal, scale, softcap, slopes, spans, d_o, lse, delta, dq, dk, dv, assign, workspace, device, stream):
// the fp32 accumulators, or, where they are None, new gradients in the dtype of q
PyObject* score_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 20);
  st_block_desc d;
  st_score m;
  Tensor q, k, t_do;
  st_tensor tq, tk, tv, tdo;
  int64_t device;
  int32_t assign;
  void *lse, *delta, *acc[3], *low[3] = {nullptr, nullptr, nullptr}, *ws, *stream;
  size_t ws_bytes;
  ST_SHORT(integer(a[18], &device) && scored(a, a + 7, device, &d, &m, &q, &k, &tq, &tk, &tv) && truth(a[16], &assign) && handle(a[19], &stream));
  ST_SHORT(view(a[10], &t_do, &tdo) && here(t_do, device) && t_do->sizes() == q->sizes() && t_do->scalar_type() == q->scalar_type() &&
           dense_of(a[11], {d.B, d.Hq, d.Sq}, at::kFloat, device, &lse) && dense_of(a[12], {d.B, d.Hq, d.Sq}, at::kFloat, device, &delta));
  const bool alone = a[13] == Py_None;
  ST_SHORT((a[14] == Py_None) == alone && (a[15] == Py_None) == alone);
  for (int i = 0; i < 3; ++i) ST_SHORT(dense_or_none(a[13 + i], i ? k->sizes() : q->sizes(), at::kFloat, device, &acc[i]));
  Made x;
  x.on = q->options();
  ST_SHORT(workspace_of(a[17], st_attn_score_workspace_bytes(&d, &m, 1), device, &x, 3, &ws, &ws_bytes));
  if (alone)
    for (int i = 0; i < 3; ++i) low[i] = x.made(i, i ? k->sizes() : q->sizes(), q->scalar_type());
  PyObject* s = call([&] {
    return st_attn_score_bwd(&d, &m, &tq, &tk, &tv, &tdo, (float*)lse, (float*)delta, assign || alone ? ST_GRAD_ASSIGN : 0, (float*)acc[0], (float*)acc[1],
                             (float*)acc[2], low[0], low[1], low[2], ws, ws_bytes, stream);
  });
  return answer(s, {given_or(a[13], x.t[0]), given_or(a[14], x.t[1]), given_or(a[15], x.t[2])});
}

// q, k, freq, where, positions, axes, pairing, norm, eps, q_weight, k_weight at a[0 .. 10]
struct Rope {
  st_rope_desc d;
  Tensor q, k = nullptr;
  st_tensor tq, tk = {nullptr, 0, 0, 0};
  void *freq, *positions, *qw, *kw;
  bool read(PyObject* const* a, int64_t device) {
    Tensor f;
    st_block_desc at_rows;
    if (!view(a[0], &q, &tq) || !here(q, device) || !dtype_code(q, &d.dtype) || !tensor(a[2], &f)) return false;
    for (int i = 0; i < 4; ++i)
      if (q->size(i) > INT32_MAX) return false;
    d.B = (int32_t)q->size(0); d.S = (int32_t)q->size(1); d.Hq = (int32_t)q->size(2); d.D = (int32_t)q->size(3);
    d.Hkv = 0;
    if (a[1] != Py_None) {
      if (!view(a[1], &k, &tk) || !here(k, device) || k->scalar_type() != q->scalar_type() || k->size(0) != d.B || k->size(1) != d.S || k->size(3) != d.D ||
          k->size(2) > INT32_MAX)
        return false;
      d.Hkv = (int32_t)k->size(2);
    }
    const int64_t half = f->numel();
    if (half > 1 << 20 || !dense_of(a[2], {half}, at::kDouble, device, &freq) || !where(a[3], &at_rows)) return false;
    d.rot = (int32_t)(2 * half);
    d.offset = at_rows.q_offset; d.seg = at_rows.q_seg; d.offset2 = at_rows.q_offset2;
    Py_ssize_t n = 1;
    int64_t sum = 0;
    memset(d.axis_pairs, 0, sizeof(d.axis_pairs));
    d.axis_pairs[0] = (int32_t)half;
    if (a[5] != Py_None && !integers(a[5], d.axis_pairs, ST_ROPE_MAX_AXES, &n)) return false;
    for (Py_ssize_t i = 0; i < n; ++i) sum += d.axis_pairs[i];
    if (n < 1 || sum != half) return false;
    d.n_axes = (int32_t)n;
    return dense_or_none(a[4], {(int64_t)n, d.B, d.S}, at::kInt, device, &positions) && integer(a[6], &d.pairing) && truth(a[7], &d.norm) && real(a[8], &d.eps) &&
           dense_or_none(a[9], {d.D}, at::kFloat, device, &qw) && dense_or_none(a[10], {d.D}, at::kFloat, device, &kw);
  }
  // an output like `t`: the one given (None: a new one)
  bool out(PyObject* o, Tensor t, int64_t device, Made* m, int slot, st_tensor* v) {
    if (o == Py_None) {
      m->made(slot, t->sizes(), t->scalar_type());
      *v = st_tensor{address(&m->t[slot]), m->t[slot].stride(0), m->t[slot].stride(1), m->t[slot].stride(2)};
      return true;
    }
    Tensor x;
    return view(o, &x, v) && here(x, device) && x->sizes() == t->sizes() && x->scalar_type() == t->scalar_type();
  }
};

// rope_fwd(..., q_out, k_out, device, stream)
PyObject* rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 15);
  Rope r;
  Made m;
  st_tensor oq, ok = {nullptr, 0, 0, 0};
  int64_t device;
  void* stream;
  ST_SHORT(integer(a[13], &device) && handle(a[14], &stream) && r.read(a, device));
  m.on = r.q->options();
  ST_SHORT(r.out(a[11], r.q, device, &m, 0, &oq) && (r.k == nullptr ? a[12] == Py_None : r.out(a[12], r.k, device, &m, 1, &ok)));
  PyObject* s = call([&] {
    return st_qk_rope_fwd(&r.d, &r.tq, &r.tk, (const float*)r.qw, (const float*)r.kw, (const double*)r.freq, (const int32_t*)r.positions, &oq, &ok, stream);
  });
  return answer(s, {given_or(a[11], m.t[0]), given_or(a[12], m.t[1])});
}

// rope_bwd(..., d_q, d_k, dx_q, dx_k, workspace, device, stream): gradients of the weights in new tensors where there are weights
PyObject* rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ST_SHORT(n == 18);
  Rope r;
  Made m, w;
  Tensor gq, gk = nullptr;
  st_tensor tgq, tgk = {nullptr, 0, 0, 0}, oq, ok = {nullptr, 0, 0, 0};
  int64_t device;
  int32_t d_dtype;
  void *ws = nullptr, *stream;
  size_t ws_bytes = 0;
  ST_SHORT(integer(a[16], &device) && handle(a[17], &stream) && r.read(a, device));
  ST_SHORT(view(a[11], &gq, &tgq) && here(gq, device) && gq->sizes() == r.q->sizes() && dtype_code(gq, &d_dtype));
  if (r.k != nullptr) ST_SHORT(view(a[12], &gk, &tgk) && here(gk, device) && gk->sizes() == r.k->sizes() && gk->scalar_type() == gq->scalar_type());
  m.on = w.on = r.q->options();
  ST_SHORT(r.out(a[13], r.q, device, &m, 0, &oq) && (r.k == nullptr ? a[14] == Py_None : r.out(a[14], r.k, device, &m, 1, &ok)));
  float *dwq = nullptr, *dwk = nullptr;
  if (r.qw) dwq = w.f32(0, {r.d.D});
  if (r.kw && r.k != nullptr) dwk = w.f32(1, {r.d.D});
  if (dwq || dwk) ST_SHORT(workspace_of(a[15], st_qk_rope_bwd_workspace_bytes(&r.d), device, &w, 2, &ws, &ws_bytes));
  PyObject* s = call([&] {
    return st_qk_rope_bwd(&r.d, &r.tq, &r.tk, &tgq, &tgk, d_dtype, (const float*)r.qw, (const float*)r.kw, (const double*)r.freq, (const int32_t*)r.positions,
                          ST_GRAD_ASSIGN, &oq, &ok, dwq, dwk, ws, ws_bytes, stream);
  });
  return answer(s, {given_or(a[13], m.t[0]), given_or(a[14], m.t[1]), given_or(Py_None, w.t[0]), given_or(Py_None, w.t[1])});
}

#define ST_METHOD(f) {#f, (PyCFunction)(void*)guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ST_METHOD(ring_fwd), ST_METHOD(ring_bwd), ST_METHOD(block_fwd), ST_METHOD(block_bwd), ST_METHOD(merge),
                         ST_METHOD(combine),  ST_METHOD(delta),    ST_METHOD(cast),
                         ST_METHOD(mask_spans), ST_METHOD(score_fwd), ST_METHOD(score_bwd), ST_METHOD(rope_fwd), ST_METHOD(rope_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "built_for", ST_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
