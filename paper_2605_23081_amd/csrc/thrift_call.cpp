// Python entry of the calls a serving loop makes for every token or prompt: checks the tensors, allocates what the caller
// left out and calls the C ABI, without a Python object per pointer and shape (ctypes: 20 us of host time for a decode
// call, as long as its kernels take on a short cache; here 2 us).
//
// Every function returns the result, or the C call's status as an int when it is not THRIFT_OK, or None when the
// arguments are not of the plain kind that is served here; the caller then takes its general path, which names what is
// wrong with them.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>

#include "thrift.h"

namespace {

using at::Tensor;

bool tensor(PyObject* o, const Tensor** t) {
  if (!THPVariable_Check(o)) return false;
  *t = &THPVariable_Unpack(o);
  return (*t)->is_cuda() && (*t)->is_contiguous();
}
bool optional(PyObject* o, const Tensor** t) {
  if (o == Py_None) { *t = nullptr; return true; }
  return tensor(o, t);
}
bool is(const Tensor& t, at::ScalarType dt, std::initializer_list<int64_t> shape) {
  return t.scalar_type() == dt && t.sizes() == at::IntArrayRef(shape.begin(), shape.size());
}
bool dtype16(const Tensor& t, thrift_dtype* dt) {
  if (t.scalar_type() == at::kHalf) *dt = THRIFT_F16;
  else if (t.scalar_type() == at::kBFloat16) *dt = THRIFT_BF16;
  else return false;
  return true;
}
bool dtype_out(const Tensor& t, thrift_dtype* dt) {
  if (t.scalar_type() == at::kFloat) { *dt = THRIFT_F32; return true; }
  return dtype16(t, dt);
}
// small sizes only: what does not fit an int takes the general path
bool integer(PyObject* o, int* x) {
  int overflow = 0;
  const long v = PyLong_Check(o) ? PyLong_AsLongAndOverflow(o, &overflow) : (overflow = 1, 0);
  *x = (int)v;
  return overflow == 0 && v == (long)*x;
}
bool real(PyObject* o, double* x) {
  if (PyFloat_Check(o)) { *x = PyFloat_AS_DOUBLE(o); return true; }
  if (!PyLong_Check(o)) return false;
  *x = PyLong_AsDouble(o);
  if (*x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}
bool stream_of(PyObject* o, void** s) {
  *s = PyLong_AsVoidPtr(o);
  if (*s == nullptr && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}
void* ptr(const Tensor* t) { return t ? t->data_ptr() : nullptr; }
template <typename P>
P* ptr_as(const Tensor* t) { return static_cast<P*>(ptr(t)); }

PyObject* answer(thrift_status s, const Tensor& out) {
  if (s != THRIFT_OK) return PyLong_FromLong((long)s);
  return THPVariable_Wrap(out);
}
// The interpreter lock, given up while this lives; also taken back when an exception passes (a tensor without storage has no
// data pointer).
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
Tensor bytes_like(const Tensor& t, size_t n) { return at::empty({(int64_t)std::max<size_t>(n, 256)}, t.options().dtype(at::kByte)); }

// the tensors of a cache: k16 v16 k4 ks v4 vs kmean
struct Cache {
  const Tensor *k16, *v16, *k4, *ks, *v4, *vs, *kmean;
  thrift_dtype dt;
  int B, Hkv, N, D;
};
bool cache(PyObject* const* a, int Bk, Cache* c) {
  if (!tensor(a[0], &c->k16) || !tensor(a[1], &c->v16) || !tensor(a[2], &c->k4) || !tensor(a[3], &c->ks) || !tensor(a[4], &c->v4) ||
      !tensor(a[5], &c->vs) || !tensor(a[6], &c->kmean) || !dtype16(*c->k16, &c->dt) || c->k16->dim() != 4 || Bk <= 0)
    return false;
  const auto s = c->k16->sizes();
  for (int i = 0; i < 4; ++i) if (s[i] > 0x7fffffff) return false;
  const int64_t B = s[0], H = s[1], N = s[2], D = s[3];
  c->B = (int)B; c->Hkv = (int)H; c->N = (int)N; c->D = (int)D;
  return is(*c->v16, c->k16->scalar_type(), {B, H, N, D}) && is(*c->k4, at::kByte, {B, H, N, D / 2}) && is(*c->ks, at::kByte, {B, H, N, D / 32}) &&
         is(*c->v4, at::kByte, {B, H, N / 64, D, 32}) && is(*c->vs, at::kByte, {B, H, N / 32, D}) && is(*c->kmean, at::kFloat, {B, H, N / Bk, D});
}

// decode(q, k16, v16, k4, ks, v4, vs, kmean, Bk, budget, fixed_k, split_blocks, scale, seqlens, out, workspace, shared, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const Tensor *q, *seqlens, *out_given, *ws_given;
  Cache c;
  int Bk, fixed_k, split, shared;
  double budget, scale;
  void* stream;
  thrift_dtype odt;
  if (n != 18 || !tensor(a[0], &q) || !integer(a[8], &Bk) || !cache(a + 1, Bk, &c) || !real(a[9], &budget) || !integer(a[10], &fixed_k) ||
      !integer(a[11], &split) || !real(a[12], &scale) || !optional(a[13], &seqlens) || !optional(a[14], &out_given) ||
      !optional(a[15], &ws_given) || !integer(a[16], &shared) || !stream_of(a[17], &stream) || q->dim() != 3 || q->size(1) > 0x7fffffff)
    Py_RETURN_NONE;
  const int Hq = (int)q->size(1);
  if (!is(*q, c.k16->scalar_type(), {c.B, Hq, c.D}) || (seqlens && !is(*seqlens, at::kInt, {c.B})) ||
      (out_given && !is(*out_given, out_given->scalar_type(), {c.B, Hq, c.D})))
    Py_RETURN_NONE;
  const Tensor out = out_given ? *out_given : at::empty({c.B, Hq, c.D}, q->options());
  if (!dtype_out(out, &odt)) Py_RETURN_NONE;
  const Tensor ws = ws_given ? *ws_given : bytes_like(*q, thrift_attn_decode_workspace(c.B, Hq, c.Hkv, c.N, c.D, Bk, split));
  const size_t ws_bytes = (size_t)ws.numel();
  thrift_status s;
  {
    const Unlocked unlocked;
    s = (shared ? thrift_attn_decode_shared : thrift_attn_decode)(
        ptr(q), c.dt, ptr(c.k16), ptr(c.v16), ptr_as<uint8_t>(c.k4), ptr_as<uint8_t>(c.ks), ptr_as<uint8_t>(c.v4), ptr_as<uint8_t>(c.vs),
        ptr_as<float>(c.kmean), ptr_as<int32_t>(seqlens), c.B, Hq, c.Hkv, c.N, c.D, Bk, budget, fixed_k, split, (float)scale,
        out.data_ptr(), odt, nullptr, nullptr, 0, ws.data_ptr(), ws_bytes, stream);
  }
  return answer(s, out);
}

// append(k_new, v_new, seqlens, new_lens, k16, v16, k4, ks, v4, vs, kmean, Bk, stream): the lengths after the call
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const Tensor *k_new, *v_new, *seqlens, *new_lens;
  Cache c;
  int Bk;
  void* stream;
  if (n != 13 || !tensor(a[0], &k_new) || !tensor(a[1], &v_new) || !tensor(a[2], &seqlens) || !optional(a[3], &new_lens) ||
      !integer(a[11], &Bk) || !cache(a + 4, Bk, &c) || !stream_of(a[12], &stream) || k_new->dim() != 4 || k_new->size(2) > 0x7fffffff)
    Py_RETURN_NONE;
  const int n_new = (int)k_new->size(2);
  const auto st = c.k16->scalar_type();
  if (!is(*k_new, st, {c.B, c.Hkv, n_new, c.D}) || !is(*v_new, st, {c.B, c.Hkv, n_new, c.D}) || !is(*seqlens, at::kInt, {c.B}) ||
      (new_lens && !is(*new_lens, at::kInt, {c.B})))
    Py_RETURN_NONE;
  const Tensor after = at::empty({c.B}, seqlens->options());
  thrift_status s;
  {
    const Unlocked unlocked;
    s = thrift_kv_cache_append_advance(ptr(k_new), ptr(v_new), c.dt, n_new, ptr_as<int32_t>(seqlens), ptr_as<int32_t>(new_lens),
                                       after.data_ptr<int32_t>(), ptr(c.k16), ptr(c.v16), ptr_as<uint8_t>(c.k4), ptr_as<uint8_t>(c.ks),
                                       ptr_as<uint8_t>(c.v4), ptr_as<uint8_t>(c.vs), ptr_as<float>(c.kmean), c.B, c.Hkv, c.N, c.D, Bk, stream);
  }
  return answer(s, after);
}

// attention(q, k, v, causal, Bq, Bk, budget, fixed_k, scale, workspace, out, lse, tile_order, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const Tensor *q, *k, *v, *ws_given, *out_given, *lse;
  int causal, Bq, Bk, fixed_k, order;
  double budget, scale;
  void* stream;
  thrift_dtype dt, odt;
  if (n != 14 || !tensor(a[0], &q) || !tensor(a[1], &k) || !tensor(a[2], &v) || !integer(a[3], &causal) || !integer(a[4], &Bq) ||
      !integer(a[5], &Bk) || !real(a[6], &budget) || !integer(a[7], &fixed_k) || !real(a[8], &scale) || !optional(a[9], &ws_given) ||
      !optional(a[10], &out_given) || !optional(a[11], &lse) || !integer(a[12], &order) || !stream_of(a[13], &stream) ||
      !dtype16(*q, &dt) || q->dim() != 4 || k->dim() != 4)
    Py_RETURN_NONE;
  const auto s = q->sizes();
  const int64_t Hkv = k->size(1);
  for (int i = 0; i < 4; ++i) if (s[i] > 0x7fffffff || k->size(i) > 0x7fffffff) Py_RETURN_NONE;
  if (!is(*k, q->scalar_type(), {s[0], Hkv, s[2], s[3]}) || !is(*v, q->scalar_type(), {s[0], Hkv, s[2], s[3]})) Py_RETURN_NONE;
  // what the C call would write past, were it of another shape or type, takes the general path
  if ((out_given && !is(*out_given, out_given->scalar_type(), {s[0], s[1], s[2], s[3]})) || (lse && !is(*lse, at::kFloat, {s[0], s[1], s[2]})) ||
      (ws_given && ws_given->scalar_type() != at::kByte))
    Py_RETURN_NONE;
  const Tensor out = out_given ? *out_given : at::empty(s, q->options());
  if (!dtype_out(out, &odt)) Py_RETURN_NONE;
  const int B = (int)s[0], Hq = (int)s[1], N = (int)s[2], D = (int)s[3];
  const Tensor ws = ws_given ? *ws_given
                             : bytes_like(*q, thrift_attention_forward_workspace(B, Hq, (int)Hkv, N, D, Bq, Bk, causal, budget, fixed_k));
  const size_t ws_bytes = (size_t)ws.numel();
  thrift_status st;
  {
    const Unlocked unlocked;
    st = thrift_attention_forward(ptr(q), ptr(k), ptr(v), dt, B, Hq, (int)Hkv, N, D, Bq, Bk, causal, budget, fixed_k, order, (float)scale,
                                  out.data_ptr(), odt, ptr_as<float>(lse), ws.data_ptr(), ws_bytes, stream);
  }
  return answer(st, out);
}

// ---- rotary positions and the paged cache; these calls also refuse tensors of another device than the current one ----

// strided heads: the channels of a head contiguous
bool heads(PyObject* o, int device, const Tensor** t) {
  if (!THPVariable_Check(o)) return false;
  *t = &THPVariable_Unpack(o);
  if (!(*t)->is_cuda() || (*t)->device().index() != device || (*t)->dim() == 0) return false;
  const auto s = (*t)->sizes();
  for (const int64_t x : s) if (x < 1 || x > 0x7fffffff) return false;
  return s.back() == 1 || (*t)->stride(-1) == 1;
}
bool plain(PyObject* o, int device, const Tensor** t) { return tensor(o, t) && (*t)->device().index() == device; }
bool plain_or_none(PyObject* o, int device, const Tensor** t) {
  if (o == Py_None) { *t = nullptr; return true; }
  return plain(o, device, t);
}
bool like(const Tensor& t, const Tensor& of, at::IntArrayRef shape) { return t.scalar_type() == of.scalar_type() && t.sizes() == shape; }
// no two elements share an address (sufficient: every stride passes what the smaller ones reach)
bool apart(const Tensor& t) {
  int64_t stride[8], size[8];
  int n = 0;
  if (t.dim() > 8) return false;
  for (int64_t d = 0; d < t.dim(); ++d) {
    if (t.size(d) <= 1) continue;
    int i = n++;
    for (; i > 0 && stride[i - 1] > t.stride(d); --i) stride[i] = stride[i - 1], size[i] = size[i - 1];
    stride[i] = t.stride(d), size[i] = t.size(d);
  }
  int64_t reach = 1;
  for (int i = 0; i < n; ++i) {
    if (stride[i] < reach) return false;
    reach += stride[i] * (size[i] - 1);
  }
  return true;
}

// rope(backward, q, k, freqs, positions, layout, gain, q_out, k_out, device, stream): (q_out, k_out)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const Tensor *q, *k = nullptr, *freqs, *positions = nullptr, *qo = nullptr, *ko = nullptr;
  int backward, layout, device;
  double gain;
  void* stream;
  thrift_dtype dt;
  if (n != 11 || !integer(a[9], &device) || !integer(a[0], &backward) || !heads(a[1], device, &q) || (a[2] != Py_None && !heads(a[2], device, &k)) ||
      !plain(a[3], device, &freqs) || (a[4] != Py_None && !heads(a[4], device, &positions)) || !integer(a[5], &layout) || !real(a[6], &gain) ||
      (a[7] != Py_None && !heads(a[7], device, &qo)) || (a[8] != Py_None && !heads(a[8], device, &ko)) || !stream_of(a[10], &stream) ||
      !dtype16(*q, &dt) || q->dim() != 4 || freqs->scalar_type() != at::kDouble || freqs->dim() != 1 || freqs->numel() > 0x3fffffff)
    Py_RETURN_NONE;
  const int64_t B = q->size(0), N = q->size(2), D = q->size(3);
  if (k ? (k->dim() != 4 || !like(*k, *q, {B, k->size(1), N, D})) : ko != nullptr) Py_RETURN_NONE;
  if ((qo && (!like(*qo, *q, q->sizes()) || !apart(*qo))) || (ko && (!like(*ko, *k, k->sizes()) || !apart(*ko)))) Py_RETURN_NONE;
  if (positions && (positions->scalar_type() != at::kInt || !(positions->sizes() == at::IntArrayRef{N} || positions->sizes() == at::IntArrayRef{B, N})))
    Py_RETURN_NONE;
  const int64_t step = positions && positions->dim() == 2 ? positions->stride(0) : 0;
  const Tensor q_out = qo ? *qo : at::empty(q->sizes(), q->options());
  const Tensor k_out = !k ? Tensor() : ko ? *ko : at::empty(k->sizes(), k->options());
  int64_t st[4][3] = {};
  for (int i = 0; i < 3; ++i) {
    st[0][i] = q->stride(i), st[1][i] = q_out.stride(i);
    if (k) st[2][i] = k->stride(i), st[3][i] = k_out.stride(i);
  }
  thrift_status r;
  {
    const Unlocked unlocked;
    r = (backward ? thrift_rope_backward : thrift_rope)(
        ptr(q), st[0], q_out.data_ptr(), st[1], (int)q->size(1), ptr(k), st[2], k ? k_out.data_ptr() : nullptr, st[3], k ? (int)k->size(1) : 0, dt,
        ptr_as<int32_t>(positions), step, ptr_as<double>(freqs), 2 * (int)freqs->numel(), layout, (float)gain, (int)B, (int)N, (int)D, stream);
  }
  if (r != THRIFT_OK) return PyLong_FromLong((long)r);
  PyObject* both = PyTuple_New(2);
  if (both == nullptr) return nullptr;
  PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(q_out));
  PyTuple_SET_ITEM(both, 1, k ? THPVariable_Wrap(k_out) : (Py_INCREF(Py_None), Py_None));
  return both;
}

// page_map(seqlens, new_lens, block_table, free_pages, free_count, page_size, n_pages, rows, device, stream): its five outputs
PyObject* page_map(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const Tensor *lens, *fresh, *table, *free, *count;
  int page, n_pages, rows, device;
  void* stream;
  if (n != 10 || !integer(a[8], &device) || !plain(a[0], device, &lens) || !plain(a[1], device, &fresh) || !plain(a[2], device, &table) ||
      !plain(a[3], device, &free) || !plain(a[4], device, &count) || !integer(a[5], &page) || !integer(a[6], &n_pages) || !integer(a[7], &rows) ||
      !stream_of(a[9], &stream) || table->dim() != 2 || free->dim() != 1 || rows < 1)
    Py_RETURN_NONE;
  const int64_t B = table->size(0), width = table->size(1);
  if (B > 0x7ffffffe || width > 0x7fffffff || free->numel() > 0x7fffffff || table->scalar_type() != at::kInt || free->scalar_type() != at::kInt ||
      !is(*lens, at::kInt, {B}) || !is(*fresh, at::kInt, {B}) || !is(*count, at::kInt, {1}))
    Py_RETURN_NONE;
  // five arrays of one allocation, 16 bytes aligned each
  Tensor out[5];
  const int64_t sizes[5] = {rows, rows, B + 1, B, 1};
  int64_t offset = 0;
  for (const int64_t x : sizes) offset += (x + 3) / 4 * 4;
  const Tensor space = at::empty({offset}, lens->options());
  offset = 0;
  for (int i = 0; i < 5; ++i) {
    out[i] = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(space.storage()), space.key_set(), space.dtype());
    out[i].unsafeGetTensorImpl()->set_storage_offset(offset);
    out[i].unsafeGetTensorImpl()->set_sizes_contiguous({sizes[i]});
    offset += (sizes[i] + 3) / 4 * 4;
  }
  const auto p = [&](int i) { return out[i].data_ptr<int32_t>(); };
  thrift_status r;
  {
    const Unlocked unlocked;
    r = thrift_page_map(ptr_as<int32_t>(lens), ptr_as<int32_t>(fresh), (int)B, page, n_pages, ptr_as<int32_t>(table), (int)width,
                                            ptr_as<int32_t>(free), (int)free->numel(), ptr_as<int32_t>(count), rows, p(0), p(1), p(2), p(3), p(4), stream);
  }
  if (r != THRIFT_OK) return PyLong_FromLong((long)r);
  PyObject* all = PyTuple_New(5);
  if (all == nullptr) return nullptr;
  for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(all, i, THPVariable_Wrap(out[i]));
  return all;
}

bool pages(PyObject* ko, PyObject* vo, int device, const Tensor** k, const Tensor** v, thrift_dtype* dt) {
  if (!plain(ko, device, k) || !plain(vo, device, v) || !dtype16(**k, dt) || (*k)->dim() != 4 || !like(**v, **k, (*k)->sizes())) return false;
  for (const int64_t x : (*k)->sizes()) if (x < 1 || x > 0x7fffffff) return false;
  return true;
}

// codes and scales of an 8-bit cache: k, k scales, v, v scales
bool pages8(PyObject* const* a, int device, const Tensor* (&p)[4]) {
  for (int i = 0; i < 4; ++i)
    if (!plain(a[i], device, &p[i]) || p[i]->scalar_type() != at::kByte) return false;
  if (p[0]->dim() != 4 || p[2]->sizes() != p[0]->sizes() || p[1]->sizes() != p[0]->sizes().slice(0, 3) || p[3]->sizes() != p[1]->sizes()) return false;
  for (const int64_t x : p[0]->sizes()) if (x < 1 || x > 0x7fffffff) return false;
  return true;
}

// paged_append(k, v, slots, k_pages, v_pages, q, q_out, positions, freqs, layout, gain, device, stream): q_out, or True without q
// paged_append8: the same with k_codes, k_scales, v_codes, v_scales for the pages
template <bool CODES>
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kPages = CODES ? 4 : 2;
  const Tensor *k, *v, *slots, *p[4] = {}, *q = nullptr, *qo, *positions, *freqs;
  int layout, device;
  double gain;
  void* stream;
  thrift_dtype dt;
  if (n != 11 + kPages) Py_RETURN_NONE;
  PyObject* const* b = a + 3 + kPages;     // behind the pages
  if (!integer(b[6], &device) || !heads(a[0], device, &k) || !heads(a[1], device, &v) || !plain(a[2], device, &slots) ||
      !(CODES ? pages8(a + 3, device, p) && dtype16(*k, &dt) : pages(a[3], a[4], device, &p[0], &p[1], &dt)) ||
      (b[0] != Py_None && !heads(b[0], device, &q)) || !plain_or_none(b[1], device, &qo) ||
      !plain_or_none(b[2], device, &positions) || !plain_or_none(b[3], device, &freqs) || !integer(b[4], &layout) || !real(b[5], &gain) ||
      !stream_of(b[7], &stream) || k->dim() != 3 || (qo && !q))
    Py_RETURN_NONE;
  const Tensor& of = CODES ? *k : *p[0];   // whose type keys, values and queries have
  const int64_t T = k->size(0), Hkv = p[0]->size(1), D = p[0]->size(3);
  if (!like(*k, of, {T, Hkv, D}) || !like(*v, of, {T, Hkv, D}) || !is(*slots, at::kInt, {T}) ||
      (q && (q->dim() != 3 || !like(*q, of, {T, q->size(1), D}))) || (qo && !like(*qo, *q, q->sizes())))
    Py_RETURN_NONE;
  if (freqs && (freqs->scalar_type() != at::kDouble || freqs->dim() != 1 || freqs->numel() < 1 || freqs->numel() > 0x3fffffff || !positions ||
                !is(*positions, at::kInt, {T})))
    Py_RETURN_NONE;
  const Tensor q_out = !q ? Tensor() : qo ? *qo : at::empty(q->sizes(), q->options());
  int64_t st[3][2];
  for (int i = 0; i < 2; ++i) {
    st[0][i] = q ? q->stride(i) : 0, st[1][i] = k->stride(i), st[2][i] = v->stride(i);
  }
  thrift_status r;
  {
    const Unlocked unlocked;
    const int Hq = q ? (int)q->size(1) : 0, rot = freqs ? 2 * (int)freqs->numel() : 0, n_pages = (int)p[0]->size(0), page = (int)p[0]->size(2);
    void* to = q ? q_out.data_ptr() : nullptr;
    if constexpr (CODES)
      r = thrift_paged_append8(ptr(q), st[0], to, Hq, ptr(k), st[1], ptr(v), st[2], (int)Hkv, dt, (int)T, ptr_as<int32_t>(slots),
                               ptr_as<int32_t>(positions), ptr_as<double>(freqs), rot, layout, (float)gain, ptr_as<uint8_t>(p[0]), ptr_as<uint8_t>(p[1]),
                               ptr_as<uint8_t>(p[2]), ptr_as<uint8_t>(p[3]), n_pages, page, (int)D, stream);
    else
      r = thrift_paged_append(ptr(q), st[0], to, Hq, ptr(k), st[1], ptr(v), st[2], (int)Hkv, dt, (int)T, ptr_as<int32_t>(slots),
                              ptr_as<int32_t>(positions), ptr_as<double>(freqs), rot, layout, (float)gain, ptr(p[0]), ptr(p[1]), n_pages, page, (int)D, stream);
  }
  if (r != THRIFT_OK) return PyLong_FromLong((long)r);
  if (!q) Py_RETURN_TRUE;
  return THPVariable_Wrap(q_out);
}

// paged_decode(q, k_pages, v_pages, block_table, seqlens, scale, out, lse, return_lse, workspace, device, stream): out, or (out, lse)
// CODES: k_codes, k_scales, v_codes, v_scales for the pages; PREFIX: group_of and group_lens behind the lengths
template <bool CODES, bool PREFIX>
PyObject* paged_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kPages = CODES ? 4 : 2, kGroups = PREFIX ? 2 : 0;
  const Tensor *q, *p[4] = {}, *table, *lens, *of = nullptr, *group_lens = nullptr, *out_given, *lse_given, *ws_given;
  int return_lse, device;
  double scale;
  void* stream;
  thrift_dtype dt, odt;
  if (n != 10 + kPages + kGroups) Py_RETURN_NONE;
  PyObject* const* b = a + 1 + kPages;     // behind the pages
  PyObject* const* c = b + 2 + kGroups;    // behind the groups
  if (!integer(c[5], &device) || !plain(a[0], device, &q) ||
      !(CODES ? pages8(a + 1, device, p) && dtype16(*q, &dt) : pages(a[1], a[2], device, &p[0], &p[1], &dt)) || !plain(b[0], device, &table) ||
      !plain(b[1], device, &lens) || (PREFIX && (!plain(b[2], device, &of) || !plain(b[3], device, &group_lens))) || !real(c[0], &scale) ||
      !plain_or_none(c[1], device, &out_given) || !plain_or_none(c[2], device, &lse_given) || !integer(c[3], &return_lse) ||
      !plain_or_none(c[4], device, &ws_given) || !stream_of(c[6], &stream) || q->dim() != 3 || table->dim() != 2)
    Py_RETURN_NONE;
  const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), width = table->size(1);
  if (B > 0x7fffffff || Hq > 0x7fffffff || width > 0x7fffffff || !like(*q, CODES ? *q : *p[0], {B, Hq, p[0]->size(3)}) || !is(*table, at::kInt, {B, width}) ||
      !is(*lens, at::kInt, {B}) || (out_given && out_given->sizes() != q->sizes()) || (lse_given && !is(*lse_given, at::kFloat, {B, Hq})) ||
      (ws_given && ws_given->scalar_type() != at::kByte))
    Py_RETURN_NONE;
  if (PREFIX && (!is(*of, at::kInt, {B}) || group_lens->scalar_type() != at::kInt || group_lens->dim() != 1 || group_lens->numel() > 0x7fffffff)) Py_RETURN_NONE;
  const Tensor out = out_given ? *out_given : at::empty({B, Hq, D}, q->options());
  if (!dtype_out(out, &odt)) Py_RETURN_NONE;
  const Tensor lse = lse_given ? *lse_given : return_lse ? at::empty({B, Hq}, q->options().dtype(at::kFloat)) : Tensor();
  const int Hkv = (int)p[0]->size(1), page = (int)p[0]->size(2), n_pages = (int)p[0]->size(0), groups = PREFIX ? (int)group_lens->numel() : 0;
  const size_t need = ws_given ? 0
                      : PREFIX ? thrift_paged_decode_prefix_workspace(CODES ? 8 : 16, (int)B, (int)Hq, Hkv, groups, (int)width, page, (int)D)
                               : (CODES ? thrift_paged_decode8_workspace : thrift_paged_decode_workspace)((int)B, (int)Hq, Hkv, (int)width, page, (int)D);
  const Tensor ws = ws_given ? *ws_given : need > 0 ? bytes_like(*q, need) : Tensor();
  thrift_status r;
  {
    const Unlocked unlocked;
    const int32_t *t = ptr_as<int32_t>(table), *l = ptr_as<int32_t>(lens), *g = ptr_as<int32_t>(of), *gl = ptr_as<int32_t>(group_lens);
    const uint8_t *kc = ptr_as<uint8_t>(p[0]), *ks = ptr_as<uint8_t>(p[1]), *vc = ptr_as<uint8_t>(p[2]), *vs = ptr_as<uint8_t>(p[3]);
    float* e = lse.defined() ? lse.data_ptr<float>() : nullptr;
    void* w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? (size_t)ws.numel() : 0;
    const int nb = (int)B, hq = (int)Hq, m = (int)width, d = (int)D;
    const float s = (float)scale;
    if constexpr (CODES && PREFIX)
      r = thrift_paged_decode_prefix8(ptr(q), dt, kc, ks, vc, vs, n_pages, t, m, l, g, gl, groups, nb, hq, Hkv, d, page, s, out.data_ptr(), odt, e, w, bytes, stream);
    else if constexpr (CODES)
      r = thrift_paged_decode8(ptr(q), dt, kc, ks, vc, vs, n_pages, t, m, l, nb, hq, Hkv, d, page, s, out.data_ptr(), odt, e, w, bytes, stream);
    else if constexpr (PREFIX)
      r = thrift_paged_decode_prefix(ptr(q), dt, ptr(p[0]), ptr(p[1]), n_pages, t, m, l, g, gl, groups, nb, hq, Hkv, d, page, s, out.data_ptr(), odt, e, w, bytes, stream);
    else
      r = thrift_paged_decode(ptr(q), dt, ptr(p[0]), ptr(p[1]), n_pages, t, m, l, nb, hq, Hkv, d, page, s, out.data_ptr(), odt, e, w, bytes, stream);
  }
  if (r != THRIFT_OK || !return_lse) return answer(r, out);
  PyObject* both = PyTuple_New(2);
  if (both == nullptr) return nullptr;
  PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(out));
  PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(lse));
  return both;
}

// paged_read(k_pages, v_pages, block_table, seqlens, n, first, k_out, v_out, device, stream): (k, v)
// CODES: k_codes, k_scales, v_codes, v_scales for the pages, and the type of the rows (a thrift_dtype) behind v_out
template <bool CODES>
PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kPages = CODES ? 4 : 2;
  const Tensor *p[4] = {}, *table, *lens, *first, *given[2];
  int N, device, code = 0;
  void* stream;
  thrift_dtype dt;
  if (n != kPages + 8 + (CODES ? 1 : 0)) Py_RETURN_NONE;
  PyObject* const* b = a + kPages;         // behind the pages
  PyObject* const* c = b + 6 + (CODES ? 1 : 0);                  // device, stream
  if (!integer(c[0], &device) || !(CODES ? pages8(a, device, p) && integer(b[6], &code) : pages(a[0], a[1], device, &p[0], &p[1], &dt)) ||
      !plain(b[0], device, &table) || !plain(b[1], device, &lens) || !integer(b[2], &N) || !plain_or_none(b[3], device, &first) ||
      !plain_or_none(b[4], device, &given[0]) || !plain_or_none(b[5], device, &given[1]) || !stream_of(c[1], &stream) || table->dim() != 2)
    Py_RETURN_NONE;
  if (CODES) {
    if (code != THRIFT_F16 && code != THRIFT_BF16) Py_RETURN_NONE;
    dt = (thrift_dtype)code;
  }
  const int64_t B = table->size(0), width = table->size(1), Hkv = p[0]->size(1), D = p[0]->size(3);
  const at::ScalarType type = dt == THRIFT_F16 ? at::kHalf : at::kBFloat16;
  if (N < 1 || B < 1 || B > 0x7fffffff || width > 0x7fffffff || !is(*table, at::kInt, {B, width}) || !is(*lens, at::kInt, {B}) ||
      (first && !is(*first, at::kInt, {B})))
    Py_RETURN_NONE;
  for (const Tensor* t : given)
    if (t && !is(*t, type, {B, Hkv, N, D})) Py_RETURN_NONE;
  Tensor out[2];
  for (int i = 0; i < 2; ++i) out[i] = given[i] ? *given[i] : at::empty({B, Hkv, N, D}, table->options().dtype(type));
  thrift_status r;
  {
    const Unlocked unlocked;
    const int32_t *t = ptr_as<int32_t>(table), *f = ptr_as<int32_t>(first), *l = ptr_as<int32_t>(lens);
    const int n_pages = (int)p[0]->size(0), page = (int)p[0]->size(2), nb = (int)B, h = (int)Hkv, m = (int)width, d = (int)D;
    if constexpr (CODES)
      r = thrift_paged_read8(ptr_as<uint8_t>(p[0]), ptr_as<uint8_t>(p[1]), ptr_as<uint8_t>(p[2]), ptr_as<uint8_t>(p[3]), n_pages, t, m, f, l, nb, h, N, d, page,
                             out[0].data_ptr(), out[1].data_ptr(), dt, stream);
    else
      r = thrift_paged_read(ptr(p[0]), ptr(p[1]), n_pages, t, m, f, l, nb, h, N, d, page, out[0].data_ptr(), out[1].data_ptr(), stream);
  }
  if (r != THRIFT_OK) return PyLong_FromLong((long)r);
  PyObject* both = PyTuple_New(2);
  if (both == nullptr) return nullptr;
  for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(both, i, THPVariable_Wrap(out[i]));
  return both;
}

// A tensor whose sizes or storage cannot be asked for (a fake one, one under a transform) throws: not a plain argument.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {
    {"decode", (PyCFunction)(void (*)(void))guarded<decode>, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))guarded<append>, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)(void))guarded<attention>, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)(void))guarded<rope>, METH_FASTCALL, nullptr},
    {"page_map", (PyCFunction)(void (*)(void))guarded<page_map>, METH_FASTCALL, nullptr},
    {"paged_append", (PyCFunction)(void (*)(void))guarded<paged_append<false>>, METH_FASTCALL, nullptr},
    {"paged_append8", (PyCFunction)(void (*)(void))guarded<paged_append<true>>, METH_FASTCALL, nullptr},
    {"paged_decode", (PyCFunction)(void (*)(void))guarded<paged_decode<false, false>>, METH_FASTCALL, nullptr},
    {"paged_decode8", (PyCFunction)(void (*)(void))guarded<paged_decode<true, false>>, METH_FASTCALL, nullptr},
    {"paged_decode_prefix", (PyCFunction)(void (*)(void))guarded<paged_decode<false, true>>, METH_FASTCALL, nullptr},
    {"paged_decode_prefix8", (PyCFunction)(void (*)(void))guarded<paged_decode<true, true>>, METH_FASTCALL, nullptr},
    {"paged_read", (PyCFunction)(void (*)(void))guarded<paged_read<false>>, METH_FASTCALL, nullptr},
    {"paged_read8", (PyCFunction)(void (*)(void))guarded<paged_read<true>>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
