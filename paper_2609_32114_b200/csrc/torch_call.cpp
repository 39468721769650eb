// The torch entry points of binding.py (ha_la_prefill, ha_la_decode) and layer.py as one native call each: tensors are unpacked,
// checked, missing outputs allocated and the C struct filled here instead of in Python (one decoding step cost its caller
// 12 us of interpreter and ctypes time around a 3 us kernel).  Nothing is computed here.  A call that is not entirely
// ordinary -- a tensor of another type, layout, size or device, the batch dimension left out -- returns None, and binding.py
// takes it through its own marshalling, which also words the errors.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <type_traits>

#include "ha_la.h"

namespace {

int (*g_prefill)(const ha_la_prefill_args*, void*) = nullptr;
int (*g_prefill_bytes)(const ha_la_prefill_args*, size_t*) = nullptr;
int (*g_decode)(const ha_la_decode_args*, void*) = nullptr;
int (*g_gla_prefill)(const ha_la_gla_args*, void*) = nullptr;
int (*g_gla_backward)(const ha_la_gla_args*, void*) = nullptr;
int (*g_gla_bytes)(const ha_la_gla_args*, int, size_t*) = nullptr;
int (*g_gla_decode)(const ha_la_decode_args*, void*) = nullptr;
int (*g_gated_norm)(const ha_la_gated_norm_args*, void*) = nullptr;
int (*g_gated_norm_backward)(const ha_la_gated_norm_args*, void*) = nullptr;
int (*g_gated_norm_bytes)(const ha_la_gated_norm_args*, size_t*) = nullptr;
int (*g_add_norm)(const ha_la_add_norm_args*, void*) = nullptr;
int (*g_add_norm_backward)(const ha_la_add_norm_args*, void*) = nullptr;
int (*g_add_norm_bytes)(const ha_la_add_norm_args*, size_t*) = nullptr;

int (*g_conv)(const ha_la_conv_args*, void*) = nullptr;
int (*g_conv_backward)(const ha_la_conv_args*, void*) = nullptr;
int (*g_conv_bytes)(const ha_la_conv_args*, size_t*) = nullptr;
int (*g_conv_decode)(const ha_la_conv_args*, void*) = nullptr;
int (*g_scan)(const ha_la_scan_args*, void*) = nullptr;
int (*g_scan_backward)(const ha_la_scan_args*, void*) = nullptr;
int (*g_scan_bytes)(const ha_la_scan_args*, int, size_t*) = nullptr;
int (*g_scan_decode)(const ha_la_scan_args*, void*) = nullptr;
int (*g_latent_prefill)(const ha_la_latent_prefill_args*, void*) = nullptr;
int (*g_latent_decode)(const ha_la_latent_decode_args*, void*) = nullptr;
int (*g_latent_decode_bytes)(const ha_la_latent_decode_args*, size_t*) = nullptr;

// a tensor, or nullptr for None; anything else is not ordinary
bool unpack(PyObject* o, const at::Tensor** t) {
  *t = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return false;
  *t = &THPVariable_Unpack(o);
  return true;
}
bool plain(const at::Tensor* t, at::ScalarType type, int64_t dim) {
  return t && t->is_cuda() && t->scalar_type() == type && t->dim() == dim && t->is_contiguous();
}
// q [rows.., HK, dk] sets the sizes of k, v [rows.., HV, dv], g [rows.., HV] (KDA: and dk) and beta [rows.., HV].  The others may
// have more rows than q where they lie one behind the other.
bool inputs(const at::Tensor* q, const at::Tensor* k, const at::Tensor* v, const at::Tensor* g, const at::Tensor* beta,
            int64_t dim, bool kda) {
  if (!q || !(q->scalar_type() == at::kBFloat16 || q->scalar_type() == at::kFloat)) return false;
  if (!plain(q, q->scalar_type(), dim) || !plain(k, q->scalar_type(), dim) || !plain(v, q->scalar_type(), dim) ||
      !plain(g, at::kFloat, kda ? dim : dim - 1) || !plain(beta, at::kFloat, dim - 1))
    return false;
  // (as arrays: a tensor's size(i) is a call and a range check each)
  const int64_t *qs = q->sizes().data(), *ks = k->sizes().data(), *vs = v->sizes().data(), *gs = g->sizes().data(), *bs = beta->sizes().data();
  const int h = (int)dim - 2;                            // (dimension of the heads)
  const auto device = q->device();
  for (const at::Tensor* t : {k, v, g, beta})
    if (t->device() != device) return false;
  for (const int64_t* ts : {ks, vs, gs, bs}) {
    if (ts[0] < qs[0]) return false;
    if (h == 2 && !(ts[1] == qs[1] || (qs[0] == 1 && ts[1] > qs[1]))) return false;
  }
  return ks[h] == qs[h] && ks[h + 1] == qs[h + 1] && gs[h] == vs[h] && bs[h] == vs[h] && (!kda || gs[h + 1] == qs[h + 1]);
}
// an optional tensor with room for n elements that the kernels can take by its address
bool room(const at::Tensor* t, const at::Tensor& q, at::ScalarType type, int64_t n) {
  return !t || (t->device() == q.device() && t->scalar_type() == type && t->is_contiguous() && t->numel() >= n);
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// The stream of a call.  Where the caller names another than torch's current one, that is the current one while this lives:
// tensors that the call allocates and fills come from that stream's pool and are filled in its order, and nothing that is
// queued on the current stream can still be using (or clear, in the status word's case) what the kernels write.  The caller
// reads them on the current stream once it has waited, so they are recorded there too and not reused before that is over.
struct CallStream {
  void* handle = nullptr;
  std::optional<c10::cuda::CUDAStream> current;          // (set: another stream's call)
  std::optional<c10::cuda::CUDAStreamGuard> guard;
  bool set(PyObject* stream, const at::Tensor& q) {      // false: Python error
    if (stream == Py_None) {
      handle = at::cuda::getCurrentCUDAStream(q.get_device()).stream();
      return true;
    }
    handle = PyLong_AsVoidPtr(stream);
    return !PyErr_Occurred();
  }
  void will_allocate(PyObject* stream, const at::Tensor& q) {
    if (stream == Py_None || current) return;
    const c10::cuda::CUDAStream c = c10::cuda::getCurrentCUDAStream(q.get_device());
    if (c.stream() == handle) return;
    current = c;
    guard.emplace(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), q.get_device()));
  }
  void allocated(const at::Tensor& t) const {
    if (current) t.record_stream(current->unwrap());
  }
};

// The library's entry points, as addresses
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 24) { PyErr_SetString(PyExc_TypeError, "twenty-four addresses"); return nullptr; }
  int i = 0;
  auto take = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(PyLong_AsVoidPtr(a[i++])); };
  take(g_prefill);
  take(g_prefill_bytes);
  take(g_decode);
  take(g_gla_prefill);
  take(g_gla_backward);
  take(g_gla_bytes);
  take(g_gla_decode);
  take(g_gated_norm);
  take(g_gated_norm_backward);
  take(g_gated_norm_bytes);
  take(g_add_norm);
  take(g_add_norm_backward);
  take(g_add_norm_bytes);
  take(g_conv);
  take(g_conv_backward);
  take(g_conv_bytes);
  take(g_conv_decode);
  take(g_scan);
  take(g_scan_backward);
  take(g_scan_bytes);
  take(g_scan_decode);
  take(g_latent_prefill);
  take(g_latent_decode);
  take(g_latent_decode_bytes);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// decode(q, k, v, g, beta, state, stream, kda, scale, o, state_out) -> (o, state_out) | status | None
PyObject* decode_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_decode) { PyErr_SetString(PyExc_TypeError, "eleven arguments"); return nullptr; }
  const at::Tensor *q, *k, *v, *g, *beta, *st, *o, *so;
  const bool kda = a[7] == Py_True;
  if (!unpack(a[0], &q) || !unpack(a[1], &k) || !unpack(a[2], &v) || !unpack(a[3], &g) || !unpack(a[4], &beta) ||
      !unpack(a[5], &st) || !unpack(a[9], &o) || !unpack(a[10], &so) || !inputs(q, k, v, g, beta, 3, kda))
    Py_RETURN_NONE;
  const int64_t state = q->size(0) * v->size(1) * q->size(2) * v->size(2);
  if (!room(st, *q, at::kFloat, state) || !room(so, *q, at::kFloat, state) ||
      !room(o, *q, q->scalar_type(), q->size(0) * v->size(1) * v->size(2)))
    Py_RETURN_NONE;
  ha_la_decode_args d{};
  d.variant = kda;
  d.dtype = q->scalar_type() == at::kFloat;
  d.num_seqs = (int32_t)q->size(0);
  d.num_qk_heads = (int32_t)q->size(1);
  d.num_v_heads = (int32_t)v->size(1);
  d.d_k = (int32_t)q->size(2);
  d.d_v = (int32_t)v->size(2);
  d.scale = (float)PyFloat_AsDouble(a[8]);
  if (PyErr_Occurred()) return nullptr;
  CallStream on;
  if (!on.set(a[6], *q)) return nullptr;
  at::Tensor o_new, s_new;
  if (!o || (!so && !st)) on.will_allocate(a[6], *q);
  if (!o) { o_new = at::empty(v->sizes(), v->options()); o = &o_new; on.allocated(o_new); }
  if (!so) {
    if (st) so = st;
    else { s_new = at::empty({d.num_seqs, d.num_v_heads, d.d_k, d.d_k}, g->options()); so = &s_new; on.allocated(s_new); }
  }
  d.q = ptr(q); d.k = ptr(k); d.v = ptr(v);
  d.g = (const float*)ptr(g); d.beta = (const float*)ptr(beta);
  d.h_in = (const float*)ptr(st); d.h_out = (float*)ptr(so); d.o = ptr(o);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_decode(&d, on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  PyObject* po = o == &o_new ? THPVariable_Wrap(o_new) : Py_NewRef(a[9]);
  PyObject* ps = so == &s_new ? THPVariable_Wrap(s_new) : Py_NewRef(so == st ? a[5] : a[10]);
  PyObject* r = PyTuple_Pack(2, po, ps);
  Py_XDECREF(po);
  Py_XDECREF(ps);
  return r;
}

// prefill(q, k, v, g, beta, h0, cu_seqlens, max_seqlen, stream, kda, scale, o, hT, want_hT, workspace, status_word)
//   -> (o, hT | None, status_word, workspace) | status | None
PyObject* prefill_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 16 || !g_prefill) { PyErr_SetString(PyExc_TypeError, "sixteen arguments"); return nullptr; }
  const at::Tensor *q, *k, *v, *g, *beta, *h0, *cu, *o, *hT, *ws, *sw;
  if (a[9] != Py_True && a[9] != Py_False) Py_RETURN_NONE;
  const bool kda = a[9] == Py_True;
  if (!unpack(a[0], &q) || !unpack(a[1], &k) || !unpack(a[2], &v) || !unpack(a[3], &g) || !unpack(a[4], &beta) ||
      !unpack(a[5], &h0) || !unpack(a[6], &cu) || !unpack(a[11], &o) || !unpack(a[12], &hT) || !unpack(a[14], &ws) ||
      !unpack(a[15], &sw) || !inputs(q, k, v, g, beta, 4, kda))
    Py_RETURN_NONE;
  if (cu && (!plain(cu, at::kInt, 1) || cu->device() != q->device() || q->size(0) != 1)) Py_RETURN_NONE;
  if (ws && (!plain(ws, at::kByte, 1) || ws->device() != q->device())) Py_RETURN_NONE;
  const int64_t N = cu ? cu->numel() - 1 : q->size(0), state = N * v->size(2) * q->size(3) * v->size(3);
  if (!room(h0, *q, at::kFloat, state) || !room(hT, *q, at::kFloat, state) ||
      !room(o, *q, q->scalar_type(), q->size(0) * q->size(1) * v->size(2) * v->size(3)) || !room(sw, *q, at::kInt, 1))
    Py_RETURN_NONE;
  ha_la_prefill_args d{};
  d.variant = kda;
  d.dtype = q->scalar_type() == at::kFloat;
  d.batch = (int32_t)q->size(0);
  d.seqlen = (int32_t)q->size(1);
  d.num_qk_heads = (int32_t)q->size(2);
  d.num_v_heads = (int32_t)v->size(2);
  d.d_k = (int32_t)q->size(3);
  d.d_v = (int32_t)v->size(3);
  d.chunk = 64;
  d.scale = (float)PyFloat_AsDouble(a[10]);
  d.num_seqs = cu ? (int32_t)N : 0;
  d.max_seqlen = (int32_t)PyLong_AsLong(a[7]);
  if (PyErr_Occurred()) return nullptr;
  d.q = ptr(q); d.k = ptr(k); d.v = ptr(v);
  d.g = (const float*)ptr(g); d.beta = (const float*)ptr(beta);
  d.h0 = (const float*)ptr(h0); d.cu_seqlens = (const int32_t*)ptr(cu);
  size_t need = 0;
  int rc = g_prefill_bytes(&d, &need);
  if (rc != HA_LA_OK) Py_RETURN_NONE;                     // (binding.py words the error)
  at::Tensor o_new, h_new, w_new, s_new;
  // (asked for its truth value only where the call has to know: when it brings no hT)
  const int want_hT = hT ? 0 : PyObject_IsTrue(a[13]);
  if (want_hT < 0) return nullptr;
  CallStream on;
  if (!on.set(a[8], *q)) return nullptr;
  if (!o || (!hT && want_hT) || !ws || !sw) on.will_allocate(a[8], *q);
  if (!o) { o_new = at::empty(v->sizes(), v->options()); o = &o_new; on.allocated(o_new); }
  if (!hT && want_hT) { h_new = at::empty({N, v->size(2), q->size(3), v->size(3)}, g->options()); hT = &h_new; on.allocated(h_new); }
  if (!ws) { w_new = at::empty({(int64_t)need + 256}, g->options().dtype(at::kByte)); ws = &w_new; on.allocated(w_new); }
  if (!sw) { s_new = at::zeros({1}, g->options().dtype(at::kInt)); sw = &s_new; on.allocated(s_new); }
  d.o = ptr(o); d.hT = (float*)ptr(hT); d.status_word = (int32_t*)ptr(sw);
  const uintptr_t base = (uintptr_t)ws->data_ptr(), al = (base + 255) / 256 * 256;
  d.workspace = (void*)al;
  const int64_t pad = (int64_t)(al - base);
  d.workspace_bytes = ws->numel() > pad ? (size_t)(ws->numel() - pad) : 0;   // (a buffer may end before its first aligned byte)
  Py_BEGIN_ALLOW_THREADS
  rc = g_prefill(&d, on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  PyObject* r = PyTuple_New(4);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, o == &o_new ? THPVariable_Wrap(o_new) : Py_NewRef(a[11]));
  PyTuple_SET_ITEM(r, 1, hT == &h_new && hT ? THPVariable_Wrap(h_new) : Py_NewRef(a[12]));
  PyTuple_SET_ITEM(r, 2, sw == &s_new ? THPVariable_Wrap(s_new) : Py_NewRef(a[15]));
  PyTuple_SET_ITEM(r, 3, ws == &w_new ? THPVariable_Wrap(w_new) : Py_NewRef(a[14]));
  return r;
}

// ---------------------------------------------------------------- layer.py: gated linear attention, norms
//
// As above; tensors have to have the very shapes that go with the first one, and its device is the current one during the call.

bool element(const at::Tensor* t) { return t && t->is_cuda() && (t->scalar_type() == at::kBFloat16 || t->scalar_type() == at::kFloat); }
bool same(const at::Tensor* t, const at::Tensor& like, at::ScalarType type, at::IntArrayRef shape) {
  return t && t->scalar_type() == type && t->device() == like.device() && t->sizes() == shape && t->is_contiguous();
}
bool number(PyObject* o, double* v) {                     // false: not an ordinary call (layer.py words the errors)
  *v = PyFloat_AsDouble(o);
  if (!PyErr_Occurred()) return *v == *v;
  PyErr_Clear();
  return false;
}

// Outputs, scratch and status word of a call: what the caller did not bring is allocated on the call's stream.
struct Outputs {
  static constexpr int kMax = 12;
  c10::cuda::CUDAGuard device;
  CallStream on;
  PyObject* stream;
  const at::Tensor& like;
  at::Tensor own[kMax];
  int n = 0;
  Outputs(PyObject* s, const at::Tensor& t) : device(t.device()), stream(s), like(t) {}
  bool set() { return on.set(stream, like); }
  const at::Tensor* take(const at::Tensor* given, at::IntArrayRef shape, at::ScalarType type, bool zeros = false) {
    if (given) return given;
    on.will_allocate(stream, like);
    at::Tensor& t = own[n++];
    t = zeros ? at::zeros(shape, like.options().dtype(type)) : at::empty(shape, like.options().dtype(type));
    on.allocated(t);
    return &t;
  }
  // the aligned part of a scratch buffer, `need` bytes if it is allocated here
  const at::Tensor* scratch(const at::Tensor* given, size_t need, void** at, size_t* bytes) {
    const at::Tensor* t = take(given, {(int64_t)need + 256}, at::kByte);
    const uintptr_t base = (uintptr_t)t->data_ptr(), al = (base + 255) / 256 * 256;
    const size_t have = (size_t)t->numel(), pad = (size_t)(al - base);
    *at = (void*)al;
    *bytes = have > pad ? have - pad : 0;
    return t;
  }
  // the caller's own object, or a new one
  PyObject* wrap(const at::Tensor* t, PyObject* given) const {
    for (int i = 0; i < n; ++i)
      if (t == &own[i]) return THPVariable_Wrap(own[i]);
    return Py_NewRef(given);
  }
};

PyObject* pack(std::initializer_list<PyObject*> items) {   // takes the references
  PyObject* r = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (r && o) PyTuple_SET_ITEM(r, i++, o);
    else { Py_XDECREF(o); Py_CLEAR(r); }
  }
  return r;
}

bool length(PyObject* o, int32_t* v) {
  const long x = PyLong_AsLong(o);
  if (PyErr_Occurred()) { PyErr_Clear(); return false; }
  *v = (int32_t)x;
  return x >= 0 && x <= INT32_MAX;
}
bool scratch_ok(const at::Tensor* ws, const at::Tensor& q) { return !ws || (plain(ws, at::kByte, 1) && ws->device() == q.device()); }

// sizes and inputs of a whole-sequence call on [B, T, heads, d]
bool gla_inputs(const at::Tensor* q, const at::Tensor* k, const at::Tensor* v, const at::Tensor* g, const at::Tensor* h0, const at::Tensor* cu,
                ha_la_gla_args* d, int64_t* seqs) {
  if (!element(q) || q->dim() != 4 || !q->is_contiguous() || !v || v->dim() != 4) return false;
  const auto qs = q->sizes(), vs = v->sizes();
  const int64_t B = qs[0], T = qs[1], HK = qs[2], D = qs[3], HV = vs[2];
  if (!same(k, *q, q->scalar_type(), qs) || !same(v, *q, q->scalar_type(), {B, T, HV, D}) || !same(g, *q, at::kFloat, {B, T, HV})) return false;
  if (cu && (!plain(cu, at::kInt, 1) || cu->device() != q->device() || B != 1 || cu->numel() < 2)) return false;
  const int64_t N = cu ? cu->numel() - 1 : B;
  if (B > INT32_MAX || T > INT32_MAX || HK > INT32_MAX || HV > INT32_MAX || D > 128 || N > INT32_MAX) return false;
  if (!room(h0, *q, at::kFloat, N * HV * D * D)) return false;
  d->dtype = q->scalar_type() == at::kFloat;
  d->batch = (int32_t)B; d->seqlen = (int32_t)T;
  d->num_qk_heads = (int32_t)HK; d->num_v_heads = (int32_t)HV; d->d_k = d->d_v = (int32_t)D;
  d->q = ptr(q); d->k = ptr(k); d->v = ptr(v); d->g = (const float*)ptr(g); d->h0 = (const float*)ptr(h0);
  d->cu_seqlens = (const int32_t*)ptr(cu);
  d->num_seqs = cu ? (int32_t)N : 0;
  *seqs = N;
  return true;
}

// gla_prefill(q, k, v, g, h0, cu_seqlens, max_seqlen, stream, scale, o, hT, want_hT, workspace, status_word) -> (o, hT, status_word, workspace) | status | None
PyObject* gla_prefill_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 14 || !g_gla_prefill) { PyErr_SetString(PyExc_TypeError, "fourteen arguments"); return nullptr; }
  const at::Tensor *q, *k, *v, *g, *h0, *cu, *o, *hT, *ws, *sw;
  ha_la_gla_args d{};
  int64_t N;
  double scale;
  if (!unpack(a[0], &q) || !unpack(a[1], &k) || !unpack(a[2], &v) || !unpack(a[3], &g) || !unpack(a[4], &h0) || !unpack(a[5], &cu) ||
      !unpack(a[9], &o) || !unpack(a[10], &hT) || !unpack(a[12], &ws) || !unpack(a[13], &sw) || !gla_inputs(q, k, v, g, h0, cu, &d, &N) ||
      !length(a[6], &d.max_seqlen) || !number(a[8], &scale))
    Py_RETURN_NONE;
  const int64_t HV = d.num_v_heads, D = d.d_k, state = N * HV * D * D;
  if (!room(o, *q, q->scalar_type(), v->numel()) || !room(hT, *q, at::kFloat, state) || !scratch_ok(ws, *q) || !room(sw, *q, at::kInt, 1)) Py_RETURN_NONE;
  d.scale = (float)scale;
  size_t need = 0;
  if (g_gla_bytes(&d, 0, &need) != HA_LA_OK) Py_RETURN_NONE;
  const int want_hT = hT ? 0 : PyObject_IsTrue(a[11]);
  if (want_hT < 0) return nullptr;
  Outputs out(a[7], *q);
  if (!out.set()) return nullptr;
  o = out.take(o, v->sizes(), q->scalar_type());
  if (want_hT) hT = out.take(hT, {N, HV, D, D}, at::kFloat);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.o = ptr(o); d.hT = (float*)ptr(hT); d.status_word = (int32_t*)ptr(sw);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gla_prefill(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(o, a[9]), out.wrap(hT, a[10]), out.wrap(sw, a[13]), out.wrap(ws, a[12])});
}

// gla_backward(do, q, k, v, g, h0, dhT, cu_seqlens, max_seqlen, stream, scale, dq, dk, dv, dg, dh0, want_dh0, workspace, status_word)
//   -> (dq, dk, dv, dg, dh0, status_word, workspace) | status | None
PyObject* gla_backward_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 19 || !g_gla_backward) { PyErr_SetString(PyExc_TypeError, "nineteen arguments"); return nullptr; }
  const at::Tensor *d_o, *q, *k, *v, *g, *h0, *dhT, *cu, *dq, *dk, *dv, *dg, *dh0, *ws, *sw;
  ha_la_gla_args d{};
  int64_t N;
  double scale;
  if (!unpack(a[0], &d_o) || !unpack(a[1], &q) || !unpack(a[2], &k) || !unpack(a[3], &v) || !unpack(a[4], &g) || !unpack(a[5], &h0) ||
      !unpack(a[6], &dhT) || !unpack(a[7], &cu) || !unpack(a[11], &dq) || !unpack(a[12], &dk) || !unpack(a[13], &dv) || !unpack(a[14], &dg) ||
      !unpack(a[15], &dh0) || !unpack(a[17], &ws) || !unpack(a[18], &sw) || !gla_inputs(q, k, v, g, h0, cu, &d, &N) ||
      !length(a[8], &d.max_seqlen) || !number(a[10], &scale))
    Py_RETURN_NONE;
  const at::ScalarType type = q->scalar_type();
  const int64_t HV = d.num_v_heads, D = d.d_k, state = N * HV * D * D;
  if (!same(d_o, *q, type, v->sizes()) || !room(dhT, *q, at::kFloat, state) || !room(dq, *q, type, q->numel()) || !room(dk, *q, type, k->numel()) ||
      !room(dv, *q, type, v->numel()) || !room(dg, *q, at::kFloat, g->numel()) || !room(dh0, *q, at::kFloat, state) || !scratch_ok(ws, *q) ||
      !room(sw, *q, at::kInt, 1))
    Py_RETURN_NONE;
  d.scale = (float)scale;
  size_t need = 0;
  if (g_gla_bytes(&d, 1, &need) != HA_LA_OK) Py_RETURN_NONE;
  const int want_dh0 = dh0 ? 0 : PyObject_IsTrue(a[16]);
  if (want_dh0 < 0) return nullptr;
  Outputs out(a[9], *q);
  if (!out.set()) return nullptr;
  dq = out.take(dq, q->sizes(), type);
  dk = out.take(dk, k->sizes(), type);
  dv = out.take(dv, v->sizes(), type);
  dg = out.take(dg, g->sizes(), at::kFloat);
  if (want_dh0) dh0 = out.take(dh0, {N, HV, D, D}, at::kFloat);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.do_ = ptr(d_o); d.dhT = (const float*)ptr(dhT);
  d.dq = ptr(dq); d.dk = ptr(dk); d.dv = ptr(dv); d.dg = (float*)ptr(dg); d.dh0 = (float*)ptr(dh0); d.status_word = (int32_t*)ptr(sw);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gla_backward(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(dq, a[11]), out.wrap(dk, a[12]), out.wrap(dv, a[13]), out.wrap(dg, a[14]), out.wrap(dh0, a[15]), out.wrap(sw, a[18]),
               out.wrap(ws, a[17])});
}

// gla_decode(q, k, v, g, state, stream, scale, o, state_out) -> (o, state_out) | status | None
PyObject* gla_decode_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 9 || !g_gla_decode) { PyErr_SetString(PyExc_TypeError, "nine arguments"); return nullptr; }
  const at::Tensor *q, *k, *v, *g, *st, *o, *so;
  double scale;
  if (!unpack(a[0], &q) || !unpack(a[1], &k) || !unpack(a[2], &v) || !unpack(a[3], &g) || !unpack(a[4], &st) || !unpack(a[7], &o) || !unpack(a[8], &so) ||
      !number(a[6], &scale) || !element(q) || q->dim() != 3 || !q->is_contiguous() || !v || v->dim() != 3)
    Py_RETURN_NONE;
  const int64_t N = q->size(0), HK = q->size(1), D = q->size(2), HV = v->size(1);
  if (N > INT32_MAX || HK > INT32_MAX || HV > INT32_MAX || D > 128) Py_RETURN_NONE;
  const int64_t state = N * HV * D * D;
  if (!same(k, *q, q->scalar_type(), q->sizes()) || !same(v, *q, q->scalar_type(), {N, HV, D}) || !same(g, *q, at::kFloat, {N, HV}) ||
      !room(st, *q, at::kFloat, state) || !room(so, *q, at::kFloat, state) || !room(o, *q, q->scalar_type(), v->numel()))
    Py_RETURN_NONE;
  ha_la_decode_args d{};
  d.dtype = q->scalar_type() == at::kFloat;
  d.num_seqs = (int32_t)N; d.num_qk_heads = (int32_t)HK; d.num_v_heads = (int32_t)HV; d.d_k = d.d_v = (int32_t)D;
  d.scale = (float)scale;
  Outputs out(a[5], *q);
  if (!out.set()) return nullptr;
  o = out.take(o, v->sizes(), q->scalar_type());
  const bool in_place = !so && st;
  if (!so) so = st ? st : out.take(nullptr, {N, HV, D, D}, at::kFloat);
  d.q = ptr(q); d.k = ptr(k); d.v = ptr(v); d.g = (const float*)ptr(g);
  d.h_in = (const float*)ptr(st); d.h_out = (float*)ptr(so); d.o = ptr(o);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gla_decode(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(o, a[7]), out.wrap(so, in_place ? a[4] : a[8])});
}

// rows of the last dimension, and the weight
bool rows_of(const at::Tensor* x, const at::Tensor* w, int64_t* rows, int32_t* cols) {
  if (!element(x) || x->dim() < 1 || !x->is_contiguous()) return false;
  const int64_t c = x->size(-1);
  if (c < 1 || c > INT32_MAX || !same(w, *x, at::kFloat, {c})) return false;
  *rows = x->numel() / c;
  *cols = (int32_t)c;
  return true;
}
bool activation_of(PyObject* o, int32_t* v) { return o != Py_None && length(o, v); }

// gated_norm(x, w, z, activation, eps, y, stream) -> y | status | None
PyObject* gated_norm_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 7 || !g_gated_norm) { PyErr_SetString(PyExc_TypeError, "seven arguments"); return nullptr; }
  const at::Tensor *x, *w, *z, *y;
  ha_la_gated_norm_args d{};
  double eps;
  if (!unpack(a[0], &x) || !unpack(a[1], &w) || !unpack(a[2], &z) || !activation_of(a[3], &d.activation) || !number(a[4], &eps) || eps < 0 ||
      !unpack(a[5], &y) || !rows_of(x, w, &d.rows, &d.cols) || (z && !same(z, *x, x->scalar_type(), x->sizes())) ||
      !room(y, *x, x->scalar_type(), x->numel()))
    Py_RETURN_NONE;
  Outputs out(a[6], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), x->scalar_type());
  d.dtype = x->scalar_type() == at::kFloat;
  d.eps = (float)eps;
  d.x = ptr(x); d.w = (const float*)ptr(w); d.z = ptr(z); d.y = ptr(y);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gated_norm(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return out.wrap(y, a[5]);
}

// gated_norm_backward(dy, x, w, z, activation, eps, dx, dw, dz, workspace, stream) -> (dx, dw, dz) | status | None
PyObject* gated_norm_backward_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_gated_norm_backward) { PyErr_SetString(PyExc_TypeError, "eleven arguments"); return nullptr; }
  const at::Tensor *dy, *x, *w, *z, *dx, *dw, *dz, *ws;
  ha_la_gated_norm_args d{};
  double eps;
  if (!unpack(a[0], &dy) || !unpack(a[1], &x) || !unpack(a[2], &w) || !unpack(a[3], &z) || !activation_of(a[4], &d.activation) || !number(a[5], &eps) ||
      eps < 0 || !unpack(a[6], &dx) || !unpack(a[7], &dw) || !unpack(a[8], &dz) || !unpack(a[9], &ws) || !rows_of(x, w, &d.rows, &d.cols))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type();
  if (!same(dy, *x, type, x->sizes()) || (z && !same(z, *x, type, x->sizes())) || !room(dx, *x, type, x->numel()) || !room(dz, *x, type, x->numel()) ||
      !room(dw, *x, at::kFloat, d.cols) || !scratch_ok(ws, *x))
    Py_RETURN_NONE;
  d.dtype = type == at::kFloat;
  d.eps = (float)eps;
  size_t need = 0;
  if (g_gated_norm_bytes(&d, &need) != HA_LA_OK) Py_RETURN_NONE;
  Outputs out(a[10], *x);
  if (!out.set()) return nullptr;
  dx = out.take(dx, x->sizes(), type);
  dw = out.take(dw, {d.cols}, at::kFloat);
  dz = z ? out.take(dz, x->sizes(), type) : nullptr;
  out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  d.x = ptr(x); d.w = (const float*)ptr(w); d.z = ptr(z); d.dy = ptr(dy); d.dx = ptr(dx); d.dz = ptr(dz); d.dw = (float*)ptr(dw);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gated_norm_backward(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(dx, a[6]), out.wrap(dw, a[7]), z ? out.wrap(dz, a[8]) : Py_NewRef(Py_None)});
}

// add_norm(x, r, w, w_post, scale, eps, y, r_out, stream) -> (y, r_out) | status | None
PyObject* add_norm_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 9 || !g_add_norm) { PyErr_SetString(PyExc_TypeError, "nine arguments"); return nullptr; }
  const at::Tensor *x, *r, *w, *wp, *y, *ro;
  ha_la_add_norm_args d{};
  double scale, eps;
  if (!unpack(a[0], &x) || !unpack(a[1], &r) || !unpack(a[2], &w) || !unpack(a[3], &wp) || !number(a[4], &scale) || !number(a[5], &eps) || eps < 0 ||
      !unpack(a[6], &y) || !unpack(a[7], &ro) || !rows_of(x, w, &d.rows, &d.cols) || !same(r, *x, x->scalar_type(), x->sizes()) ||
      (wp && !same(wp, *x, at::kFloat, {d.cols})) || !room(y, *x, x->scalar_type(), x->numel()) || !room(ro, *x, x->scalar_type(), x->numel()))
    Py_RETURN_NONE;
  Outputs out(a[8], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), x->scalar_type());
  ro = out.take(ro, x->sizes(), x->scalar_type());
  d.dtype = x->scalar_type() == at::kFloat;
  d.scale = (float)scale; d.eps = (float)eps;
  d.x = ptr(x); d.r = ptr(r); d.w = (const float*)ptr(w); d.w_post = (const float*)ptr(wp); d.y = ptr(y); d.r_out = ptr(ro);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_add_norm(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(y, a[6]), out.wrap(ro, a[7])});
}

// add_norm_backward(dy, dr_out, x, r_out, w, w_post, scale, eps, dx, dr, dw, dw_post, workspace, stream) -> (dx, dr, dw, dw_post) | status | None
PyObject* add_norm_backward_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 14 || !g_add_norm_backward) { PyErr_SetString(PyExc_TypeError, "fourteen arguments"); return nullptr; }
  const at::Tensor *dy, *dro, *x, *ro, *w, *wp, *dx, *dr, *dw, *dwp, *ws;
  ha_la_add_norm_args d{};
  double scale, eps;
  if (!unpack(a[0], &dy) || !unpack(a[1], &dro) || !unpack(a[2], &x) || !unpack(a[3], &ro) || !unpack(a[4], &w) || !unpack(a[5], &wp) ||
      !number(a[6], &scale) || !number(a[7], &eps) || eps < 0 || !unpack(a[8], &dx) || !unpack(a[9], &dr) || !unpack(a[10], &dw) || !unpack(a[11], &dwp) ||
      !unpack(a[12], &ws) || !rows_of(x, w, &d.rows, &d.cols))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type();
  if (!same(dy, *x, type, x->sizes()) || !same(ro, *x, type, x->sizes()) || (dro && !same(dro, *x, type, x->sizes())) ||
      (wp && !same(wp, *x, at::kFloat, {d.cols})) || !room(dx, *x, type, x->numel()) || !room(dr, *x, type, x->numel()) ||
      !room(dw, *x, at::kFloat, d.cols) || !room(dwp, *x, at::kFloat, d.cols) || !scratch_ok(ws, *x))
    Py_RETURN_NONE;
  d.dtype = type == at::kFloat;
  d.scale = (float)scale; d.eps = (float)eps;
  d.w_post = (const float*)ptr(wp);
  size_t need = 0;
  if (g_add_norm_bytes(&d, &need) != HA_LA_OK) Py_RETURN_NONE;
  Outputs out(a[13], *x);
  if (!out.set()) return nullptr;
  dx = out.take(dx, x->sizes(), type);
  dr = out.take(dr, x->sizes(), type);
  dw = out.take(dw, {d.cols}, at::kFloat);
  dwp = wp ? out.take(dwp, {d.cols}, at::kFloat) : nullptr;
  out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  d.x = ptr(x); d.r_out = ptr(ro); d.w = (const float*)ptr(w); d.dy = ptr(dy); d.dr_out = ptr(dro);
  d.dx = ptr(dx); d.dr = ptr(dr); d.dw = (float*)ptr(dw); d.dw_post = (float*)ptr(dwp);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_add_norm_backward(&d, out.on.handle);
  Py_END_ALLOW_THREADS
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(dx, a[8]), out.wrap(dr, a[9]), out.wrap(dw, a[10]), wp ? out.wrap(dwp, a[11]) : Py_NewRef(Py_None)});
}

// ---------------------------------------------------------------- mixer.py: short convolution, selective scan, attention over latent rows
//
// As above; inputs with a row to a token may be rows of a wider tensor.

// t is [*lead, *inner] of like's type and device, contiguous within a token, tokens at one distance: that distance, in elements
bool token_rows(const at::Tensor* t, const at::Tensor& like, at::IntArrayRef lead, std::initializer_list<int64_t> inner, int64_t* step) {
  if (!t || t->scalar_type() != like.scalar_type() || t->device() != like.device() || t->dim() != (int64_t)(lead.size() + inner.size())) return false;
  const auto size = t->sizes(), stride = t->strides();
  int64_t d = t->dim() - 1, width = 1;
  for (auto i = inner.end(); i != inner.begin(); --d) {
    const int64_t n = *--i;
    if (size[d] != n || (n != 1 && stride[d] != width)) return false;
    width *= n;
  }
  *step = width;
  int64_t tokens = 1;
  for (; d >= 0; --d) {
    if (size[d] != lead[d]) return false;
    if (lead[d] > 1) {
      if (tokens == 1) *step = stride[d];
      if (stride[d] != *step * tokens) return false;
    }
    tokens *= lead[d];
  }
  if (tokens == 0) *step = width;
  return *step >= width;
}
// ... [*lead, H, d], contiguous within a head, heads at one distance too
bool head_rows(const at::Tensor* t, const at::Tensor& like, at::IntArrayRef lead, int64_t H, int64_t* step, int64_t* head, int64_t* d) {
  if (!t || t->scalar_type() != like.scalar_type() || t->device() != like.device() || t->dim() != (int64_t)lead.size() + 2) return false;
  const auto size = t->sizes(), stride = t->strides();
  const int64_t k = lead.size();
  *d = size[k + 1];
  if (size[k] != H || *d < 1 || (*d > 1 && stride[k + 1] != 1)) return false;
  *head = H > 1 ? stride[k] : *d;
  *step = H * *d;
  int64_t tokens = 1;
  for (int64_t i = k - 1; i >= 0; --i) {
    if (size[i] != lead[i]) return false;
    if (lead[i] > 1) {
      if (tokens == 1) *step = stride[i];
      if (stride[i] != *step * tokens) return false;
    }
    tokens *= lead[i];
  }
  return tokens > 0 && *head >= *d && *step >= *d;
}
bool vector(const at::Tensor* t, const at::Tensor& like, at::IntArrayRef shape) { return !t || same(t, like, at::kFloat, shape); }
bool offsets(const at::Tensor* cu, const at::Tensor& like, int64_t batch) {
  return !cu || (plain(cu, at::kInt, 1) && cu->device() == like.device() && batch == 1 && cu->numel() >= 2 && cu->numel() <= INT32_MAX);
}
template <typename F, typename A> int without_lock(F f, const A* args, void* stream) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f(args, stream);
  Py_END_ALLOW_THREADS
  return rc;
}

// an optional contiguous tensor whose elements are in that shape's order as far as its own shape tells: from the last one on dimensions agree, but for the outermost
// (in front of which there are only ones), which has at least what the wanted ones that are left come to
bool laid_out(const at::Tensor* t, const at::Tensor& like, at::ScalarType type, at::IntArrayRef shape) {
  if (!t) return true;
  if (t->device() != like.device() || t->scalar_type() != type || !t->is_contiguous()) return false;
  const auto have = t->sizes();
  int64_t i = (int64_t)have.size() - 1, j = (int64_t)shape.size() - 1;
  for (; i > 0 && j >= 0 && have[i] == shape[j]; --i) --j;
  if (i < 0 || t->numel() < c10::multiply_integers(shape)) return false;
  int64_t least = 1;
  for (int64_t k = 0; k <= j; ++k) least *= shape[k];
  for (int64_t k = 0; j >= 0 && k < i; ++k)
    if (have[k] != 1) return false;
  return j < 0 || have[i] >= least;
}

// x [B, T, C] (`token`: [N, C]), w, bias, activation, cu_seqlens
bool conv_inputs(const at::Tensor* x, const at::Tensor* w, const at::Tensor* bias, PyObject* act, const at::Tensor* cu, bool token, ha_la_conv_args* d, int64_t* N) {
  if (!element(x) || x->dim() != (token ? 2 : 3) || !w || w->dim() != 2) return false;
  const auto s = x->sizes();
  const int64_t B = s[0], T = token ? 1 : s[1], C = s[token ? 1 : 2], K = w->size(1);
  if (B > INT32_MAX || T > INT32_MAX || C > INT32_MAX || C < 1 || K < 2 || K > 4) return false;
  if (!same(w, *x, at::kFloat, {C, K}) || !vector(bias, *x, {C}) || !activation_of(act, &d->activation) || !offsets(cu, *x, B)) return false;
  if (!token_rows(x, *x, s.slice(0, token ? 1 : 2), {C}, &d->x_stride)) return false;
  d->dtype = x->scalar_type() == at::kFloat;
  d->batch = (int32_t)B; d->seqlen = (int32_t)T; d->channels = (int32_t)C; d->taps = (int32_t)K;
  *N = cu ? cu->numel() - 1 : B;
  d->num_seqs = cu ? (int32_t)*N : 0;
  d->x = ptr(x); d->w = (const float*)ptr(w); d->bias = (const float*)ptr(bias); d->cu_seqlens = (const int32_t*)ptr(cu);
  return true;
}

// conv(x, w, bias, activation, h0, cu_seqlens, max_seqlen, y, hT, want_hT, status_word, stream) -> (y, hT, status_word) | status | None
PyObject* conv_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 12 || !g_conv) { PyErr_SetString(PyExc_TypeError, "twelve arguments"); return nullptr; }
  const at::Tensor *x, *w, *bias, *h0, *cu, *y, *hT, *sw;
  ha_la_conv_args d{};
  int64_t N;
  if (!unpack(a[0], &x) || !unpack(a[1], &w) || !unpack(a[2], &bias) || !unpack(a[4], &h0) || !unpack(a[5], &cu) || !unpack(a[7], &y) || !unpack(a[8], &hT) ||
      !unpack(a[10], &sw) || !conv_inputs(x, w, bias, a[3], cu, false, &d, &N) || !length(a[6], &d.max_seqlen))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type();
  const int64_t C = d.channels, K = d.taps - 1;
  if (!laid_out(h0, *x, type, {N, K, C}) || !laid_out(y, *x, type, x->sizes()) || !laid_out(hT, *x, type, {N, K, C}) || !room(sw, *x, at::kInt, 1)) Py_RETURN_NONE;
  const int want = hT ? 0 : PyObject_IsTrue(a[9]);
  if (want < 0) return nullptr;
  Outputs out(a[11], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), type);
  if (want) hT = out.take(hT, {N, K, C}, type);
  sw = out.take(sw, {1}, at::kInt, true);
  d.h0 = ptr(h0); d.y = ptr(y); d.hT = ptr(hT); d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_conv, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(y, a[7]), out.wrap(hT, a[8]), out.wrap(sw, a[10])});
}

// conv_backward(dy, x, w, bias, activation, h0, dhT, cu_seqlens, max_seqlen, dx, dw, db, dh0, want_dh0, workspace, status_word, stream)
//   -> (dx, dw, db, dh0, status_word, workspace) | status | None
PyObject* conv_backward_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 17 || !g_conv_backward) { PyErr_SetString(PyExc_TypeError, "seventeen arguments"); return nullptr; }
  const at::Tensor *dy, *x, *w, *bias, *h0, *dhT, *cu, *dx, *dw, *db, *dh0, *ws, *sw;
  ha_la_conv_args d{};
  int64_t N;
  if (!unpack(a[0], &dy) || !unpack(a[1], &x) || !unpack(a[2], &w) || !unpack(a[3], &bias) || !unpack(a[5], &h0) || !unpack(a[6], &dhT) || !unpack(a[7], &cu) ||
      !unpack(a[9], &dx) || !unpack(a[10], &dw) || !unpack(a[11], &db) || !unpack(a[12], &dh0) || !unpack(a[14], &ws) || !unpack(a[15], &sw) ||
      !conv_inputs(x, w, bias, a[4], cu, false, &d, &N) || !length(a[8], &d.max_seqlen))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type();
  const int64_t C = d.channels, K = d.taps - 1;
  if (!same(dy, *x, type, x->sizes()) || !laid_out(h0, *x, type, {N, K, C}) || !laid_out(dhT, *x, type, {N, K, C}) || !laid_out(dx, *x, type, x->sizes()) ||
      !laid_out(dw, *x, at::kFloat, {C, K + 1}) || !laid_out(db, *x, at::kFloat, {C}) || !laid_out(dh0, *x, type, {N, K, C}) || !scratch_ok(ws, *x) || !room(sw, *x, at::kInt, 1))
    Py_RETURN_NONE;
  size_t need = 0;
  if (g_conv_bytes(&d, &need) != HA_LA_OK) Py_RETURN_NONE;
  const int want = dh0 ? 0 : PyObject_IsTrue(a[13]);
  if (want < 0) return nullptr;
  Outputs out(a[16], *x);
  if (!out.set()) return nullptr;
  dx = out.take(dx, x->sizes(), type);
  dw = out.take(dw, {C, K + 1}, at::kFloat);
  db = bias ? out.take(db, {C}, at::kFloat) : nullptr;
  if (want) dh0 = out.take(dh0, {N, K, C}, type);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.h0 = ptr(h0); d.dy = ptr(dy); d.dhT = ptr(dhT); d.dx = ptr(dx); d.dw = (float*)ptr(dw); d.db = (float*)ptr(db); d.dh0 = ptr(dh0);
  d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_conv_backward, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(dx, a[9]), out.wrap(dw, a[10]), db ? out.wrap(db, a[11]) : Py_NewRef(Py_None), out.wrap(dh0, a[12]), out.wrap(sw, a[15]), out.wrap(ws, a[14])});
}

// conv_decode(x, w, state, bias, activation, y, state_out, stream) -> (y, state) | status | None
PyObject* conv_decode_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !g_conv_decode) { PyErr_SetString(PyExc_TypeError, "eight arguments"); return nullptr; }
  const at::Tensor *x, *w, *st, *bias, *y, *so;
  ha_la_conv_args d{};
  int64_t N;
  if (!unpack(a[0], &x) || !unpack(a[1], &w) || !unpack(a[2], &st) || !unpack(a[3], &bias) || !unpack(a[5], &y) || !unpack(a[6], &so) ||
      !conv_inputs(x, w, bias, a[4], nullptr, true, &d, &N))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type();
  const int64_t C = d.channels, K = d.taps - 1;
  if (!laid_out(st, *x, type, {N, K, C}) || !laid_out(so, *x, type, {N, K, C}) || !laid_out(y, *x, type, x->sizes())) Py_RETURN_NONE;
  Outputs out(a[7], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), type);
  const bool in_place = !so && st;
  if (!so) so = st ? st : out.take(nullptr, {N, K, C}, type);
  d.h0 = ptr(st); d.y = ptr(y); d.hT = ptr(so);
  const int rc = without_lock(g_conv_decode, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(y, a[5]), out.wrap(so, in_place ? a[2] : a[6])});
}

// x, dt, z [B, T, channels] (`token`: [N, channels]), A, B, C, D, dt_bias, cu_seqlens
bool scan_inputs(const at::Tensor* x, const at::Tensor* dt, const at::Tensor* A, const at::Tensor* B, const at::Tensor* C, const at::Tensor* D, const at::Tensor* z,
                 const at::Tensor* bias, PyObject* softplus, const at::Tensor* cu, bool token, ha_la_scan_args* d, int64_t* N) {
  const int64_t k = token ? 1 : 2;
  if (!element(x) || x->dim() != k + 1 || !A || A->dim() != 2 || !B || B->dim() != k + 2 || (softplus != Py_True && softplus != Py_False)) return false;
  const auto s = x->sizes(), lead = s.slice(0, k);
  const int64_t batch = s[0], T = token ? 1 : s[1], ch = s[k], G = B->size(k), S = B->size(k + 1);
  if (batch > INT32_MAX || T > INT32_MAX || ch > INT32_MAX || ch < 1 || G < 1 || S < 1 || S > 64 || ch % G) return false;
  if (!same(A, *x, at::kFloat, {ch, S}) || !vector(D, *x, {ch}) || !vector(bias, *x, {ch}) || !offsets(cu, *x, batch)) return false;
  if (!token_rows(x, *x, lead, {ch}, &d->x_stride) || !token_rows(dt, *x, lead, {ch}, &d->dt_stride) || !token_rows(B, *x, lead, {G, S}, &d->b_stride) ||
      !token_rows(C, *x, lead, {G, S}, &d->c_stride) || (z && !token_rows(z, *x, lead, {ch}, &d->z_stride)))
    return false;
  d->dtype = x->scalar_type() == at::kFloat;
  d->batch = (int32_t)batch; d->seqlen = (int32_t)T; d->channels = (int32_t)ch; d->states = (int32_t)S; d->groups = (int32_t)G;
  d->softplus = softplus == Py_True;
  *N = cu ? cu->numel() - 1 : batch;
  d->num_seqs = cu ? (int32_t)*N : 0;
  d->cu_seqlens = (const int32_t*)ptr(cu);
  d->x = ptr(x); d->dt = ptr(dt); d->B = ptr(B); d->C = ptr(C); d->z = ptr(z);
  d->A = (const float*)ptr(A); d->D = (const float*)ptr(D); d->dt_bias = (const float*)ptr(bias);
  return true;
}

// scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, cu_seqlens, max_seqlen, y, hT, want_hT, workspace, status_word, stream) -> (y, hT, status_word, workspace) | status | None
PyObject* scan_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 18 || !g_scan) { PyErr_SetString(PyExc_TypeError, "eighteen arguments"); return nullptr; }
  const at::Tensor *x, *dt, *A, *B, *C, *D, *z, *bias, *h0, *cu, *y, *hT, *ws, *sw;
  ha_la_scan_args d{};
  int64_t N;
  if (!unpack(a[0], &x) || !unpack(a[1], &dt) || !unpack(a[2], &A) || !unpack(a[3], &B) || !unpack(a[4], &C) || !unpack(a[5], &D) || !unpack(a[6], &z) ||
      !unpack(a[7], &bias) || !unpack(a[9], &h0) || !unpack(a[10], &cu) || !unpack(a[12], &y) || !unpack(a[13], &hT) || !unpack(a[15], &ws) || !unpack(a[16], &sw) ||
      !scan_inputs(x, dt, A, B, C, D, z, bias, a[8], cu, false, &d, &N) || !length(a[11], &d.max_seqlen))
    Py_RETURN_NONE;
  const int64_t ch = d.channels, S = d.states;
  const int64_t state[3] = {N, ch, S};
  if (!laid_out(h0, *x, at::kFloat, state) || !laid_out(y, *x, x->scalar_type(), x->sizes()) || !laid_out(hT, *x, at::kFloat, state) || !scratch_ok(ws, *x) || !room(sw, *x, at::kInt, 1))
    Py_RETURN_NONE;
  size_t need = 0;
  if (g_scan_bytes(&d, 0, &need) != HA_LA_OK) Py_RETURN_NONE;
  const int want = hT ? 0 : PyObject_IsTrue(a[14]);
  if (want < 0) return nullptr;
  Outputs out(a[17], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), x->scalar_type());
  if (want) hT = out.take(hT, {N, ch, S}, at::kFloat);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.h0 = (const float*)ptr(h0); d.y = ptr(y); d.hT = (float*)ptr(hT); d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_scan, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(y, a[12]), out.wrap(hT, a[13]), out.wrap(sw, a[16]), out.wrap(ws, a[15])});
}

// scan_backward(dy, x, dt, A, B, C, D, z, dt_bias, softplus, h0, dhT, cu_seqlens, max_seqlen, dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0, want_dh0, workspace,
//   status_word, stream) -> (dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0, status_word, workspace) | status | None
PyObject* scan_backward_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 27 || !g_scan_backward) { PyErr_SetString(PyExc_TypeError, "twenty-seven arguments"); return nullptr; }
  const at::Tensor *dy, *x, *dt, *A, *B, *C, *D, *z, *bias, *h0, *dhT, *cu, *dx, *ddt, *dA, *dB, *dC, *dD, *dz, *dbias, *dh0, *ws, *sw;
  ha_la_scan_args d{};
  int64_t N;
  if (!unpack(a[0], &dy) || !unpack(a[1], &x) || !unpack(a[2], &dt) || !unpack(a[3], &A) || !unpack(a[4], &B) || !unpack(a[5], &C) || !unpack(a[6], &D) ||
      !unpack(a[7], &z) || !unpack(a[8], &bias) || !unpack(a[10], &h0) || !unpack(a[11], &dhT) || !unpack(a[12], &cu) || !unpack(a[14], &dx) || !unpack(a[15], &ddt) ||
      !unpack(a[16], &dA) || !unpack(a[17], &dB) || !unpack(a[18], &dC) || !unpack(a[19], &dD) || !unpack(a[20], &dz) || !unpack(a[21], &dbias) || !unpack(a[22], &dh0) ||
      !unpack(a[24], &ws) || !unpack(a[25], &sw) || !scan_inputs(x, dt, A, B, C, D, z, bias, a[9], cu, false, &d, &N) || !length(a[13], &d.max_seqlen))
    Py_RETURN_NONE;
  const at::ScalarType type = x->scalar_type(), f32 = at::kFloat;
  const int64_t ch = d.channels, S = d.states;
  const int64_t state[3] = {N, ch, S};
  if (!same(dy, *x, type, x->sizes()) || !laid_out(h0, *x, f32, state) || !laid_out(dhT, *x, f32, state) || !laid_out(dx, *x, type, x->sizes()) || !laid_out(ddt, *x, type, x->sizes()) ||
      !laid_out(dA, *x, f32, {ch, S}) || !laid_out(dB, *x, type, B->sizes()) || !laid_out(dC, *x, type, B->sizes()) || !laid_out(dD, *x, f32, {ch}) ||
      !laid_out(dz, *x, type, x->sizes()) || !laid_out(dbias, *x, f32, {ch}) || !laid_out(dh0, *x, f32, state) || !scratch_ok(ws, *x) || !room(sw, *x, at::kInt, 1))
    Py_RETURN_NONE;
  size_t need = 0;
  if (g_scan_bytes(&d, 1, &need) != HA_LA_OK) Py_RETURN_NONE;
  const int want = dh0 ? 0 : PyObject_IsTrue(a[23]);
  if (want < 0) return nullptr;
  Outputs out(a[26], *x);
  if (!out.set()) return nullptr;
  dx = out.take(dx, x->sizes(), type);
  ddt = out.take(ddt, x->sizes(), type);
  dA = out.take(dA, {ch, S}, f32);
  dB = out.take(dB, B->sizes(), type);
  dC = out.take(dC, B->sizes(), type);
  dD = D ? out.take(dD, {ch}, f32) : nullptr;
  dz = z ? out.take(dz, x->sizes(), type) : nullptr;
  dbias = bias ? out.take(dbias, {ch}, f32) : nullptr;
  if (want) dh0 = out.take(dh0, {N, ch, S}, f32);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.h0 = (const float*)ptr(h0); d.dy = ptr(dy); d.dhT = (const float*)ptr(dhT); d.dx = ptr(dx); d.ddt = ptr(ddt); d.dA = (float*)ptr(dA); d.dB = ptr(dB); d.dC = ptr(dC);
  d.dD = (float*)ptr(dD); d.dz = ptr(dz); d.ddt_bias = (float*)ptr(dbias); d.dh0 = (float*)ptr(dh0); d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_scan_backward, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  auto given = [&](const at::Tensor* t, PyObject* o) { return t ? out.wrap(t, o) : Py_NewRef(Py_None); };
  return pack({out.wrap(dx, a[14]), out.wrap(ddt, a[15]), out.wrap(dA, a[16]), out.wrap(dB, a[17]), out.wrap(dC, a[18]), given(dD, a[19]), given(dz, a[20]),
               given(dbias, a[21]), out.wrap(dh0, a[22]), out.wrap(sw, a[25]), out.wrap(ws, a[24])});
}

// scan_decode(x, dt, A, B, C, state, D, z, dt_bias, softplus, y, state_out, stream) -> (y, state) | status | None
PyObject* scan_decode_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 13 || !g_scan_decode) { PyErr_SetString(PyExc_TypeError, "thirteen arguments"); return nullptr; }
  const at::Tensor *x, *dt, *A, *B, *C, *st, *D, *z, *bias, *y, *so;
  ha_la_scan_args d{};
  int64_t N;
  if (!unpack(a[0], &x) || !unpack(a[1], &dt) || !unpack(a[2], &A) || !unpack(a[3], &B) || !unpack(a[4], &C) || !unpack(a[5], &st) || !unpack(a[6], &D) ||
      !unpack(a[7], &z) || !unpack(a[8], &bias) || !unpack(a[10], &y) || !unpack(a[11], &so) || !scan_inputs(x, dt, A, B, C, D, z, bias, a[9], nullptr, true, &d, &N))
    Py_RETURN_NONE;
  const int64_t ch = d.channels, S = d.states;
  const int64_t state[3] = {N, ch, S};
  if (!laid_out(st, *x, at::kFloat, state) || !laid_out(so, *x, at::kFloat, state) || !laid_out(y, *x, x->scalar_type(), x->sizes())) Py_RETURN_NONE;
  Outputs out(a[12], *x);
  if (!out.set()) return nullptr;
  y = out.take(y, x->sizes(), x->scalar_type());
  const bool in_place = !so && st;
  if (!so) so = st ? st : out.take(nullptr, {N, ch, S}, at::kFloat);
  d.h0 = (const float*)ptr(st); d.y = ptr(y); d.hT = (float*)ptr(so);
  const int rc = without_lock(g_scan_decode, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(y, a[10]), out.wrap(so, in_place ? a[5] : a[11])});
}

// latent_prefill(q, kn, kr, v, scale, cu_seqlens, cu_seqlens_k, max_seqlen, o, lse, status_word, stream) -> (o, lse, status_word) | status | None
PyObject* latent_prefill_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 12 || !g_latent_prefill) { PyErr_SetString(PyExc_TypeError, "twelve arguments"); return nullptr; }
  const at::Tensor *q, *kn, *kr, *v, *cu, *cuk, *o, *lse, *sw;
  ha_la_latent_prefill_args d{};
  double scale;
  if (!unpack(a[0], &q) || !unpack(a[1], &kn) || !unpack(a[2], &kr) || !unpack(a[3], &v) || !unpack(a[5], &cu) || !unpack(a[6], &cuk) || !unpack(a[8], &o) ||
      !unpack(a[9], &lse) || !unpack(a[10], &sw) || !number(a[4], &scale) || !length(a[7], &d.max_seqlen) || !element(q) || q->dim() != 4 || !kr || kr->dim() != 3 ||
      (!cu && cuk))
    Py_RETURN_NONE;
  const auto qs = q->sizes();
  const int64_t B = qs[0], T = qs[1], H = qs[2], dq = qs[3], Tk = kr->size(1), dr = kr->size(2), keys[2] = {B, Tk};
  if (B > INT32_MAX || T > INT32_MAX || Tk > INT32_MAX || H > INT32_MAX || H < 1 || dr >= dq || dq > 4096 || !offsets(cu, *q, B)) Py_RETURN_NONE;
  if (cu && !cuk) {
    if (Tk != T) Py_RETURN_NONE;
    cuk = cu;
  }
  int64_t dn, dv;
  const at::IntArrayRef lead_k(keys, 2);
  if (!token_rows(q, *q, qs.slice(0, 2), {H, dq}, &d.q_stride) || !token_rows(kr, *q, lead_k, {dr}, &d.kr_stride) ||
      !head_rows(kn, *q, lead_k, H, &d.kn_stride, &d.kn_head_stride, &dn) || !head_rows(v, *q, lead_k, H, &d.v_stride, &d.v_head_stride, &dv) || dn + dr != dq ||
      (cuk && !same(cuk, *q, at::kInt, cu->sizes())) || dv > 4096 || !laid_out(o, *q, q->scalar_type(), {B, T, H, dv}) || !laid_out(lse, *q, at::kFloat, {B, T, H}) ||
      !room(sw, *q, at::kInt, 1))
    Py_RETURN_NONE;
  d.dtype = q->scalar_type() == at::kFloat;
  d.batch = (int32_t)B; d.seqlen = (int32_t)T; d.seqlen_k = (int32_t)Tk; d.num_heads = (int32_t)H;
  d.d_nope = (int32_t)dn; d.d_rope = (int32_t)dr; d.d_v = (int32_t)dv; d.scale = (float)scale;
  d.num_seqs = cu ? (int32_t)(cu->numel() - 1) : 0;
  Outputs out(a[11], *q);
  if (!out.set()) return nullptr;
  o = out.take(o, {B, T, H, dv}, q->scalar_type());
  lse = out.take(lse, {B, T, H}, at::kFloat);
  sw = out.take(sw, {1}, at::kInt, true);
  d.cu_seqlens = (const int32_t*)ptr(cu); d.cu_seqlens_k = (const int32_t*)ptr(cuk);
  d.q = ptr(q); d.kn = ptr(kn); d.kr = ptr(kr); d.v = ptr(v); d.o = ptr(o); d.lse = (float*)ptr(lse); d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_latent_prefill, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(o, a[8]), out.wrap(lse, a[9]), out.wrap(sw, a[10])});
}

// latent_decode(q, cache, page_table, lengths, scale, o, lse, d_latent, workspace, status_word, stream) -> (o, lse, status_word, workspace) | status | None
PyObject* latent_decode_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_latent_decode) { PyErr_SetString(PyExc_TypeError, "eleven arguments"); return nullptr; }
  const at::Tensor *q, *cache, *table, *lengths, *o, *lse, *ws, *sw;
  ha_la_latent_decode_args d{};
  double scale;
  if (!unpack(a[0], &q) || !unpack(a[1], &cache) || !unpack(a[2], &table) || !unpack(a[3], &lengths) || !unpack(a[5], &o) || !unpack(a[6], &lse) ||
      !unpack(a[8], &ws) || !unpack(a[9], &sw) || !number(a[4], &scale) || !element(q) || q->dim() != 4 || !q->is_contiguous() || !cache || cache->dim() != 3 ||
      !table || table->dim() != 2 || (a[7] != Py_None && !length(a[7], &d.d_latent)))
    Py_RETURN_NONE;
  const int64_t N = q->size(0), T = q->size(1), H = q->size(2), D = q->size(3), P = cache->size(0), page = cache->size(1), M = table->size(1);
  if (N > INT32_MAX || T > INT32_MAX || H > INT32_MAX || D > 4096 || P > INT32_MAX || page > INT32_MAX || M > INT32_MAX || T < 1 || H < 1 || page < 1 || (page & (page - 1)))
    Py_RETURN_NONE;
  if (a[7] == Py_None) d.d_latent = (int32_t)D - 64;
  if (d.d_latent < 1 || d.d_latent > D) Py_RETURN_NONE;
  const int64_t dl = d.d_latent;
  if (!same(cache, *q, q->scalar_type(), {P, page, D}) || !same(table, *q, at::kInt, {N, M}) || !same(lengths, *q, at::kInt, {N}) ||
      !laid_out(o, *q, q->scalar_type(), {N, T, H, dl}) || !laid_out(lse, *q, at::kFloat, {N, T, H}) || !scratch_ok(ws, *q) || !room(sw, *q, at::kInt, 1))
    Py_RETURN_NONE;
  d.dtype = q->scalar_type() == at::kFloat;
  d.num_seqs = (int32_t)N; d.new_tokens = (int32_t)T; d.num_heads = (int32_t)H; d.d_rope = (int32_t)(D - dl);
  d.page_size = (int32_t)page; d.num_pages = (int32_t)P; d.max_pages = (int32_t)M; d.scale = (float)scale;
  size_t need = 0;
  Outputs out(a[10], *q);                                  // (the workspace is for the device's SMs)
  if (!out.set()) return nullptr;
  if (g_latent_decode_bytes(&d, &need) != HA_LA_OK) Py_RETURN_NONE;
  o = out.take(o, {N, T, H, dl}, q->scalar_type());
  lse = out.take(lse, {N, T, H}, at::kFloat);
  ws = out.scratch(ws, need, &d.workspace, &d.workspace_bytes);
  sw = out.take(sw, {1}, at::kInt, true);
  d.q = ptr(q); d.cache = ptr(cache); d.page_table = (const int32_t*)ptr(table); d.lengths = (const int32_t*)ptr(lengths);
  d.o = ptr(o); d.lse = (float*)ptr(lse); d.status_word = (int32_t*)ptr(sw);
  const int rc = without_lock(g_latent_decode, &d, out.on.handle);
  if (rc != HA_LA_OK) return PyLong_FromLong(rc);
  return pack({out.wrap(o, a[5]), out.wrap(lse, a[6]), out.wrap(sw, a[9]), out.wrap(ws, a[8])});
}

// torch's C++ calls throw (no memory, no driver, a tensor without storage).  An exception that left these functions would go
// through the interpreter's C frames and end the process; torch's own translation gives the caller the type that the same
// call raises in Python.
template <PyObject* (*call)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return call(a, n);
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&bind)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<decode_call>)), METH_FASTCALL, nullptr},
    {"prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<prefill_call>)), METH_FASTCALL, nullptr},
    {"gla_prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<gla_prefill_call>)), METH_FASTCALL, nullptr},
    {"gla_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<gla_backward_call>)), METH_FASTCALL, nullptr},
    {"gla_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<gla_decode_call>)), METH_FASTCALL, nullptr},
    {"gated_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<gated_norm_call>)), METH_FASTCALL, nullptr},
    {"gated_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<gated_norm_backward_call>)), METH_FASTCALL, nullptr},
    {"add_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<add_norm_call>)), METH_FASTCALL, nullptr},
    {"add_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<add_norm_backward_call>)), METH_FASTCALL, nullptr},
    {"conv", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<conv_call>)), METH_FASTCALL, nullptr},
    {"conv_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<conv_backward_call>)), METH_FASTCALL, nullptr},
    {"conv_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<conv_decode_call>)), METH_FASTCALL, nullptr},
    {"scan", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<scan_call>)), METH_FASTCALL, nullptr},
    {"scan_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<scan_backward_call>)), METH_FASTCALL, nullptr},
    {"scan_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<scan_decode_call>)), METH_FASTCALL, nullptr},
    {"latent_prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<latent_prefill_call>)), METH_FASTCALL, nullptr},
    {"latent_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<latent_decode_call>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "ha_la_torch_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ha_la_torch_call(void) { return PyModule_Create(&kModule); }
