// The host part of the calls a layer makes per pass (mask, forward, the two in one, backward) as a CPython
// module: sizes, checks of the tensors, allocation of what the caller did not pass, and the call of
// the C ABI.  A small layer is bound by this part, not by its kernels (one training step
// of 2 heads x 1110 tokens, d = 128: 191 -> 126 us, of 2 x 1024 floats, d = 64, 186 -> 109; mask and forward
// of 3 x 902, d = 64, 44 -> 28).
//
// The module decides nothing by itself.  Whatever it does not know exactly -- a tensor subclass, a
// tensor that does not fit the parameters, parameters the library refuses -- it hands back (None), and
// binding.py goes through its own checks and raises what it always raised.  An error code of the
// library comes back as an integer.  Nothing is kept between calls.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>

#include <ATen/ATen.h>
#include <ATen/TracerMode.h>
#include <c10/core/DeviceGuard.h>

#include "../../include/sla.h"

namespace {

PyObject *g_device = nullptr, *g_stream = nullptr;   // torch's accessors of the current device and its raw stream

struct Call {
  const sla_params* p;
  sla_sizes_t z;
  at::ScalarType dt;
};

bool open_call(PyObject* addr, Call& c) {
  c.p = static_cast<const sla_params*>(PyLong_AsVoidPtr(addr));
  if (!c.p || sla_sizes(c.p, &c.z) != SLA_OK) return false;
  c.dt = c.p->dtype == SLA_F32 ? at::kFloat : at::kBFloat16;
  return true;
}

// a plain tensor (no subclass with functions of its own), or null
const at::Tensor* plain(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// Q, K, V, O, dO, dQ, dK, dV: type, shape and memory order as the parameters state
bool dense(const at::Tensor* t, const Call& c) {
  const sla_params& p = *c.p;
  if (!t || !t->is_cuda() || t->scalar_type() != c.dt || t->dim() != 4) return false;
  const auto s = t->sizes();
  if (p.layout == SLA_BNHD) return s[0] == p.B && s[1] == p.N && s[2] == p.H && s[3] == p.d && t->is_contiguous();
  if (s[0] != p.B || s[1] != p.H || s[2] != p.N || s[3] != p.d) return false;
  if (p.layout != SLA_STRIDED) return t->is_contiguous();
  const auto st = t->strides();
  return st[0] == p.stride_b && st[1] == p.stride_h && st[2] == p.stride_n && st[3] == 1;
}
bool packed(const at::Tensor* t, at::IntArrayRef shape, at::ScalarType dt) {
  return t && t->is_cuda() && t->scalar_type() == dt && t->sizes() == shape && t->is_contiguous();
}
bool bytes(const at::Tensor* t, uint64_t need) {
  return t && t->is_cuda() && t->scalar_type() == at::kByte && t->dim() == 1 && t->is_contiguous() &&
         (uint64_t)t->numel() >= need;
}
bool mask(const at::Tensor* t, const Call& c) {
  return packed(t, {c.p->B, c.p->H, c.z.Tq, c.z.T}, at::kChar);
}

// An output or buffer of a call: the caller's, which has to fit, or a new one.
class Slot {
 public:
  explicit Slot(PyObject* o) : given_(o != Py_None ? o : nullptr), t_(given_ ? plain(given_) : nullptr) {}
  template <class Fits>
  bool ok(Fits fits) const { return !given_ || (t_ && fits(t_)); }
  template <class Make>
  void fill(Make make) {
    if (given_) return;
    own_ = make();
    t_ = &own_;
  }
  void* ptr() const { return t_->data_ptr(); }
  size_t size() const { return (size_t)t_->numel(); }
  PyObject* object() const {   // a new reference
    if (!given_) return THPVariable_Wrap(own_);
    Py_INCREF(given_);
    return given_;
  }

 private:
  PyObject* given_;
  at::Tensor own_;
  const at::Tensor* t_;
};

// Allocations and launches run without the interpreter lock, as they do when Python calls them one by one.
class NoGil {
 public:
  NoGil() : s_(PyEval_SaveThread()) {}
  ~NoGil() { PyEval_RestoreThread(s_); }
 private:
  PyThreadState* s_;
};

at::Tensor new_bytes(uint64_t n, const at::Tensor& like) {
  return at::empty({(int64_t)(n < 256 ? 256 : n)}, like.options().dtype(at::kByte).requires_grad(false));
}
at::Tensor new_like(const at::Tensor& t, const Call& c) {
  const auto o = t.options().requires_grad(false);
  return c.p->layout == SLA_STRIDED ? at::empty_strided(t.sizes(), t.strides(), o) : at::empty(t.sizes(), o);
}

bool current_stream(void** out) {
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) return false;
  PyObject* st = PyObject_CallFunctionObjArgs(g_stream, dev, nullptr);
  Py_DECREF(dev);
  if (!st) return false;
  *out = PyLong_AsVoidPtr(st);
  Py_DECREF(st);
  return !PyErr_Occurred();
}

PyObject* pack(std::initializer_list<PyObject*> items) {
  PyObject* t = PyTuple_New((Py_ssize_t)items.size());
  bool ok = t != nullptr;
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    ok = ok && o;
    if (t) PyTuple_SET_ITEM(t, i++, o);
    else Py_XDECREF(o);
  }
  if (ok) return t;
  Py_XDECREF(t);
  return nullptr;
}

// build_mask(params address, Q, K, workspace, Mc, luts) -> (Mc, luts, workspace)
PyObject* build_mask(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Call c;
  if (n != 6 || !open_call(a[0], c)) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[1]), *K = plain(a[2]);
  Slot ws(a[3]), Mc(a[4]), luts(a[5]);
  if (!dense(Q, c) || !dense(K, c) || !Mc.ok([&](auto t) { return mask(t, c); }) ||
      !luts.ok([&](auto t) { return bytes(t, c.z.luts_bytes); }) || !ws.ok([&](auto t) { return bytes(t, c.z.ws_mask_bytes); }))
    Py_RETURN_NONE;
  void* st;
  if (!current_stream(&st)) return nullptr;
  int rc;
  {
    NoGil free;
    Mc.fill([&] {
      return at::empty({c.p->B, c.p->H, c.z.Tq, c.z.T}, Q->options().dtype(at::kChar).requires_grad(false));
    });
    luts.fill([&] { return new_bytes(c.z.luts_bytes, *Q); });
    ws.fill([&] { return new_bytes(c.z.ws_mask_bytes, *Q); });
    rc = sla_build_mask(c.p, Q->data_ptr(), K->data_ptr(), (int8_t*)Mc.ptr(), luts.ptr(), ws.ptr(), ws.size(), st);
  }
  if (rc != SLA_OK) return PyLong_FromLong(rc);
  return pack({Mc.object(), luts.object(), ws.object()});
  END_HANDLE_TH_ERRORS
}

// forward(params address, Q, K, V, W, Mc, luts, O, saved, workspace, need_saved) -> (O, saved or None)
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Call c;
  if (n != 11 || !open_call(a[0], c)) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[1]), *K = plain(a[2]), *V = plain(a[3]), *W = plain(a[4]), *Mc = plain(a[5]),
                   *luts = plain(a[6]);
  Slot O(a[7]), saved(a[8]), ws(a[9]);
  if (!dense(Q, c) || !dense(K, c) || !dense(V, c) || !packed(W, {c.p->d, c.p->d}, c.dt) || !mask(Mc, c) ||
      !bytes(luts, c.z.luts_bytes) || !O.ok([&](auto t) { return dense(t, c); }) ||
      !saved.ok([&](auto t) { return bytes(t, c.z.saved_bytes); }) ||
      !ws.ok([&](auto t) { return bytes(t, c.z.ws_forward_bytes); }))
    Py_RETURN_NONE;
  const int need = PyObject_IsTrue(a[10]);
  if (need < 0) return nullptr;
  const bool save = need || a[8] != Py_None;
  void* st;
  if (!current_stream(&st)) return nullptr;
  int rc;
  {
    NoGil free;
    O.fill([&] { return new_like(*Q, c); });
    if (save) saved.fill([&] { return new_bytes(c.z.saved_bytes, *Q); });
    ws.fill([&] { return new_bytes(c.z.ws_forward_bytes, *Q); });
    rc = sla_forward(c.p, Q->data_ptr(), K->data_ptr(), V->data_ptr(), W->data_ptr(), (const int8_t*)Mc->data_ptr(),
                     luts->data_ptr(), O.ptr(), save ? saved.ptr() : nullptr, ws.ptr(), ws.size(), st);
  }
  if (rc != SLA_OK) return PyLong_FromLong(rc);
  if (!save) Py_INCREF(Py_None);
  return pack({O.object(), save ? saved.object() : Py_None});
  END_HANDLE_TH_ERRORS
}

// mask_forward(params address, Q, K, V, W, need_saved) -> (Mc, luts, O, saved or None)
PyObject* mask_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Call c;
  if (n != 6 || !open_call(a[0], c)) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[1]), *K = plain(a[2]), *V = plain(a[3]), *W = plain(a[4]);
  if (!dense(Q, c) || !dense(K, c) || !dense(V, c) || !packed(W, {c.p->d, c.p->d}, c.dt)) Py_RETURN_NONE;
  const int save = PyObject_IsTrue(a[5]);
  if (save < 0) return nullptr;
  void* st;
  if (!current_stream(&st)) return nullptr;
  at::Tensor Mc, luts, O, saved;
  int rc;
  {
    NoGil free;
    Mc = at::empty({c.p->B, c.p->H, c.z.Tq, c.z.T}, Q->options().dtype(at::kChar).requires_grad(false));
    luts = new_bytes(c.z.luts_bytes, *Q);
    O = new_like(*Q, c);
    if (save) saved = new_bytes(c.z.saved_bytes, *Q);
    const at::Tensor wm = new_bytes(c.z.ws_mask_bytes, *Q), wf = new_bytes(c.z.ws_forward_bytes, *Q);
    rc = sla_mask_forward(c.p, Q->data_ptr(), K->data_ptr(), V->data_ptr(), W->data_ptr(), (int8_t*)Mc.data_ptr(),
                          luts.data_ptr(), wm.data_ptr(), (size_t)wm.numel(), O.data_ptr(), save ? saved.data_ptr() : nullptr,
                          wf.data_ptr(), (size_t)wf.numel(), st);
  }
  if (rc != SLA_OK) return PyLong_FromLong(rc);
  if (!save) Py_INCREF(Py_None);
  return pack({THPVariable_Wrap(Mc), THPVariable_Wrap(luts), THPVariable_Wrap(O), save ? THPVariable_Wrap(saved) : Py_None});
  END_HANDLE_TH_ERRORS
}

// backward(params address, Q, K, V, W, Mc, luts, saved, dO, workspace, dQ, dK, dV, dW, dW in bf16) -> (dQ, dK, dV, dW)
PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Call c;
  if (n != 15 || !open_call(a[0], c)) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[1]), *K = plain(a[2]), *V = plain(a[3]), *W = plain(a[4]), *Mc = plain(a[5]),
                   *luts = plain(a[6]), *saved = plain(a[7]), *dO = plain(a[8]);
  Slot ws(a[9]), dQ(a[10]), dK(a[11]), dV(a[12]), dW(a[13]);
  const int w16 = PyObject_IsTrue(a[14]);
  if (w16 < 0) return nullptr;
  const at::ScalarType wt = w16 ? at::kBFloat16 : at::kFloat;
  const auto fits = [&](auto t) { return dense(t, c); };
  if (!dense(Q, c) || !dense(K, c) || !dense(V, c) || !dense(dO, c) || !packed(W, {c.p->d, c.p->d}, c.dt) ||
      !mask(Mc, c) || !bytes(luts, c.z.luts_bytes) || !bytes(saved, c.z.saved_bytes) || !dQ.ok(fits) || !dK.ok(fits) ||
      !dV.ok(fits) || !dW.ok([&](auto t) { return packed(t, {c.p->d, c.p->d}, wt); }) ||
      !ws.ok([&](auto t) { return bytes(t, c.z.ws_backward_bytes); }))
    Py_RETURN_NONE;
  void* st;
  if (!current_stream(&st)) return nullptr;
  int rc;
  {
    NoGil free;
    dQ.fill([&] { return new_like(*Q, c); });
    dK.fill([&] { return new_like(*K, c); });
    dV.fill([&] { return new_like(*V, c); });
    dW.fill([&] { return at::empty({c.p->d, c.p->d}, Q->options().dtype(wt).requires_grad(false)); });
    ws.fill([&] { return new_bytes(c.z.ws_backward_bytes, *Q); });
    rc = sla_backward_typed(c.p, Q->data_ptr(), K->data_ptr(), V->data_ptr(), W->data_ptr(),
                            (const int8_t*)Mc->data_ptr(), luts->data_ptr(), saved->data_ptr(), dO->data_ptr(),
                            dQ.ptr(), dK.ptr(), dV.ptr(), dW.ptr(), w16 ? SLA_BF16 : SLA_F32, ws.ptr(), ws.size(), st);
  }
  if (rc != SLA_OK) return PyLong_FromLong(rc);
  return pack({dQ.object(), dK.object(), dV.object(), dW.object()});
  END_HANDLE_TH_ERRORS
}

// ---- softmax attention

bool stream_of(const at::Tensor& t, void** out) {   // the current stream of the tensor's device
  PyObject* dev = PyLong_FromLong(t.get_device());
  if (!dev) return false;
  PyObject* st = PyObject_CallFunctionObjArgs(g_stream, dev, nullptr);
  Py_DECREF(dev);
  if (!st) return false;
  *out = PyLong_AsVoidPtr(st);
  Py_DECREF(st);
  return !PyErr_Occurred();
}

struct AttnCall {
  const sla_attn_params* p;
  uint64_t fwd, bwd;
  at::ScalarType dt, tt;
  bool token;   // [B, N, H, d] tensors
  at::Device dev = at::kCPU;

  bool open(const sla_attn_params* params, bool token_major, const at::Tensor* Q) {
    p = params;
    if (!p || !Q || !Q->is_cuda() || sla_attn_sizes(p, &fwd, &bwd) != SLA_OK) return false;
    dt = p->dtype == SLA_F32 ? at::kFloat : at::kBFloat16;
    tt = p->table_dtype == SLA_F32 ? at::kFloat : at::kBFloat16;
    token = token_major;
    dev = Q->device();
    return true;
  }
  bool here(const at::Tensor* t, at::ScalarType type) const { return t && t->device() == dev && t->scalar_type() == type; }
  bool rows(const at::Tensor* t, int heads, int n, sla_tensor* out) const {
    if (!here(t, dt) || t->dim() != 4) return false;
    const auto s = t->sizes(), st = t->strides();
    const int hx = token ? 2 : 1, nx = token ? 1 : 2;
    if (s[0] != p->B || s[hx] != heads || s[nx] != n || s[3] != p->d || st[3] != 1) return false;
    *out = sla_tensor{t->data_ptr(), st[0], st[hx], st[nx]};
    return true;
  }
  bool prefix(const at::Tensor* t, sla_tensor* out) const {
    if (!here(t, dt) || t->dim() != 3) return false;
    const auto s = t->sizes(), st = t->strides();
    const int hx = token ? 1 : 0, nx = token ? 0 : 1;
    if (s[hx] != p->Hkv || s[nx] != p->Np || s[2] != p->d || st[2] != 1) return false;
    *out = sla_tensor{t->data_ptr(), 0, st[hx], st[nx]};
    return true;
  }
  bool flat(const at::Tensor* t, at::IntArrayRef shape, at::ScalarType type) const {
    return here(t, type) && t->sizes() == shape && t->is_contiguous();
  }
  // lengths [B] and the table: absent (None) or as stated
  bool lengths(const at::Tensor* t, const int32_t** out) const {
    *out = nullptr;
    if (!t) return true;
    if (!flat(t, {p->B}, at::kInt)) return false;
    *out = t->const_data_ptr<int32_t>();
    return true;
  }
  bool table(const at::Tensor* t, const void** out) const {
    *out = nullptr;
    if (!t) return p->buckets.n_buckets == 0;
    if (!flat(t, {p->buckets.n_buckets, p->H}, tt)) return false;
    *out = t->const_data_ptr();
    return true;
  }
  at::Tensor fresh(const at::Tensor& like, int heads, int n, sla_tensor* out) const {
    const int64_t B = p->B, h = heads, m = n, d = p->d;
    at::Tensor t = at::empty(token ? at::IntArrayRef{B, m, h, d} : at::IntArrayRef{B, h, m, d},
                             like.options().requires_grad(false));
    rows(&t, heads, n, out);
    return t;
  }
};

// The whole of dense_attention and cached_attention for plain tensors: parameters, checks, forward call and, where a
// gradient is wanted, the node of the graph, in one call from Python and none in the backward pass.
struct Attend {   // what a call is given beside its tensors
  const sla_buckets* buckets;
  bool causal, token, cached;
  double scale;   // 0: 1 / sqrt(d)
};

// an input of forward-mode differentiation, which the kernels would take for a constant
bool tangent(const at::Tensor& t) { return t._fw_grad(0).defined(); }

const at::Tensor* defined(const at::Tensor& t) { return t.defined() ? &t : nullptr; }

bool attend_params(const Attend& a, const at::Tensor& Q, const at::Tensor& K, const at::Tensor* Kp, const at::Tensor* table,
                   sla_attn_params* p) {
  if (Q.dim() != 4 || K.dim() != 4 || (table != nullptr) != (a.buckets != nullptr) || (Kp && Kp->dim() != 3)) return false;
  const int hx = a.token ? 2 : 1, nx = a.token ? 1 : 2;
  const auto q = Q.sizes(), k = K.sizes();
  for (int64_t x : {q[0], q[1], q[2], q[3], k[1], k[2]})
    if (x > 0x7fffffff) return false;
  auto code = [](at::ScalarType t) { return t == at::kFloat ? (int)SLA_F32 : t == at::kBFloat16 ? (int)SLA_BF16 : -1; };
  memset(p, 0, sizeof(*p));
  p->B = (int)q[0];
  p->H = (int)q[hx];
  p->Hkv = (int)k[hx];
  p->Nq = (int)q[nx];
  p->Nk = (int)k[nx];
  p->Np = Kp ? (int)Kp->size(a.token ? 0 : 1) : 0;
  p->d = (int)q[3];
  p->dtype = code(Q.scalar_type());
  p->causal = a.causal;
  p->q_pos = a.cached ? -p->Nq : p->Nk - p->Nq;
  p->q_from_end = a.cached;
  p->table_dtype = table ? code(table->scalar_type()) : (int)SLA_F32;
  p->scale = (float)(a.scale != 0.0 ? a.scale : 1.0 / std::sqrt((double)p->d));
  if (a.buckets) p->buckets = *a.buckets;
  return true;
}

// the forward call; false where anything does not fit
bool attend_forward(const sla_attn_params& p, bool token, const at::Tensor& Q, const at::Tensor& K, const at::Tensor& V,
                    const at::Tensor* Kp, const at::Tensor* Vp, const at::Tensor* table, const at::Tensor* q_len,
                    const at::Tensor* k_len, void* st, at::Tensor* O, at::Tensor* L) {
  AttnCall c;
  sla_tensor q, k, v, kp, vp, o;
  const void* tb;
  const int32_t *ql, *kl;
  if (!c.open(&p, token, &Q) || !c.rows(&Q, p.H, p.Nq, &q) || !c.rows(&K, p.Hkv, p.Nk, &k) || !c.rows(&V, p.Hkv, p.Nk, &v) ||
      !c.table(table, &tb) || !c.lengths(q_len, &ql) || !c.lengths(k_len, &kl))
    return false;
  if (p.Np && (!c.prefix(Kp, &kp) || !c.prefix(Vp, &vp))) return false;
  const c10::DeviceGuard guard(c.dev);
  *O = c.fresh(Q, p.H, p.Nq, &o);
  if (L) *L = at::empty({p.B, p.H, p.Nq}, Q.options().dtype(at::kFloat).requires_grad(false));
  at::Tensor ws;
  if (c.fwd) ws = new_bytes(c.fwd, Q);
  return sla_attn_forward(&p, &q, &k, &v, p.Np ? &kp : nullptr, p.Np ? &vp : nullptr, tb, ql, kl, &o,
                          L ? L->data_ptr<float>() : nullptr, c.fwd ? ws.data_ptr() : nullptr, c.fwd, st) == SLA_OK;
}

struct DenseAttention : torch::autograd::Function<DenseAttention> {
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& Q, const at::Tensor& K,
                                                const at::Tensor& V, const std::optional<at::Tensor>& table,
                                                const at::Tensor* q_len, const at::Tensor* k_len, const sla_attn_params* p,
                                                bool token, const at::Tensor* O, const at::Tensor* L) {   // (the call is made already)
    const at::Tensor none;
    ctx->save_for_backward({Q, K, V, table ? *table : none, *O, *L, q_len ? *q_len : none, k_len ? *k_len : none});
    ctx->saved_data["p"] = std::string(reinterpret_cast<const char*>(p), sizeof(*p));
    ctx->saved_data["token"] = token;
    return {*O};
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    const auto s = ctx->get_saved_variables();
    const at::Tensor &Q = s[0], &K = s[1], &V = s[2], &table = s[3], &O = s[4], &L = s[5];
    sla_attn_params p;
    const std::string bytes = ctx->saved_data["p"].toStringRef();
    memcpy(&p, bytes.data(), sizeof(p));
    at::Tensor dO = grads[0], dQ, dK, dV, dT;
    {
      const at::NoGradGuard none;
      AttnCall c;
      const bool opened = c.open(&p, ctx->saved_data["token"].toBool(), &Q);
      sla_tensor q, k, v, o, go, gq, gk, gv;
      const void* tb;
      const int32_t *ql, *kl;
      auto whole = [](const sla_tensor& t, int64_t esz) {   // (what the library's own check of dO would refuse)
        return (reinterpret_cast<uintptr_t>(t.data) | (t.stride_b * esz) | (t.stride_h * esz) | (t.stride_n * esz)) % 16 == 0 &&
               t.stride_n * esz <= 1 << 24;
      };
      TORCH_CHECK(!tangent(dO), "dense_attention's backward pass has no forward-mode derivative");
      const int64_t esz = dO.element_size();
      if (!c.rows(&dO, p.H, p.Nq, &go) || !whole(go, esz) || go.stride_n < p.d) {
        dO = dO.clone(at::MemoryFormat::Contiguous);   // (contiguous() would hand back a tensor at an odd address)
        TORCH_CHECK(c.rows(&dO, p.H, p.Nq, &go), "dense_attention: the output's gradient has another type or shape");
      }
      TORCH_CHECK(opened && c.rows(&Q, p.H, p.Nq, &q) && c.rows(&K, p.Hkv, p.Nk, &k) && c.rows(&V, p.Hkv, p.Nk, &v) &&
                      c.rows(&O, p.H, p.Nq, &o) && c.flat(&L, {p.B, p.H, p.Nq}, at::kFloat) && c.table(defined(table), &tb) &&
                      c.lengths(defined(s[6]), &ql) && c.lengths(defined(s[7]), &kl),
                  "dense_attention: the saved tensors have changed");
      const PyGILState_STATE gil = PyGILState_Ensure();
      void* st = nullptr;
      const bool have = stream_of(Q, &st);
      if (!have) PyErr_Clear();
      PyGILState_Release(gil);
      TORCH_CHECK(have, "no current stream");
      const c10::DeviceGuard guard(c.dev);
      dQ = c.fresh(Q, p.H, p.Nq, &gq);
      dK = c.fresh(Q, p.Hkv, p.Nk, &gk);
      dV = c.fresh(Q, p.Hkv, p.Nk, &gv);
      if (tb) dT = at::empty({p.buckets.n_buckets, p.H}, Q.options().dtype(c.tt).requires_grad(false));
      const at::Tensor ws = new_bytes(c.bwd, Q);
      const int rc = sla_attn_backward(&p, &q, &k, &v, &o, &go, L.data_ptr<float>(), tb, ql, kl, &gq, &gk, &gv,
                                       tb ? dT.data_ptr() : nullptr, ws.data_ptr(), (size_t)ws.numel(), st);
      TORCH_CHECK(rc == SLA_OK, "sla_attn_backward failed: ", sla_strerror(rc), " (code ", rc, ")");
    }
    if (c10::GradMode::is_enabled()) {   // a graph of the gradients: differentiating them raises
      torch::autograd::variable_list in;
      for (at::Tensor* t : {&dQ, &dK, &dV, &dT})
        if (t->defined()) in.push_back(t->requires_grad_(true));
      const auto out = (*std::make_shared<torch::autograd::DelayedError>(
          "dense_attention: its gradients cannot be differentiated", (int64_t)in.size()))(std::move(in));
      dQ = out[0], dK = out[1], dV = out[2];
      if (out.size() > 3) dT = out[3];
    }
    const at::Tensor no;
    return {dQ, dK, dV, dT, no, no, no, no, no, no};
  }
};

// attend(Q, K, V, prefix K, prefix V, table, q_len, k_len, address of the buckets or 0, causal, scale or None, token_major,
//        cached) -> O, or None where the Python code has to lay out, check or refuse
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 13 || at::tracer::impl::is_dispatch_enabled()) Py_RETURN_NONE;   // (a traced call is refused there)
  const at::Tensor* t[8];
  for (int i = 0; i < 8; ++i) {
    t[i] = a[i] == Py_None ? nullptr : plain(a[i]);
    if (!t[i] && (a[i] != Py_None || i < 3)) Py_RETURN_NONE;
    if (t[i] && tangent(*t[i])) Py_RETURN_NONE;   // (refused there)
  }
  const at::Tensor &Q = *t[0], &K = *t[1], &V = *t[2];
  if (!Q.is_cuda() || (t[3] != nullptr) != (t[4] != nullptr)) Py_RETURN_NONE;
  Attend at_;
  at_.buckets = static_cast<const sla_buckets*>(PyLong_AsVoidPtr(a[8]));
  at_.causal = PyObject_IsTrue(a[9]) == 1;
  at_.scale = a[10] == Py_None ? 0.0 : PyFloat_AsDouble(a[10]);
  at_.token = PyObject_IsTrue(a[11]) == 1;
  at_.cached = a[12] == Py_True;
  if (PyErr_Occurred()) return nullptr;
  if (a[10] != Py_None && !(at_.scale > 0.0)) Py_RETURN_NONE;
  sla_attn_params p;
  if (!attend_params(at_, Q, K, t[3], t[5], &p)) Py_RETURN_NONE;
  void* st;
  if (!stream_of(Q, &st)) return nullptr;
  at::Tensor O;
  bool grad = false;
  if (!at_.cached && c10::GradMode::is_enabled())
    for (int i : {0, 1, 2, 5}) grad = grad || (t[i] && t[i]->requires_grad());
  at::Tensor L;
  {
    const at::NoGradGuard no;
    NoGil free;
    if (!attend_forward(p, at_.token, Q, K, V, t[3], t[4], t[5], t[6], t[7], st, &O, grad ? &L : nullptr)) O = at::Tensor();
  }
  if (!O.defined()) Py_RETURN_NONE;
  if (grad)
    O = DenseAttention::apply(Q, K, V, t[5] ? std::optional<at::Tensor>(*t[5]) : std::nullopt, t[6], t[7],
                              static_cast<const sla_attn_params*>(&p), at_.token, static_cast<const at::Tensor*>(&O),
                              static_cast<const at::Tensor*>(&L))[0];
  return THPVariable_Wrap(O);
  END_HANDLE_TH_ERRORS
}

PyMethodDef g_methods[] = {
    {"build_mask", (PyCFunction)(void (*)(void))build_mask, METH_FASTCALL, nullptr},
    {"forward", (PyCFunction)(void (*)(void))forward, METH_FASTCALL, nullptr},
    {"mask_forward", (PyCFunction)(void (*)(void))mask_forward, METH_FASTCALL, nullptr},
    {"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_sla_host", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sla_host(void) {
  PyObject* tc = PyImport_ImportModule("torch._C");
  if (!tc) return nullptr;
  g_device = PyObject_GetAttrString(tc, "_cuda_getDevice");
  g_stream = g_device ? PyObject_GetAttrString(tc, "_cuda_getCurrentRawStream") : nullptr;
  Py_DECREF(tc);
  return g_stream ? PyModule_Create(&g_module) : nullptr;
}
