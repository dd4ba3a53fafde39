// The block operators under autograd in native code: what block.py's functions do, for the calls that need nothing of Python.
//
// A small operator's pass is host time (attention of four sequences of 16 tokens, forward and backward: 70 us through the Python
// functions).  Here a forward pass is one call from Python and a backward pass none.  Whatever these functions do not take -- what
// sk_torch.cpp's leave out, tensors that have to be copied first, arguments that are to be refused -- gives None, and block.py goes on from there.
#include "sk_torch_block.h"

#include <functional>

#include "../../include/sk_block.h"

namespace sk_torch {
namespace {

bool floating(const Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
bool same(const Tensor& x, const Tensor& t) { return t.scalar_type() == x.scalar_type() && t.device() == x.device() && no_tangent(t); }
bool dense(const Tensor& t) { return t.is_contiguous() && aligned(t); }
Tensor made_dense(const Tensor& t) { return dense(t) ? t : t.clone(at::MemoryFormat::Contiguous); }
bool integers(const Tensor& t, const at::Device& device) { return (t.scalar_type() == at::kInt || t.scalar_type() == at::kLong) && t.device() == device; }

// Strides that the library takes in place (block.py's _strided)
bool strided(const Tensor& t, int64_t token) {
  if (!aligned(t) || (t.stride(-1) != 1 && t.size(-1) != 1)) return false;
  const int64_t unit = 16 / (int64_t)t.element_size();
  for (int64_t d = 0; d < t.dim() - 1; ++d)
    if (t.size(d) > 1 && (t.stride(d) % unit != 0 || t.stride(d) < 0 || t.stride(d) >= (d == token ? (int64_t)1 << 22 : (int64_t)1 << 40))) return false;
  return true;
}

// Tokens that do not overlap in memory (block.py's _apart)
bool apart(const Tensor& t) { return t.size(1) <= 1 || t.stride(1) >= t.size(3); }

// Results that depend on something, with no rule for how (block.py's _Underivable).
struct Underivable : torch::autograd::Function<Underivable> {
  static variable_list forward(AutogradContext*, const Tensor&, const std::function<variable_list()>& compute) { return compute(); }
  static variable_list backward(AutogradContext*, variable_list) {
    TORCH_CHECK(false, "libsk: a gradient of a gradient was asked for; these operators are differentiated once, not twice");
  }
};
// A backward pass's gradients; where a graph of it is made they refuse to be differentiated.
template <typename Compute>
variable_list once(const Compute& compute) {
  if (!at::GradMode::is_enabled()) return compute();
  return Underivable::apply(at::empty({0}, at::kFloat).set_requires_grad(true), std::function<variable_list()>(compute));
}

// (a function's arguments are tensors that are there, or options)
std::optional<Tensor> given(const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; }

bool number(PyObject* o, double& v) {
  if (PyFloat_Check(o)) { v = PyFloat_AS_DOUBLE(o); return true; }
  if (!PyLong_Check(o)) return false;
  v = PyLong_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}
bool word(PyObject* o, uint64_t& v) {
  if (!PyLong_Check(o)) return false;
  v = PyLong_AsUnsignedLongLong(o);
  if (v == (uint64_t)-1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}

// ---- attention ----

struct AttentionCall {
  sk_attention_shape s{};
  AttentionCall(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& ql, const Tensor& kl, bool causal, double scale) {
    s.batch = q.size(0); s.q_len = q.size(1); s.k_len = k.size(1);
    s.heads = (int32_t)q.size(2); s.kv_heads = (int32_t)k.size(2); s.head_dim = (int32_t)q.size(3);
    s.causal = causal; s.scale = (float)scale; s.dtype = dtype_of(q);
    for (int i = 0; i < 3; ++i) { s.q_strides[i] = q.stride(i); s.k_strides[i] = k.stride(i); s.v_strides[i] = v.stride(i); }
    s.q_lengths = ql.defined() ? ql.data_ptr<int32_t>() : nullptr;
    s.k_lengths = kl.defined() ? kl.data_ptr<int32_t>() : nullptr;
  }
};

Tensor attention_forward(const Tensor& q, const Tensor& k, const Tensor& v, const AttentionCall& c, Tensor* lse, Tensor* rest) {
  const c10::DeviceGuard guard(q.device());
  Tensor o = at::empty(q.sizes(), q.options());
  if (lse) *lse = at::empty({q.size(0), q.size(2), q.size(1)}, q.options().dtype(at::kFloat));
  if (rest && c.s.dtype == SK_BF16) *rest = at::empty(q.sizes(), q.options());
  void* const stream = stream_of(q.device());
  const size_t need = sk_attention_workspace_bytes(&c.s, 0);
  Workspaces& w = workspaces();
  sk_status st;
  {
    const std::lock_guard<std::mutex> lock(w.mutex);
    const Tensor ws = w.get(q.device(), stream, need);
    st = sk_attention_fwd(&c.s, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse ? lse->data_ptr<float>() : nullptr,
                          rest && rest->defined() ? rest->data_ptr() : nullptr, ws.data_ptr(), (size_t)ws.numel(), stream);
  }
  check(st);
  return o;
}

struct Attention : torch::autograd::Function<Attention> {
  static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const std::optional<Tensor>& ql, const std::optional<Tensor>& kl, bool causal,
                        double scale) {
    Tensor lse, rest;
    const Tensor n = ql.value_or(Tensor()), m = kl.value_or(Tensor());
    const Tensor o = attention_forward(q, k, v, AttentionCall(q, k, v, n, m, causal, scale), &lse, &rest);
    ctx->save_for_backward({q, k, v, o, lse, rest, n, m});
    ctx->saved_data["causal"] = causal;
    ctx->saved_data["scale"] = scale;
    return o;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list out = once([&] { return gradients(ctx, grads); });
    return {out[0], out[1], out[2], Tensor(), Tensor(), Tensor(), Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &q = saved[0], &k = saved[1], &v = saved[2];
    const c10::DeviceGuard guard(q.device());
    const Tensor dO = made_dense(grads[0]);
    const AttentionCall c(q, k, v, saved[6], saved[7], ctx->saved_data["causal"].toBool(), ctx->saved_data["scale"].toDouble());
    const Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(k.sizes(), q.options()), dv = at::empty(k.sizes(), q.options());
    void* const stream = stream_of(q.device());
    const size_t need = sk_attention_workspace_bytes(&c.s, 1);
    Workspaces& w = workspaces();
    sk_status st;
    {
      const std::lock_guard<std::mutex> lock(w.mutex);
      const Tensor ws = w.get(q.device(), stream, need);
      st = sk_attention_bwd(&c.s, q.data_ptr(), k.data_ptr(), v.data_ptr(), saved[3].data_ptr(), saved[4].data_ptr<float>(), saved[5].defined() ? saved[5].data_ptr() : nullptr, dO.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                            dv.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), stream);
    }
    check(st);
    return {dq, dk, dv};
  }
};

// ---- norms with the rotation ----

struct NormRopeCall {
  sk_norm_rope_shape s{};
  NormRopeCall(const Tensor& q, const Tensor& k, const Tensor& cos, const Tensor& positions, double eps, bool interleaved) {
    s.tokens = q.size(0); s.heads = (int32_t)q.size(1); s.kv_heads = (int32_t)k.size(1); s.head_dim = (int32_t)q.size(2);
    s.rotary_dim = (int32_t)(2 * cos.size(1)); s.table_rows = cos.size(0);
    s.interleaved = interleaved; s.position_bytes = (int32_t)positions.element_size(); s.eps = (float)eps; s.dtype = dtype_of(q);
    for (int i = 0; i < 2; ++i) { s.q_strides[i] = q.stride(i); s.k_strides[i] = k.stride(i); }
    s.q_out_strides[0] = q.size(1) * q.size(2); s.k_out_strides[0] = k.size(1) * k.size(2);
    s.q_out_strides[1] = s.k_out_strides[1] = q.size(2);
  }
};

variable_list norm_rope_forward(const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, const Tensor& cos, const Tensor& sin, const Tensor& positions,
                                const NormRopeCall& c) {
  const c10::DeviceGuard guard(q.device());
  Tensor qo = at::empty(q.sizes(), q.options()), ko = at::empty(k.sizes(), q.options());
  check(sk_norm_rope_fwd(&c.s, q.data_ptr(), k.data_ptr(), wq.data_ptr(), wk.data_ptr(), cos.data_ptr<float>(), sin.data_ptr<float>(), positions.data_ptr(), qo.data_ptr(),
                         ko.data_ptr(), stream_of(q.device())));
  return {qo, ko};
}

struct NormRope : torch::autograd::Function<NormRope> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, const Tensor& cos, const Tensor& sin,
                               const Tensor& positions, double eps, bool interleaved) {
    ctx->save_for_backward({q, k, wq, wk, cos, sin, positions});
    ctx->saved_data["eps"] = eps;
    ctx->saved_data["interleaved"] = interleaved;
    return norm_rope_forward(q, k, wq, wk, cos, sin, positions, NormRopeCall(q, k, cos, positions, eps, interleaved));
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list out = once([&] { return gradients(ctx, grads); });
    return {out[0], out[1], out[2], out[3], Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads) {
    const variable_list t = ctx->get_saved_variables();
    const Tensor &q = t[0], &k = t[1], &wq = t[2], &wk = t[3];
    const c10::DeviceGuard guard(q.device());
    const NormRopeCall c(q, k, t[4], t[6], ctx->saved_data["eps"].toDouble(), ctx->saved_data["interleaved"].toBool());
    const Tensor dqo = made_dense(grads[0]), dko = made_dense(grads[1]);   // (zeros for a result that nobody used)
    const Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(k.sizes(), q.options()), dwq = at::empty(wq.sizes(), q.options()), dwk = at::empty(wk.sizes(), q.options());
    void* const stream = stream_of(q.device());
    const size_t need = sk_norm_rope_workspace_bytes(&c.s);
    Workspaces& w = workspaces();
    sk_status st;
    {
      const std::lock_guard<std::mutex> lock(w.mutex);
      const Tensor ws = w.get(q.device(), stream, need);
      st = sk_norm_rope_bwd(&c.s, q.data_ptr(), k.data_ptr(), wq.data_ptr(), wk.data_ptr(), t[4].data_ptr<float>(), t[5].data_ptr<float>(), t[6].data_ptr(), dqo.data_ptr(),
                            dko.data_ptr(), dq.data_ptr(), dk.data_ptr(), dwq.data_ptr(), dwk.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), stream);
    }
    check(st);
    return {dq, dk, dwq, dwk};
  }
};

// ---- embedding ----

Tensor embedding_forward(const Tensor& ids, const Tensor& table, double scale) {
  const c10::DeviceGuard guard(table.device());
  std::vector<int64_t> shape = ids.sizes().vec();
  shape.push_back(table.size(1));
  Tensor y = at::empty(shape, table.options());
  check(sk_embedding_fwd(ids.data_ptr(), (int32_t)ids.element_size(), table.data_ptr(), y.data_ptr(), ids.numel(), table.size(0), table.size(1), (float)scale, dtype_of(table),
                         stream_of(table.device())));
  return y;
}

struct Embedding : torch::autograd::Function<Embedding> {
  static Tensor forward(AutogradContext* ctx, const Tensor& ids, const Tensor& table, double scale) {
    ctx->save_for_backward({ids});
    ctx->saved_data["rows"] = table.size(0);
    ctx->saved_data["scale"] = scale;
    return embedding_forward(ids, table, scale);
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    return {Tensor(), once([&] { return gradients(ctx, grads); })[0], Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads) {
    const Tensor ids = ctx->get_saved_variables()[0];
    const c10::DeviceGuard guard(ids.device());
    const Tensor dy = made_dense(grads[0]);
    const int64_t rows = ctx->saved_data["rows"].toInt(), width = dy.size(-1);
    const Tensor dtable = at::empty({rows, width}, dy.options());
    void* const stream = stream_of(ids.device());
    const size_t need = sk_embedding_workspace_bytes(ids.numel(), rows, width, dtype_of(dy));
    Workspaces& w = workspaces();
    sk_status st;
    {
      const std::lock_guard<std::mutex> lock(w.mutex);
      const Tensor ws = w.get(ids.device(), stream, need);
      st = sk_embedding_bwd(ids.data_ptr(), (int32_t)ids.element_size(), dy.data_ptr(), dtable.data_ptr(), ids.numel(), rows, width, (float)ctx->saved_data["scale"].toDouble(),
                            dtype_of(dy), ws.data_ptr(), (size_t)ws.numel(), stream);
    }
    check(st);
    return {dtable};
  }
};

// ---- dropout ----

Tensor dropout_forward(const Tensor& x, const Tensor& residual, double p, int64_t seed, int64_t offset) {
  const c10::DeviceGuard guard(x.device());
  Tensor y = at::empty(x.sizes(), x.options());
  check(sk_dropout(x.data_ptr(), residual.defined() ? residual.data_ptr() : nullptr, y.data_ptr(), x.numel(), (float)p, (uint64_t)seed, (uint64_t)offset, dtype_of(x),
                   stream_of(x.device())));
  return y;
}

struct Dropout : torch::autograd::Function<Dropout> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const std::optional<Tensor>& residual, double p, int64_t seed, int64_t offset) {
    ctx->saved_data["p"] = p;
    ctx->saved_data["seed"] = seed;
    ctx->saved_data["offset"] = offset;
    ctx->saved_data["residual"] = residual.has_value() && residual->requires_grad();
    return dropout_forward(x, residual.value_or(Tensor()), p, seed, offset);
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const Tensor dy = made_dense(grads[0]);
    const double p = ctx->saved_data["p"].toDouble();
    const int64_t seed = ctx->saved_data["seed"].toInt(), offset = ctx->saved_data["offset"].toInt();
    Tensor dx;
    if (ctx->needs_input_grad(0))   // (linear: its own gradient's gradient)
      dx = at::GradMode::is_enabled() && dy.requires_grad() ? Dropout::apply(dy, std::nullopt, p, seed, offset) : dropout_forward(dy, Tensor(), p, seed, offset);
    return {dx, ctx->saved_data["residual"].toBool() ? grads[0] : Tensor(), Tensor(), Tensor(), Tensor()};
  }
};

}  // namespace

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !PyBool_Check(a[5]) || !unwatched()) Py_RETURN_NONE;
  const Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]);
  if (!q || !k || !v || !floating(*q) || !no_tangent(*q) || !same(*q, *k) || !same(*q, *v)) Py_RETURN_NONE;
  if (q->dim() != 4 || k->dim() != 4 || v->dim() != 4 || q->numel() == 0 || k->numel() == 0 || k->sizes() != v->sizes() || q->size(0) != k->size(0) || q->size(3) != k->size(3))
    Py_RETURN_NONE;
  if (q->size(2) > INT32_MAX || q->size(3) > INT32_MAX || !strided(*q, 1) || !strided(*k, 1) || !strided(*v, 1) || !apart(*k) || !apart(*v)) Py_RETURN_NONE;
  Tensor lengths[2];
  for (int i = 0; i < 2; ++i) {
    if (a[3 + i] == Py_None) continue;
    const Tensor* t = plain(a[3 + i]);
    if (!t || t->scalar_type() != at::kInt || t->device() != q->device() || t->dim() != 1 || t->size(0) != q->size(0) || !t->is_contiguous()) Py_RETURN_NONE;
    lengths[i] = *t;
  }
  double scale = 1.0 / std::sqrt((double)q->size(3));
  if (a[6] != Py_None && !number(a[6], scale)) Py_RETURN_NONE;
  const bool causal = a[5] == Py_True;
  const AttentionCall c(*q, *k, *v, lengths[0], lengths[1], causal, scale);
  if (sk_attention_workspace_bytes(&c.s, 0) == (size_t)-1) Py_RETURN_NONE;
  Tensor o;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && (q->requires_grad() || k->requires_grad() || v->requires_grad()))
      o = Attention::apply(*q, *k, *v, given(lengths[0]), given(lengths[1]), causal, scale);
    else
      o = attention_forward(*q, *k, *v, c, nullptr, nullptr);
  }
  return THPVariable_Wrap(std::move(o));
  END_HANDLE_TH_ERRORS
}

PyObject* head_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  double eps;
  if (n != 9 || !PyBool_Check(a[8]) || !number(a[7], eps) || !unwatched()) Py_RETURN_NONE;
  const Tensor* t[7];
  for (int i = 0; i < 7; ++i)
    if (!(t[i] = plain(a[i])) || !no_tangent(*t[i])) Py_RETURN_NONE;
  const Tensor &q = *t[0], &k = *t[1], &wq = *t[2], &wk = *t[3], &cos = *t[4], &sin = *t[5], &positions = *t[6];
  if (!floating(q) || !same(q, k) || !same(q, wq) || !same(q, wk) || q.dim() != 3 || k.dim() != 3 || q.numel() == 0 || k.numel() == 0) Py_RETURN_NONE;
  const int64_t D = q.size(2);
  if (k.size(0) != q.size(0) || k.size(2) != D || wq.dim() != 1 || wk.dim() != 1 || wq.size(0) != D || wk.size(0) != D || D > INT32_MAX || q.size(1) > INT32_MAX ||
      k.size(1) > INT32_MAX || !dense(wq) || !dense(wk) || !strided(q, -1) || !strided(k, -1))
    Py_RETURN_NONE;
  if (cos.scalar_type() != at::kFloat || sin.scalar_type() != at::kFloat || cos.device() != q.device() || sin.device() != q.device() || cos.dim() != 2 || cos.numel() == 0 ||
      cos.sizes() != sin.sizes() || 2 * cos.size(1) > D || !dense(cos) || !dense(sin) || !integers(positions, q.device()) || positions.dim() != 1 ||
      positions.size(0) != q.size(0) || !dense(positions) || (at::GradMode::is_enabled() && (cos.requires_grad() || sin.requires_grad())))
    Py_RETURN_NONE;
  const bool interleaved = a[8] == Py_True;
  const NormRopeCall c(q, k, cos, positions, eps, interleaved);
  if (sk_norm_rope_workspace_bytes(&c.s) == (size_t)-1) Py_RETURN_NONE;
  variable_list out;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && (q.requires_grad() || k.requires_grad() || wq.requires_grad() || wk.requires_grad()))
      out = NormRope::apply(q, k, wq, wk, cos, sin, positions, eps, interleaved);
    else
      out = norm_rope_forward(q, k, wq, wk, cos, sin, positions, c);
  }
  PyObject* const pair = PyTuple_New(2);
  if (pair == nullptr) return nullptr;
  for (int i = 0; i < 2; ++i) {
    PyObject* const o = THPVariable_Wrap(std::move(out[i]));
    if (o == nullptr) { Py_DECREF(pair); return nullptr; }
    PyTuple_SET_ITEM(pair, i, o);
  }
  return pair;
  END_HANDLE_TH_ERRORS
}

PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  double scale;
  if (n != 3 || !number(a[2], scale) || !unwatched()) Py_RETURN_NONE;
  const Tensor *ids = plain(a[0]), *table = plain(a[1]);
  if (!ids || !table || !floating(*table) || !no_tangent(*table) || table->dim() != 2 || table->numel() == 0 || !dense(*table) || !integers(*ids, table->device()) ||
      ids->numel() == 0 || !dense(*ids))
    Py_RETURN_NONE;
  if (!std::isfinite(scale) || sk_embedding_workspace_bytes(ids->numel(), table->size(0), table->size(1), dtype_of(*table)) == (size_t)-1) Py_RETURN_NONE;
  Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && table->requires_grad()) y = Embedding::apply(*ids, *table, scale);
    else y = embedding_forward(*ids, *table, scale);
  }
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  double p;
  uint64_t seed, offset;
  if (n != 5 || !number(a[1], p) || !(p >= 0.0 && p <= 1.0) || !word(a[2], seed) || !word(a[3], offset) || !unwatched()) Py_RETURN_NONE;
  const Tensor* x = plain(a[0]);
  if (!x || !floating(*x) || !no_tangent(*x) || x->numel() == 0 || !dense(*x)) Py_RETURN_NONE;
  Tensor residual;
  if (a[4] != Py_None) {
    const Tensor* r = plain(a[4]);
    if (!r || !same(*x, *r) || r->sizes() != x->sizes() || !dense(*r)) Py_RETURN_NONE;
    residual = *r;
  }
  Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && (x->requires_grad() || (residual.defined() && residual.requires_grad())))
      y = Dropout::apply(*x, given(residual), p, (int64_t)seed, (int64_t)offset);
    else
      y = dropout_forward(*x, residual, p, (int64_t)seed, (int64_t)offset);
  }
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

}  // namespace sk_torch
