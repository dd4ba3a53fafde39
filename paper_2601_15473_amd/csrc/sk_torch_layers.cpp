// Layer norm, dense layers and the distillation loss under autograd in native code: as sk_torch_block.cpp, and like it giving None for whatever block.py's
// functions have to look at.
#include "sk_torch_block.h"

#include "../../include/sk_block.h"

namespace sk_torch {
namespace {

// Which inputs' gradients a backward pass forms: those that had one at the forward pass; where a graph of it is made, every one (a function's results are all there).
// (With them, in one number: what else there was, and a dense layer's activation.)
enum Wanted : int64_t { WANT_X = 1, WANT_WEIGHT = 2, WANT_BIAS = 4, WANT_RESIDUAL = 8, HAS_BIAS = 16, HAS_REST = 32, ACTIVATION = 256 };
bool wants(const std::optional<Tensor>& t) { return t.has_value() && t->requires_grad(); }
int64_t wanted(const Tensor& x, const std::optional<Tensor>& weight, const std::optional<Tensor>& bias, const std::optional<Tensor>& residual) {
  return (x.requires_grad() ? WANT_X : 0) | (wants(weight) ? WANT_WEIGHT : 0) | (wants(bias) ? WANT_BIAS : 0) | (wants(residual) ? WANT_RESIDUAL : 0) | (bias.has_value() ? HAS_BIAS : 0);
}

// Rows that the library takes in place: of a dense tensor, or of a matrix with a stride between them.
bool rows_in_place(const Tensor& t, int64_t least, int64_t most) {
  if (dense(t)) return true;
  return t.dim() == 2 && t.stride(1) == 1 && aligned(t) && t.stride(0) * (int64_t)t.element_size() % 16 == 0 && t.stride(0) >= least && t.stride(0) <= most;
}
int64_t row_stride(const Tensor& t) { return t.is_contiguous() ? t.size(-1) : t.stride(0); }
void* data(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// What was saved, as the kernels take it: hooks may have laid it out differently.
Tensor saved_dense(const Tensor& t) { return t.defined() ? made_dense(t) : t; }
Tensor saved_rows(const Tensor& t, int64_t least, int64_t most) { return rows_in_place(t, least, most) ? t : made_dense(t); }

template <typename Call>
void with_workspace(const Tensor& t, size_t bytes, const Call& call) {
  void* const stream = stream_of(t.device());
  Workspaces& w = workspaces();
  sk_status st;
  {
    const std::lock_guard<std::mutex> lock(w.mutex);
    const Tensor ws = w.get(t.device(), stream, bytes);
    st = call(ws.data_ptr(), (size_t)ws.numel(), stream);
  }
  check(st);
}

// A tensor that is not there, or one of the type, device and shape of `like`'s last dimension
bool vector_like(PyObject* o, const Tensor& like, int64_t n, Tensor& out) {
  if (o == Py_None) return true;
  const Tensor* t = plain(o);
  if (!t || !same(like, *t) || t->dim() != 1 || t->size(0) != n || !dense(*t)) return false;
  out = *t;
  return true;
}

// ---- layer norm ----

sk_layer_norm_shape norm_shape(const Tensor& x, const Tensor& residual, double eps) {
  sk_layer_norm_shape s{};
  s.width = x.size(-1); s.rows = x.numel() / s.width;
  s.eps = (float)eps; s.dtype = dtype_of(x);
  s.x_stride = row_stride(x); s.residual_stride = residual.defined() ? row_stride(residual) : s.width;
  return s;
}

// What a sum's rounding left off stands behind the rows' statistics, from a boundary on: the values ahead of it.
int64_t rest_at(const sk_layer_norm_shape& s) { return (s.rows + 1) / 2 * 4; }

variable_list norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& residual, const sk_layer_norm_shape& s, Tensor* stats, bool rest) {
  const c10::DeviceGuard guard(x.device());
  Tensor y = at::empty(x.sizes(), x.options()), sum;
  if (residual.defined()) sum = at::empty(x.sizes(), x.options());
  if (stats) *stats = at::empty({rest ? rest_at(s) + s.rows * (s.width / 8) : s.rows * 2}, x.options().dtype(at::kFloat));
  float* const kept = stats ? stats->data_ptr<float>() : nullptr;
  check(sk_layer_norm_fwd(&s, x.data_ptr(), data(residual), data(weight), data(bias), y.data_ptr(), data(sum), rest ? kept + rest_at(s) : nullptr, kept, stream_of(x.device())));
  return residual.defined() ? variable_list{y, sum} : variable_list{y};
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
  static variable_list forward(AutogradContext* ctx, const Tensor& x, const std::optional<Tensor>& weight, const std::optional<Tensor>& bias, const std::optional<Tensor>& residual,
                               double eps) {
    const Tensor w = weight.value_or(Tensor()), r = residual.value_or(Tensor());
    Tensor stats;
    const bool rest = r.defined() && wants(weight) && x.scalar_type() == at::kBFloat16;
    const variable_list out = norm_forward(x, w, bias.value_or(Tensor()), r, norm_shape(x, r, eps), &stats, rest);
    ctx->save_for_backward({r.defined() ? out[1] : x, w, stats});
    ctx->saved_data["wanted"] = wanted(x, weight, bias, residual) | (rest ? HAS_REST : 0);
    ctx->set_materialize_grads(false);
    return out;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool all = at::GradMode::is_enabled();   // (off inside)
    const int64_t want = ctx->saved_data["wanted"].toInt();
    const variable_list out = once([&] { return gradients(ctx, grads, want, all); });
    return {want & WANT_X ? out[0] : Tensor(), want & WANT_WEIGHT ? out[1] : Tensor(), want & WANT_BIAS ? out[2] : Tensor(), want & WANT_RESIDUAL ? out[0] : Tensor(), Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads, int64_t want, bool all) {
    const variable_list saved = ctx->get_saved_variables();
    const c10::DeviceGuard guard(saved[0].device());
    const Tensor x = saved_rows(saved[0], 0, (int64_t)1 << 40), w = saved_dense(saved[1]), stats = saved_dense(saved[2]);
    const Tensor dy = grads[0].defined() ? made_dense(grads[0]) : at::zeros(x.sizes(), x.options());
    const Tensor ds = grads.size() > 1 && grads[1].defined() ? made_dense(grads[1]) : Tensor();
    const sk_layer_norm_shape s = norm_shape(x, Tensor(), 0.0);
    float* const kept = stats.data_ptr<float>();
    const Tensor none = all ? at::zeros({0}, x.options()) : Tensor();
    const Tensor dx = at::empty(x.sizes(), x.options());
    const Tensor dw = w.defined() && (all || (want & WANT_WEIGHT)) ? at::empty({s.width}, x.options()) : none;
    const Tensor db = (want & HAS_BIAS) && (all || (want & WANT_BIAS)) ? at::empty({s.width}, x.options()) : none;
    with_workspace(x, sk_layer_norm_workspace_bytes(&s), [&](void* ws, size_t n, void* stream) {
      return sk_layer_norm_bwd(&s, x.data_ptr(), want & HAS_REST ? kept + rest_at(s) : nullptr, data(w), kept, dy.data_ptr(), data(ds), dx.data_ptr(), data(dw), data(db), ws, n, stream);
    });
    return {dx, dw, db};
  }
};

// ---- dense layers ----

sk_dense_shape layer_shape(const Tensor& x, const Tensor& weight, const Tensor& residual, int64_t activation) {
  sk_dense_shape s{};
  s.in = weight.size(1); s.out = weight.size(0); s.tokens = x.numel() / s.in;
  s.activation = (int32_t)activation; s.dtype = dtype_of(x);
  s.x_stride = row_stride(x); s.residual_stride = residual.defined() ? row_stride(residual) : s.out;
  return s;
}

Tensor layer_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& residual, const sk_dense_shape& s, Tensor* z) {
  const c10::DeviceGuard guard(x.device());
  std::vector<int64_t> shape = x.sizes().vec();
  shape.back() = s.out;
  Tensor y = at::empty(shape, x.options());
  if (z && s.activation != SK_ACT_NONE) *z = at::empty({s.tokens, s.out}, x.options());
  with_workspace(x, sk_dense_workspace_bytes(&s, 0), [&](void* ws, size_t n, void* stream) {
    return sk_dense_fwd(&s, x.data_ptr(), weight.data_ptr(), data(bias), data(residual), y.data_ptr(), z ? data(*z) : nullptr, ws, n, stream);
  });
  return y;
}

struct Dense : torch::autograd::Function<Dense> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, const std::optional<Tensor>& bias, const std::optional<Tensor>& residual, int64_t activation) {
    const Tensor r = residual.value_or(Tensor());
    Tensor z;
    const Tensor y = layer_forward(x, weight, bias.value_or(Tensor()), r, layer_shape(x, weight, r, activation), &z);
    ctx->save_for_backward({x, weight, z});
    ctx->saved_data["wanted"] = wanted(x, weight, bias, residual) | activation * ACTIVATION;
    return y;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const int64_t want = ctx->saved_data["wanted"].toInt();
    variable_list out{Tensor(), Tensor(), Tensor()};
    const bool all = at::GradMode::is_enabled();   // (off inside)
    if (want & (WANT_X | WANT_WEIGHT | WANT_BIAS)) out = once([&] { return gradients(ctx, grads, want, all); });
    return {want & WANT_X ? out[0] : Tensor(), want & WANT_WEIGHT ? out[1] : Tensor(), want & WANT_BIAS ? out[2] : Tensor(), want & WANT_RESIDUAL ? grads[0] : Tensor(), Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads, int64_t want, bool all) {
    const variable_list saved = ctx->get_saved_variables();
    const c10::DeviceGuard guard(saved[0].device());
    const Tensor x = saved_rows(saved[0], saved[0].size(-1), 1 << 20), w = saved_dense(saved[1]), z = saved_dense(saved[2]);
    const Tensor dy = made_dense(grads[0]);
    const sk_dense_shape s = layer_shape(x, w, Tensor(), want / ACTIVATION);
    const Tensor none = all ? at::zeros({0}, x.options()) : Tensor();
    const Tensor dx = all || (want & WANT_X) ? at::empty(x.sizes(), x.options()) : none;
    const Tensor dw = all || (want & WANT_WEIGHT) ? at::empty(w.sizes(), x.options()) : none;
    const Tensor db = (want & HAS_BIAS) && (all || (want & WANT_BIAS)) ? at::empty({s.out}, x.options()) : none;
    with_workspace(x, sk_dense_workspace_bytes(&s, 1), [&](void* ws, size_t n, void* stream) {
      return sk_dense_bwd(&s, x.data_ptr(), w.data_ptr(), data(z), dy.data_ptr(), data(dx), data(dw), data(db), ws, n, stream);
    });
    return {dx, dw, db};
  }
};

// ---- the distillation loss ----

bool logits_in_place(const Tensor& z) {
  return z.is_contiguous() || (z.dim() == 2 && z.stride(1) == 1 && z.stride(0) > 0 && z.stride(0) <= (int64_t)1 << 40);
}

struct DistillCall {
  sk_distill_shape s{};
  DistillCall(const Tensor& z, const Tensor& ids, const Tensor& labels, double temperature, double label_weight) {
    s.vocabulary = z.size(-1); s.rows = z.numel() / s.vocabulary; s.logits_stride = row_stride(z);
    s.top = (int32_t)ids.size(-1); s.id_bytes = (int32_t)ids.element_size(); s.label_bytes = labels.defined() ? (int32_t)labels.element_size() : 8;
    s.temperature = (float)temperature; s.label_weight = (float)label_weight; s.dtype = dtype_of(z);
  }
};

Tensor distill_forward(const Tensor& z, const Tensor& t, const Tensor& ids, const Tensor& labels, const sk_distill_shape& s, Tensor* stats) {
  const c10::DeviceGuard guard(z.device());
  const at::TensorOptions f32 = z.options().dtype(at::kFloat);
  Tensor loss = at::empty(z.sizes().slice(0, z.dim() - 1), f32);
  if (stats) *stats = at::empty({s.rows, 8}, f32);
  check(sk_distill_fwd(&s, z.data_ptr(), data(t), data(ids), data(labels), loss.data_ptr<float>(), stats ? stats->data_ptr<float>() : nullptr, stream_of(z.device())));
  return loss;
}

struct Distill : torch::autograd::Function<Distill> {
  static Tensor forward(AutogradContext* ctx, const Tensor& z, const Tensor& t, const Tensor& ids, const std::optional<Tensor>& labels, double temperature, double label_weight) {
    const Tensor l = labels.value_or(Tensor());
    Tensor stats;
    const Tensor loss = distill_forward(z, t, ids, l, DistillCall(z, ids, l, temperature, label_weight).s, &stats);
    ctx->save_for_backward({z, t, ids, l, stats});
    ctx->saved_data["temperature"] = temperature;
    ctx->saved_data["label_weight"] = label_weight;
    return loss;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    return {once([&] { return gradients(ctx, grads); })[0], Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
  }

  static variable_list gradients(AutogradContext* ctx, const variable_list& grads) {
    const variable_list saved = ctx->get_saved_variables();
    const c10::DeviceGuard guard(saved[0].device());
    const Tensor z = logits_in_place(saved[0]) ? saved[0] : made_dense(saved[0]);
    const Tensor t = saved_dense(saved[1]), ids = saved_dense(saved[2]), labels = saved_dense(saved[3]), stats = saved_dense(saved[4]);
    const Tensor dloss = made_dense(grads[0]), dz = at::empty(z.sizes(), z.options());
    const DistillCall c(z, ids, labels, ctx->saved_data["temperature"].toDouble(), ctx->saved_data["label_weight"].toDouble());
    check(sk_distill_bwd(&c.s, z.data_ptr(), data(t), data(ids), data(labels), stats.data_ptr<float>(), dloss.data_ptr<float>(), dz.data_ptr(), stream_of(z.device())));
    return {dz};
  }
};

PyObject* wrapped(variable_list out) {
  if (out.size() == 1) return THPVariable_Wrap(std::move(out[0]));
  PyObject* const pair = PyTuple_New((Py_ssize_t)out.size());
  if (pair == nullptr) return nullptr;
  for (size_t i = 0; i < out.size(); ++i) {
    PyObject* const o = THPVariable_Wrap(std::move(out[i]));
    if (o == nullptr) { Py_DECREF(pair); return nullptr; }
    PyTuple_SET_ITEM(pair, (Py_ssize_t)i, o);
  }
  return pair;
}

}  // namespace

PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  double eps;
  if (n != 5 || !number(a[4], eps) || !unwatched()) Py_RETURN_NONE;
  const Tensor* x = plain(a[0]);
  if (!x || !floating(*x) || !no_tangent(*x) || x->dim() < 1 || x->numel() == 0 || !rows_in_place(*x, 0, (int64_t)1 << 40)) Py_RETURN_NONE;
  Tensor weight, bias, residual;
  if (!vector_like(a[1], *x, x->size(-1), weight) || !vector_like(a[2], *x, x->size(-1), bias)) Py_RETURN_NONE;
  if (a[3] != Py_None) {
    const Tensor* r = plain(a[3]);
    if (!r || !same(*x, *r) || r->sizes() != x->sizes() || !rows_in_place(*r, 0, (int64_t)1 << 40)) Py_RETURN_NONE;
    residual = *r;
  }
  const sk_layer_norm_shape s = norm_shape(*x, residual, eps);
  if (sk_layer_norm_workspace_bytes(&s) == (size_t)-1) Py_RETURN_NONE;
  variable_list out;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && (x->requires_grad() || wants(given(weight)) || wants(given(bias)) || wants(given(residual))))
      out = LayerNorm::apply(*x, given(weight), given(bias), given(residual), eps);
    else
      out = norm_forward(*x, weight, bias, residual, s, nullptr, false);
  }
  return wrapped(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyObject* dense_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  uint64_t activation;
  if (n != 5 || !word(a[4], activation) || activation > SK_ACT_SILU || !unwatched()) Py_RETURN_NONE;
  const Tensor *x = plain(a[0]), *w = plain(a[1]);
  if (!x || !w || !floating(*x) || !no_tangent(*x) || !same(*x, *w) || w->dim() != 2 || w->numel() == 0 || !dense(*w) || x->dim() < 1 || x->numel() == 0 ||
      x->size(-1) != w->size(1) || !rows_in_place(*x, w->size(1), 1 << 20))
    Py_RETURN_NONE;
  Tensor bias, residual;
  if (!vector_like(a[2], *x, w->size(0), bias)) Py_RETURN_NONE;
  if (a[3] != Py_None) {
    const Tensor* r = plain(a[3]);
    if (!r || !same(*x, *r) || r->dim() != x->dim() || r->size(-1) != w->size(0) || r->sizes().slice(0, r->dim() - 1) != x->sizes().slice(0, x->dim() - 1) ||
        !rows_in_place(*r, w->size(0), 1 << 20))
      Py_RETURN_NONE;
    residual = *r;
  }
  const sk_dense_shape s = layer_shape(*x, *w, residual, (int64_t)activation);
  if (sk_dense_workspace_bytes(&s, 0) == (size_t)-1) Py_RETURN_NONE;
  Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && (x->requires_grad() || w->requires_grad() || wants(given(bias)) || wants(given(residual))))
      y = Dense::apply(*x, *w, given(bias), given(residual), (int64_t)activation);
    else
      y = layer_forward(*x, *w, bias, residual, s, nullptr);
  }
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

PyObject* distillation_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  double temperature, label_weight;
  if (n != 6 || !number(a[4], temperature) || !number(a[5], label_weight) || !unwatched()) Py_RETURN_NONE;
  const Tensor *z = plain(a[0]), *t = plain(a[1]), *ids = plain(a[2]);
  if (!z || !t || !ids || !floating(*z) || !no_tangent(*z) || !same(*z, *t) || !integers(*ids, z->device()) || z->dim() < 1 || z->numel() == 0) Py_RETURN_NONE;
  if (!logits_in_place(*z)) Py_RETURN_NONE;
  if (t->dim() != z->dim() || ids->sizes() != t->sizes() || t->sizes().slice(0, t->dim() - 1) != z->sizes().slice(0, z->dim() - 1) || t->numel() == 0 || t->size(-1) > 1 << 16 || !dense(*t) || !dense(*ids) ||
      (at::GradMode::is_enabled() && t->requires_grad()))
    Py_RETURN_NONE;
  Tensor labels;
  if (a[3] != Py_None) {
    const Tensor* l = plain(a[3]);
    if (!l || !integers(*l, z->device()) || l->sizes() != z->sizes().slice(0, z->dim() - 1) || !dense(*l)) Py_RETURN_NONE;
    labels = *l;
  }
  const DistillCall c(*z, *ids, labels, temperature, label_weight);
  if (!(temperature >= 1e-3 && temperature <= 1e3 && label_weight >= 0.0 && label_weight <= 1.0) || c.s.rows >= 1 << 23 || c.s.vocabulary > 1 << 24) Py_RETURN_NONE;
  Tensor loss;
  {
    pybind11::gil_scoped_release no_gil;
    if (at::GradMode::is_enabled() && z->requires_grad()) loss = Distill::apply(*z, *t, *ids, given(labels), temperature, label_weight);
    else loss = distill_forward(*z, *t, *ids, labels, c.s, nullptr);
  }
  return THPVariable_Wrap(std::move(loss));
  END_HANDLE_TH_ERRORS
}

}  // namespace sk_torch
