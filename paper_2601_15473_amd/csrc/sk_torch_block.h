// The block operators' native functions (sk_torch_block.cpp, sk_torch_layers.cpp), as the module's table calls them, and what they share.
#pragma once
#include <functional>

#include "sk_torch.h"

namespace sk_torch {

inline bool floating(const Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
inline bool same(const Tensor& x, const Tensor& t) { return t.scalar_type() == x.scalar_type() && t.device() == x.device() && no_tangent(t); }
inline bool dense(const Tensor& t) { return t.is_contiguous() && aligned(t); }
inline Tensor made_dense(const Tensor& t) { return dense(t) ? t : t.clone(at::MemoryFormat::Contiguous); }
inline bool integers(const Tensor& t, const at::Device& device) { return (t.scalar_type() == at::kInt || t.scalar_type() == at::kLong) && t.device() == device; }

// Strides that the library takes in place (block.py's _strided)
inline bool strided(const Tensor& t, int64_t token) {
  if (!aligned(t) || (t.stride(-1) != 1 && t.size(-1) != 1)) return false;
  const int64_t unit = 16 / (int64_t)t.element_size();
  for (int64_t d = 0; d < t.dim() - 1; ++d)
    if (t.size(d) > 1 && (t.stride(d) % unit != 0 || t.stride(d) < 0 || t.stride(d) >= (d == token ? (int64_t)1 << 22 : (int64_t)1 << 40))) return false;
  return true;
}

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
inline std::optional<Tensor> given(const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; }

inline bool number(PyObject* o, double& v) {
  if (PyFloat_Check(o)) { v = PyFloat_AS_DOUBLE(o); return true; }
  if (!PyLong_Check(o)) return false;
  v = PyLong_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}
inline bool word(PyObject* o, uint64_t& v) {
  if (!PyLong_Check(o)) return false;
  v = PyLong_AsUnsignedLongLong(o);
  if (v == (uint64_t)-1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n);        // q, k, v, q_lengths, k_lengths (or None), causal, scale or None
PyObject* head_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n);   // q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n);        // ids, table, scale
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n);          // x, p, seed, offset, residual or None
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n);       // x, weight or None, bias or None, residual or None, eps
PyObject* dense_layer(PyObject*, PyObject* const* a, Py_ssize_t n);      // x, weight, bias or None, residual or None, activation (a number)
PyObject* distillation_loss(PyObject*, PyObject* const* a, Py_ssize_t n);   // logits, teacher_logits, teacher_ids, labels or None, temperature, label_weight
}  // namespace sk_torch
