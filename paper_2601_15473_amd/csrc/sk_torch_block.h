// The block operators' native functions (sk_torch_block.cpp), as the module's table calls them.
#pragma once
#include "sk_torch.h"

namespace sk_torch {
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n);        // q, k, v, q_lengths, k_lengths (or None), causal, scale or None
PyObject* head_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n);   // q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n);        // ids, table, scale
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n);          // x, p, seed, offset, residual or None
}  // namespace sk_torch
