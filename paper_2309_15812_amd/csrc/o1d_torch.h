// What the native calls from torch tensors share (included by o1d_torch.cpp and o1d_torch_train.cpp).
//
// A call returns None where its case is not the common one (a tensor of other strides or one that does not match, no
// rows, an error status): the caller then takes its checked path, which also names what is wrong.  Outputs are
// new tensors; kernels run on the current stream of the first tensor's device, which is made the current one
// for the call (the default stream's handle means the current device's).
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <optional>

#include "o1d.h"

namespace {

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
PyObject* none() { Py_RETURN_NONE; }
PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

// Rows on a GPU: M x C of a type that the kernels have, contiguous or a matrix whose rows lie ld apart.
struct Rows {
  const at::Tensor* t = nullptr;
  long long M = 0;
  int C = 0;
  long long ld = 0;
  o1d_dtype_t dt = O1D_F32;
  void* data() const { return t->data_ptr(); }
};
std::optional<o1d_dtype_t> type_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return O1D_F32;
  if (t.scalar_type() == at::kBFloat16) return O1D_BF16;
  return std::nullopt;
}
bool rows_of(PyObject* o, Rows& r) {
  r.t = tensor(o);
  if (!r.t || !r.t->is_cuda() || r.t->dim() < 1) return false;
  const auto dt = type_of(*r.t);
  const int64_t C = r.t->size(-1), n = r.t->numel();
  if (!dt || C < 1 || n < 1 || C > INT32_MAX || n / C > INT32_MAX) return false;
  r.dt = *dt;
  r.C = (int)C;
  r.M = n / C;
  r.ld = C;
  if (r.t->is_contiguous()) return true;
  if (r.t->dim() != 2 || r.M < 2 || (C > 1 && r.t->stride(1) != 1) || r.t->stride(0) < C) return false;
  r.ld = r.t->stride(0);
  return true;
}
bool like(const at::Tensor& t, const Rows& r) {
  return t.is_cuda() && t.scalar_type() == r.t->scalar_type() && t.get_device() == r.t->get_device();
}
[[maybe_unused]] bool matches(const Rows& a, const Rows& r, int C) { return like(*a.t, r) && a.M == r.M && a.C == C; }
[[maybe_unused]] const at::Tensor* vector(PyObject* o, const Rows& r, int64_t n) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == 1 && t->size(0) == n && like(*t, r) && t->is_contiguous() ? t : nullptr;
}
[[maybe_unused]] const at::Tensor* matrix(PyObject* o, const Rows& r) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == 2 && t->size(0) > 0 && t->size(0) <= INT32_MAX && t->size(1) <= INT32_MAX && like(*t, r) &&
                 t->is_contiguous()
             ? t
             : nullptr;
}

void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }
at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}
// r's leading axes and C features
[[maybe_unused]] at::Tensor empty_rows(const Rows& r, int C) {
  c10::SmallVector<int64_t, 6> shape(r.t->sizes().begin(), r.t->sizes().end());
  shape.back() = C;
  return empty(shape, *r.t, r.t->scalar_type());
}
// Workspace.  Calls that need none ask for 256 bytes, to which nothing is
// written (those that write ask for 512 at least): one such tensor per device,
// never freed, serves them all, on whichever streams they run.
[[maybe_unused]] at::Tensor space(size_t need, const at::Tensor& like) {
  if (need > 256) return empty({(int64_t)need}, like, at::kByte);
  static std::array<at::Tensor*, 64> held{};
  const int d = like.get_device();
  if (d < 0 || d >= (int)held.size()) return empty({256}, like, at::kByte);
  if (!held[d]) held[d] = new at::Tensor(empty({256}, like, at::kByte));
  return *held[d];
}

template <typename F>
o1d_status_t call(F&& f) {
  o1d_status_t s;
  Py_BEGIN_ALLOW_THREADS;
  s = f();
  Py_END_ALLOW_THREADS;
  return s;
}
[[maybe_unused]] PyObject* result(std::initializer_list<PyObject*> items) {
  PyObject* t = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (!t || !o) {
      for (PyObject* p : items) Py_XDECREF(p);
      if (t) Py_DECREF(t);
      return nullptr;
    }
    ++i;
  }
  i = 0;
  for (PyObject* o : items) PyTuple_SET_ITEM(t, i++, o);
  return t;
}

}  // namespace
