// The row operators' calls for the common case, from torch tensors to the C ABI
// without Python in between.  Most of these calls are short: in Python the checks,
// the outputs and the argument list took longer than the launch: 49 x 768 layer
// norm 9.0 us per call, of which the launch 3; 5.1 this way.
//
// Each function returns None where its case is not the common one (a tensor of
// other strides or one that does not match, no rows, an error status): the caller
// then takes its checked path, which also names what is wrong.  Outputs are new
// tensors; kernels run on the current stream of the first tensor's device, which is
// made the current one for the call (the default stream's handle means the current device's).
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

// The library's entry points, as the loader of the library found them.
decltype(&o1d_ln_fwd) p_ln_fwd;
decltype(&o1d_ln_bwd) p_ln_bwd;
decltype(&o1d_ln_bwd_workspace_bytes) p_ln_bytes;
decltype(&o1d_linear_fwd) p_linear_fwd;
decltype(&o1d_linear_bwd_input) p_linear_bwd_input;
decltype(&o1d_linear_bwd_weight) p_linear_bwd_weight;
decltype(&o1d_linear_bwd_weight_workspace_bytes) p_linear_bytes;
decltype(&o1d_pack) p_pack;
decltype(&o1d_unpack) p_unpack;

constexpr int kGroup = 64;

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
bool matches(const Rows& a, const Rows& r, int C) { return like(*a.t, r) && a.M == r.M && a.C == C; }
const at::Tensor* vector(PyObject* o, const Rows& r, int64_t n) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == 1 && t->size(0) == n && like(*t, r) && t->is_contiguous() ? t : nullptr;
}
const at::Tensor* matrix(PyObject* o, const Rows& r) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == 2 && t->size(0) > 0 && t->size(0) <= INT32_MAX && t->size(1) <= INT32_MAX && like(*t, r) &&
                 t->is_contiguous()
             ? t
             : nullptr;
}

// A tensor of r's rows of C features, or (scale not None) a checkpoint (q, scale) of
// `cols` features, which have to be C.
struct Source {
  const void* x = nullptr;
  const signed char* q = nullptr;
  const float* scale = nullptr;
  long long ld = 0;
};
bool source_of(PyObject* x, PyObject* scale, PyObject* cols, const Rows& r, int C, Source& s) {
  if (scale == Py_None) {
    Rows a;
    if (!rows_of(x, a) || !matches(a, r, C)) return false;
    s.x = a.data();
    s.ld = a.ld;
    return true;
  }
  // (the checkpoint's own constructor has checked its tensors against each other)
  const at::Tensor *q = tensor(x), *f = tensor(scale);
  if (PyLong_AsLong(cols) != C || !q || !f || q->dim() != 2 || f->dim() != 2) return false;
  for (const at::Tensor* t : {q, f})
    if (t->size(0) != r.M || t->get_device() != r.t->get_device() || !t->is_contiguous()) return false;
  if (q->scalar_type() != at::kChar || f->scalar_type() != at::kFloat || q->size(1) != (C + 15) / 16 * 16 ||
      f->size(1) != (C + kGroup - 1) / kGroup)
    return false;
  s.ld = C;
  s.q = static_cast<const signed char*>(q->data_ptr());
  s.scale = static_cast<const float*>(f->data_ptr());
  return true;
}

void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }
at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}
// r's leading axes and C features
at::Tensor empty_rows(const Rows& r, int C) {
  c10::SmallVector<int64_t, 6> shape(r.t->sizes().begin(), r.t->sizes().end());
  shape.back() = C;
  return empty(shape, *r.t, r.t->scalar_type());
}
// Workspace.  Calls that need none ask for 256 bytes, to which nothing is
// written (those that write ask for 512 at least): one such tensor per device,
// never freed, serves them all, on whichever streams they run.
at::Tensor space(size_t need, const at::Tensor& like) {
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
PyObject* result(std::initializer_list<PyObject*> items) {
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

// (x, w, b, eps) -> (y, mean, rstd)
PyObject* ln_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x;
  if (n != 4 || !rows_of(a[0], x)) return none();
  const at::Tensor *w = vector(a[1], x, x.C), *b = vector(a[2], x, x.C);
  const double eps = PyFloat_Check(a[3]) ? PyFloat_AS_DOUBLE(a[3]) : -1.;
  if (!w || !b || eps < 0.) return none();
  at::Tensor y = empty_rows(x, x.C), mean = empty({x.M}, *x.t, at::kFloat), rstd = empty({x.M}, *x.t, at::kFloat);
  const c10::DeviceGuard guard(x.t->device());
  void* s = stream_of(*x.t);
  const auto st = call([&] {
    return p_ln_fwd(x.data(), x.ld, w->data_ptr(), b->data_ptr(), y.data_ptr(), x.C, (float*)mean.data_ptr(),
                    (float*)rstd.data_ptr(), (int)x.M, x.C, (float)eps, x.dt, s);
  });
  return st ? none() : result({wrap(y), wrap(mean), wrap(rstd)});
  END_HANDLE_TH_ERRORS
}

// (x or q, scale or None, cols, dy, mean, rstd, w) -> (dx, dw, db)
PyObject* ln_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows dy;
  Source x;
  if (n != 7 || !rows_of(a[3], dy) || !source_of(a[0], a[1], a[2], dy, dy.C, x)) return none();
  const at::Tensor *mean = tensor(a[4]), *rstd = tensor(a[5]), *w = vector(a[6], dy, dy.C);
  for (const at::Tensor* t : {mean, rstd})
    if (!t || t->dim() != 1 || t->size(0) != dy.M || t->scalar_type() != at::kFloat || !t->is_contiguous() ||
        !t->is_cuda() || t->get_device() != dy.t->get_device())
      return none();
  if (!w) return none();
  at::Tensor dx = empty_rows(dy, dy.C), dw = empty({dy.C}, *w, w->scalar_type()),
             db = empty({dy.C}, *w, w->scalar_type());
  const size_t need = p_ln_bytes((int)dy.M, dy.C, dy.dt);
  at::Tensor ws = space(need, *dy.t);
  const c10::DeviceGuard guard(dy.t->device());
  void* s = stream_of(*dy.t);
  const auto st = call([&] {
    return p_ln_bwd(x.x, x.ld, x.q, x.scale, dy.data(), dy.ld, (const float*)mean->data_ptr(),
                    (const float*)rstd->data_ptr(), w->data_ptr(), dx.data_ptr(), dy.C, dw.data_ptr(), db.data_ptr(),
                    (int)dy.M, dy.C, dy.dt, ws.data_ptr(),
                    (size_t)ws.numel(), s);
  });
  return st ? none() : result({wrap(dx), wrap(dw), wrap(db)});
  END_HANDLE_TH_ERRORS
}

// (x, w, b or None, act, residual or None, save: 0 nothing, 1 whole, 2 in 8 bits)
// -> y, (y, pre) or (y, q, scale)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x, res;
  if (n != 6 || !rows_of(a[0], x)) return none();
  const at::Tensor *w = matrix(a[1], x), *b = nullptr;
  if (!w || w->size(1) != x.C) return none();
  const int O = (int)w->size(0);
  if (a[2] != Py_None && !(b = vector(a[2], x, O))) return none();
  if (a[4] != Py_None && (!rows_of(a[4], res) || !matches(res, x, O))) return none();
  const long act = PyLong_AsLong(a[3]), save = PyLong_AsLong(a[5]);
  at::Tensor y = empty_rows(x, O), pre, q, scale;
  if (save == 1) pre = empty_rows(x, O);
  if (save == 2) {
    q = empty({x.M, (O + 15) / 16 * 16}, *x.t, at::kChar);
    scale = empty({x.M, (O + kGroup - 1) / kGroup}, *x.t, at::kFloat);
  }
  const c10::DeviceGuard guard(x.t->device());
  void* s = stream_of(*x.t);
  const auto st = call([&] {
    return p_linear_fwd(x.data(), x.ld, w->data_ptr(), b ? b->data_ptr() : nullptr, (o1d_act_t)act,
                        res.t ? res.data() : nullptr, res.t ? res.ld : O, y.data_ptr(), O,
                        save == 1 ? pre.data_ptr() : nullptr, O,
                        save == 2 ? (signed char*)q.data_ptr() : nullptr, save == 2 ? (float*)scale.data_ptr() : nullptr,
                        (int)x.M, x.C, O, x.dt, s);
  });
  if (st) return none();
  if (save == 1) return result({wrap(y), wrap(pre)});
  if (save == 2) return result({wrap(y), wrap(q), wrap(scale)});
  return wrap(y);
  END_HANDLE_TH_ERRORS
}

// (dy, w, pre or q or None, scale or None, cols, act) -> dx
PyObject* linear_bwd_input(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows dy;
  if (n != 6 || !rows_of(a[0], dy)) return none();
  const at::Tensor* w = matrix(a[1], dy);
  if (!w || w->size(0) != dy.C) return none();
  const int I = (int)w->size(1);
  const long act = PyLong_AsLong(a[5]);
  Source pre;
  if (I < 1 || (a[2] == Py_None) != (act == O1D_ACT_NONE)) return none();
  if (a[2] != Py_None && !source_of(a[2], a[3], a[4], dy, I, pre)) return none();
  at::Tensor dx = empty_rows(dy, I);
  const c10::DeviceGuard guard(dy.t->device());
  void* s = stream_of(*dy.t);
  const auto st = call([&] {
    return p_linear_bwd_input(dy.data(), dy.ld, w->data_ptr(), (o1d_act_t)act, pre.x, pre.x ? pre.ld : I, pre.q,
                              pre.scale, dx.data_ptr(), I,
                              (int)dy.M, I, dy.C, dy.dt, s);
  });
  return st ? none() : wrap(dx);
  END_HANDLE_TH_ERRORS
}

// (x or q, scale or None, cols, dy, act, bias) -> (dw, db or None)
PyObject* linear_bwd_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows dy;
  Source x;
  if (n != 6 || !rows_of(a[3], dy)) return none();
  const long I = PyLong_AsLong(a[2]), act = PyLong_AsLong(a[4]);
  const bool bias = a[5] == Py_True;
  if (I < 1 || I > INT32_MAX || !source_of(a[0], a[1], a[2], dy, (int)I, x)) return none();
  const int O = dy.C;
  at::Tensor dw = empty({O, I}, *dy.t, dy.t->scalar_type()), db;
  if (bias) db = empty({O}, *dy.t, dy.t->scalar_type());
  const size_t need = p_linear_bytes((int)dy.M, (int)I, O, (o1d_act_t)act, x.q != nullptr, dy.dt);
  at::Tensor ws = space(need, *dy.t);
  const c10::DeviceGuard guard(dy.t->device());
  void* s = stream_of(*dy.t);
  const auto st = call([&] {
    return p_linear_bwd_weight(x.x, x.ld, x.q, x.scale, (o1d_act_t)act, dy.data(), dy.ld, dw.data_ptr(),
                               bias ? db.data_ptr() : nullptr, (int)dy.M, (int)I, O, dy.dt, ws.data_ptr(),
                               (size_t)ws.numel(), s);
  });
  if (st) return none();
  PyObject* second = bias ? wrap(db) : none();
  return result({wrap(dw), second});
  END_HANDLE_TH_ERRORS
}

// (x) -> (q, scale)
PyObject* pack8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x;
  if (n != 1 || !rows_of(a[0], x)) return none();
  at::Tensor q = empty({x.M, (x.C + 15) / 16 * 16}, *x.t, at::kChar),
             scale = empty({x.M, (x.C + kGroup - 1) / kGroup}, *x.t, at::kFloat);
  const c10::DeviceGuard guard(x.t->device());
  void* s = stream_of(*x.t);
  const auto st = call([&] {
    return p_pack(x.data(), x.ld, (signed char*)q.data_ptr(), (float*)scale.data_ptr(), (int)x.M, x.C, x.dt, s);
  });
  return st ? none() : result({wrap(q), wrap(scale)});
  END_HANDLE_TH_ERRORS
}

// (q, scale, cols, type, act) -> y
PyObject* unpack8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *q = n == 5 ? tensor(a[0]) : nullptr, *scale = n == 5 ? tensor(a[1]) : nullptr;
  if (!q || !scale || !q->is_cuda() || q->dim() != 2 || q->size(0) < 1 || q->size(0) > INT32_MAX) return none();
  const long C = PyLong_AsLong(a[2]), dt = PyLong_AsLong(a[3]), act = PyLong_AsLong(a[4]);
  if (C < 1 || q->size(1) != (C + 15) / 16 * 16) return none();
  at::Tensor y = empty({q->size(0), C}, *q, dt == O1D_F32 ? at::kFloat : at::kBFloat16);
  const c10::DeviceGuard guard(q->device());
  void* s = stream_of(*q);
  const auto st = call([&] {
    return p_unpack((const signed char*)q->data_ptr(), (const float*)scale->data_ptr(), (o1d_act_t)act, y.data_ptr(), C,
                    (int)q->size(0), (int)C, (o1d_dtype_t)dt, s);
  });
  return st ? none() : wrap(y);
  END_HANDLE_TH_ERRORS
}

// (addresses of the nine entry points, in the order above)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void** to[] = {(void**)&p_ln_fwd,       (void**)&p_ln_bwd,      (void**)&p_ln_bytes,
                 (void**)&p_linear_fwd,   (void**)&p_linear_bwd_input, (void**)&p_linear_bwd_weight,
                 (void**)&p_linear_bytes, (void**)&p_pack,        (void**)&p_unpack};
  if (n != (Py_ssize_t)(sizeof(to) / sizeof(to[0]))) {
    PyErr_SetString(PyExc_TypeError, "nine addresses expected");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    *to[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  return none();
}

#define O1D_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {O1D_METHOD(ln_fwd),        O1D_METHOD(ln_bwd),  O1D_METHOD(linear_fwd),
                         O1D_METHOD(linear_bwd_input), O1D_METHOD(linear_bwd_weight), O1D_METHOD(pack8),
                         O1D_METHOD(unpack8),       O1D_METHOD(bind),    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows(void) { return PyModule_Create(&module); }
