// Group norm, products of 8-bit operands and AdamW for the common case, from torch
// tensors to the C ABI without Python in between.  In Python a step over 63 tensors took 120 us of
// checks and argument lists, longer than its kernels.
#include "o1d_torch.h"

#include <c10/util/SmallVector.h>

#include <vector>

namespace {

decltype(&o1d_gn_fwd) p_gn_fwd;
decltype(&o1d_gn_fwd_workspace_bytes) p_gn_fwd_bytes;
decltype(&o1d_gn_bwd) p_gn_bwd;
decltype(&o1d_gn_bwd_workspace_bytes) p_gn_bwd_bytes;
decltype(&o1d_pack_scaled) p_pack;
decltype(&o1d_pack_scaled_workspace_bytes) p_pack_bytes;
decltype(&o1d_scaled_linear_fwd) p_fwd;
decltype(&o1d_scaled_linear_bwd_input) p_bwd_input;
decltype(&o1d_scaled_linear_bwd_weight) p_bwd_weight;
decltype(&o1d_scaled_linear_bwd_weight_workspace_bytes) p_bwd_weight_bytes;
decltype(&o1d_adamw) p_adamw;
decltype(&o1d_adamw_workspace_bytes) p_adamw_bytes;

constexpr int64_t kGroup = 128;
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A whole number, or -1 where it is none of C's: the checked path says what is wrong.
long number(PyObject* o) {
  const long k = PyLong_AsLong(o);
  if (k == -1) PyErr_Clear();
  return k;
}

// Samples of rows: (N, ..., C).
bool samples_of(PyObject* o, Rows& r, int& N, int& P) {
  if (!rows_of(o, r) || r.t->dim() < 2 || r.t->size(0) > INT32_MAX) return false;
  N = (int)r.t->size(0);
  P = (int)(r.M / N);
  return true;
}

// (x, w, b, groups, eps, act) -> (y, mean, rstd)
PyObject* gn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x;
  int N, P;
  if (n != 6 || !samples_of(a[0], x, N, P)) return none();
  const at::Tensor *w = vector(a[1], x, x.C), *b = vector(a[2], x, x.C);
  const long G = number(a[3]), act = number(a[5]);
  const double eps = PyFloat_Check(a[4]) ? PyFloat_AS_DOUBLE(a[4]) : -1.;
  if (!w || !b || G < 1 || G > x.C || x.C % G || eps < 0.) return none();
  at::Tensor y = empty_rows(x, x.C), mean = empty({N, G}, *x.t, at::kFloat), rstd = empty({N, G}, *x.t, at::kFloat);
  const size_t need = p_gn_fwd_bytes(N, P, x.C, (int)G, x.dt);
  at::Tensor ws = space(need, *x.t);
  const c10::DeviceGuard guard(x.t->device());
  void* s = stream_of(*x.t);
  const auto st = call([&] {
    return p_gn_fwd(x.data(), x.ld, w->data_ptr(), b->data_ptr(), (o1d_act_t)act, y.data_ptr(), x.C,
                    (float*)mean.data_ptr(), (float*)rstd.data_ptr(), N, P, x.C, (int)G, (float)eps, x.dt, ws.data_ptr(),
                    (size_t)ws.numel(), s);
  });
  return st ? none() : result({wrap(y), wrap(mean), wrap(rstd)});
  END_HANDLE_TH_ERRORS
}

// (x, dy, mean, rstd, w, b, act) -> (dx, dw, db)
PyObject* gn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x, dy;
  int N, P;
  if (n != 7 || !samples_of(a[1], dy, N, P) || !rows_of(a[0], x) || !matches(x, dy, dy.C)) return none();
  const at::Tensor *mean = tensor(a[2]), *rstd = tensor(a[3]), *w = vector(a[4], dy, dy.C), *b = vector(a[5], dy, dy.C);
  const long act = PyLong_AsLong(a[6]);
  if (!mean || !rstd || !w || !b || mean->dim() != 2) return none();
  const int64_t G = mean->size(1);
  for (const at::Tensor* t : {mean, rstd})
    if (t->dim() != 2 || t->size(0) != N || t->size(1) != G || t->scalar_type() != at::kFloat || !t->is_contiguous() ||
        !t->is_cuda() || t->get_device() != dy.t->get_device())
      return none();
  if (G < 1 || G > dy.C || dy.C % G) return none();
  at::Tensor dx = empty_rows(dy, dy.C), dw = empty({dy.C}, *w, w->scalar_type()), db = empty({dy.C}, *w, w->scalar_type());
  const size_t need = p_gn_bwd_bytes(N, P, dy.C, (int)G, dy.dt);
  at::Tensor ws = space(need, *dy.t);
  const c10::DeviceGuard guard(dy.t->device());
  void* s = stream_of(*dy.t);
  const auto st = call([&] {
    return p_gn_bwd(x.data(), x.ld, dy.data(), dy.ld, (const float*)mean->data_ptr(), (const float*)rstd->data_ptr(),
                    w->data_ptr(), b->data_ptr(), (o1d_act_t)act, dx.data_ptr(), dy.C, dw.data_ptr(), db.data_ptr(), N, P,
                    dy.C, (int)G, dy.dt, ws.data_ptr(), (size_t)ws.numel(), s);
  });
  return st ? none() : result({wrap(dx), wrap(dw), wrap(db)});
  END_HANDLE_TH_ERRORS
}

at::ScalarType scaled_type(long type) { return type == O1D_E5M2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn; }

// A packed operand: (q, e) of R rows of K values.
struct Packed {
  const at::Tensor *q = nullptr, *e = nullptr;
  int R = 0, K = 0;
  o1d_scaled_t type = O1D_E4M3;
  const unsigned char* values() const { return static_cast<const unsigned char*>(q->data_ptr()); }
  const unsigned char* exponents() const { return static_cast<const unsigned char*>(e->data_ptr()); }
};
bool packed_of(PyObject* q, PyObject* e, PyObject* cols, Packed& p) {
  p.q = tensor(q);
  p.e = tensor(e);
  const long K = number(cols);
  if (!p.q || !p.e || K < 1 || K > INT32_MAX || !p.q->is_cuda() || p.q->dim() != 2 || p.q->size(0) < 1 ||
      p.q->size(0) > INT32_MAX)
    return false;
  const auto t = p.q->scalar_type();
  if (t != at::kFloat8_e4m3fn && t != at::kFloat8_e5m2) return false;
  p.R = (int)p.q->size(0);
  p.K = (int)K;
  p.type = t == at::kFloat8_e5m2 ? O1D_E5M2 : O1D_E4M3;
  return p.q->size(1) == up(K, kGroup) && p.q->is_contiguous() && p.e->dim() == 2 && p.e->scalar_type() == at::kByte &&
         p.e->size(0) == up(K, kGroup) / kGroup && p.e->size(1) == up(p.R, 16) && p.e->is_contiguous() && p.e->is_cuda() &&
         p.e->get_device() == p.q->get_device();
}
bool goes_with(const Packed& b, const Packed& a) {
  return b.K == a.K && b.type == O1D_E4M3 && b.q->get_device() == a.q->get_device();
}
// A tensor of M rows of C features of type dt on a's device.
bool rows_like(PyObject* o, const Packed& a, long long M, int C, o1d_dtype_t dt, Rows& r) {
  return rows_of(o, r) && r.M == M && r.C == C && r.dt == dt && r.t->get_device() == a.q->get_device();
}
at::ScalarType stored(o1d_dtype_t dt) { return dt == O1D_F32 ? at::kFloat : at::kBFloat16; }

// (x, type, along: 1 features, 2 rows, 3 both, sums) -> the operands' (q, e) one behind the other, then the sums
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Rows x;
  if (n != 4 || !rows_of(a[0], x)) return none();
  const long type = PyLong_AsLong(a[1]), along = PyLong_AsLong(a[2]);
  const bool sums = a[3] == Py_True;
  at::Tensor q, e, qt, et, total, ws;
  if (along & 1) {
    q = empty({x.M, up(x.C, kGroup)}, *x.t, scaled_type(type));
    e = empty({up(x.C, kGroup) / kGroup, up(x.M, 16)}, *x.t, at::kByte);
  }
  if (along & 2) {
    qt = empty({x.C, up(x.M, kGroup)}, *x.t, scaled_type(type));
    et = empty({up(x.M, kGroup) / kGroup, up(x.C, 16)}, *x.t, at::kByte);
  }
  if (sums) {
    total = empty({x.C}, *x.t, x.t->scalar_type());
    ws = space(p_pack_bytes((int)x.M, x.C, 1), *x.t);
  }
  auto at = [](const at::Tensor& t) { return t.defined() ? static_cast<unsigned char*>(t.data_ptr()) : nullptr; };
  const c10::DeviceGuard guard(x.t->device());
  void* s = stream_of(*x.t);
  const auto st = call([&] {
    return p_pack(x.data(), x.ld, (o1d_scaled_t)type, at(q), at(e), at(qt), at(et), at(total), (int)x.M, x.C, x.dt, at(ws),
                  ws.defined() ? (size_t)ws.numel() : 0, s);
  });
  if (st) return none();
  if (along == 3) return sums ? result({wrap(q), wrap(e), wrap(qt), wrap(et), wrap(total)}) : result({wrap(q), wrap(e), wrap(qt), wrap(et)});
  if (along == 2) return sums ? result({wrap(qt), wrap(et), wrap(total)}) : result({wrap(qt), wrap(et)});
  return result({wrap(q), wrap(e)});
  END_HANDLE_TH_ERRORS
}

// (xq, xe, wq, we, cols, b or None, act, residual or None, save, dtype) -> y or (y, pre)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed x, w;
  if (n != 10 || !packed_of(a[0], a[1], a[4], x) || !packed_of(a[2], a[3], a[4], w) || !goes_with(w, x)) return none();
  const long act = PyLong_AsLong(a[6]), dt = PyLong_AsLong(a[9]);
  const bool save = a[8] == Py_True;
  Rows res, b;
  if (a[5] != Py_None && !(rows_like(a[5], x, 1, w.R, (o1d_dtype_t)dt, b) && b.t->dim() == 1 && b.t->is_contiguous())) return none();
  if (a[7] != Py_None && !rows_like(a[7], x, x.R, w.R, (o1d_dtype_t)dt, res)) return none();
  at::Tensor y = empty({x.R, w.R}, *x.q, stored((o1d_dtype_t)dt)), pre;
  if (save) pre = empty({x.R, w.R}, *x.q, stored((o1d_dtype_t)dt));
  const c10::DeviceGuard guard(x.q->device());
  void* s = stream_of(*x.q);
  const auto st = call([&] {
    return p_fwd(x.values(), x.exponents(), x.type, w.values(), w.exponents(), b.t ? b.data() : nullptr, (o1d_act_t)act,
                 res.t ? res.data() : nullptr, res.t ? res.ld : w.R, y.data_ptr(), w.R, save ? pre.data_ptr() : nullptr, w.R,
                 x.R, x.K, w.R, (o1d_dtype_t)dt, s);
  });
  if (st) return none();
  return save ? result({wrap(y), wrap(pre)}) : wrap(y);
  END_HANDLE_TH_ERRORS
}

// (dyq, dye, wtq, wte, cols, pre or None, act, dtype) -> dx
PyObject* linear_bwd_input(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed dy, w;
  if (n != 8 || !packed_of(a[0], a[1], a[4], dy) || !packed_of(a[2], a[3], a[4], w) || !goes_with(w, dy)) return none();
  const long act = PyLong_AsLong(a[6]), dt = PyLong_AsLong(a[7]);
  Rows pre;
  if ((a[5] == Py_None) != (act == O1D_ACT_NONE)) return none();
  if (a[5] != Py_None && !rows_like(a[5], dy, dy.R, w.R, (o1d_dtype_t)dt, pre)) return none();
  at::Tensor dx = empty({dy.R, w.R}, *dy.q, stored((o1d_dtype_t)dt));
  const c10::DeviceGuard guard(dy.q->device());
  void* s = stream_of(*dy.q);
  const auto st = call([&] {
    return p_bwd_input(dy.values(), dy.exponents(), dy.type, w.values(), w.exponents(), (o1d_act_t)act,
                       pre.t ? pre.data() : nullptr, pre.t ? pre.ld : w.R, dx.data_ptr(), w.R, dy.R, w.R, dy.K,
                       (o1d_dtype_t)dt, s);
  });
  return st ? none() : wrap(dx);
  END_HANDLE_TH_ERRORS
}

// (dytq, dyte, xtq, xte, cols, dtype) -> dw
PyObject* linear_bwd_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed dy, x;
  if (n != 6 || !packed_of(a[0], a[1], a[4], dy) || !packed_of(a[2], a[3], a[4], x) || !goes_with(x, dy)) return none();
  const long dt = PyLong_AsLong(a[5]);
  at::Tensor dw = empty({dy.R, x.R}, *dy.q, stored((o1d_dtype_t)dt));
  at::Tensor ws = space(p_bwd_weight_bytes(dy.K, x.R, dy.R, (o1d_dtype_t)dt), *dy.q);
  const c10::DeviceGuard guard(dy.q->device());
  void* s = stream_of(*dy.q);
  const auto st = call([&] {
    return p_bwd_weight(dy.values(), dy.exponents(), dy.type, x.values(), x.exponents(), dw.data_ptr(), dy.K, x.R, dy.R,
                        (o1d_dtype_t)dt, ws.data_ptr(), (size_t)ws.numel(), s);
  });
  return st ? none() : wrap(dw);
  END_HANDLE_TH_ERRORS
}

const at::Tensor* flat(PyObject* o, int64_t n, at::ScalarType type, const at::Tensor* like) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == 1 && t->size(0) == n && t->scalar_type() == type && t->is_cuda() && t->is_contiguous() &&
                 (!like || t->get_device() == like->get_device())
             ? t
             : nullptr;
}

// (sizes, m, v, step, ms or None, vs or None, master or None) -> where each tensor's part starts, or None where the
// states do not have these sizes
PyObject* adam_starts(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !PyList_Check(a[0])) return none();
  const Py_ssize_t count = PyList_GET_SIZE(a[0]);
  int64_t total = 0;
  PyObject* starts = PyList_New(count);
  if (!starts) return nullptr;
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyList_SET_ITEM(starts, i, PyLong_FromLongLong(total));
    const long long k = PyLong_AsLongLong(PyList_GET_ITEM(a[0], i));
    if (k < 0) {
      Py_DECREF(starts);
      return PyErr_Occurred() ? nullptr : none();
    }
    total += up(k, kGroup);
  }
  const at::Tensor* m = tensor(a[1]);
  const bool held = m && m->scalar_type() == at::kFloat8_e4m3fn;
  const auto type = held ? at::kFloat8_e4m3fn : at::kFloat;
  bool good = flat(a[1], total, type, nullptr) && flat(a[2], total, type, m) && flat(a[3], 2, at::kInt, m);
  for (int k : {4, 5})
    good = good && (held ? flat(a[k], total / kGroup, at::kFloat, m) != nullptr : a[k] == Py_None);
  good = good && (a[6] == Py_None || flat(a[6], total, at::kFloat, m));
  if (good) return starts;
  Py_DECREF(starts);
  return none();
  END_HANDLE_TH_ERRORS
}

// (params, grads, sizes, (m, v, step, ms, vs, master), lr, beta1, beta2, eps, weight_decay, max_norm or 0., follow) -> the
// gradients' norm, or True
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11 || !PyList_Check(a[0]) || !PyList_Check(a[1]) || !PyList_Check(a[2]) || !PyTuple_Check(a[3]) ||
      PyTuple_GET_SIZE(a[3]) != 6)
    return none();
  const Py_ssize_t count = PyList_GET_SIZE(a[0]);
  if (PyList_GET_SIZE(a[1]) != count || PyList_GET_SIZE(a[2]) != count) return none();
  const at::Tensor* s[6];
  for (int k = 0; k < 6; ++k) s[k] = tensor(PyTuple_GET_ITEM(a[3], k));
  if (!s[0] || !s[1] || !s[2] || !s[0]->is_cuda()) return none();
  const auto device = s[0]->device();
  c10::SmallVector<o1d_adamw_tensor_t, 128> list;
  c10::SmallVector<const at::Tensor*, 128> written;
  std::optional<o1d_dtype_t> pdt, gdt;
  int64_t start = 0;
  for (Py_ssize_t i = 0; i < count; ++i) {
    const at::Tensor* p = tensor(PyList_GET_ITEM(a[0], i));
    const long long size = PyLong_AsLongLong(PyList_GET_ITEM(a[2], i));
    PyObject* go = PyList_GET_ITEM(a[1], i);
    if (!p || size < 0 || p->numel() != size || p->device() != device || !p->is_contiguous()) return none();
    const auto t = type_of(*p);
    if (!t || (pdt && *pdt != *t)) return none();
    pdt = t;
    if (go != Py_None && size) {
      const at::Tensor* g = tensor(go);
      if (!g || g->sizes() != p->sizes() || g->device() != device || !g->is_contiguous()) return none();
      const auto u = type_of(*g);
      if (!u || (gdt && *gdt != *u)) return none();
      gdt = u;
      list.push_back({p->data_ptr(), g->data_ptr(), size, start});
      written.push_back(p);
    }
    start += up(size, kGroup);
  }
  if (s[0]->numel() != start || list.empty()) return none();
  const at::Tensor* lr = tensor(a[4]);
  if (lr && (lr->numel() != 1 || lr->scalar_type() != at::kFloat || lr->device() != device)) return none();
  double h[6];
  for (int k = 0; k < 6; ++k) {
    h[k] = k == 0 && lr ? 0. : PyFloat_AsDouble(a[4 + k]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      return none();
    }
  }
  auto data = [](const at::Tensor* t) { return t ? t->data_ptr() : nullptr; };
  const o1d_adamw_state_t state{data(s[0]), data(s[1]), (float*)data(s[3]), (float*)data(s[4]), (float*)data(s[5]),
                                (int*)data(s[2]), s[3] ? 8 : 32};
  const o1d_adamw_options_t options{h[0], h[1], h[2], h[3], h[4], h[5], (const float*)data(lr), a[10] == Py_True};
  at::Tensor norm, ws = space(p_adamw_bytes(h[5]), *s[0]);
  if (h[5] > 0.) norm = empty({}, *s[0], at::kFloat);
  const c10::DeviceGuard guard(device);
  void* stream = stream_of(*s[0]);
  const auto st = call([&] {
    return p_adamw(list.data(), (int)list.size(), *pdt, *gdt, &state, &options, norm.defined() ? (float*)norm.data_ptr() : nullptr,
                   ws.data_ptr(), (size_t)ws.numel(), stream);
  });
  if (st) return none();
  // (a backward that was recorded before the step refuses what it kept of them)
  for (const at::Tensor* p : written)
    if (!p->is_inference()) p->unsafeGetTensorImpl()->bump_version();
  if (norm.defined()) return wrap(norm);
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// (addresses of the twelve entry points, in the order above)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void** to[] = {(void**)&p_gn_fwd, (void**)&p_gn_fwd_bytes, (void**)&p_gn_bwd, (void**)&p_gn_bwd_bytes,
                 (void**)&p_pack, (void**)&p_pack_bytes, (void**)&p_fwd, (void**)&p_bwd_input,
                 (void**)&p_bwd_weight, (void**)&p_bwd_weight_bytes, (void**)&p_adamw, (void**)&p_adamw_bytes};
  if (n != (Py_ssize_t)(sizeof(to) / sizeof(to[0]))) {
    PyErr_SetString(PyExc_TypeError, "twelve addresses expected");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    *to[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  return none();
}

#define O1D_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {O1D_METHOD(gn_fwd),           O1D_METHOD(gn_bwd),            O1D_METHOD(pack),  O1D_METHOD(linear_fwd),
                         O1D_METHOD(linear_bwd_input), O1D_METHOD(linear_bwd_weight), O1D_METHOD(adamw), O1D_METHOD(adam_starts),
                         O1D_METHOD(bind),             {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train(void) { return PyModule_Create(&module); }
