// Short way from Python to the operators on tensors: what gcpsl.py does for a
// call with regular arguments on the current stream, in one native call.  A
// small call is bound by the host, and there attribute by attribute in Python
// with a foreign call took 2 to 5 us of 6.5 to 11 beside the launch's 3.
//
// Every function returns its result, or None where an argument is not what it
// expects (gcpsl.py's own checks then say what is wrong, or take it), or the
// library's error code.  The library's entries are handed over by address, so
// that there is one copy of it in the process.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>

#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "../../include/gcpsl.h"

namespace {

using at::Tensor;

struct {
  decltype(&gcpsl_group_forward) group_forward;
  decltype(&gcpsl_group_input_grad) group_input_grad;
  decltype(&gcpsl_group_workspace_bytes) group_workspace_bytes;
  decltype(&gcpsl_group_weight_grad) group_weight_grad;
  decltype(&gcpsl_dropout) dropout;
  decltype(&gcpsl_score_workspace_bytes) score_workspace_bytes;
  decltype(&gcpsl_score) score;
  decltype(&gcpsl_score_grad) score_grad;
} entry;
PyObject *get_device, *get_stream;  // torch's own: the current device, a device's current stream as a number
PyTypeObject *scores_type;          // gcpsl.Scores

struct Irregular {};  // thrown: gcpsl.py takes the call

const Tensor &tensor(PyObject *o) {
  if (!THPVariable_Check(o)) throw Irregular();
  return THPVariable_Unpack(o);
}
const Tensor *optional(PyObject *o) { return o == Py_None ? nullptr : &tensor(o); }

long long integer(PyObject *o) {
  if (!PyLong_Check(o)) throw Irregular();
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow) throw Irregular();
  return v;
}
int32_t int32(int64_t v) {
  if (v < INT32_MIN || v > INT32_MAX) throw Irregular();
  return (int32_t)v;
}
uint64_t seed_of(PyObject *o) {
  if (!PyLong_Check(o)) throw Irregular();
  const uint64_t v = PyLong_AsUnsignedLongLong(o);
  if (PyErr_Occurred()) {  // negative or past 64 bits
    PyErr_Clear();
    throw Irregular();
  }
  return v;
}
double number(PyObject *o) {
  if (PyFloat_Check(o)) return PyFloat_AS_DOUBLE(o);
  return (double)integer(o);
}
long long result_of(PyObject *o) {  // of one of torch's functions
  if (!o) throw python_error();
  const long long v = PyLong_AsLongLong(o);
  Py_DECREF(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}

// Type, device and stream of a call, from its first tensor.
struct Call {
  at::ScalarType type;
  int32_t code;
  at::Device device;
  void *stream;
  explicit Call(const Tensor &t) : type(t.scalar_type()), code(type == at::kFloat ? GCPSL_F32 : GCPSL_BF16), device(t.device()) {
    if ((type != at::kFloat && type != at::kBFloat16) || !device.is_cuda()) throw Irregular();
    if (result_of(PyObject_CallNoArgs(get_device)) != device.index()) throw Irregular();
    PyObject *index = PyLong_FromLong(device.index());
    if (!index) throw python_error();
    PyObject *handle = PyObject_CallOneArg(get_stream, index);
    Py_DECREF(index);
    if (!handle) throw python_error();
    stream = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!stream && PyErr_Occurred()) throw python_error();
  }
  Tensor empty(at::IntArrayRef shape, at::ScalarType t) const {
    return at::empty(shape, at::TensorOptions().dtype(t).device(device));
  }
};

struct Rows {
  void *p;
  int64_t ld, rows, cols;
  Rows() : p(nullptr), ld(0), rows(0), cols(0) {}
  Rows(const Call &c, const Tensor &t) {
    if (t.dim() != 2 || t.scalar_type() != c.type || t.device() != c.device) throw Irregular();
    rows = t.size(0);
    cols = t.size(1);
    if (cols > 1 && t.stride(1) != 1) throw Irregular();
    ld = rows > 1 ? t.stride(0) : cols;
    p = t.data_ptr();
  }
  Rows(const Call &c, const Tensor &t, int64_t r, int64_t n) : Rows(c, t) {
    if (rows != r || cols != n) throw Irregular();
  }
};

// The result: `out`, or a new tensor.
Tensor result(const Call &c, PyObject *out, int64_t rows, int64_t cols, Rows &r) {
  Tensor t = out == Py_None ? c.empty({rows, cols}, c.type) : tensor(out);
  r = Rows(c, t, rows, cols);
  return t;
}

template <typename T> T *vector(const Call &c, const Tensor *t, at::ScalarType type, int64_t n) {
  if (!t) return nullptr;
  if (t->dim() != 1 || t->size(0) != n || t->scalar_type() != type || t->device() != c.device || !t->is_contiguous())
    throw Irregular();
  return (T *)t->data_ptr();
}

struct Groups {
  const int32_t *offsets;
  int32_t n;
  Groups(const Call &c, const Tensor &t) {
    if (t.dim() != 1 || t.size(0) < 2) throw Irregular();
    offsets = vector<int32_t>(c, &t, at::kInt, t.size(0));
    n = int32(t.size(0) - 1);
  }
};

// [G][n][k] weights or (k 0) [G][n] biases, a group's entries consecutive.
struct Weights {
  void *p = nullptr;
  int64_t stride = 0;
  Weights(const Call &c, const Tensor *t, at::ScalarType type, int64_t G, int64_t n, int64_t k) {
    if (!t) return;
    const bool matrix = k > 0;
    if (t->dim() != (matrix ? 3 : 2) || t->scalar_type() != type || t->device() != c.device || t->size(0) != G ||
        t->size(1) != n)
      throw Irregular();
    if (matrix && (t->size(2) != k || (n > 1 && t->stride(1) != k))) throw Irregular();
    if ((matrix ? k : n) > 1 && t->stride(matrix ? 2 : 1) != 1) throw Irregular();
    stride = G > 1 ? t->stride(0) : n * (matrix ? k : 1);
    p = t->data_ptr();
  }
};

// A library call without the interpreter's lock; its error code, if it gives one, ends the function.
struct Failed {
  int code;
};
template <typename F, typename... A> void call(F f, A... a) {
  int code;
  Py_BEGIN_ALLOW_THREADS
  code = f(a...);
  Py_END_ALLOW_THREADS
  if (code != GCPSL_OK) throw Failed{code};
}

// f's result with the three ways out.
template <typename F> PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
  HANDLE_TH_ERRORS
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", wanted, given);
    return nullptr;
  }
  try {
    return f();
  } catch (const Irregular &) {
    Py_RETURN_NONE;
  } catch (const Failed &e) {
    return PyLong_FromLong(e.code);
  }
  END_HANDLE_TH_ERRORS
}

// group_forward(x, offsets, w, bias, relu, p, seed, out)
PyObject *group_forward(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 8, [&] {
    const Tensor &xt = tensor(a[0]), &wt = tensor(a[2]);
    const Call c(xt);
    const Rows x(c, xt);
    const Groups g(c, tensor(a[1]));
    if (wt.dim() != 3 || x.cols < 1) throw Irregular();
    const int64_t n = wt.size(1);
    const Weights w(c, &wt, c.type, g.n, n, x.cols), b(c, optional(a[3]), at::kFloat, g.n, n, 0);
    const int relu = PyObject_IsTrue(a[4]);
    if (relu < 0) throw python_error();
    const double p = number(a[5]);
    const uint64_t seed = seed_of(a[6]);
    Rows y;
    const Tensor out = result(c, a[7], x.rows, n, y);
    call(entry.group_forward, c.code, g.n, x.rows, int32(n), int32(x.cols), g.offsets, x.p, x.ld, w.p, w.stride,
         (const float *)b.p, b.stride, relu, p, seed, y.p, y.ld, c.stream);
    return THPVariable_Wrap(out);
  });
}

// group_input_grad(dy, offsets, w, gate, p, out)
PyObject *group_input_grad(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 6, [&] {
    const Tensor &dt = tensor(a[0]), &wt = tensor(a[2]);
    const Call c(dt);
    const Rows dy(c, dt);
    const Groups g(c, tensor(a[1]));
    if (wt.dim() != 3 || wt.size(2) < 1) throw Irregular();
    const int64_t k = wt.size(2);
    const Weights w(c, &wt, c.type, g.n, dy.cols, k);
    const Tensor *gate = optional(a[3]);
    const Rows gt = gate ? Rows(c, *gate, dy.rows, k) : Rows();
    const double p = number(a[4]);
    Rows dx;
    const Tensor out = result(c, a[5], dy.rows, k, dx);
    call(entry.group_input_grad, c.code, g.n, dy.rows, int32(dy.cols), int32(k), g.offsets, dy.p, dy.ld, w.p, w.stride,
         gt.p, gt.ld, p, dx.p, dx.ld, c.stream);
    return THPVariable_Wrap(out);
  });
}

PyObject *tuple(std::initializer_list<const Tensor *> items, PyTypeObject *type) {
  const Py_ssize_t n = (Py_ssize_t)items.size();
  PyObject *t = type == &PyTuple_Type ? PyTuple_New(n) : type->tp_alloc(type, n);  // (a subclass of tuple)
  if (!t) throw python_error();
  Py_ssize_t i = 0;
  for (const Tensor *v : items) {
    PyObject *o = v ? THPVariable_Wrap(*v) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(t);
      throw python_error();
    }
    PyTuple_SET_ITEM(t, i++, o);
  }
  return t;
}

// group_weight_grad(dy, x, offsets, dw, db, bias)
PyObject *group_weight_grad(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 6, [&] {
    const Tensor &dt = tensor(a[0]), &xt = tensor(a[1]);
    const Call c(dt);
    const Rows dy(c, dt), x(c, xt);
    const Groups g(c, tensor(a[2]));
    const int64_t rows = dy.rows, n = dy.cols, k = x.cols;
    if (x.rows != rows || n < 1 || k < 1) throw Irregular();
    const int bias = PyObject_IsTrue(a[5]);
    if (bias < 0) throw python_error();
    const bool with_db = a[4] != Py_None || bias;
    size_t need = 0;
    call(entry.group_workspace_bytes, c.code, g.n, rows, int32(n), int32(k), &need);
    const Tensor dw = a[3] == Py_None ? c.empty({g.n, n, k}, at::kFloat) : tensor(a[3]);
    const Tensor db = a[4] != Py_None ? tensor(a[4]) : with_db ? c.empty({g.n, n}, at::kFloat) : Tensor();
    const Weights w(c, &dw, at::kFloat, g.n, n, k), b(c, with_db ? &db : nullptr, at::kFloat, g.n, n, 0);
    const Tensor work = need ? c.empty({(int64_t)need}, at::kByte) : Tensor();
    call(entry.group_weight_grad, c.code, g.n, rows, int32(n), int32(k), g.offsets, dy.p, dy.ld, x.p, x.ld, (float *)w.p,
         w.stride, (float *)b.p, b.stride, need ? work.data_ptr() : nullptr, need, c.stream);
    return tuple({&dw, with_db ? &db : nullptr}, &PyTuple_Type);
  });
}

// dropout(x, p, seed, out)
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 4, [&] {
    const Tensor &xt = tensor(a[0]);
    const Call c(xt);
    const Rows x(c, xt);
    const double p = number(a[1]);
    const uint64_t seed = seed_of(a[2]);
    Rows y;
    const Tensor out = result(c, a[3], x.rows, x.cols, y);
    call(entry.dropout, c.code, x.rows, x.cols, x.p, x.ld, p, seed, y.p, y.ld, c.stream);
    return THPVariable_Wrap(out);
  });
}

// Entries [first, ..) of a vector of 4-byte entries as a tensor of its own (five allocations took 1.3 us longer).
Tensor part(const Tensor &held, int64_t first, at::IntArrayRef shape, at::ScalarType type) {
  Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(held.storage()), held.key_set(),
                                                      c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_storage_offset(first);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  return t;
}

// score(logits, labels, top)
PyObject *score(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 3, [&] {
    const Tensor &zt = tensor(a[0]);
    const Call c(zt);
    const Rows z(c, zt);
    const int32_t *labels = vector<int32_t>(c, optional(a[1]), at::kInt, z.rows);
    const bool given = a[1] != Py_None;
    const int32_t top = int32(integer(a[2])), L = int32(z.cols);
    size_t need = 0;
    call(entry.score_workspace_bytes, c.code, z.rows, L, top, &need);  // (refuses a top that is not a size)
    const Tensor work = need ? c.empty({(int64_t)need}, at::kByte) : Tensor();
    const int64_t n = z.rows;
    const Tensor held = c.empty({n * (3 + 2 * (int64_t)top)}, at::kFloat);
    const Tensor logp = given ? part(held, 0, {n}, at::kFloat) : Tensor(), entropy = part(held, n, {n}, at::kFloat),
                 lse = part(held, 2 * n, {n}, at::kFloat), top_logp = part(held, 3 * n, {n, top}, at::kFloat),
                 top_class = part(held, (3 + top) * n, {n, top}, at::kInt);
    call(entry.score, c.code, z.rows, L, z.p, z.ld, labels, top, given ? (float *)logp.data_ptr() : nullptr,
         (float *)entropy.data_ptr(), (float *)lse.data_ptr(), (float *)top_logp.data_ptr(),
         (int32_t *)top_class.data_ptr(), need ? work.data_ptr() : nullptr, need, c.stream);
    return tuple({given ? &logp : nullptr, &entropy, &lse, &top_logp, &top_class}, scores_type);
  });
}

// score_grad(logits, labels, lse, entropy, g_logp, g_entropy, out)
PyObject *score_grad(PyObject *, PyObject *const *a, Py_ssize_t na) {
  return guarded(na, 7, [&] {
    const Tensor &zt = tensor(a[0]);
    const Call c(zt);
    const Rows z(c, zt);
    const auto row = [&](PyObject *o) { return (const float *)vector<float>(c, optional(o), at::kFloat, z.rows); };
    const int32_t *labels = vector<int32_t>(c, optional(a[1]), at::kInt, z.rows);
    const float *lse = row(a[2]), *entropy = row(a[3]), *g_logp = row(a[4]), *g_entropy = row(a[5]);
    Rows dz;
    const Tensor out = result(c, a[6], z.rows, z.cols, dz);
    call(entry.score_grad, c.code, z.rows, int32(z.cols), z.p, z.ld, labels, lse, entropy, g_logp, g_entropy, dz.p, dz.ld,
         c.stream);
    return THPVariable_Wrap(out);
  });
}

// init(entries' addresses in the order of `entry`, get_device, get_stream, Scores)
PyObject *init(PyObject *, PyObject *args) {
  PyObject *addresses, *device, *stream, *scores;
  if (!PyArg_ParseTuple(args, "O!OOO!", &PyTuple_Type, &addresses, &device, &stream, &PyType_Type, &scores)) return nullptr;
  void *p[sizeof(entry) / sizeof(void *)];
  constexpr Py_ssize_t n = sizeof(p) / sizeof(p[0]);
  if (PyTuple_GET_SIZE(addresses) != n || !PyType_IsSubtype((PyTypeObject *)scores, &PyTuple_Type)) {
    PyErr_SetString(PyExc_ValueError, "addresses of the entries and a tuple type expected");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (PyErr_Occurred()) return nullptr;
  }
  memcpy(&entry, p, sizeof(entry));
  get_device = Py_NewRef(device);  // kept for the process's life
  get_stream = Py_NewRef(stream);
  scores_type = (PyTypeObject *)Py_NewRef(scores);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, nullptr},
    {"group_forward", (PyCFunction)(void (*)(void))group_forward, METH_FASTCALL, nullptr},
    {"group_input_grad", (PyCFunction)(void (*)(void))group_input_grad, METH_FASTCALL, nullptr},
    {"group_weight_grad", (PyCFunction)(void (*)(void))group_weight_grad, METH_FASTCALL, nullptr},
    {"dropout", (PyCFunction)(void (*)(void))dropout, METH_FASTCALL, nullptr},
    {"score", (PyCFunction)(void (*)(void))score, METH_FASTCALL, nullptr},
    {"score_grad", (PyCFunction)(void (*)(void))score_grad, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() { return PyModule_Create(&module); }
