// The binding's host half, the module `_tensors` of the package: a table of many tensors, several outputs allocated at
// once, and the training operators' calls whole (checks, outputs, workspace, entry point) for the plain case, in which a
// small call's time is the host's. A call that is not plain (an argument of another type, shape, layout or device), or that
// the entry point's checks refuse, gives None and leaves nothing behind: the Python binding then takes it, and says what is
// wrong with it. A failed launch raises the binding's error here and is not made again: part of its work may be on the
// stream. Plain host code against torch's C++ interface.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstring>
#include <vector>

#include "maestro_train.h"

namespace {

constexpr int32_t kF32 = MAESTRO_F32, kBf16 = MAESTRO_BF16;

PyObject* bytes_of(const void* p, size_t n) {
  return PyBytes_FromStringAndSize(static_cast<const char*>(p), static_cast<Py_ssize_t>(n));
}

// table(tensors: list, name: str) -> (addresses int64, element counts int64, maestro_dtype int32), each as bytes
PyObject* table(PyObject*, PyObject* args) {
  PyObject* list;
  const char* name;
  if (!PyArg_ParseTuple(args, "O!s", &PyList_Type, &list, &name)) return nullptr;
  HANDLE_TH_ERRORS
  const Py_ssize_t n = PyList_GET_SIZE(list);
  std::vector<int64_t> at(n), size(n);
  std::vector<int32_t> code(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* o = PyList_GET_ITEM(list, i);
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda())
      return PyErr_Format(PyExc_TypeError, "%s must be CUDA (HIP) tensors", name);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || !t.is_contiguous())
      return PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16)
      return PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %s", name, c10::toString(t.scalar_type()));
    at[i] = reinterpret_cast<int64_t>(t.data_ptr());
    size[i] = t.numel();
    code[i] = t.scalar_type() == at::kFloat ? kF32 : kBf16;
  }
  return Py_BuildValue("NNN", bytes_of(at.data(), n * sizeof(int64_t)), bytes_of(size.data(), n * sizeof(int64_t)),
                       bytes_of(code.data(), n * sizeof(int32_t)));
  END_HANDLE_TH_ERRORS
}

// empties(like: tensor, *(shape: tuple, type: int) or None) -> tuple of uninitialised tensors on like's device, None where
// None was given; type 0: float32, 1: int32, 2: like's
PyObject* empties(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 1 || !THPVariable_Check(args[0])) return PyErr_Format(PyExc_TypeError, "a tensor is needed");
  HANDLE_TH_ERRORS
  THPObjectPtr out(PyTuple_New(n - 1));
  if (!out) return nullptr;
  const at::Tensor& like = THPVariable_Unpack(args[0]);
  const at::TensorOptions on = at::TensorOptions().device(like.device());
  for (Py_ssize_t i = 1; i < n; ++i) {
    if (args[i] == Py_None) {
      Py_INCREF(Py_None);
      PyTuple_SET_ITEM(out.get(), i - 1, Py_None);
      continue;
    }
    if (!PyTuple_Check(args[i]) || PyTuple_GET_SIZE(args[i]) != 2 || !PyTuple_Check(PyTuple_GET_ITEM(args[i], 0)))
      return PyErr_Format(PyExc_TypeError, "(shape, type) is needed");
    PyObject* shape = PyTuple_GET_ITEM(args[i], 0);
    const long type = PyLong_AsLong(PyTuple_GET_ITEM(args[i], 1));
    const Py_ssize_t dims = PyTuple_GET_SIZE(shape);
    if (dims > 2) return PyErr_Format(PyExc_ValueError, "at most two dimensions");
    int64_t size[2];
    for (Py_ssize_t d = 0; d < dims; ++d) size[d] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, d));
    if (PyErr_Occurred()) return nullptr;
    if (type < 0 || type > 2) return PyErr_Format(PyExc_ValueError, "type must be 0, 1 or 2");
    const at::ScalarType dtype = type == 0 ? at::kFloat : type == 1 ? at::kInt : like.scalar_type();
    PyObject* t = THPVariable_Wrap(at::empty(c10::IntArrayRef(size, static_cast<size_t>(dims)), on.dtype(dtype)));
    if (!t) return nullptr;
    PyTuple_SET_ITEM(out.get(), i - 1, t);
  }
  return out.release();
  END_HANDLE_TH_ERRORS
}

// --- whole calls ------------------------------------------------------------------------------------

struct Entries {
  decltype(&maestro_layer) layer;
  decltype(&maestro_layer_grad_workspace) layer_grad_workspace;
  decltype(&maestro_layer_grad) layer_grad;
  decltype(&maestro_logprobs_workspace) logprobs_workspace;
  decltype(&maestro_logprobs) logprobs;
  decltype(&maestro_logprobs_grad) logprobs_grad;
  decltype(&maestro_clip_gradients_workspace) clip_workspace;
  decltype(&maestro_clip_gradients) clip;
} entries;
PyObject* error;                     // the binding's exception of (entry point, status)

// bind(layer, layer_grad_workspace, ..., error): the addresses of libmaestro.so's entry points, in the order of Entries,
// and the exception that a failed launch raises
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* at[8];
  static_assert(sizeof(at) == sizeof(entries), "one address an entry point");
  if (n != 9 || !PyExceptionClass_Check(args[8])) return PyErr_Format(PyExc_TypeError, "eight addresses and an exception are needed");
  for (int i = 0; i < 8; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  memcpy(&entries, at, sizeof(at));
  Py_INCREF(args[8]);
  Py_XSETREF(error, args[8]);
  Py_RETURN_NONE;
}

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
bool strided(const at::Tensor* t) { return t && t->is_cuda() && t->layout() == at::kStrided; }
bool is(const at::Tensor* t, at::ScalarType type, at::IntArrayRef shape) {
  return strided(t) && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
}
// given: None, or a tensor as is() wants it; `t` is nullptr for None
bool given(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor*& t) {
  t = o == Py_None ? nullptr : tensor(o);
  return o == Py_None || is(t, type, shape);
}
void* at_of(const at::Tensor* t) { return t && t->defined() ? t->data_ptr() : nullptr; }
int32_t code_of(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? kF32 : t.scalar_type() == at::kBFloat16 ? kBf16 : -1; }

at::Tensor fresh(const at::Tensor& like, at::ScalarType type, at::IntArrayRef shape) {
  return at::empty(shape, at::TensorOptions().device(like.device()).dtype(type));
}
at::Tensor scratch(const at::Tensor& like, size_t bytes) {
  return bytes ? fresh(like, at::kByte, {static_cast<int64_t>(bytes)}) : at::Tensor();
}
PyObject* wrap(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

template <class F>
maestro_status unlocked(const F& f) {
  maestro_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return st;
}

// The result of a call that `entry` did not take: None, for the binding, where its checks refused it.
PyObject* refused(const char* entry, maestro_status st) {
  if (st == MAESTRO_ERR_INVALID_ARG || st == MAESTRO_ERR_UNSUPPORTED || st == MAESTRO_ERR_WORKSPACE) Py_RETURN_NONE;
  THPObjectPtr e(PyObject_CallFunction(error, "si", entry, static_cast<int>(st)));
  if (e) PyErr_SetObject(error, e.get());
  return nullptr;
}

// x [n][d_in] and weight [d_out][d_in] of one type
bool layer_shapes(const at::Tensor* x, const at::Tensor* w) {
  if (!strided(x) || !strided(w) || x->dim() != 2 || w->dim() != 2 || code_of(*w) < 0) return false;
  return x->scalar_type() == w->scalar_type() && x->size(1) == w->size(1) && x->is_contiguous() && w->is_contiguous() &&
         w->size(0) <= INT32_MAX && w->size(1) <= INT32_MAX;
}

// layer(x, weight, bias, relu, stream)
PyObject* layer(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 5) return PyErr_Format(PyExc_TypeError, "five arguments are needed");
  HANDLE_TH_ERRORS
  const at::Tensor *x = tensor(a[0]), *w = tensor(a[1]), *b = tensor(a[2]);
  if (!layer_shapes(x, w) || !is(b, at::kFloat, {w->size(0)})) Py_RETURN_NONE;
  const int relu = PyObject_IsTrue(a[3]);
  void* stream = PyLong_AsVoidPtr(a[4]);
  if (PyErr_Occurred()) return nullptr;
  const int64_t n = x->size(0), o = w->size(0), i = w->size(1);
  const at::Tensor y = fresh(*x, x->scalar_type(), {n, o});
  void *xp = at_of(x), *wp = at_of(w), *yp = at_of(&y);
  const float* bp = static_cast<float*>(at_of(b));
  const maestro_status st = unlocked([&] { return entries.layer(n, i, o, code_of(*w), xp, wp, bp, relu, yp, stream); });
  if (st != MAESTRO_OK) return refused("maestro_layer", st);
  return wrap(y);
  END_HANDLE_TH_ERRORS
}

// layer_grad(x, weight, g_z, relu_input, want_x, stream) -> (g_x or None, g_weight, g_bias)
PyObject* layer_grad(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) return PyErr_Format(PyExc_TypeError, "six arguments are needed");
  HANDLE_TH_ERRORS
  const at::Tensor *x = tensor(a[0]), *w = tensor(a[1]), *gz = tensor(a[2]);
  if (!layer_shapes(x, w) || !is(gz, w->scalar_type(), {x->size(0), w->size(0)})) Py_RETURN_NONE;
  const int relu = PyObject_IsTrue(a[3]), want_x = PyObject_IsTrue(a[4]);
  void* stream = PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  const int64_t n = x->size(0), o = w->size(0), i = w->size(1);
  const int32_t code = code_of(*w);
  const at::Tensor gx = want_x ? fresh(*x, x->scalar_type(), {n, i}) : at::Tensor(), gw = fresh(*x, at::kFloat, {o, i}),
                   gb = fresh(*x, at::kFloat, {o});
  const size_t need = entries.layer_grad_workspace(n, i, o, code);
  const at::Tensor work = scratch(*x, need);
  void *xp = at_of(x), *wp = at_of(w), *gp = at_of(gz), *gxp = at_of(&gx), *workp = at_of(&work);
  float *gwp = static_cast<float*>(at_of(&gw)), *gbp = static_cast<float*>(at_of(&gb));
  const maestro_status st = unlocked([&] { return entries.layer_grad(n, i, o, code, xp, wp, gp, relu, gxp, gwp, gbp, workp, need, stream); });
  if (st != MAESTRO_OK) return refused("maestro_layer_grad", st);
  return Py_BuildValue("NNN", wrap(gx), wrap(gw), wrap(gb));
  END_HANDLE_TH_ERRORS
}

// rows of [n][v] that are contiguous and do not overlap, and their stride
bool rows(const at::Tensor* t, int64_t& stride) {
  if (!strided(t) || code_of(*t) < 0 || t->dim() != 2) return false;
  const int64_t n = t->size(0), v = t->size(1);
  if (v < 1 || v > INT32_MAX) return false;
  stride = n <= 1 ? v : t->stride(0);
  return (v == 1 || t->stride(1) == 1) && stride >= v;
}

// logprobs(logits, token or None, k, want_entropy, want_stats, stream) -> (logprob or None, entropy or None, top_id, top_logprob, stats or None)
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) return PyErr_Format(PyExc_TypeError, "six arguments are needed");
  HANDLE_TH_ERRORS
  const at::Tensor *x = tensor(a[0]), *token;
  int64_t stride;
  if (!rows(x, stride) || !PyLong_Check(a[2])) Py_RETURN_NONE;
  const int64_t n = x->size(0), v = x->size(1);
  if (!given(a[1], at::kInt, {n}, token)) Py_RETURN_NONE;
  const long k = PyLong_AsLong(a[2]);
  const int want_entropy = PyObject_IsTrue(a[3]), want_stats = PyObject_IsTrue(a[4]);
  void* stream = PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  if (k < 0 || k > MAESTRO_MAX_ALTERNATIVES) Py_RETURN_NONE;
  const at::Tensor lp = token ? fresh(*x, at::kFloat, {n}) : at::Tensor(), h = want_entropy ? fresh(*x, at::kFloat, {n}) : at::Tensor(),
                   id = fresh(*x, at::kInt, {n, k}), top = fresh(*x, at::kFloat, {n, k}),
                   stats = want_stats ? fresh(*x, at::kFloat, {n, 2}) : at::Tensor();
  const int32_t code = code_of(*x);
  const size_t need = entries.logprobs_workspace(n, v, k, code);
  const at::Tensor work = scratch(*x, need);
  void *xp = at_of(x), *workp = at_of(&work);
  auto f = [](const at::Tensor& t) { return static_cast<float*>(at_of(&t)); };
  const int32_t* tp = static_cast<int32_t*>(at_of(token));
  int32_t* idp = static_cast<int32_t*>(at_of(&id));
  float *lpp = f(lp), *hp = f(h), *topp = f(top), *sp = f(stats);
  const maestro_status st = unlocked([&] { return entries.logprobs(n, v, xp, stride, code, tp, k, lpp, hp, idp, topp, sp, workp, need, stream); });
  if (st != MAESTRO_OK) return refused("maestro_logprobs", st);
  return Py_BuildValue("NNNNN", wrap(lp), wrap(h), wrap(id), wrap(top), wrap(stats));
  END_HANDLE_TH_ERRORS
}

// logprobs_grad(logits, token or None, stats, entropy or None, g_logprob or None, g_entropy or None, stream)
PyObject* logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 7) return PyErr_Format(PyExc_TypeError, "seven arguments are needed");
  HANDLE_TH_ERRORS
  const at::Tensor *x = tensor(a[0]), *token, *stats = tensor(a[2]), *h, *g, *ge;
  int64_t stride;
  if (!rows(x, stride)) Py_RETURN_NONE;
  const int64_t n = x->size(0), v = x->size(1);
  if (!given(a[1], at::kInt, {n}, token) || !is(stats, at::kFloat, {n, 2}) || !given(a[3], at::kFloat, {n}, h) ||
      !given(a[4], at::kFloat, {n}, g) || !given(a[5], at::kFloat, {n}, ge))
    Py_RETURN_NONE;
  if (!token != !g || (!g && !ge) || (ge && !h)) Py_RETURN_NONE;
  void* stream = PyLong_AsVoidPtr(a[6]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor out = fresh(*x, x->scalar_type(), {n, v});
  auto f = [](const at::Tensor* t) { return static_cast<float*>(at_of(t)); };
  void *xp = at_of(x), *op = at_of(&out);
  const int32_t* tp = static_cast<int32_t*>(at_of(token));
  const float *sp = f(stats), *hp = f(h), *gp = f(g), *gep = f(ge);
  const maestro_status st = unlocked([&] { return entries.logprobs_grad(n, v, xp, stride, code_of(*x), tp, sp, hp, gp, gep, op, v, stream); });
  if (st != MAESTRO_OK) return refused("maestro_logprobs_grad", st);
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

struct Table {
  std::vector<void*> at;
  std::vector<int64_t> size;
  std::vector<int32_t> code;
  bool fill(PyObject* list) {
    const Py_ssize_t n = PyList_GET_SIZE(list);
    at.reserve(n), size.reserve(n), code.reserve(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
      const at::Tensor* t = tensor(PyList_GET_ITEM(list, i));
      if (!strided(t) || code_of(*t) < 0 || !t->is_contiguous()) return false;
      at.push_back(t->data_ptr()), size.push_back(t->numel()), code.push_back(code_of(*t));
    }
    return true;
  }
};

// clip(tensors: list, max_norm: float, out: list or None, stream) -> norm
PyObject* clip(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 4) return PyErr_Format(PyExc_TypeError, "four arguments are needed");
  HANDLE_TH_ERRORS
  if (!PyList_Check(a[0]) || !PyFloat_Check(a[1]) || (a[2] != Py_None && !PyList_Check(a[2]))) Py_RETURN_NONE;
  Table in, out;
  if (!in.fill(a[0]) || in.at.empty() || in.at.size() > INT32_MAX) Py_RETURN_NONE;
  if (a[2] != Py_None && (!out.fill(a[2]) || out.size != in.size || out.code != in.code)) Py_RETURN_NONE;
  const float max_norm = static_cast<float>(PyFloat_AS_DOUBLE(a[1]));
  void* stream = PyLong_AsVoidPtr(a[3]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor& like = *tensor(PyList_GET_ITEM(a[0], 0));
  const int32_t n = static_cast<int32_t>(in.at.size());
  const size_t need = entries.clip_workspace(n);
  const at::Tensor norm = fresh(like, at::kFloat, {1}), work = scratch(like, need);
  float* np = static_cast<float*>(at_of(&norm));
  void* workp = at_of(&work);
  void* const* op = a[2] != Py_None ? out.at.data() : nullptr;
  const maestro_status st = unlocked([&] { return entries.clip(n, in.at.data(), op, in.size.data(), in.code.data(), max_norm, np, workp, need, stream); });
  if (st != MAESTRO_OK) return refused("maestro_clip_gradients", st);
  return wrap(norm);
  END_HANDLE_TH_ERRORS
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    {"table", table, METH_VARARGS, "addresses, sizes and dtype codes of contiguous float32 or bfloat16 tensors on a GPU"},
    FAST(empties), FAST(bind), FAST(layer), FAST(layer_grad), FAST(logprobs), FAST(logprobs_grad), FAST(clip),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() {
  PyObject* m = PyModule_Create(&module);
  // the torch whose interface this was compiled against: the binding refuses another
  if (m && PyModule_AddStringConstant(m, "torch_version", MAESTRO_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
