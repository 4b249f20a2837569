// What the binding does for every tensor of a call, where Python takes longer over it than the GPU over the work: a
// table of many tensors, and several outputs allocated at once. Plain host code against torch's C++ interface; the
// module `_tensors` of the package.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <vector>

namespace {

constexpr int32_t kF32 = 0, kBf16 = 1;      // maestro_dtype

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

PyMethodDef methods[] = {
    {"table", table, METH_VARARGS, "addresses, sizes and dtype codes of contiguous float32 or bfloat16 tensors on a GPU"},
    {"empties", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(empties)), METH_FASTCALL, "several uninitialised tensors"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
