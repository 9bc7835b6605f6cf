// tensors.cpp -- lists of tensors for the binding: a list of hundreds costs Python
// half a microsecond a tensor and check, more than the kernels of a small step take.
//
// gather(list, dims, dtype, device, table, stride, sizes) -> bool
//     writes each tensor's address to table[i * stride] (an address of int64 words)
//     and, with sizes, its number of elements to the word behind; False, if one is
//     not a contiguous tensor of this dtype on this GPU, or, where dims is not 0, not
//     of the sizes there (of each tensor how many, and the sizes)
// own(table, count, copies) -> int
//     of rows n, w, g, w_out, copy, ... (eight words): 0, or 1: two outputs begin at
//     the same address, 2: an output and a gradient, 3: an output and another
//     tensor's weight
// changed(list)
//     counts a change of each tensor (None is skipped), for autograd
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <vector>

namespace {

int64_t* words(PyObject* o) { return reinterpret_cast<int64_t*>(PyLong_AsUnsignedLongLong(o)); }

bool fits(PyObject* o, at::ScalarType dtype, long device, const int64_t** dims, at::Tensor* out) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.scalar_type() != dtype || t.layout() != at::kStrided || !t.is_contiguous())
    return false;
  if (*dims) {
    const int64_t n = *(*dims)++;
    if (t.dim() != n || !std::equal(t.sizes().begin(), t.sizes().end(), *dims)) return false;
    *dims += n;
  }
  *out = t;
  return true;
}

PyObject* gather(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 7 || !PyList_Check(arg[0]) || !THPDtype_Check(arg[2])) {
    PyErr_SetString(PyExc_TypeError, "gather(list, dims, dtype, device, table, stride, sizes)");
    return nullptr;
  }
  const int64_t* dims = words(arg[1]);
  const at::ScalarType dtype = reinterpret_cast<THPDtype*>(arg[2])->scalar_type;
  const long device = PyLong_AsLong(arg[3]), stride = PyLong_AsLong(arg[5]), sizes = PyLong_AsLong(arg[6]);
  int64_t* table = words(arg[4]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const Py_ssize_t count = PyList_GET_SIZE(arg[0]);
    at::Tensor t;
    for (Py_ssize_t i = 0; i < count; ++i) {
      if (!fits(PyList_GET_ITEM(arg[0], i), dtype, device, &dims, &t)) Py_RETURN_FALSE;
      table[i * stride] = reinterpret_cast<int64_t>(t.data_ptr());
      if (sizes) table[i * stride + 1] = t.numel();
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  Py_RETURN_TRUE;
}

PyObject* own(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "own(table, count, copies)");
    return nullptr;
  }
  const int64_t* table = words(arg[0]);
  const long count = PyLong_AsLong(arg[1]), copies = PyLong_AsLong(arg[2]);
  if (PyErr_Occurred()) return nullptr;
  try {
    std::vector<int64_t> outs;
    outs.reserve(2 * count);
    for (long i = 0; i < count; ++i) {
      const int64_t* r = table + 8 * i;
      if (!r[0]) continue;
      outs.push_back(r[3]);
      if (copies) outs.push_back(r[4]);
    }
    std::sort(outs.begin(), outs.end());
    if (std::adjacent_find(outs.begin(), outs.end()) != outs.end()) return PyLong_FromLong(1);
    auto in = [&](int64_t p) { return std::binary_search(outs.begin(), outs.end(), p); };
    for (long i = 0; i < count; ++i) {
      const int64_t* r = table + 8 * i;
      if (!r[0]) continue;
      if (in(r[2])) return PyLong_FromLong(2);
      if (r[1] != r[3] && in(r[1])) return PyLong_FromLong(3);
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  return PyLong_FromLong(0);
}

PyObject* changed(PyObject*, PyObject* list) {
  if (!PyList_Check(list)) {
    PyErr_SetString(PyExc_TypeError, "changed(list)");
    return nullptr;
  }
  try {
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
      PyObject* o = PyList_GET_ITEM(list, i);
      if (o == Py_None) continue;
      if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "changed(list of tensors)");
        return nullptr;
      }
      const at::Tensor& t = THPVariable_Unpack(o);
      if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gather)), METH_FASTCALL, "addresses of a list of tensors"},
                         {"own", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(own)), METH_FASTCALL, "whether outputs are each their own"},
                         {"changed", changed, METH_O, "counts a change of each tensor"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "lists of tensors for the binding", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
