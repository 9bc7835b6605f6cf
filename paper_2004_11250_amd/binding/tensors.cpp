// tensors.cpp -- lists of tensors for the binding: a list of hundreds costs Python
// half a microsecond a tensor and check, more than the kernels of a small step take.
//
// Addresses of the library's functions and of memory come as numbers.  A list "fits"
// if its tensors are contiguous, of the dtype and on the GPU that is asked for, and,
// where dims is not 0, of the sizes there (of each tensor how many, and the sizes).
//
// adamw(lists, dtypes, device, dims, table, fn, desc, stream, buffers) -> int
//     lists: weights, grads, new weights and copies (None: weights; none), of the
//     table's length; their addresses go to the table (rows n, w, g, w_out, copy, ...
//     of eight int64), and fn is pp_adamw_step.  Counts a change of what was written,
//     the buffers among it.  0; 1: two outputs begin at the same address, 2: an output
//     and a gradient, 3: an output and another tensor's weight; 10 + k: list k does
//     not fit; a pp_status
// grad_norm(list, dtype, device, max_norm, workspace_fn, fn, stream) -> (norm, scale)
//     with pp_grad_norm_workspace and pp_grad_norm; 10: the list does not fit; a pp_status
// own(table, rows, copies) -> int
//     0 to 3 as above, of a filled table
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ops/empty.h>
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

// addresses of a list's tensors to table[stride i] (and their elements behind them)
bool gather(PyObject* list, at::ScalarType dtype, long device, const int64_t* dims, int64_t* table, Py_ssize_t stride, bool sizes) {
  at::Tensor t;
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
    if (!fits(PyList_GET_ITEM(list, i), dtype, device, &dims, &t)) return false;
    table[i * stride] = reinterpret_cast<int64_t>(t.data_ptr());
    if (sizes) table[i * stride + 1] = t.numel();
  }
  return true;
}

// 0, or which rule the outputs break
int own_of(const int64_t* table, Py_ssize_t count, bool copies) {
  std::vector<int64_t> outs;
  outs.reserve(2 * count);
  for (Py_ssize_t i = 0; i < count; ++i) {
    const int64_t* r = table + 8 * i;
    if (!r[0]) continue;
    outs.push_back(r[3]);
    if (copies) outs.push_back(r[4]);
  }
  std::sort(outs.begin(), outs.end());
  if (std::adjacent_find(outs.begin(), outs.end()) != outs.end()) return 1;
  auto in = [&](int64_t p) { return std::binary_search(outs.begin(), outs.end(), p); };
  for (Py_ssize_t i = 0; i < count; ++i) {
    const int64_t* r = table + 8 * i;
    if (!r[0]) continue;
    if (in(r[2])) return 2;
    if (r[1] != r[3] && in(r[1])) return 3;
  }
  return 0;
}

void bump(PyObject* o) {
  if (o == Py_None || !THPVariable_Check(o)) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

PyObject* refuse(const char* what) {
  PyErr_SetString(PyExc_TypeError, what);
  return nullptr;
}

// f(), whose C++ exceptions become Python's
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* adamw(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 9 || !PyTuple_Check(arg[0]) || PyTuple_GET_SIZE(arg[0]) != 4 || !PyTuple_Check(arg[1]) || PyTuple_GET_SIZE(arg[1]) != 2 ||
      !PyBytes_Check(arg[6]) || !PyTuple_Check(arg[8]))
    return refuse("adamw(lists, dtypes, device, dims, table, fn, desc, stream, buffers)");
  PyObject* lists[4];
  at::ScalarType dtypes[4];
  for (int k = 0; k < 4; ++k) {
    lists[k] = PyTuple_GET_ITEM(arg[0], k);
    if (!(k > 1 && lists[k] == Py_None) && (!PyList_Check(lists[k]) || PyList_GET_SIZE(lists[k]) != PyList_GET_SIZE(lists[0])))
      return refuse("lists of one length");
  }
  for (int k = 0; k < 2; ++k) {
    PyObject* o = PyTuple_GET_ITEM(arg[1], k);
    if (!THPDtype_Check(o)) return refuse("two dtypes");
    dtypes[k] = reinterpret_cast<THPDtype*>(o)->scalar_type;
  }
  dtypes[2] = dtypes[0], dtypes[3] = at::kBFloat16;
  const long device = PyLong_AsLong(arg[2]);
  const int64_t* dims = words(arg[3]);
  int64_t* table = words(arg[4]);
  auto fn = reinterpret_cast<int32_t (*)(const void*, int32_t, const void*, void*)>(words(arg[5]));
  void* stream = words(arg[7]);
  if (PyErr_Occurred()) return nullptr;
  return guarded([&]() -> PyObject* {
    const Py_ssize_t count = PyList_GET_SIZE(lists[0]);
    for (int k = 0; k < 4; ++k)
      if (lists[k] != Py_None && !gather(lists[k], dtypes[k], device, dims, table + 1 + k, 8, false)) return PyLong_FromLong(10 + k);
    if (lists[2] == Py_None)
      for (Py_ssize_t i = 0; i < count; ++i) table[8 * i + 3] = table[8 * i + 1];
    const int wrong = own_of(table, count, lists[3] != Py_None);
    if (wrong) return PyLong_FromLong(wrong);
    const int32_t status = fn(table, static_cast<int32_t>(count), PyBytes_AS_STRING(arg[6]), stream);
    if (status) return PyLong_FromLong(status);
    for (PyObject* list : {lists[2] == Py_None ? lists[0] : lists[2], lists[3]})
      if (list != Py_None)
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) bump(PyList_GET_ITEM(list, i));
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(arg[8]); ++i) bump(PyTuple_GET_ITEM(arg[8], i));
    return PyLong_FromLong(0);
  });
}

PyObject* grad_norm(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 7 || !PyList_Check(arg[0]) || !THPDtype_Check(arg[1]))
    return refuse("grad_norm(list, dtype, device, max_norm, workspace_fn, fn, stream)");
  const at::ScalarType dtype = reinterpret_cast<THPDtype*>(arg[1])->scalar_type;
  const long device = PyLong_AsLong(arg[2]);
  const double most = PyFloat_AsDouble(arg[3]);
  auto need = reinterpret_cast<int32_t (*)(const void*, int32_t, int32_t, size_t*)>(words(arg[4]));
  auto fn = reinterpret_cast<int32_t (*)(const void*, int32_t, int32_t, float, float*, void*, size_t, void*)>(words(arg[5]));
  void* stream = words(arg[6]);
  if (PyErr_Occurred()) return nullptr;
  return guarded([&]() -> PyObject* {
    const Py_ssize_t count = PyList_GET_SIZE(arg[0]);
    std::vector<int64_t> table(2 * count + 2);
    if (!gather(arg[0], dtype, device, nullptr, table.data(), 2, true)) return PyLong_FromLong(10);
    const int32_t code = dtype == at::kBFloat16;
    size_t bytes = 0;
    int32_t status = need(table.data(), static_cast<int32_t>(count), code, &bytes);
    if (status) return PyLong_FromLong(status);
    const auto on = at::TensorOptions().device(at::kCUDA, static_cast<c10::DeviceIndex>(device));
    const at::Tensor both = at::empty({2}, on.dtype(at::kFloat));
    const at::Tensor ws = at::empty({static_cast<int64_t>(std::max<size_t>(bytes, 256))}, on.dtype(at::kByte));
    status = fn(table.data(), static_cast<int32_t>(count), code, static_cast<float>(most), both.data_ptr<float>(), ws.data_ptr(),
                static_cast<size_t>(ws.numel()), stream);
    if (status) return PyLong_FromLong(status);
    PyObject *x = THPVariable_Wrap(both.select(0, 0)), *y = THPVariable_Wrap(both.select(0, 1));
    PyObject* got = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return got;
  });
}

PyObject* own(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 3) return refuse("own(table, rows, copies)");
  const int64_t* table = words(arg[0]);
  const long count = PyLong_AsLong(arg[1]), copies = PyLong_AsLong(arg[2]);
  if (PyErr_Occurred()) return nullptr;
  return guarded([&] { return PyLong_FromLong(own_of(table, count, copies != 0)); });
}

template <class F>
PyCFunction method(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}
PyMethodDef methods[] = {{"adamw", method(adamw), METH_FASTCALL, "pp_adamw_step of lists of tensors"},
                         {"grad_norm", method(grad_norm), METH_FASTCALL, "pp_grad_norm of a list of tensors"},
                         {"own", method(own), METH_FASTCALL, "whether outputs are each their own"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "lists of tensors for the binding", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
