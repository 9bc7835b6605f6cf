// tensors.cpp -- calls of the binding whose checks cost Python more than the kernels
// take: lists of tensors (half a microsecond a tensor and check), and single tokens.
//
// Addresses of the library's functions come as numbers, tables as buffers of int64.  A
// list "fits" if its tensors are contiguous, of the dtype and on the device that is
// asked for, and, where dims is given, of the sizes there (of each tensor how many, and
// the sizes).
//
// adamw(lists, dtypes, device, dims, table, weight_decay, elements, buffers, desc, fn,
//       stream) -> int
//     lists: weights, grads, new weights, copies and tap masks (None: weights; none;
//     none, as may be one of the masks), of the table's length.  table: rows of
//     pp_adamw_tensor (weight_decay: of all, or None: the rows' own); desc: a
//     pp_adamw_desc without moments; buffers: m, v, m_scale and v_scale of the state
//     and of the new one, of `elements`; fn: pp_adamw_step.
//     Counts a change of what was written.  0; 1: two outputs begin at the same
//     address, 2: an output and a gradient, 3: an output and another tensor's weight;
//     10 + k: list k does not fit; 20: the buffers do not; 30: device is below 0 (the
//     CPU); a pp_status
// grad_norm(list, dtype, device, max_norm, workspace_fn, fn, stream) -> (norm, scale)
//     with pp_grad_norm_workspace and pp_grad_norm; 10: the list does not fit; a pp_status
// embed_fwd(ids, w, dtype, scale, ignore_index, fn, stream) -> features
//     with pp_embed_fwd, of contiguous tensors on one GPU, dtype None: w's
// embed_bwd(ids, dy, v, dtype, scale, ignore_index, add, workspace_fn, fn, stream)
//     -> gradient
//     with pp_embed_workspace and pp_embed_bwd, likewise (add: or None).  Both: None,
//     with nothing done, where an argument is another than these; a pp_status
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <limits>
#include <vector>

#include "pp.h"

namespace {

int64_t* words(PyObject* o) { return reinterpret_cast<int64_t*>(PyLong_AsUnsignedLongLong(o)); }

// What a buffer of int64 holds.
struct Words {
  Py_buffer b = {};
  explicit Words(PyObject* o) { PyObject_GetBuffer(o, &b, PyBUF_SIMPLE); }
  ~Words() { PyBuffer_Release(&b); }
  Words(const Words&) = delete;
  const int64_t* begin() const { return static_cast<const int64_t*>(b.buf); }
  Py_ssize_t size() const { return b.len / 8; }
};

// The GPU of a number, or the CPU.
at::Device on(long device) { return device < 0 ? at::Device(at::kCPU) : at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(device)); }

// A contiguous tensor of some axes, or nullptr.
const at::Tensor* whole(PyObject* o, int64_t least, int64_t most) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.layout() == at::kStrided && t.is_contiguous() && t.dim() >= least && t.dim() <= most ? &t : nullptr;
}

bool fits(PyObject* o, at::ScalarType dtype, at::Device device, const int64_t** dims, at::Tensor* out) {
  const at::Tensor* p = whole(o, 0, std::numeric_limits<int64_t>::max());
  if (!p || p->device() != device || p->scalar_type() != dtype) return false;
  const at::Tensor& t = *p;
  if (*dims) {
    const int64_t n = *(*dims)++;
    if (t.dim() != n || !std::equal(t.sizes().begin(), t.sizes().end(), *dims)) return false;
    *dims += n;
  }
  *out = t;
  return true;
}

constexpr Py_ssize_t kRow = sizeof(pp_adamw_tensor) / 8;   // words: n, w, g, w_out, copy, ...

// addresses of a list's tensors to table[stride i] (and their elements behind them)
bool gather(PyObject* list, at::ScalarType dtype, at::Device device, const int64_t* dims, int64_t* table, Py_ssize_t stride, bool sizes) {
  at::Tensor t;
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
    if (!fits(PyList_GET_ITEM(list, i), dtype, device, &dims, &t)) return false;
    table[i * stride] = reinterpret_cast<int64_t>(t.data_ptr());
    if (sizes) table[i * stride + 1] = t.numel();
  }
  return true;
}

// Whether a buffer has the sizes of `count` tensors.
bool sized(const Words& dims, Py_ssize_t count) {
  Py_ssize_t at = 0;
  for (Py_ssize_t i = 0; i < count; ++i) {
    if (at >= dims.size() || dims.begin()[at] < 0 || dims.begin()[at] > dims.size()) return false;
    at += 1 + dims.begin()[at];
  }
  return at <= dims.size();
}

// addresses of tap masks to the table: int16, of the first two sizes of a tensor that
// has nine values for each
bool masks(PyObject* list, at::Device device, const int64_t* dims, pp_adamw_tensor* table) {
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i, dims += dims[0] + 1) {
    PyObject* o = PyList_GET_ITEM(list, i);
    if (o == Py_None) continue;
    const at::Tensor* t = whole(o, 2, 2);
    if (!t || t->device() != device || t->scalar_type() != at::kShort || dims[0] < 2 || t->size(0) != dims[1] || t->size(1) != dims[2] ||
        table[i].n != 9 * t->numel())
      return false;
    table[i].keep = static_cast<const uint16_t*>(t->data_ptr());
  }
  return true;
}

// 0, or which rule the outputs break
int own_of(const int64_t* table, Py_ssize_t count, bool copies) {
  std::vector<int64_t> outs;
  outs.reserve(2 * count);
  for (Py_ssize_t i = 0; i < count; ++i) {
    const int64_t* r = table + kRow * i;
    if (!r[0]) continue;
    outs.push_back(r[3]);
    if (copies) outs.push_back(r[4]);
  }
  std::sort(outs.begin(), outs.end());
  if (std::adjacent_find(outs.begin(), outs.end()) != outs.end()) return 1;
  auto in = [&](int64_t p) { return std::binary_search(outs.begin(), outs.end(), p); };
  for (Py_ssize_t i = 0; i < count; ++i) {
    const int64_t* r = table + kRow * i;
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
  HANDLE_TH_ERRORS
  return f();
  END_HANDLE_TH_ERRORS
}

PyObject* adamw(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 11 || !PyTuple_Check(arg[0]) || PyTuple_GET_SIZE(arg[0]) != 5 || !PyTuple_Check(arg[1]) || PyTuple_GET_SIZE(arg[1]) != 2 ||
      !PyTuple_Check(arg[7]) || PyTuple_GET_SIZE(arg[7]) != 8 || !PyBytes_Check(arg[8]) || PyBytes_GET_SIZE(arg[8]) != sizeof(pp_adamw_desc))
    return refuse("adamw(lists, dtypes, device, dims, table, weight_decay, elements, buffers, desc, fn, stream)");
  PyObject* lists[5];
  at::ScalarType dtypes[4];
  for (int k = 0; k < 5; ++k) {
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
  const Words sizes(arg[3]), table_in(arg[4]);
  const double decay = arg[5] == Py_None ? 0. : PyFloat_AsDouble(arg[5]);
  const int64_t elements = PyLong_AsLongLong(arg[6]);
  auto fn = reinterpret_cast<decltype(&pp_adamw_step)>(words(arg[9]));
  void* stream = words(arg[10]);
  if (PyErr_Occurred()) return nullptr;
  const Py_ssize_t count = PyList_GET_SIZE(lists[0]);
  if (table_in.size() != kRow * count || !sized(sizes, count)) return refuse("tables of the lists' length");
  return guarded([&]() -> PyObject* {
    const int64_t* dims = sizes.begin();
    const auto* rows = reinterpret_cast<const pp_adamw_tensor*>(table_in.begin());
    pp_adamw_desc d;
    std::memcpy(&d, PyBytes_AS_STRING(arg[8]), sizeof(d));
    void* at[8] = {};
    for (int k = 0; k < 8; ++k) {
      PyObject* o = PyTuple_GET_ITEM(arg[7], k);
      const bool scale = k % 4 > 1;
      if (scale && d.bits == 32) {
        if (o != Py_None) return PyLong_FromLong(20);
        continue;
      }
      const at::Tensor* t = whole(o, 0, 64);
      const auto dtype = scale || d.bits == 32 ? at::kFloat : k % 4 ? at::kHalf : at::kFloat8_e4m3fn;
      if (!t || t->scalar_type() != dtype || t->device() != on(device) || t->numel() != (scale ? elements / PP_ADAMW_BLOCK : elements))
        return PyLong_FromLong(20);
      at[k] = t->data_ptr();
    }
    d.m = at[0], d.v = at[1], d.m_scale = static_cast<float*>(at[2]), d.v_scale = static_cast<float*>(at[3]);
    d.m_out = at[4], d.v_out = at[5], d.m_scale_out = static_cast<float*>(at[6]), d.v_scale_out = static_cast<float*>(at[7]);
    std::vector<pp_adamw_tensor> all(rows, rows + count);
    int64_t* table = reinterpret_cast<int64_t*>(all.data());
    for (int k = 0; k < 4; ++k)
      if (lists[k] != Py_None && !gather(lists[k], dtypes[k], on(device), dims, table + 1 + k, kRow, false)) return PyLong_FromLong(10 + k);
    if (lists[4] != Py_None && !masks(lists[4], on(device), dims, all.data())) return PyLong_FromLong(14);
    for (Py_ssize_t i = 0; i < count; ++i) {
      if (lists[2] == Py_None) table[kRow * i + 3] = table[kRow * i + 1];
      if (arg[5] != Py_None) all[i].weight_decay = decay;
    }
    const int wrong = own_of(table, count, lists[3] != Py_None);
    if (wrong) return PyLong_FromLong(wrong);
    if (device < 0) return PyLong_FromLong(30);
    const int32_t status = fn(all.data(), static_cast<int32_t>(count), &d, stream);
    if (status) return PyLong_FromLong(status);
    for (PyObject* list : {lists[2] == Py_None ? lists[0] : lists[2], lists[3]})
      if (list != Py_None)
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) bump(PyList_GET_ITEM(list, i));
    for (int k = 4; k < 8; ++k) bump(PyTuple_GET_ITEM(arg[7], k));
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
    if (!gather(arg[0], dtype, on(device), nullptr, table.data(), 2, true)) return PyLong_FromLong(10);
    const int32_t code = dtype == at::kBFloat16;
    size_t bytes = 0;
    int32_t status = need(table.data(), static_cast<int32_t>(count), code, &bytes);
    if (status) return PyLong_FromLong(status);
    const auto opt = at::TensorOptions().device(on(device));
    const at::Tensor both = at::empty({2}, opt.dtype(at::kFloat));
    const at::Tensor ws = at::empty({static_cast<int64_t>(std::max<size_t>(bytes, 256))}, opt.dtype(at::kByte));
    status = fn(table.data(), static_cast<int32_t>(count), code, static_cast<float>(most), both.data_ptr<float>(), ws.data_ptr(),
                static_cast<size_t>(ws.numel()), stream);
    if (status) return PyLong_FromLong(status);
    const at::AutoDispatchBelowADInplaceOrView plain;   // (no autograd's part of two views: 1 us)
    PyObject *x = THPVariable_Wrap(both.select(0, 0)), *y = THPVariable_Wrap(both.select(0, 1));
    PyObject* got = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return got;
  });
}

// Type code of float32 and bfloat16, or -1.
int code_of(at::ScalarType t) { return t == at::kBFloat16 ? PP_BF16 : t == at::kFloat ? PP_F32 : -1; }
int code_of(PyObject* dtype, int otherwise) {
  return dtype == Py_None ? otherwise : THPDtype_Check(dtype) ? code_of(reinterpret_cast<THPDtype*>(dtype)->scalar_type) : -1;
}

bool number(PyObject* o, float* x) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  const double d = PyFloat_AsDouble(o);
  *x = static_cast<float>(d);
  if (!PyErr_Occurred() && (std::abs(d) <= std::numeric_limits<float>::max() || !(std::abs(d) < std::numeric_limits<double>::infinity())))
    return true;
  PyErr_Clear();
  return false;
}
bool number(PyObject* o, int64_t* x) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *x = PyLong_AsLongLongAndOverflow(o, &over);
  return !over;
}

at::Tensor rows_of(at::IntArrayRef shape, int code, const at::Tensor& like) {
  return at::empty(shape, at::TensorOptions().device(like.device()).dtype(code == PP_BF16 ? at::kBFloat16 : at::kFloat));
}

PyObject* embed_fwd(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 7) return refuse("embed_fwd(ids, w, dtype, scale, ignore_index, fn, stream)");
  auto fn = reinterpret_cast<decltype(&pp_embed_fwd)>(words(arg[5]));
  void* stream = words(arg[6]);
  if (PyErr_Occurred()) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *ids = whole(arg[0], 0, 64), *w = whole(arg[1], 2, 2);
    pp_embed_desc d = {};
    if (!ids || !w || ids->scalar_type() != at::kLong || !ids->is_cuda() || ids->device() != w->device() || w->numel() == 0 ||
        (d.w_dtype = code_of(w->scalar_type())) < 0 || (d.y_dtype = code_of(arg[2], d.w_dtype)) < 0 || !number(arg[3], &d.scale) ||
        !number(arg[4], &d.ignore_index))
      Py_RETURN_NONE;
    d.t = ids->numel(), d.v = w->size(0), d.d = d.w_ld = d.y_ld = w->size(1);
    std::vector<int64_t> shape(ids->sizes().begin(), ids->sizes().end());
    shape.push_back(d.d);
    const at::Tensor y = rows_of(shape, d.y_dtype, *ids);
    const int32_t status = fn(&d, ids->data_ptr<int64_t>(), w->data_ptr(), y.data_ptr(), stream);
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(y);
  });
}

PyObject* embed_bwd(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  if (n != 10) return refuse("embed_bwd(ids, dy, v, dtype, scale, ignore_index, add, workspace_fn, fn, stream)");
  auto need = reinterpret_cast<decltype(&pp_embed_workspace)>(words(arg[7]));
  auto fn = reinterpret_cast<decltype(&pp_embed_bwd)>(words(arg[8]));
  void* stream = words(arg[9]);
  if (PyErr_Occurred()) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *ids = whole(arg[0], 0, 63), *dy = whole(arg[1], 1, 64);
    pp_embed_desc d = {};
    if (!ids || !dy || ids->scalar_type() != at::kLong || !ids->is_cuda() || ids->device() != dy->device() || dy->dim() != ids->dim() + 1 ||
        !std::equal(ids->sizes().begin(), ids->sizes().end(), dy->sizes().begin()) || dy->size(-1) < 1 || !number(arg[2], &d.v) || d.v < 1 ||
        (d.y_dtype = code_of(dy->scalar_type())) < 0 || (d.w_dtype = code_of(arg[3], d.y_dtype)) < 0 || !number(arg[4], &d.scale) ||
        !number(arg[5], &d.ignore_index))
      Py_RETURN_NONE;
    d.t = ids->numel(), d.d = d.w_ld = d.y_ld = dy->size(-1);
    const at::Tensor* add = nullptr;
    if (arg[6] != Py_None) {
      add = whole(arg[6], 2, 2);
      if (!add || add->device() != ids->device() || add->size(0) != d.v || add->size(1) != d.d ||
          (d.w_dtype = code_of(add->scalar_type())) < 0 || code_of(arg[3], d.w_dtype) != d.w_dtype)
        Py_RETURN_NONE;
    }
    size_t bytes = 0;
    int32_t status = need(&d, &bytes);
    if (status) return PyLong_FromLong(status);
    const at::Tensor dw = rows_of({d.v, d.d}, d.w_dtype, *ids);
    const at::Tensor ws = at::empty({static_cast<int64_t>(bytes)}, at::TensorOptions().device(ids->device()).dtype(at::kByte));
    status = fn(&d, ids->data_ptr<int64_t>(), dy->data_ptr(), add ? add->data_ptr() : nullptr, dw.data_ptr(), ws.data_ptr(), bytes, stream);
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(dw);
  });
}

template <class F>
PyCFunction method(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}
PyMethodDef methods[] = {{"adamw", method(adamw), METH_FASTCALL, "pp_adamw_step of lists of tensors"},
                         {"grad_norm", method(grad_norm), METH_FASTCALL, "pp_grad_norm of a list of tensors"},
                         {"embed_fwd", method(embed_fwd), METH_FASTCALL, "pp_embed_fwd of whole tensors"},
                         {"embed_bwd", method(embed_bwd), METH_FASTCALL, "pp_embed_bwd of whole tensors"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "lists of tensors for the binding", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
