// Argument marshalling for the calls that take a list of tensors: reads address, size, type and
// layout of every torch tensor of a Python list and hands the descriptors to the C ABI
// (include/efcp.h).  A model has hundreds of gradients; in Python the same takes longer than
// the kernels of a small model.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "efcp.h"

namespace {

enum class Use { kRead, kWrite, kGather };

// One entry of the list: a tensor on `device`, or the number of elements of an absent gradient.
// False with a Python error set when it is neither, or of a kind the library does not take.
bool describe(PyObject* o, long device, Use use, Py_ssize_t i, efcp_tensor* out) {
  const bool absent_ok = use == Use::kGather;
  if (!THPVariable_Check(o)) {
    if (!absent_ok || !PyLong_Check(o)) {
      PyErr_Format(PyExc_TypeError, "entry %zd is not a tensor%s", i,
                   absent_ok ? " (or an element count)" : "");
      return false;
    }
    const long long n = PyLong_AsLongLong(o);
    if (n == -1 && PyErr_Occurred()) return false;
    out->data = nullptr;
    out->numel = n;
    out->dtype = EFCP_F32;
    out->rank = 0;
    return true;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) {
    PyErr_Format(PyExc_ValueError, "entry %zd is not a dense tensor on cuda:%ld", i, device);
    return false;
  }
  switch (t.scalar_type()) {
    case at::kFloat: out->dtype = EFCP_F32; break;
    case at::kBFloat16: out->dtype = EFCP_BF16; break;
    case at::kHalf: out->dtype = EFCP_F16; break;
    default:
      PyErr_Format(PyExc_ValueError, "entry %zd: fp32, bfloat16 or fp16 expected", i);
      return false;
  }
  if (t.is_neg()) {
    PyErr_Format(PyExc_ValueError, "entry %zd is a lazily negated view", i);
    return false;
  }
  out->numel = t.numel();
  out->rank = 0;
  out->data = nullptr;
  if (out->numel && use == Use::kWrite) {
    out->data = t.mutable_data_ptr();
    t.unsafeGetTensorImpl()->bump_version();  // autograd's record of changes in place
  } else if (out->numel) {
    out->data = const_cast<void*>(t.const_data_ptr());
  }
  if (out->numel && !t.is_contiguous()) {
    const int64_t nd = t.dim();
    if (nd > EFCP_MAX_RANK) {
      PyErr_Format(PyExc_ValueError, "entry %zd: more than %d dimensions", i, EFCP_MAX_RANK);
      return false;
    }
    out->rank = int32_t(nd);
    for (int64_t k = 0; k < nd; ++k) {
      out->size[k] = t.size(k);
      out->stride[k] = t.stride(k);
    }
  }
  return true;
}

bool describe_list(PyObject* seq, long device, Use use, std::vector<efcp_tensor>* out) {
  if (!PyList_Check(seq) && !PyTuple_Check(seq)) {
    PyErr_SetString(PyExc_TypeError, "a list or tuple of tensors expected");
    return false;
  }
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject** items = PySequence_Fast_ITEMS(seq);
  out->resize(size_t(n));
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!describe(items[i], device, use, i, &(*out)[size_t(i)])) return false;
  return true;
}

void* ptr_of(unsigned long long v) { return reinterpret_cast<void*>(uintptr_t(v)); }

// Every function returns the EFCP_* code of the C call; no C++ exception leaves it.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

PyObject* grads_norm(PyObject*, PyObject* args) {
  PyObject* seq;
  long device;
  float scale;
  unsigned long long norm, ws, stream;
  if (!PyArg_ParseTuple(args, "OlfKKK", &seq, &device, &scale, &norm, &ws, &stream)) return nullptr;
  return guarded([&]() -> PyObject* {
    std::vector<efcp_tensor> list;
    if (!describe_list(seq, device, Use::kRead, &list)) return nullptr;
    return PyLong_FromLong(efcp_grads_norm(list.data(), int32_t(list.size()), scale,
                                           static_cast<float*>(ptr_of(norm)), ptr_of(ws),
                                           ptr_of(stream)));
  });
}

PyObject* grads_clip(PyObject*, PyObject* args) {
  PyObject* seq;
  long device;
  float max_norm, scale;
  unsigned long long norm, ws, stream;
  if (!PyArg_ParseTuple(args, "OlffKKK", &seq, &device, &max_norm, &scale, &norm, &ws, &stream))
    return nullptr;
  return guarded([&]() -> PyObject* {
    std::vector<efcp_tensor> list;
    if (!describe_list(seq, device, Use::kWrite, &list)) return nullptr;
    return PyLong_FromLong(efcp_grads_clip(list.data(), int32_t(list.size()), max_norm, scale,
                                           static_cast<float*>(ptr_of(norm)), ptr_of(ws),
                                           ptr_of(stream)));
  });
}

PyObject* grads_gather(PyObject*, PyObject* args) {
  PyObject* seq;
  long device;
  long long d;
  float max_norm, scale;
  unsigned long long flat, norm, ws, stream;
  if (!PyArg_ParseTuple(args, "OlKLffKKK", &seq, &device, &flat, &d, &max_norm, &scale, &norm, &ws,
                        &stream))
    return nullptr;
  return guarded([&]() -> PyObject* {
    std::vector<efcp_tensor> list;
    if (!describe_list(seq, device, Use::kGather, &list)) return nullptr;
    return PyLong_FromLong(efcp_grads_gather(list.data(), int32_t(list.size()),
                                             static_cast<float*>(ptr_of(flat)), d, max_norm, scale,
                                             static_cast<float*>(ptr_of(norm)), ptr_of(ws),
                                             ptr_of(stream)));
  });
}

PyMethodDef methods[] = {
    {"grads_norm", grads_norm, METH_VARARGS, "efcp_grads_norm on a list of tensors"},
    {"grads_clip", grads_clip, METH_VARARGS, "efcp_grads_clip on a list of tensors"},
    {"grads_gather", grads_gather, METH_VARARGS, "efcp_grads_gather on a list of tensors"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
