// Argument marshalling for the calls on lists of gradients and on activations: checks torch tensors,
// makes the outputs and the scratch memory, and hands addresses and layouts to the C ABI
// (include/efcp.h) on the current stream.  The same in Python takes longer than the kernels of a
// small model: 23 us a call, 7 to 10 here, 3 to 10 on the device.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/InferenceMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <map>
#include <optional>
#include <utility>
#include <vector>

#include "efcp.h"

namespace {

// A refusal, raised as the Python exception of that kind.
struct Refused {
  PyObject* kind;
  std::string what;
};
[[noreturn]] void refuse(PyObject* kind, const std::string& what) { throw Refused{kind, what}; }
void require(bool ok, const char* what) {
  if (!ok) refuse(PyExc_ValueError, what);
}
struct PythonError {};  // one is set already

// No C++ exception leaves a function of this module.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const PythonError&) {
  } catch (const Refused& r) {
    PyErr_SetString(r.kind, r.what.c_str());
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* kind = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(kind ? kind : PyExc_RuntimeError, e.what_without_backtrace());
    Py_XDECREF(kind);
    Py_XDECREF(torch);
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

int dtype_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return EFCP_F32;
    case at::kBFloat16: return EFCP_BF16;
    case at::kHalf: return EFCP_F16;
    default: return -1;
  }
}

const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + ": a tensor expected");
  return THPVariable_Unpack(o);
}
// None: an empty optional
std::optional<at::Tensor> maybe_tensor(PyObject* o, const char* name) {
  if (o == Py_None) return std::nullopt;
  return tensor_of(o, name);
}

// Runs with the tensor's device current and knows its current stream.
struct Place {
  c10::cuda::CUDAGuard guard;
  c10::cuda::CUDAStream stream;
  explicit Place(c10::Device d)
      : guard(d), stream(c10::cuda::getCurrentCUDAStream(d.index())) {}

  // An output, without the way through the operators' dispatch (a call makes up to four).
  at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type = at::kFloat) const {
    return at::detail::empty_cuda(sizes, type, stream.device(), std::nullopt);
  }
  // Scratch memory until the end of the call, in the stream's order like a tensor's.
  c10::DataPtr scratch(int64_t bytes) const {
    return c10::cuda::CUDACachingAllocator::get()->allocate(size_t(bytes));
  }
};

// ------------------------------------------------------------------ lists of gradients
enum class Use { kRead, kWrite, kGather };

// One entry of the list: a tensor on `device`, or the number of elements of an absent gradient.
void describe(PyObject* o, c10::Device device, Use use, Py_ssize_t i, efcp_tensor* out) {
  const auto at = [&] { return "entry " + std::to_string(i) + ": "; };
  if (!THPVariable_Check(o)) {
    if (use != Use::kGather || !PyLong_Check(o))
      refuse(PyExc_TypeError, at() + (use == Use::kGather ? "a tensor or an element count expected"
                                                           : "a tensor expected"));
    const long long n = PyLong_AsLongLong(o);
    if (n == -1 && PyErr_Occurred()) throw PythonError{};
    out->data = nullptr;
    out->numel = n;
    out->dtype = EFCP_F32;
    out->rank = 0;
    return;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || t.device() != device)
    refuse(PyExc_ValueError, at() + "a dense tensor on " + device.str() + " expected");
  out->dtype = dtype_of(t);
  if (out->dtype < 0) refuse(PyExc_ValueError, at() + "fp32, bfloat16 or fp16 expected");
  if (t.is_neg()) refuse(PyExc_ValueError, at() + "a lazily negated view");
  out->numel = t.numel();
  out->rank = 0;
  out->data = nullptr;
  if (!out->numel) return;
  if (use == Use::kWrite) {
    if (t.is_inference() && !c10::InferenceMode::is_enabled())
      refuse(PyExc_RuntimeError, at() + "an inference tensor changed outside of inference mode");
    out->data = t.mutable_data_ptr();
  } else {
    out->data = const_cast<void*>(t.const_data_ptr());
  }
  if (!t.is_contiguous()) {
    const int64_t nd = t.dim();
    if (nd > EFCP_MAX_RANK) refuse(PyExc_ValueError, at() + "too many dimensions");
    out->rank = int32_t(nd);
    for (int64_t k = 0; k < nd; ++k) {
      out->size[k] = t.size(k);
      out->stride[k] = t.stride(k);
    }
  }
}

// Autograd's record of a change in place, once the call has succeeded.  (Inference tensors have none.)
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(const std::optional<at::Tensor>& t) {
  if (t) written(*t);
}

// The list's device: that of `first` if given, else of its first tensor, else the current one.
c10::Device list_device(PyObject* seq, const std::optional<at::Tensor>& first) {
  if (!PyList_Check(seq) && !PyTuple_Check(seq))
    refuse(PyExc_TypeError, "a list or tuple of tensors expected");
  c10::Device d(c10::kCUDA, 0);
  bool found = false;
  if (first) {
    d = first->device();
    found = true;
  }
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject** items = PySequence_Fast_ITEMS(seq);
  for (Py_ssize_t i = 0; i < n && !found; ++i) {
    if (THPVariable_Check(items[i])) {
      d = THPVariable_Unpack(items[i]).device();
      found = true;
    }
  }
  if (!found) d = c10::Device(c10::kCUDA, c10::cuda::current_device());
  require(d.is_cuda(), "CUDA tensors expected");
  return d;
}

std::vector<efcp_tensor> describe_list(PyObject* seq, c10::Device device, Use use) {
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject** items = PySequence_Fast_ITEMS(seq);
  std::vector<efcp_tensor> out{size_t(n)};
  for (Py_ssize_t i = 0; i < n; ++i) describe(items[i], device, use, i, &out[size_t(i)]);
  return out;
}

// Scratch memory for the list calls on one stream; a graph being captured gets its own, since it may be
// replayed on any stream.  (Never freed: streams live as long as the process.)
at::Tensor list_workspace(const Place& place) {
  static const int64_t bytes = efcp_grads_workspace_bytes();
  const auto fresh = [&] {
    return at::zeros({bytes}, at::TensorOptions().dtype(at::kByte).device(place.stream.device()));
  };
  if (c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None)
    return fresh();
  static auto* known = new std::map<std::pair<int, void*>, at::Tensor>;  // (under the GIL)
  at::Tensor& ws = (*known)[{place.stream.device_index(), place.stream.stream()}];
  if (!ws.defined()) ws = fresh();
  return ws;
}

at::Tensor norm_out(const std::optional<at::Tensor>& out, const Place& place) {
  if (!out) return place.empty({});
  require(out->scalar_type() == at::kFloat && out->numel() == 1 &&
              out->device() == place.stream.device(),
          "out: one fp32 value on the gradients' device expected");
  return *out;
}

// A tensor, or the EFCP_* code of the call when it is not EFCP_OK.
PyObject* result(int rc, const at::Tensor& t) {
  return rc == EFCP_OK ? THPVariable_Wrap(t) : PyLong_FromLong(rc);
}

PyObject* grads_norm(PyObject*, PyObject* args) {
  PyObject *seq, *out_;
  float scale;
  if (!PyArg_ParseTuple(args, "OfO", &seq, &scale, &out_)) return nullptr;
  return guarded([&] {
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, out));
    const auto list = describe_list(seq, place.stream.device(), Use::kRead);
    const at::Tensor norm = norm_out(out, place), ws = list_workspace(place);
    const int rc = efcp_grads_norm(list.data(), int32_t(list.size()), scale,
                                   norm.mutable_data_ptr<float>(), ws.mutable_data_ptr(),
                                   place.stream.stream());
    if (rc == EFCP_OK) written(out);
    return result(rc, norm);
  });
}

PyObject* grads_clip(PyObject*, PyObject* args) {
  PyObject *seq, *out_;
  float max_norm, scale;
  if (!PyArg_ParseTuple(args, "OffO", &seq, &max_norm, &scale, &out_)) return nullptr;
  return guarded([&] {
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, out));
    const auto list = describe_list(seq, place.stream.device(), Use::kWrite);
    const at::Tensor norm = norm_out(out, place), ws = list_workspace(place);
    const int rc = efcp_grads_clip(list.data(), int32_t(list.size()), max_norm, scale,
                                   norm.mutable_data_ptr<float>(), ws.mutable_data_ptr(),
                                   place.stream.stream());
    if (rc == EFCP_OK) {
      for (Py_ssize_t i = 0; i < Py_ssize_t(list.size()); ++i)
        if (list[size_t(i)].numel) written(THPVariable_Unpack(PySequence_Fast_GET_ITEM(seq, i)));
      written(out);
    }
    return result(rc, norm);
  });
}

PyObject* grads_gather(PyObject*, PyObject* args) {
  PyObject *seq, *flat_, *out_;
  float max_norm, scale;
  int want;
  if (!PyArg_ParseTuple(args, "OOffpO", &seq, &flat_, &max_norm, &scale, &want, &out_))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& flat = tensor_of(flat_, "flat");
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, flat));
    require(flat.scalar_type() == at::kFloat && flat.is_contiguous(),
            "flat: a contiguous fp32 tensor expected");
    const auto list = describe_list(seq, place.stream.device(), Use::kGather);
    at::Tensor norm, ws;
    if (want || out) norm = norm_out(out, place);
    if (norm.defined() || max_norm > 0.f) ws = list_workspace(place);
    const int rc = efcp_grads_gather(
        list.data(), int32_t(list.size()), flat.mutable_data_ptr<float>(), flat.numel(), max_norm,
        scale, norm.defined() ? norm.mutable_data_ptr<float>() : nullptr,
        ws.defined() ? ws.mutable_data_ptr() : nullptr, place.stream.stream());
    if (rc == EFCP_OK) {
      written(flat);
      written(out);
      if (!norm.defined()) Py_RETURN_NONE;
    }
    return result(rc, norm);
  });
}

// ------------------------------------------------------------------ group normalisation
struct Rows {
  int64_t batch, row;  // elements between samples and between positions
};

// Whether the channels of x (n, channels, *positions) lie side by side and its positions at one
// distance, and which.
std::optional<Rows> rows_of(const at::Tensor& x) {
  const int64_t channels = x.size(1);
  if (x.numel() == 0) return Rows{channels, channels};
  if (channels != 1 && x.stride(1) != 1) return std::nullopt;
  int64_t row = 0, count = 1;  // the merged positions so far, from the last dimension on
  for (int64_t k = x.dim() - 1; k >= 2; --k) {
    if (x.size(k) == 1) continue;
    if (count == 1) row = x.stride(k);
    else if (x.stride(k) != row * count) return std::nullopt;
    count *= x.size(k);
  }
  if (count == 1) row = channels;
  if (row < channels) return std::nullopt;
  return Rows{x.size(0) != 1 ? x.stride(0) : row * count, row};
}

// x itself, or a channels-last copy when its layout is another.
at::Tensor channels_last(const at::Tensor& x, Rows* rows) {
  if (const auto r = rows_of(x)) {
    *rows = *r;
    return x;
  }
  std::vector<int64_t> to{0}, back{0, x.dim() - 1};
  for (int64_t k = 2; k < x.dim(); ++k) {
    to.push_back(k);
    back.push_back(k - 1);
  }
  to.push_back(1);
  // (clone, not contiguous(): a tensor of overlapping rows may count as contiguous)
  const at::Tensor y = x.permute(to).clone(at::MemoryFormat::Contiguous).permute(back);
  *rows = *rows_of(y);
  return y;
}

// An empty channels-last tensor of x's shape and type.
at::Tensor new_channels_last(const at::Tensor& x, Rows* rows) {
  const int64_t nd = x.dim();
  std::vector<int64_t> strides(static_cast<size_t>(nd));
  int64_t step = x.size(1);
  for (int64_t k = nd - 1; k >= 2; --k) {
    strides[size_t(k)] = step;
    step *= x.size(k);
  }
  strides[0] = step;
  strides[1] = 1;
  *rows = Rows{step, x.size(1)};
  if (x.is_cuda())
    return at::detail::empty_strided_cuda(x.sizes(), strides, x.scalar_type(), x.device());
  return at::empty_strided(x.sizes(), strides, x.options());
}

efcp_group_norm group_norm_desc(const at::Tensor& x, int groups,
                                const std::optional<at::Tensor>& weight,
                                const std::optional<at::Tensor>& bias, float eps, const char* act) {
  require(x.layout() == at::kStrided && x.dim() >= 2 && dtype_of(x) >= 0 && !x.is_neg(),
          "x: (n, channels, ...) in fp32, bfloat16 or fp16 expected");
  require(x.is_cuda(), "x: a CUDA tensor expected");
  efcp_group_norm d{};
  d.act = !std::strcmp(act, "none")   ? EFCP_ACT_NONE
          : !std::strcmp(act, "relu") ? EFCP_ACT_RELU
          : !std::strcmp(act, "silu") ? EFCP_ACT_SILU
                                      : -1;
  require(d.act >= 0, "act: one of none, relu, silu expected");
  int param = -1;
  for (const auto* t : {&weight, &bias}) {
    if (!*t) continue;
    const at::Tensor& v = **t;
    const int dt = dtype_of(v);
    require(v.layout() == at::kStrided && v.device() == x.device() && dt >= 0 &&
                (param < 0 || dt == param) && v.numel() == x.size(1) && v.is_contiguous() &&
                !v.is_neg(),
            "weight, bias: contiguous, one value per channel, one type (fp32, bfloat16 or fp16), "
            "on x's device");
    param = dt;
  }
  d.n = x.size(0);
  d.channels = x.size(1);
  d.rows = 1;
  for (int64_t k = 2; k < x.dim(); ++k) d.rows *= x.size(k);
  d.groups = groups;
  d.dtype = dtype_of(x);
  d.param_dtype = param < 0 ? EFCP_F32 : param;
  d.eps = eps;
  return d;
}

const void* data_of(const std::optional<at::Tensor>& t) {
  return t ? t->const_data_ptr() : nullptr;
}

PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

PyObject* triple(int rc, const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
  if (rc != EFCP_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("(NNN)", wrap_or_none(a), wrap_or_none(b), wrap_or_none(c));
}

PyObject* group_norm_forward(PyObject*, PyObject* args) {
  PyObject *x_, *w_, *b_;
  int groups;
  float eps;
  const char* act;
  if (!PyArg_ParseTuple(args, "OiOOfs", &x_, &groups, &w_, &b_, &eps, &act)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& given = tensor_of(x_, "x");
    const auto weight = maybe_tensor(w_, "weight"), bias = maybe_tensor(b_, "bias");
    efcp_group_norm d = group_norm_desc(given, groups, weight, bias, eps, act);
    const Place place(given.device());
    const int64_t bytes = efcp_group_norm_workspace_bytes(&d, false);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    Rows in, out;
    const at::Tensor x = channels_last(given, &in), y = new_channels_last(x, &out);
    d.x_batch = in.batch;
    d.x_row = in.row;
    d.y_batch = out.batch;
    d.y_row = out.row;
    const at::Tensor mean = place.empty({d.n, groups});
    const at::Tensor rstd = place.empty({d.n, groups});
    const int rc = efcp_group_norm_forward(
        &d, x.const_data_ptr(), data_of(weight), data_of(bias), y.mutable_data_ptr(),
        mean.mutable_data_ptr<float>(), rstd.mutable_data_ptr<float>(), ws.get(), bytes,
        place.stream.stream());
    return triple(rc, y, mean, rstd);
  });
}

PyObject* group_norm_backward(PyObject*, PyObject* args) {
  PyObject *dy_, *x_, *m_, *r_, *w_, *b_;
  int groups;
  const char* act;
  if (!PyArg_ParseTuple(args, "OOOOiOOs", &dy_, &x_, &m_, &r_, &groups, &w_, &b_, &act))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor &given = tensor_of(x_, "x"), &given_dy = tensor_of(dy_, "dy");
    const at::Tensor &mean = tensor_of(m_, "mean"), &rstd = tensor_of(r_, "rstd");
    const auto weight = maybe_tensor(w_, "weight"), bias = maybe_tensor(b_, "bias");
    efcp_group_norm d = group_norm_desc(given, groups, weight, bias, 0.f, act);
    require(given_dy.layout() == at::kStrided && given_dy.sizes() == given.sizes() &&
                given_dy.scalar_type() == given.scalar_type() &&
                given_dy.device() == given.device() && !given_dy.is_neg(),
            "dy: x's shape, type and device expected");
    for (const at::Tensor* t : {&mean, &rstd})
      require(t->scalar_type() == at::kFloat && t->numel() == d.n * groups && t->is_contiguous() &&
                  t->device() == given.device(),
              "mean, rstd: as group_norm_forward returned them");
    const Place place(given.device());
    const int64_t bytes = efcp_group_norm_workspace_bytes(&d, true);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    Rows in, grad, out;
    const at::Tensor x = channels_last(given, &in), dy = channels_last(given_dy, &grad);
    const at::Tensor dx = new_channels_last(x, &out);
    d.x_batch = in.batch;
    d.x_row = in.row;
    d.dy_batch = grad.batch;
    d.dy_row = grad.row;
    d.y_batch = out.batch;
    d.y_row = out.row;
    const at::Tensor dw = weight ? place.empty(weight->sizes(), weight->scalar_type()) : at::Tensor();
    const at::Tensor db = bias ? place.empty(bias->sizes(), bias->scalar_type()) : at::Tensor();
    const int rc = efcp_group_norm_backward(
        &d, dy.const_data_ptr(), x.const_data_ptr(), mean.const_data_ptr<float>(),
        rstd.const_data_ptr<float>(), data_of(weight), data_of(bias), dx.mutable_data_ptr(),
        dw.defined() ? dw.mutable_data_ptr() : nullptr,
        db.defined() ? db.mutable_data_ptr() : nullptr, ws.get(), bytes,
        place.stream.stream());
    return triple(rc, dx, dw, db);
  });
}

// rows_layout(x): (elements between samples, between positions), or None when a copy would be made;
// as_channels_last(x): x or that copy; like_channels_last(x): an empty output for x.  What the calls
// above do to layouts, on tensors of any device.
PyObject* rows_layout(PyObject*, PyObject* x) {
  return guarded([&]() -> PyObject* {
    const auto r = rows_of(tensor_of(x, "x"));
    if (!r) Py_RETURN_NONE;
    return Py_BuildValue("(LL)", (long long)r->batch, (long long)r->row);
  });
}
PyObject* as_channels_last(PyObject*, PyObject* x) {
  return guarded([&] {
    Rows r;
    return THPVariable_Wrap(channels_last(tensor_of(x, "x"), &r));
  });
}
PyObject* like_channels_last(PyObject*, PyObject* x) {
  return guarded([&] {
    Rows r;
    return THPVariable_Wrap(new_channels_last(tensor_of(x, "x"), &r));
  });
}

PyMethodDef methods[] = {
    {"grads_norm", grads_norm, METH_VARARGS, "efcp_grads_norm"},
    {"grads_clip", grads_clip, METH_VARARGS, "efcp_grads_clip"},
    {"grads_gather", grads_gather, METH_VARARGS, "efcp_grads_gather"},
    {"group_norm_forward", group_norm_forward, METH_VARARGS, "efcp_group_norm_forward"},
    {"group_norm_backward", group_norm_backward, METH_VARARGS, "efcp_group_norm_backward"},
    {"rows_layout", rows_layout, METH_O, "strides of samples and positions, or None"},
    {"as_channels_last", as_channels_last, METH_O, "the tensor, or a channels-last copy"},
    {"like_channels_last", like_channels_last, METH_O, "an empty channels-last tensor"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
